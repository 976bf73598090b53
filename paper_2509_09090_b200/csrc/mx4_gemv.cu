// Product of two microscaled 4-bit matrices for one to four tokens: a weight stream on CUDA cores.
//
// Bounded by HBM: 0.5625 (MXFP4 0.53) bytes per weight, read once. The tensor-core kernel (mx4_linear.cu) needs tensor memory,
// a cluster's exchange and two launches for what is a few microseconds of streaming (1 x 12288 x 4096: 11.1 us, 2.6 TB/s; the
// quantization that every CTA does first and some 2 instructions per code are what is left). Here a code's doubled value (0, 1, 2, 3, 4,
// 6, 8, 12, with a sign) is an int8, so a block's sum of products is exact in integers:
//   sum over the block of x w = (1/4) dp4a(...),  then the two block scales in fp32 (the quarter is in the tokens').
// Four nibbles become four bytes by one byte permute of an 8-byte table with the nibbles as selectors: the selector's top bit
// (the code's sign) replaces the byte by its sign bit, 0 here, so one permute gives the positive codes and a second, with the
// signs flipped, the negative ones.
// The tokens are quantized by every CTA itself (a few hundred instructions, while its first weights travel) where the call
// brings them as rows; they lie in shared memory as int8, with their scales. Two CTAs to an SM walk the rows, so that this is
// done once for many of them.
// Rows: a 32-byte sector of the scale tiles holds rows r, r + 1 and those 32, 64 and 96 further down, so four warps take those
// eight together, a warp two of them (which share the tokens' reads).
#include <type_traits>

#include "mx4_device.cuh"

namespace sqap {
namespace mx4v {

constexpr int WARPS = 8, TEAMS = WARPS / 4, THREADS = 32 * WARPS;   // a team of four warps takes eight rows
constexpr int AHEAD = 4;               // steps (1024 elements: 32 a lane, one 16-byte load per row) whose loads are in flight together

struct GemvArgs {
    const void* x;                     // rows to be quantized, or null
    int64_t ldx;
    const int32_t* row_index;
    const uint8_t *x_codes, *x_scales;
    const uint8_t *w_codes, *w_scales;
    const float *gx, *gw;
    void* out;
    int64_t ldo;
    int N, K, k_tiles, out_dtype;
};

// Bytes of the four nibbles in the low half of w: magnitudes times two of the positive codes, 0 for the negative ones (and the
// other way round for w ^ 0x8888).
__device__ __forceinline__ uint32_t magnitudes(uint32_t w) {
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(0x03020100u), "r"(0x0C080604u), "r"(w));
    return r;
}
// p - n, byte by byte, of what the two permutes give (at most 12, one of them 0).
__device__ __forceinline__ uint32_t minus(uint32_t p, uint32_t n) { return ((p | 0x80808080u) - n) ^ 0x80808080u; }

// Eight codes as two words of int8 (doubled values).
__device__ __forceinline__ uint2 codes_to_int8(uint32_t w) {
    const uint32_t f = w ^ 0x88888888u;
    return make_uint2(minus(magnitudes(w), magnitudes(f)), minus(magnitudes(w >> 16), magnitudes(f >> 16)));
}

// T = void: the tokens come as codes and scales.
template <typename T, int FMT, int MM>
__global__ void __launch_bounds__(THREADS, 2) mx4_gemv_kernel(GemvArgs a) {
    constexpr int BLK = FMT == SQAP_MX_NVFP4 ? 16 : 32;
    extern __shared__ uint8_t smem[];
    const int K = a.K, groups = K / 32;                  // 32 elements: a lane's share of a step
    // int8 tokens: of each 32 elements the first 16 and the second 16 in arrays of their own (no bank conflicts)
    auto lo = [&](int m) { return reinterpret_cast<uint4*>(smem) + (2 * m) * groups; };
    auto hi = [&](int m) { return reinterpret_cast<uint4*>(smem) + (2 * m + 1) * groups; };
    float* const xs = reinterpret_cast<float*>(smem + MM * K);            // [MM][K / BLK]: a quarter of the scales (codes are doubled)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_launch_dependents();
    pdl_wait();

    // The rows of this team, eight at a time; this warp's share r, r + 1 of a 128-row tile. Loads run AHEAD steps in front of
    // the sums, across the change of rows.
    const int total = (a.N + 127) / 128 * 16, steps = (groups + 31) / 32;
    const int stride = gridDim.x * TEAMS, team = blockIdx.x * TEAMS + (warp >> 2);
    uint4 c[AHEAD][2];
    uint32_t s[AHEAD][2];
    int f_rows = team, f_step = 0;                       // what is fetched next
    const uint4 *w0 = nullptr, *w1 = nullptr;
    const uint8_t* sc = nullptr;
    auto aim = [&]() {
        const int tile = f_rows >> 4, r = (f_rows & 15) * 2 + (warp & 3) * 32, n0 = tile * 128 + r;
        w0 = reinterpret_cast<const uint4*>(a.w_codes + static_cast<size_t>(n0 < a.N ? n0 : 0) * (K / 2));
        w1 = reinterpret_cast<const uint4*>(a.w_codes + static_cast<size_t>(n0 + 1 < a.N ? n0 + 1 : 0) * (K / 2));
        // scale bytes of rows r and r + 1 of the tile: 16 bytes apart
        sc = a.w_scales + static_cast<size_t>(tile) * a.k_tiles * 512 + (r & 31) * 16 + (r >> 5) * 4;
    };
    auto fetch = [&](int i) {
        if (f_rows >= total) return;
        const int g = lane + 32 * f_step;                // the lane's 32 elements
        if (g < groups) {
            c[i][0] = __ldg(w0 + g);
            c[i][1] = __ldg(w1 + g);
            if (FMT == SQAP_MX_NVFP4) {
                const uint8_t* p = sc + static_cast<size_t>(g >> 1) * 512 + (g & 1) * 2;
                s[i][0] = __ldg(reinterpret_cast<const uint16_t*>(p));
                s[i][1] = __ldg(reinterpret_cast<const uint16_t*>(p + 16));
            } else {
                const uint8_t* p = sc + static_cast<size_t>(g >> 2) * 512 + (g & 3);
                s[i][0] = __ldg(p);
                s[i][1] = __ldg(p + 16);
            }
        }
        if (++f_step == steps) {
            f_step = 0;
            f_rows += stride;
            if (f_rows < total) aim();
        }
    };
    if (f_rows < total) aim();
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fetch(i);

    // the tokens
    const float gs = a.gx ? __ldg(a.gx) : 1.0f;
    for (int m = 0; m < MM; ++m) {
        // 16 elements a thread; the count is even, so that the lanes that share a block of 32 run together
        for (int h0 = 0; h0 < 2 * groups; h0 += THREADS) {
            const int h = h0 + threadIdx.x;
            uint2 q;
            float scale;
            if constexpr (!std::is_same<T, void>::value) {
                float v[16], amax = 0.0f;
                if (h < 2 * groups) {
                    const int64_t src = a.row_index ? __ldg(a.row_index + m) : m;
                    amax = load16<T>(static_cast<const T*>(a.x) + src * a.ldx + 16 * h, v);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = 0.0f;
                }
                scale = scale_value<FMT>(quantize16<FMT>(v, amax, gs));
                q = make_uint2(to_e2m1x8(v), to_e2m1x8(v + 8));
            } else if (h < 2 * groups) {
                q = __ldg(reinterpret_cast<const uint2*>(a.x_codes + static_cast<size_t>(m) * (K / 2)) + h);
                scale = scale_value<FMT>(__ldg(a.x_scales + scale_offset(m, 16 * h / BLK, a.k_tiles)));
            }
            if (h < 2 * groups) {
                const uint2 p0 = codes_to_int8(q.x), p1 = codes_to_int8(q.y);
                ((h & 1) ? hi(m) : lo(m))[h >> 1] = make_uint4(p0.x, p0.y, p1.x, p1.y);
                if (FMT == SQAP_MX_NVFP4 || (h & 1) == 0) xs[m * (K / BLK) + 16 * h / BLK] = 0.25f * scale;
            }
        }
    }
    __syncthreads();

    const float alpha = FMT == SQAP_MX_NVFP4 ? __fmul_rn(gs, a.gw ? __ldg(a.gw) : 1.0f) : 1.0f;
    float acc[2][MM] = {};
    int rows = team, step = 0;
    while (rows < total) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (rows >= total) break;
            const int g = lane + 32 * step;
            if (g < groups) {
            uint4 xl[MM], xh[MM];
#pragma unroll
            for (int m = 0; m < MM; ++m) {
                xl[m] = lo(m)[g];
                xh[m] = hi(m)[g];
            }
#pragma unroll
            for (int row = 0; row < 2; ++row) {
                const uint32_t cw[4] = {c[i][row].x, c[i][row].y, c[i][row].z, c[i][row].w};
                int dot[MM][2] = {}, minus_dot[MM][2] = {};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t f = cw[q] ^ 0x88888888u;
                    const uint32_t pos[2] = {magnitudes(cw[q]), magnitudes(cw[q] >> 16)}, neg[2] = {magnitudes(f), magnitudes(f >> 16)};
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t both = MM > 2 ? minus(pos[e], neg[e]) : 0;   // one or two tokens: two dp4a are fewer instructions
#pragma unroll
                        for (int m = 0; m < MM; ++m) {
                            const uint4 x = q < 2 ? xl[m] : xh[m];
                            const int xw = static_cast<int>((q & 1) ? (e ? x.w : x.z) : (e ? x.y : x.x));
                            int* d = &dot[m][q >> 1];
                            if (MM > 2) {
                                *d = __dp4a(static_cast<int>(both), xw, *d);
                            } else {
                                *d = __dp4a(static_cast<int>(pos[e]), xw, *d);
                                minus_dot[m][q >> 1] = __dp4a(static_cast<int>(neg[e]), xw, minus_dot[m][q >> 1]);
                            }
                        }
                    }
                }
                if (MM <= 2)
#pragma unroll
                    for (int m = 0; m < MM; ++m) {
                        dot[m][0] -= minus_dot[m][0];
                        dot[m][1] -= minus_dot[m][1];
                    }
                if (FMT == SQAP_MX_NVFP4) {
                    const float s0 = scale_value<FMT>(s[i][row] & 0xFFu), s1 = scale_value<FMT>(s[i][row] >> 8);
#pragma unroll
                    for (int m = 0; m < MM; ++m) {
                        const float2 x = *reinterpret_cast<const float2*>(xs + m * (K / 16) + 2 * g);
                        acc[row][m] = fmaf(static_cast<float>(dot[m][0]) * x.x, s0, acc[row][m]);
                        acc[row][m] = fmaf(static_cast<float>(dot[m][1]) * x.y, s1, acc[row][m]);
                    }
                } else {
                    const float s0 = scale_value<FMT>(s[i][row]);
                    // The scales reach over the whole range of fp32: they meet before the sum of products does (which is up to 2^12),
                    // bounded, so that a sum of 0 stays 0.
#pragma unroll
                    for (int m = 0; m < MM; ++m)
                        acc[row][m] = fmaf(static_cast<float>(dot[m][0] + dot[m][1]), fminf(xs[m * (K / 32) + g] * s0, 3.4028235e38f), acc[row][m]);
                }
            }
            }
            fetch(i);
            if (++step < steps) continue;
            const int n0 = (rows >> 4) * 128 + (rows & 15) * 2 + (warp & 3) * 32;
#pragma unroll
            for (int row = 0; row < 2; ++row)
#pragma unroll
                for (int m = 0; m < MM; ++m) {
                    float y = acc[row][m];
                    acc[row][m] = 0.0f;
#pragma unroll
                    for (int o = 16; o; o >>= 1) y += __shfl_xor_sync(0xffffffffu, y, o);
                    if (lane == 0 && n0 + row < a.N) {
                        y *= alpha;
                        const int64_t at = m * a.ldo + n0 + row;
                        if (a.out_dtype == SQAP_FP16) static_cast<__half*>(a.out)[at] = __float2half_rn(y);
                        else if (a.out_dtype == SQAP_BF16) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(y);
                        else static_cast<float*>(a.out)[at] = y;
                    }
                }
            step = 0;
            rows += stride;
        }
    }
}

template <typename T, int FMT, int MM>
static sqap_status launch_as(const GemvArgs& a, cudaStream_t s) {
    static PerDevice<int> setup;
    const sqap_status st = setup.run([](int*) { return set_max_dynamic_smem(mx4_gemv_kernel<T, FMT, MM>, 227 * 1024); });
    if (st != SQAP_OK) return st;
    const size_t smem = static_cast<size_t>(MM) * a.K + static_cast<size_t>(MM) * (a.K / mx4_block(FMT)) * sizeof(float);
    const unsigned teams = static_cast<unsigned>((a.N + 127) / 128) * 16u, most = 2u * static_cast<unsigned>(sm_count());
    const unsigned grid = teams / TEAMS < most ? teams / TEAMS : most;
    const cudaError_t e = launch_dependent(mx4_gemv_kernel<T, FMT, MM>, dim3(grid), dim3(THREADS), smem, s, a);
    if (e != cudaSuccess) {
        note_cuda_error(e);
        cudaGetLastError();
        return SQAP_ERR_CUDA;
    }
    count_launch();
    return check_launch();
}
template <typename T, int FMT>
static sqap_status launch_rows(const GemvArgs& a, int M, cudaStream_t s) {
    switch (M) {
        case 1: return launch_as<T, FMT, 1>(a, s);
        case 2: return launch_as<T, FMT, 2>(a, s);
        case 3: return launch_as<T, FMT, 3>(a, s);
        default: return launch_as<T, FMT, 4>(a, s);
    }
}
template <typename T>
static sqap_status launch_format(const GemvArgs& a, int M, int format, cudaStream_t s) {
    return format == SQAP_MX_NVFP4 ? launch_rows<T, SQAP_MX_NVFP4>(a, M, s) : launch_rows<T, SQAP_MX_MXFP4>(a, M, s);
}

}  // namespace mx4v

// One token, or up to four with few elements and few products: their quantization is repeated by every CTA and the integer products
// grow with them, where the tensor-core kernels take four tokens in the time of one. Measured with the quantizer, weights from HBM, this /
// those in a graph, us (called one by one, those take 12 to 18 us for their two launches up to 4096 x 11008). NVFP4, one token: 4096 x 1024
// (rows x K) 3.0 / 6.0, 4096 x 4096 6.1 / 9.6, 12288 x 4096 11.1 / 11.5, 22016 x 4096 16.3 / 17.5, 4096 x 11008 11.7 / 13.5, 8192 x 8192
// 14.3 / 14.5, 4096 x 16384 15.4 / 14.8; two: 4096 x 4096 7.5 / 9.6; four: 1024 x 4096 7.5 / 7.5, 4096 x 1024 5.8 / 6.4.
// MXFP4, one token: 4096 x 4096 5.4 / 9.3, 4096 x 11008 12.3 / 12.5, but 12288 x 4096 12.0 / 11.1, 8192 x 8192 16.1 / 13.9 and
// 22016 x 4096 18.4 / 16.8.
// The tokens as int8 and their scales have to fit shared memory, with room for a second CTA.
bool mx4_gemv_takes(int M, int N, int K, int format) {
    if (M > MX4_GEMV_MAX_ROWS || static_cast<int64_t>(M) * (K + K / mx4_block(format) * 4) > 100 * 1024) return false;
    const int64_t products = static_cast<int64_t>(M) * N * K;
    if (M == 1) return format == SQAP_MX_NVFP4 || products < 48 << 20;
    return static_cast<int64_t>(M) * K <= 12 * 1024 && products <= 48 << 20;
}

sqap_status launch_mx4_gemv(const Mx4Product& q, const void* x, int x_dtype, int64_t ldx, const int32_t* row_index, cudaStream_t s) {
    using namespace mx4v;
    const GemvArgs a = {x, ldx, row_index, q.x_codes, q.x_scales, q.w_codes, q.w_scales, q.gx, q.gw, q.out, q.ldo, q.N, q.K,
                        mx4_k_tiles(q.K, q.format), q.out_dtype};
    if (!x) return launch_format<void>(a, q.M, q.format, s);
    if (x_dtype == SQAP_FP16) return launch_format<__half>(a, q.M, q.format, s);
    if (x_dtype == SQAP_BF16) return launch_format<__nv_bfloat16>(a, q.M, q.format, s);
    return launch_format<float>(a, q.M, q.format, s);
}

}  // namespace sqap
