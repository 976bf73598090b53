// Attention of many query rows (prompts) over the paged 8-bit cache, head_dim 256, on register matrix instructions. (head_dim 64 and 128:
// kv_prefill_tc.cu, whose items of 256 rows do not fit: 512 columns of tensor memory for the output alone. Items of 128 rows would, 256
// columns of output and two tiles of scores, with 64 KB of queries and two stages of 64 keys and values; that form is not built.)
//
// One CTA takes 128 rows (query x head of the group, packed: the heads that share a key/value head share its tiles) of one
// sequence and key/value head and walks the keys in tiles. A tile's codes are fetched one tile ahead into registers,
// turned into fp16 once per CTA and kept in shared memory, from where the eight warps (16 rows each) feed
// register matrix instructions: scores, running maximum and denominator, weights times values. Bounded by their rate, an
// eighth of tcgen05's, and by the registers that allow one CTA an SM (16 prompts' last 9 tokens behind 290, 32 heads: 73 us, 78 MB).
#include "kv_attention.cuh"

namespace sqap {
namespace kv {
namespace {

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void ldmatrix4(uint32_t* r, uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t* r, uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

constexpr int D = 256;
constexpr int WARPS = 8, THREADS = WARPS * 32;
constexpr int KEYS = 32;                             // keys per tile
constexpr int LD = D + 8;                            // halves per row in shared memory: rows 16 bytes apart in the banks
constexpr int CHUNKS = KEYS * D / 16 / THREADS;      // 16-byte pieces of codes per thread
constexpr int GROUPS = KEYS / 16;
static_assert(WARPS * 16 == PREFILL_ROWS && CHUNKS >= 1, "tile shape");

template <typename T, int TYPE>
__global__ void __launch_bounds__(THREADS, 1) kv_prefill_kernel(AttnArgs a) {
    __shared__ alignas(16) __half sk[KEYS][LD];
    __shared__ alignas(16) __half sv[KEYS][LD];
    __shared__ float s_ks[GROUPS], s_lv[GROUPS], s_iv[GROUPS];   // a missing page has lv = -inf

    pdl_launch_dependents();
    pdl_wait();
    Where w = locate(a, blockIdx.x, a.tiles);
    w.tile = a.tiles - 1 - w.tile;                       // the rows that see the most first
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int G = a.group;
    const int nq = w.n_q < a.max_q ? w.n_q : a.max_q;
    const int rows = nq * G;
    const int r_first = w.tile * PREFILL_ROWS;
    if (r_first >= rows) return;
    const int key0 = w.split * a.chunk;
    const int key1 = a.splits > 1 ? min(key0 + a.chunk, w.len) : w.len;
    const int last_row = min(rows, r_first + PREFILL_ROWS) - 1;
    const int end = a.c.pages > 0 ? min(key1, visible(a, w, last_row / G)) : 0;

    // queries: A operands of the warp's 16 rows, scaled row by row to fit fp16
    const int r_warp = r_first + warp * 16;
    uint32_t qf[D / 16][4];
    float fac[2];
    int lim[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int r = r_warp + g + 8 * e;
        const bool real = r < rows;
        const T* src = static_cast<const T*>(a.q) + (static_cast<int64_t>(w.row0) + (real ? r / G : 0)) * a.ldq +
                       static_cast<int64_t>(w.h * G + (real ? r % G : 0)) * D;
        // lane (g, t) holds elements 2t, 2t+1, 2t+8, 2t+9 of every sixteen
        float amax = 0.0f;
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {
            const uint32_t u = real ? __ldg(reinterpret_cast<const uint32_t*>(src + 8 * k + 2 * t)) : 0u;
            qf[k >> 1][(k & 1) * 2 + e] = u;
            const T* x = reinterpret_cast<const T*>(&u);
            amax = fmaxf(amax, fmaxf(fabsf(to_f<T>(x[0])), fabsf(to_f<T>(x[1]))));
        }
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        float back;
        const float up = fit_exponent(amax, &back);
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {
            const uint32_t u = qf[k >> 1][(k & 1) * 2 + e];
            const T* x = reinterpret_cast<const T*>(&u);
            qf[k >> 1][(k & 1) * 2 + e] = half2_of(to_f<T>(x[0]) * up, to_f<T>(x[1]) * up);
        }
        fac[e] = back * a.scale_log2;
        lim[e] = real ? min(visible(a, w, r / G), end) : 0;
    }

    float o[D / 8][4];
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] = 0.0f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};

    const int32_t* table = a.table + w.b * a.ldt;
    const int shift = a.c.page_shift, mask = (1 << shift) - 1;
    auto page_at = [&](int key) {
        const int j = key >> shift;
        return key < end && j < a.ldt ? checked_page(a.c, __ldg(table + j)) : -1;
    };
    uint4 kc[CHUNKS], vc[CHUNKS];
    float next_ks = 0.0f, next_vs = 0.0f;
    int next_page = -1;
    auto fetch = [&](int k0) {
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int x = threadIdx.x + i * THREADS, row = x / (D / 16), col = x % (D / 16) * 16;
            const int key = k0 + row;
            const int page = page_at(key);
            kc[i] = vc[i] = make_uint4(0, 0, 0, 0);       // behind the end: zero codes, whatever lies there
            if (page >= 0) {
                const int64_t at = (page_codes(a.c, page, w.h) + (key & mask)) * D + col;
                kc[i] = __ldg(reinterpret_cast<const uint4*>(a.c.k.codes + at));
                vc[i] = __ldg(reinterpret_cast<const uint4*>(a.c.v.codes + at));
            }
        }
        if (threadIdx.x < GROUPS) {
            next_page = page_at(k0 + 16 * threadIdx.x);
            next_ks = next_vs = 0.0f;
            if (next_page >= 0) {
                const int64_t s = static_cast<int64_t>(next_page) * a.c.kv_heads + w.h;
                next_ks = __ldg(a.c.k.scales + s);
                next_vs = __ldg(a.c.v.scales + s);
            }
        }
    };
    auto put16 = [&](__half* to, uint4 u) {
        const uint32_t in[4] = {u.x, u.y, u.z, u.w};
        uint32_t out[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (TYPE == SQAP_KV_INT8) {
                out[2 * i] = biased_to_half2<0>(in[i] ^ 0x80808080u);
                out[2 * i + 1] = biased_to_half2<1>(in[i] ^ 0x80808080u);
            } else {
                out[2 * i] = e4m3x2_to_half2(in[i] & 0xFFFFu);
                out[2 * i + 1] = e4m3x2_to_half2(in[i] >> 16);
            }
        }
        reinterpret_cast<uint4*>(to)[0] = make_uint4(out[0], out[1], out[2], out[3]);
        reinterpret_cast<uint4*>(to)[1] = make_uint4(out[4], out[5], out[6], out[7]);
    };

    if (key0 < end) fetch(key0);
    for (int k0 = key0; k0 < end; k0 += KEYS) {
        __syncthreads();                                  // the tile before has been read
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int x = threadIdx.x + i * THREADS, row = x / (D / 16), col = x % (D / 16) * 16;
            put16(&sk[row][col], kc[i]);
            put16(&sv[row][col], vc[i]);
        }
        if (threadIdx.x < GROUPS) {
            const float x = next_vs > 0.0f ? next_vs : ZERO_PAGE_SCALE;
            const float lv = __log2f(x);
            s_ks[threadIdx.x] = next_ks;
            s_lv[threadIdx.x] = next_page >= 0 ? lv : -INFINITY;
            s_iv[threadIdx.x] = fast_exp2(-lv);
        }
        __syncthreads();
        if (k0 + KEYS < end) fetch(k0 + KEYS);

        float sc[KEYS / 8][4];
#pragma unroll
        for (int j = 0; j < KEYS / 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[j][e] = 0.0f;
        // lane x of an ldmatrix names row x % 8 of matrix x / 8: four matrices = 32 elements of 8 keys
#pragma unroll
        for (int j = 0; j < KEYS / 8; ++j)
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                uint32_t b[4];
                ldmatrix4(b, smem_addr(&sk[8 * j + (lane & 7)][32 * k + 8 * (lane >> 3)]));
                mma_16816(sc[j], qf[2 * k], b[0], b[1]);
                mma_16816(sc[j], qf[2 * k + 1], b[2], b[3]);
            }
        float top[2] = {m[0], m[1]};
#pragma unroll
        for (int j = 0; j < KEYS / 8; ++j) {
            const float ks = s_ks[j >> 1], lv = s_lv[j >> 1];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int key = k0 + 8 * j + 2 * t + (e & 1);
                // lv = -inf for a missing page: its scores (of zero codes) become -inf as well
                sc[j][e] = key < lim[e >> 1] ? fmaf(sc[j][e], fac[e >> 1] * ks, lv) : -INFINITY;
                top[e >> 1] = fmaxf(top[e >> 1], sc[j][e]);
            }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 1));
            top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 2));
            const float ref = top[e] == -INFINITY ? 0.0f : top[e];
            const float fade = fast_exp2(m[e] - ref);
            m[e] = top[e];
            l[e] *= fade;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                o[i][2 * e] *= fade;
                o[i][2 * e + 1] *= fade;
            }
#pragma unroll
            for (int j = 0; j < KEYS / 8; ++j) {
                sc[j][2 * e] = fast_exp2(sc[j][2 * e] - ref);
                sc[j][2 * e + 1] = fast_exp2(sc[j][2 * e + 1] - ref);
                l[e] = fmaf(sc[j][2 * e] + sc[j][2 * e + 1], s_iv[j >> 1], l[e]);
            }
        }
#pragma unroll
        for (int kk = 0; kk < KEYS / 16; ++kk) {
            const uint32_t p[4] = {half2_of(sc[2 * kk][0], sc[2 * kk][1]), half2_of(sc[2 * kk][2], sc[2 * kk][3]),
                                   half2_of(sc[2 * kk + 1][0], sc[2 * kk + 1][1]), half2_of(sc[2 * kk + 1][2], sc[2 * kk + 1][3])};
            // four matrices: keys 0-7 and 8-15 of two runs of 8 elements
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                uint32_t b[4];
                ldmatrix4_trans(b, smem_addr(&sv[16 * kk + (lane & 15)][16 * i + 8 * (lane >> 4)]));
                mma_16816(o[2 * i], p, b[0], b[1]);
                mma_16816(o[2 * i + 1], p, b[2], b[3]);
            }
        }
    }

#pragma unroll
    for (int e = 0; e < 2; ++e) {
        l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
        l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
        const int r = r_warp + g + 8 * e;
        if (r >= rows) continue;
        const int i = r / G, head = w.h * G + r % G;
        if (a.splits > 1) {
            const int64_t at = part_index(a, w.b, head, i, w.split);
            if (t == 0) a.part_ml[at] = make_float2(m[e], l[e]);
            float* po = a.part_o + at * D + 2 * t;
#pragma unroll
            for (int x = 0; x < D / 8; ++x) *reinterpret_cast<float2*>(po + 8 * x) = make_float2(o[x][2 * e], o[x][2 * e + 1]);
        } else {
            const float inv = l[e] != 0.0f ? 1.0f / l[e] : 0.0f;
            const int64_t row = static_cast<int64_t>(w.row0) + i;
            T* out = static_cast<T*>(a.out) + row * a.ldo + static_cast<int64_t>(head) * D + 2 * t;
#pragma unroll
            for (int x = 0; x < D / 8; ++x) *reinterpret_cast<uint32_t*>(out + 8 * x) = pack2<T>(o[x][2 * e] * inv, o[x][2 * e + 1] * inv);
            if (t == 0 && a.lse) a.lse[row * a.heads + head] = l[e] != 0.0f ? log_sum(m[e], l[e]) : -INFINITY;
        }
    }
}

template <typename T, int TYPE>
cudaError_t launch_as(const AttnArgs& a, unsigned grid, cudaStream_t s) {
    return launch_dependent(kv_prefill_kernel<T, TYPE>, dim3(grid), dim3(THREADS), 0, s, a);
}

}  // namespace

sqap_status launch_kv_prefill(const AttnArgs& a, int type, int dtype, cudaStream_t s) {
    const unsigned grid = static_cast<unsigned>(static_cast<int64_t>(a.batch) * a.c.kv_heads * a.splits * a.tiles);
    if (dtype == SQAP_FP16)
        return finish_launch(type == SQAP_KV_INT8 ? launch_as<__half, SQAP_KV_INT8>(a, grid, s) : launch_as<__half, SQAP_KV_E4M3>(a, grid, s));
    return finish_launch(type == SQAP_KV_INT8 ? launch_as<__nv_bfloat16, SQAP_KV_INT8>(a, grid, s)
                                              : launch_as<__nv_bfloat16, SQAP_KV_E4M3>(a, grid, s));
}

}  // namespace kv
}  // namespace sqap
