// Attention of a few query rows (n_q x group <= 16 per key/value head, 8 at D = 256) over the paged 8-bit cache.
//
// Bounded by HBM: every code of the history is read once, 2 D bytes per token and head, for 4 D group operations. So the
// codes go from global memory straight to registers in the order in which the matrix instructions want them (no shared
// memory, no transposition): the order of the elements within a contraction is free as long as both operands agree.
//   scores  S[token][row] = K q:  A = 16 tokens x 16 elements. Lane (g, t) loads 16 consecutive bytes of the keys of tokens g
//           and g + 8, elements 64 c + 16 t ...; MMA j of chunk c takes bytes 4 j .. 4 j + 3 of them, and the queries are laid
//           out to match.
//   output  O[element][row] = V^T w:  lane (g, t) loads D/8 consecutive bytes of the values of tokens 2t, 2t+1, 2t+8, 2t+9; byte
//           permutes pair up the tokens of an element. The weights turn from the score layout (token down, row across)
//           into the operand layout by one transposition of 8 x 8 halves (movmatrix) per eight tokens.
// A warp keeps a running maximum, denominator and output of its own over steps of 16 or 32 tokens (see launch_rows); the warps of a
// CTA take the steps of their piece of the history in turn and meet in shared memory once at the end. Histories that are
// too few to fill the device are cut into pieces, joined by kv_combine_kernel. 32 uneven histories of up to 16384 tokens, 8 heads of
// 128 in e4m3, groups of 4: 126 us, 4.8 TB/s; what is left is the start and end of uneven pieces and 16 warps an SM.
#include "kv_attention.cuh"

namespace sqap {
namespace kv {
namespace {

constexpr int WARPS = 4;

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

template <int BYTES>
struct Bytes {
    uint32_t w[BYTES / 4];
};
template <int BYTES>
__device__ __forceinline__ Bytes<BYTES> load_bytes(const uint8_t* p) {
    Bytes<BYTES> r;
    if (BYTES == 8) {
        const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
        r.w[0] = u.x;
        r.w[1] = u.y;
    } else {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const uint4 u = __ldg(reinterpret_cast<const uint4*>(p) + i);
            r.w[4 * i] = u.x;
            r.w[4 * i + 1] = u.y;
            r.w[4 * i + 2] = u.z;
            r.w[4 * i + 3] = u.w;
        }
    }
    return r;
}

// Two fp16x2 from a word of four codes: elements 0, 1 and elements 2, 3.
template <int TYPE>
__device__ __forceinline__ void word_to_half2x2(uint32_t w, uint32_t* lo, uint32_t* hi) {
    if (TYPE == SQAP_KV_INT8) {
        w ^= 0x80808080u;
        *lo = biased_to_half2<0>(w);
        *hi = biased_to_half2<1>(w);
    } else {
        *lo = e4m3x2_to_half2(w & 0xFFFFu);
        *hi = e4m3x2_to_half2(w >> 16);
    }
}

template <typename T, int TYPE, int D, int NT, int GROUPS>
__global__ void __launch_bounds__(WARPS * 32, D <= 128 && NT == 1 && GROUPS == 1 ? 4 : 1) kv_decode_kernel(AttnArgs a) {
    constexpr int STEP = 16 * GROUPS;
    constexpr int KC = D / 64;                     // 16-byte chunks of a key row per lane
    constexpr int VB = D / 8;                      // bytes of a value row per lane
    constexpr int MT = D / 16;                     // MMA rows of 16 elements of the output
    __shared__ float red_m[WARPS][8 * NT], red_l[WARPS][8 * NT];
    __shared__ alignas(16) float red_o[WARPS][8 * NT][D + 4];

    pdl_launch_dependents();
    pdl_wait();
    const Where w = locate(a, blockIdx.x, 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int G = a.group;
    const int nq = w.n_q < a.max_q ? w.n_q : a.max_q;
    const int rows = nq * G;                       // row r: query r / G, head h G + r % G
    if (rows == 0) return;
    const int key0 = w.split * a.chunk;
    const int key1 = a.splits > 1 ? min(key0 + a.chunk, w.len) : w.len;

    // the queries as B operands, scaled row by row to fit fp16
    uint32_t qf[NT][KC][4][2];
    float fac[NT][2];                              // back-scaling of the rows of this lane's columns (2t, 2t + 1)
    int lim[NT][2];                                // keys that those rows may see
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = 8 * n + g;
        const bool real = r < rows;
        const T* src = static_cast<const T*>(a.q) + (static_cast<int64_t>(w.row0) + (real ? r / G : 0)) * a.ldq +
                       static_cast<int64_t>(w.h * G + (real ? r % G : 0)) * D;
        float v[KC][16];
        float amax = 0.0f;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                unpack8<T>(__ldg(reinterpret_cast<const uint4*>(src + 64 * c + 16 * t) + i), v[c] + 8 * i);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (!real) v[c][i] = 0.0f;
                amax = fmaxf(amax, fabsf(v[c][i]));
            }
        }
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        float back;
        const float up = fit_exponent(amax, &back);
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                qf[n][c][j][0] = half2_of(v[c][4 * j] * up, v[c][4 * j + 1] * up);
                qf[n][c][j][1] = half2_of(v[c][4 * j + 2] * up, v[c][4 * j + 3] * up);
            }
        // lane (g, t) needs the factors of rows 2t and 2t + 1, held by lanes (2t, *) and (2t + 1, *)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            fac[n][e] = __shfl_sync(0xffffffffu, back, (2 * t + e) * 4) * a.scale_log2;
            const int rr = 8 * n + 2 * t + e;
            lim[n][e] = rr < rows ? visible(a, w, rr / G) : 0;
        }
    }
    const int lim_max = visible(a, w, nq - 1);     // the last row sees the most
    const int end = a.c.pages > 0 ? min(key1, lim_max) : 0;

    float o[NT][MT][4];
    float m[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][i][e] = 0.0f;
        m[n][0] = m[n][1] = -INFINITY;
        l[n][0] = l[n][1] = 0.0f;
    }
    const int32_t* table = a.table + w.b * a.ldt;
    const int shift = a.c.page_shift, mask = (1 << shift) - 1;

    // A step's loads are issued as soon as their registers are free: the next keys during this step's softmax, the next values
    // at its end, the pages' numbers a step earlier still.
    int entry[GROUPS], page[GROUPS] = {};
    Bytes<16> kw[GROUPS][2][KC];
    Bytes<VB> vw[GROUPS][4];
    float ks[GROUPS], vs[GROUPS];
    auto entries = [&](int k0) {
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
            const int key = k0 + 16 * u, j = key >> shift;
            entry[u] = -1;
            if (key < end && j < a.ldt) entry[u] = __ldg(table + j);
        }
    };
    // a page that does not exist is read as page 0 and masked
    auto token_at = [&](int k0, int u) { return page_codes(a.c, max(page[u], 0), w.h) + ((k0 + 16 * u) & mask); };
    auto load_keys = [&](int k0) {
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
            page[u] = checked_page(a.c, entry[u]);
            const uint8_t* kp = a.c.k.codes + (token_at(k0, u) + g) * D + 16 * t;
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                kw[u][0][c] = load_bytes<16>(kp + 64 * c);
                kw[u][1][c] = load_bytes<16>(kp + 8 * D + 64 * c);
            }
            const int64_t s = static_cast<int64_t>(max(page[u], 0)) * a.c.kv_heads + w.h;
            ks[u] = __ldg(a.c.k.scales + s);
            vs[u] = 0.0f;                          // not page 0's: its reciprocal times a weight of 0 need not be 0
            if (page[u] >= 0) vs[u] = __ldg(a.c.v.scales + s);
        }
    };
    auto load_values = [&](int k0) {
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
            const uint8_t* vp = a.c.v.codes + (token_at(k0, u) + 2 * t) * D + (VB > 16 ? 16 : VB) * g;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint8_t* p = vp + ((i & 1) + (i >> 1) * 8) * D;
                if (VB <= 16) {
                    vw[u][i] = load_bytes<VB>(p);
                } else {
#pragma unroll
                    for (int c = 0; c < VB / 16; ++c) {
                        const Bytes<16> x = load_bytes<16>(p + 128 * c);
#pragma unroll
                        for (int q = 0; q < 4; ++q) vw[u][i].w[4 * c + q] = x.w[q];
                    }
                }
            }
        }
    };
    const int first = key0 + warp * STEP;
    if (first < end) {
        entries(first);
        load_keys(first);
        load_values(first);
        entries(first + WARPS * STEP);
    }
    for (int k0 = first; k0 < end; k0 += WARPS * STEP) {
        const bool more = k0 + WARPS * STEP < end;
        // scores
        float sc[GROUPS][NT][4];
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[u][n][e] = 0.0f;
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t af[4];
                    word_to_half2x2<TYPE>(kw[u][0][c].w[j], &af[0], &af[2]);
                    word_to_half2x2<TYPE>(kw[u][1][c].w[j], &af[1], &af[3]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma_16816(sc[u][n], af, qf[n][c][j][0], qf[n][c][j][1]);
                }
        }
        // (the page and scales of this step, before the next step's take their place)
        bool there[GROUPS];
        float this_ks[GROUPS], lv[GROUPS], iv[GROUPS];
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
            there[u] = page[u] >= 0;
            this_ks[u] = ks[u];
            lv[u] = __log2f(vs[u] > 0.0f ? vs[u] : ZERO_PAGE_SCALE);
            iv[u] = fast_exp2(-lv[u]);             // the reciprocal of what lv stands for: the weights use lv
        }
        if (more) load_keys(k0 + WARPS * STEP);
        // scale, mask, maximum
        float top[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            top[n][0] = m[n][0];
            top[n][1] = m[n][1];
        }
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
            const int base = k0 + 16 * u;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = base + g + (e >> 1) * 8;
                    const bool seen = there[u] && key < min(lim[n][e & 1], end);
                    sc[u][n][e] = seen ? fmaf(sc[u][n][e], fac[n][e & 1] * this_ks[u], lv[u]) : -INFINITY;
                    top[n][e & 1] = fmaxf(top[n][e & 1], sc[u][n][e]);
                }
            if (!there[u] || base + 16 > end) {
                // what lies behind the end of a history may be anything, not-a-numbers included: weight 0 is not enough
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!there[u] || base + 2 * t + (i & 1) + (i >> 1) * 8 >= end)
#pragma unroll
                        for (int q = 0; q < VB / 4; ++q) vw[u][i].w[q] = 0;
            }
        }
        // weights
        uint32_t pf[GROUPS][NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) top[n][e] = fmaxf(top[n][e], __shfl_xor_sync(0xffffffffu, top[n][e], x));
                const float ref = top[n][e] == -INFINITY ? 0.0f : top[n][e];
                const float fade = fast_exp2(m[n][e] - ref);   // m = -inf gives 0
                m[n][e] = top[n][e];
                l[n][e] *= fade;
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    o[n][i][e] *= fade;
                    o[n][i][e + 2] *= fade;
                }
#pragma unroll
                for (int u = 0; u < GROUPS; ++u) {
                    sc[u][n][e] = fast_exp2(sc[u][n][e] - ref);
                    sc[u][n][e + 2] = fast_exp2(sc[u][n][e + 2] - ref);
                    l[n][e] = fmaf(sc[u][n][e] + sc[u][n][e + 2], iv[u], l[n][e]);
                }
            }
#pragma unroll
            for (int u = 0; u < GROUPS; ++u) {
                pf[u][n][0] = transpose_8x8(half2_of(sc[u][n][0], sc[u][n][1]));
                pf[u][n][1] = transpose_8x8(half2_of(sc[u][n][2], sc[u][n][3]));
            }
        }
        // output
#pragma unroll
        for (int u = 0; u < GROUPS; ++u)
#pragma unroll
            for (int q = 0; q < VB / 4; ++q) {
                // four elements of the four tokens: pairs (2t, 2t+1) and (2t+8, 2t+9)
                uint32_t x[2][2], f[2][4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    x[i][0] = __byte_perm(vw[u][2 * i].w[q], vw[u][2 * i + 1].w[q], 0x5140);
                    x[i][1] = __byte_perm(vw[u][2 * i].w[q], vw[u][2 * i + 1].w[q], 0x7362);
                    word_to_half2x2<TYPE>(x[i][0], &f[i][0], &f[i][1]);
                    word_to_half2x2<TYPE>(x[i][1], &f[i][2], &f[i][3]);
                }
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const uint32_t af[4] = {f[0][2 * p], f[0][2 * p + 1], f[1][2 * p], f[1][2 * p + 1]};
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma_16816(o[n][2 * q + p], af, pf[u][n][0], pf[u][n][1]);
                }
            }
        if (more) {
            load_values(k0 + WARPS * STEP);
            entries(k0 + 2 * WARPS * STEP);
        }
    }

    // the warps of the CTA meet
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float x = l[n][e];
#pragma unroll
            for (int s = 4; s < 32; s <<= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
            const int r = 8 * n + 2 * t + e;
            if (r < rows) {
                if (g == 0) {
                    red_m[warp][r] = m[n][e];
                    red_l[warp][r] = x;
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    // MMA row i holds elements 2 i and 2 i + 1 of the lane's run; runs of 16 (8 at D = 64) bytes per g
                    const int el = 2 * i;
                    const int d = VB <= 16 ? VB * g + el : 128 * (el / 16) + 16 * g + el % 16;
                    *reinterpret_cast<float2*>(&red_o[warp][r][d]) = make_float2(o[n][i][e], o[n][i][e + 2]);
                }
            }
        }
    __syncthreads();
    for (int x = threadIdx.x; x < rows * (D / 8); x += WARPS * 32) {
        const int r = x / (D / 8), d = x % (D / 8) * 8;
        float mm = -INFINITY;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) mm = fmaxf(mm, red_m[i][r]);
        const float ref = mm == -INFINITY ? 0.0f : mm;
        float ll = 0.0f, y[8] = {};
#pragma unroll
        for (int i = 0; i < WARPS; ++i) {
            const float f = fast_exp2(red_m[i][r] - ref);
            ll = fmaf(red_l[i][r], f, ll);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = fmaf(red_o[i][r][d + e], f, y[e]);
        }
        const int i = r / G, head = w.h * G + r % G;
        if (a.splits > 1) {
            const int64_t at = part_index(a, w.b, head, i, w.split);
            if (d == 0) a.part_ml[at] = make_float2(mm, ll);
            float4* po = reinterpret_cast<float4*>(a.part_o + at * D + d);
            po[0] = make_float4(y[0], y[1], y[2], y[3]);
            po[1] = make_float4(y[4], y[5], y[6], y[7]);
        } else {
            const float inv = ll != 0.0f ? 1.0f / ll : 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= inv;
            const int64_t row = static_cast<int64_t>(w.row0) + i;
            *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + row * a.ldo + static_cast<int64_t>(head) * D + d) = pack8<T>(y);
            if (d == 0 && a.lse) a.lse[row * a.heads + head] = ll != 0.0f ? log_sum(mm, ll) : -INFINITY;
        }
    }
}

template <typename T, int TYPE, int D>
cudaError_t launch_rows(const AttnArgs& a, unsigned grid, cudaStream_t s) {
    // 16-token groups per step. With one group of 128 elements a fourth CTA fits an SM, at 64 elements a second group's loads in
    // flight count for more. Measured, one / two groups, us: D = 128, 16 x 290 tokens x 32 heads 11.6 / 13.5, 16 x 2048 51.6 / 53.4,
    // 32 sequences of up to 16384 x 8 heads 126 / 137; D = 64, the same, 9.1 / 8.7, 35.0 / 32.7, 83 / 76.
    constexpr int GROUPS = D == 64 ? 2 : 1;
    if constexpr (D != 256)                         // 8 rows at most: decode_max_rows()
        // 9 to 16 rows: one / two groups, 32 x 8192 tokens x 8 heads of 128, 12 rows, 134 / 115; 16 x 2048, 16 rows, 35 / 31.
        if (static_cast<int64_t>(a.max_q) * a.group > 8)
            return launch_dependent(kv_decode_kernel<T, TYPE, D, 2, 2>, dim3(grid), dim3(WARPS * 32), 0, s, a);
    return launch_dependent(kv_decode_kernel<T, TYPE, D, 1, GROUPS>, dim3(grid), dim3(WARPS * 32), 0, s, a);
}
template <typename T, int TYPE>
cudaError_t launch_dim(const AttnArgs& a, unsigned grid, cudaStream_t s) {
    if (a.c.head_dim == 64) return launch_rows<T, TYPE, 64>(a, grid, s);
    if (a.c.head_dim == 128) return launch_rows<T, TYPE, 128>(a, grid, s);
    return launch_rows<T, TYPE, 256>(a, grid, s);
}

}  // namespace

sqap_status launch_kv_decode(const AttnArgs& a, int type, int dtype, cudaStream_t s) {
    const unsigned grid = static_cast<unsigned>(static_cast<int64_t>(a.batch) * a.c.kv_heads * a.splits);
    if (dtype == SQAP_FP16)
        return finish_launch(type == SQAP_KV_INT8 ? launch_dim<__half, SQAP_KV_INT8>(a, grid, s) : launch_dim<__half, SQAP_KV_E4M3>(a, grid, s));
    return finish_launch(type == SQAP_KV_INT8 ? launch_dim<__nv_bfloat16, SQAP_KV_INT8>(a, grid, s)
                                              : launch_dim<__nv_bfloat16, SQAP_KV_E4M3>(a, grid, s));
}

}  // namespace kv
}  // namespace sqap
