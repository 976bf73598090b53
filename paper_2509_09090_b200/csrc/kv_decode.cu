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
// 128 in e4m3, groups of 4: 124 us, 4.9 TB/s; what is left is the start and end of uneven pieces and 16 warps an SM.
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

template <typename T, int TYPE, int D, int NT, int GROUPS, int VIEW>
__global__ void __launch_bounds__(WARPS * 32, D <= 128 && NT == 1 && GROUPS == 1 ? 4 : 1) kv_decode_kernel(AttnArgs a) {
    constexpr int STEP = 16 * GROUPS;
    constexpr bool WHOLE = VIEW == VIEW_ALL || VIEW == VIEW_SCORES;
    constexpr int KC = D / 64;                     // 16-byte chunks of a key row per lane
    constexpr int VB = D / 8;                      // bytes of a value row per lane
    constexpr int MT = D / 16;                     // MMA rows of 16 elements of the output
    __shared__ float red_m[WARPS][8 * NT], red_l[WARPS][8 * NT];
    __shared__ alignas(16) float red_o[WARPS][8 * NT][D + 4];

    pdl_launch_dependents();
    pdl_wait();
    const Where w = locate_view<VIEW>(a, blockIdx.x, of_several<VIEW> ? a.tiles : 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int G = a.group;
    const int rows_all = rows_of<VIEW>(a, w);      // row r: query r / G, head h G + r % G
    const int r_first = of_several<VIEW> ? w.tile * 8 * NT : 0;
    const int rows = min(rows_all - r_first, 8 * NT);
    if (rows <= 0) return;
    const Span span = span_of<VIEW, STEP>(a, w, 0);
    // VIEW_SHARED: the keys are the prefix, then the own tokens of each sequence that has rows here, in runs of 16; lane 0 knows the
    // prefix, lane s the s-th of the sequences: the run it begins with, its first token less 16 times that, and its last
    int seg_run = 0x7FFFFFFF, seg_base = 0, seg_end = 0, seg0 = 0, runs = 0;
    if constexpr (of_several<VIEW>) {
        const int per = a.max_q * G;
        seg0 = r_first / per;
        const int segments = (r_first + rows - 1) / per - seg0 + 2;
        int mine = 0, first = 0;
        if (lane == 0) {
            seg_end = w.prefix;
            mine = VIEW == VIEW_SHARED ? (w.prefix + 15) >> 4 : 0;
        } else if (lane < segments) {
            seg_end = min(max(a.lens[w.b + seg0 + lane - 1], 0), a.max_len);
            first = w.prefix & ~15;
            mine = seg_end > w.prefix ? (seg_end - first + 15) >> 4 : 0;
        }
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        runs = __shfl_sync(0xffffffffu, upto, 31);
        if (lane < segments) seg_run = upto - mine;
        seg_base = first - 16 * (upto - mine);
    }
    auto segment_of = [&](int k) { return of_several<VIEW> ? __popc(__ballot_sync(0xffffffffu, seg_run <= k >> 4)) - 1 : 0; };
    auto token_of = [&](int k, int seg) { return of_several<VIEW> ? __shfl_sync(0xffffffffu, seg_base, seg) + k : span.token(k); };
    const int len = of_several<VIEW> ? 16 * runs : w.len - span.gap;
    const int chunk = chunk_of<VIEW>(a, len);
    const int key0 = w.split * chunk;              // keys: tokens without the gap
    const int key1 = a.splits > 1 ? min(key0 + chunk, len) : len;

    // the queries as B operands, scaled row by row to fit fp16
    uint32_t qf[NT][KC][4][2];
    float fac[NT][2];                              // back-scaling of the rows of this lane's columns (2t, 2t + 1)
    int lim[NT][2], low[NT][2];                    // tokens that those rows may see: below lim, and from low on or below a.sinks
                                                   // (VIEW_SHARED: low is the segment of the row's own tokens)
    int lim_all = 0x7FFFFFFF, low_all = 0;         // tokens that all rows see: below lim_all, from low_all on
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const Row row = row_at<VIEW>(a, w, rows_all, r_first + 8 * n + g);
        const bool real = row.real;
        const T* src = static_cast<const T*>(a.q) + row.at * a.ldq + static_cast<int64_t>(row.head) * D;
        float v[KC][16];
        float amax = 0.0f;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint4 u = make_uint4(0, 0, 0, 0);
                if (!of_several<VIEW> || real) u = __ldg(reinterpret_cast<const uint4*>(src + 64 * c + 16 * t) + i);
                unpack8<T>(u, v[c] + 8 * i);
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
            const Row seen_by = row_at<VIEW>(a, w, rows_all, r_first + 8 * n + 2 * t + e);
            lim[n][e] = seen_by.sees;
            low[n][e] = of_several<VIEW> ? seen_by.b - w.b - seg0 + 1 : first_seen<VIEW>(a, w, seen_by.i);
            if (seen_by.real) {
                lim_all = min(lim_all, lim[n][e]);
                low_all = max(low_all, low[n][e]);
            }
        }
    }
    lim_all = __reduce_min_sync(0xffffffffu, lim_all);
    low_all = __reduce_max_sync(0xffffffffu, low_all);
    // the last row sees the most
    const int lim_max = of_several<VIEW> ? len : visible(a, w, rows / G - 1) - span.gap;
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
    const int per_token = a.max_q * G;
    float* scores = VIEW == VIEW_SCORES ? a.scores + (static_cast<int64_t>(w.b) * a.c.kv_heads + w.h) * a.max_len * per_token : nullptr;
    const int32_t* table = a.table + w.b * a.ldt;
    const int from = first_seen<VIEW>(a, w, 0);
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
            const int key = k0 + 16 * u, seg = segment_of(key), token = token_of(key, seg), j = token >> shift;
            entry[u] = -1;
            if (key < end && j < a.ldt && run_counts<VIEW>(a, token, from)) entry[u] = __ldg(table + (of_several<VIEW> && seg > 0 ? (seg0 + seg - 1) * a.ldt : 0) + j);
        }
    };
    // a page that does not exist is read as page 0 and masked
    auto token_at = [&](int k0, int u) {
        return page_codes(a.c, max(page[u], 0), w.h) + (token_of(k0 + 16 * u, segment_of(k0 + 16 * u)) & mask);
    };
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
        // scale, mask, maximum of what this lane holds
        float top[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) top[n][0] = top[n][1] = -INFINITY;
#pragma unroll
        for (int u = 0; u < GROUPS; ++u) {
            const int base = k0 + 16 * u;
            // the run's first token, and those of it that are the segment's: from .. until - 1
            const int seg = segment_of(base), token0 = WHOLE ? base : token_of(base, seg);
            const int begin = VIEW == VIEW_OWN || (of_several<VIEW> && seg > 0) ? w.prefix : 0;
            const int until = of_several<VIEW> ? (base < end ? __shfl_sync(0xffffffffu, seg_end, seg) : 0) : end - base + token0;
            // most runs are seen by all rows as they are
            const bool plain = there[u] && token0 + 16 <= min(until, lim_all) && (VIEW != VIEW_OWN || token0 >= begin) && (!of_several<VIEW> || seg == 0) &&
                               (VIEW != VIEW_WINDOW || token0 >= low_all);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float f[2] = {fac[n][0] * this_ks[u], fac[n][1] * this_ks[u]};
                if (VIEW == VIEW_SCORES) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[u][n][e] *= f[e & 1];
                    if (!plain) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!there[u] || token0 + g + (e >> 1) * 8 >= min(lim[n][e & 1], until)) sc[u][n][e] = -INFINITY;
                    }
                    const int r = 8 * n + 2 * t;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int token = token0 + g + half * 8;
                        float* to = scores + static_cast<int64_t>(token) * per_token + r;
                        if (token < end && r < rows) {
                            if ((per_token & 1) == 0) {
                                *reinterpret_cast<float2*>(to) = make_float2(sc[u][n][2 * half], sc[u][n][2 * half + 1]);
                            } else {
                                to[0] = sc[u][n][2 * half];
                                if (r + 1 < rows) to[1] = sc[u][n][2 * half + 1];
                            }
                        }
                        sc[u][n][2 * half] += lv[u];
                        sc[u][n][2 * half + 1] += lv[u];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[u][n][e] = fmaf(sc[u][n][e], f[e & 1], lv[u]);
                    if (!plain) {
                        int limit[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            limit[e] = there[u] ? min(lim[n][e], until) : 0;
                            if (of_several<VIEW> && seg > 0 && seg != low[n][e]) limit[e] = 0;       // another sequence's tokens
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (token0 + g + (e >> 1) * 8 >= limit[e & 1]) sc[u][n][e] = -INFINITY;
                        if ((VIEW == VIEW_OWN || of_several<VIEW>) && token0 < begin) {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (token0 + g + (e >> 1) * 8 < begin) sc[u][n][e] = -INFINITY;
                        }
                        if (VIEW == VIEW_WINDOW && token0 < low_all) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int token = token0 + g + (e >> 1) * 8;
                                if (token < low[n][e & 1] && token >= a.sinks) sc[u][n][e] = -INFINITY;
                            }
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) top[n][e & 1] = fmaxf(top[n][e & 1], sc[u][n][e]);
            }
            if (!there[u] || token0 + 16 > until || token0 < begin) {
                // what lies behind the end of a history may be anything, not-a-numbers included: weight 0 is not enough
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!there[u] || token0 + 2 * t + (i & 1) + (i >> 1) * 8 >= until || token0 + 2 * t + (i & 1) + (i >> 1) * 8 < begin)
#pragma unroll
                        for (int q = 0; q < VB / 4; ++q) vw[u][i].w[q] = 0;
            }
        }
        // where a maximum grows, the rows are brought down to the new one
        bool raise = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) raise = raise || top[n][0] > m[n][0] || top[n][1] > m[n][1];
        if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = fmaxf(m[n][e], top[n][e]);
#pragma unroll
                    for (int y = 4; y < 32; y <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, y));
                    const float fade = fast_exp2(m[n][e] - (x == -INFINITY ? 0.0f : x));   // m = -inf gives 0
                    m[n][e] = x;
                    l[n][e] *= fade;
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        o[n][i][e] *= fade;
                        o[n][i][e + 2] *= fade;
                    }
                }
        }
        // weights
        uint32_t pf[GROUPS][NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float ref = m[n][e] == -INFINITY ? 0.0f : m[n][e];
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
        const Row row = row_at<VIEW>(a, w, rows_all, r_first + r);
        if (of_several<VIEW> && !row.real) continue;
        if ((VIEW == VIEW_OWN || VIEW == VIEW_OWN_ROWS) && a.join > 0) {
            // the pieces of the prefix are there: joined here
            const int64_t at = part_index(a, row.b, row.head, row.i, 0);
            float top = mm;
#pragma unroll 8
            for (int s = 0; s < a.join; ++s) top = fmaxf(top, a.part_ml[at + s].x);
            const float base = top == -INFINITY ? 0.0f : top, f = fast_exp2(mm - base);
            ll *= f;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= f;
#pragma unroll 8
            for (int s = 0; s < a.join; ++s) {
                const float2 ml = a.part_ml[at + s];
                const float c = fast_exp2(ml.x - base);
                const float4* p = reinterpret_cast<const float4*>(a.part_o + (at + s) * D + d);
                const float4 p0 = p[0], p1 = p[1];
                ll = fmaf(ml.y, c, ll);
                y[0] = fmaf(p0.x, c, y[0]);
                y[1] = fmaf(p0.y, c, y[1]);
                y[2] = fmaf(p0.z, c, y[2]);
                y[3] = fmaf(p0.w, c, y[3]);
                y[4] = fmaf(p1.x, c, y[4]);
                y[5] = fmaf(p1.y, c, y[5]);
                y[6] = fmaf(p1.z, c, y[6]);
                y[7] = fmaf(p1.w, c, y[7]);
            }
            mm = top;
        }
        if (a.parts > 1 && !((VIEW == VIEW_OWN || VIEW == VIEW_OWN_ROWS) && a.join > 0)) {
            const int64_t at = part_index(a, row.b, row.head, row.i, w.split);
            if (d == 0) a.part_ml[at] = make_float2(mm, ll);
            float4* po = reinterpret_cast<float4*>(a.part_o + at * D + d);
            po[0] = make_float4(y[0], y[1], y[2], y[3]);
            po[1] = make_float4(y[4], y[5], y[6], y[7]);
        } else {
            const float inv = ll != 0.0f ? 1.0f / ll : 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= inv;
            *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + row.at * a.ldo + static_cast<int64_t>(row.head) * D + d) = pack8<T>(y);
            if (d == 0 && a.lse) a.lse[row.at * a.heads + row.head] = ll != 0.0f ? log_sum(mm, ll) : -INFINITY;
        }
    }
}

template <typename T, int TYPE, int D, int VIEW>
cudaError_t launch_rows(const AttnArgs& a, unsigned grid, cudaStream_t s) {
    // 16-token groups per step. With one group of 128 elements a fourth CTA fits an SM, at 64 elements a second group's loads in
    // flight count for more. Measured, one / two groups, us: D = 128, 16 x 290 tokens x 32 heads 11.6 / 13.5, 16 x 2048 51.6 / 53.4,
    // 32 sequences of up to 16384 x 8 heads 126 / 137; D = 64, the same, 9.1 / 8.7, 35.0 / 32.7, 83 / 76.
    constexpr int GROUPS = D == 64 ? 2 : 1;
    // D = 256: 8 rows at most (decode_max_rows()); the rows of a group are always taken in tiles of 8
    if constexpr (D != 256 && !of_several<VIEW>)
        // 9 to 16 rows: one / two groups, 32 x 8192 tokens x 8 heads of 128, 12 rows, 134 / 115; 16 x 2048, 16 rows, 35 / 31.
        if (a.row_tile > 8)
            return launch_dependent(kv_decode_kernel<T, TYPE, D, 2, 2, VIEW>, dim3(grid), dim3(WARPS * 32), 0, s, a);
    return launch_dependent(kv_decode_kernel<T, TYPE, D, 1, GROUPS, VIEW>, dim3(grid), dim3(WARPS * 32), 0, s, a);
}
template <typename T, int TYPE, int VIEW>
cudaError_t launch_dim(const AttnArgs& a, unsigned grid, cudaStream_t s) {
    if (a.c.head_dim == 64) return launch_rows<T, TYPE, 64, VIEW>(a, grid, s);
    if (a.c.head_dim == 128) return launch_rows<T, TYPE, 128, VIEW>(a, grid, s);
    return launch_rows<T, TYPE, 256, VIEW>(a, grid, s);
}
template <int VIEW>
cudaError_t launch_view(const AttnArgs& a, int type, int dtype, unsigned grid, cudaStream_t s) {
    if (dtype == SQAP_FP16)
        return type == SQAP_KV_INT8 ? launch_dim<__half, SQAP_KV_INT8, VIEW>(a, grid, s) : launch_dim<__half, SQAP_KV_E4M3, VIEW>(a, grid, s);
    return type == SQAP_KV_INT8 ? launch_dim<__nv_bfloat16, SQAP_KV_INT8, VIEW>(a, grid, s)
                                : launch_dim<__nv_bfloat16, SQAP_KV_E4M3, VIEW>(a, grid, s);
}

}  // namespace

sqap_status launch_kv_decode(const AttnArgs& a, View view, int64_t units, int type, int dtype, cudaStream_t s) {
    const unsigned grid = static_cast<unsigned>(units * a.c.kv_heads * a.splits * a.tiles);
    switch (view) {
        case VIEW_WINDOW: return finish_launch(launch_view<VIEW_WINDOW>(a, type, dtype, grid, s));
        case VIEW_SHARED: return finish_launch(launch_view<VIEW_SHARED>(a, type, dtype, grid, s));
        case VIEW_OWN_ROWS: return finish_launch(launch_view<VIEW_OWN_ROWS>(a, type, dtype, grid, s));
        case VIEW_OWN: return finish_launch(launch_view<VIEW_OWN>(a, type, dtype, grid, s));
        case VIEW_SCORES: return finish_launch(launch_view<VIEW_SCORES>(a, type, dtype, grid, s));
        default: return finish_launch(launch_view<VIEW_ALL>(a, type, dtype, grid, s));
    }
}

}  // namespace kv
}  // namespace sqap
