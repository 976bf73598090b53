// Attention with the weight that each token received. Few rows (decoding, see keeps_scores): the register kernel keeps its scores, 4 bytes for
// each row beside the 2 D bytes of the keys and values that it reads, and a second kernel turns them into weights once the
// log-sum-exps are there. More rows: their scores would be more than the keys; those of the rows that count are computed once more.
//
// A warp holds 16 tokens' keys of a head as the A operand (from codes in registers, as in kv_decode.cu) and goes over the
// query rows, eight at a time, as the B operand: S[token][row], p = 2^(s scale log2 e - lse log2 e), summed over the row in the lane that
// holds it. Codes are exact in fp16 and in bf16, so the queries enter in the type that they have. A CTA's four warps
// take neighbouring tokens and share the query rows, staged 32 at a time in shared memory; heads are shared out over CTAs where tokens are few,
// and their sums added by a second kernel, in the order of the heads. Measured, calls in a graph: 16 x 290 single tokens 15 us, 32 uneven
// histories of up to 16384 148 us (few rows: the attention's reads bound it); 16 prompts of 288, the last 32 queries, 76.5 us, most of it attention;
// this kernel alone 16 us with cold caches, bound by instruction latency (issue 48 %, tensor pipe 18 %).
#include "kv_attention.cuh"

namespace sqap {
namespace kv {
namespace {

constexpr int WARPS = 4, TOKENS = 16 * WARPS;

struct MassArgs {
    AttnArgs a;
    int last_q;
    const float* past;
    float* mass;
    int64_t ldm;
    int tiles, parts;          // token tiles of a sequence; pieces that its heads are cut into
    float* sums;               // [parts][batch][tiles * TOKENS], where there are several
};

template <typename T>
__device__ __forceinline__ void mma_rows(float* d, const uint32_t* a, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma_rows<__half>(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) { mma_16816(d, a, b0, b1); }
template <>
__device__ __forceinline__ void mma_rows<__nv_bfloat16>(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Four codes as two pairs of T; exact.
template <typename T, int TYPE>
__device__ __forceinline__ void word_to_pairs(uint32_t w, uint32_t* lo, uint32_t* hi) {
    if (TYPE == SQAP_KV_INT8) {
        w ^= 0x80808080u;
        *lo = biased_to_half2<0>(w);
        *hi = biased_to_half2<1>(w);
    } else {
        *lo = e4m3x2_to_half2(w & 0xFFFFu);
        *hi = e4m3x2_to_half2(w >> 16);
    }
    if (!std::is_same<T, __half>::value) {
        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(lo)), y = __half22float2(*reinterpret_cast<const __half2*>(hi));
        *lo = pack2<T>(x.x, x.y);
        *hi = pack2<T>(y.x, y.y);
    }
}

// The sum of a token's weights joins what it had.
__device__ __forceinline__ void add_to_past(const MassArgs& m, int b, int token, int tokens, int n_q, float sum) {
    const int64_t at = b * m.ldm + token;
    if (token >= m.ldm) return;
    m.mass[at] = (m.past && token < tokens - n_q ? m.past[at] : 0.0f) + sum;
}

__device__ __forceinline__ void copy_async_16(void* to, const void* from, bool real) {      // zeros where there is nothing to copy
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(to))), "l"(from), "r"(real ? 16 : 0)
                 : "memory");
}
__device__ __forceinline__ void copy_async_4(void* to, const void* from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(to))), "l"(from) : "memory");
}

constexpr int ROWS = 32;               // query rows of a stage
template <typename T, int TYPE, int D>
__global__ void __launch_bounds__(WARPS * 32, D <= 128 ? 5 : 2) kv_mass_kernel(MassArgs m) {
    constexpr int KC = D / 64, LD = D + 8;           // halves of a row in shared memory: 16 bytes on in the banks from row to row
    __shared__ alignas(16) T s_q[2][ROWS][LD];
    __shared__ alignas(8) float s_lse[2][ROWS];
    __shared__ alignas(8) int s_sees[2][ROWS];    // tokens that the row sees, 0 for no row
    pdl_launch_dependents();
    pdl_wait();
    const AttnArgs& a = m.a;
    unsigned id = blockIdx.x;
    Where w = {};
    w.tile = static_cast<int>(id % m.tiles);
    id /= m.tiles;
    const int part = static_cast<int>(id % m.parts);
    w.b = static_cast<int>(id / m.parts);
    w.row0 = a.cu[w.b];
    w.n_q = max(a.cu[w.b + 1] - w.row0, 0);
    w.tokens = max(a.lens[w.b], 0);
    w.len = min(w.tokens, a.max_len);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, G = a.group;
    if (w.tile * TOKENS >= w.len) return;
    const int t0 = w.tile * TOKENS + 16 * warp;
    const int heads_each = (a.c.kv_heads + m.parts - 1) / m.parts, h0 = part * heads_each, h1 = min(h0 + heads_each, a.c.kv_heads);
    const int i0 = max(0, w.n_q - m.last_q), rows = (min(w.n_q, a.max_q) - i0) * G;
    const int j = t0 >> a.c.page_shift;
    const int page = a.c.pages > 0 && t0 < w.len && j < a.ldt ? checked_page(a.c, a.table[w.b * a.ldt + j]) : -1;
    float sum[2] = {0.0f, 0.0f};
    // A stage: ROWS rows of a head, with their log-sum-exps. Rows in front of those that see the CTA's first token give nothing.
    const int64_t blind = a.causal ? static_cast<int64_t>(w.tile) * TOKENS - (static_cast<int64_t>(w.tokens) - w.n_q + i0) : 0;
    const int stages = (rows + ROWS - 1) / ROWS, stage0 = blind <= 0 ? 0 : blind * G / ROWS < stages ? static_cast<int>(blind * G / ROWS) : stages;
    if (stage0 < stages) {
        auto fetch = [&](int h, int stage, int buffer) {
            constexpr int PIECES = D / 8;
#pragma unroll
            for (int x = threadIdx.x; x < ROWS * PIECES; x += WARPS * 32) {
                const int k = x / PIECES, piece = x % PIECES, r = stage * ROWS + k, i = r / G;
                const bool real = r < rows;
                const T* src = static_cast<const T*>(a.q) + (static_cast<int64_t>(w.row0) + i0 + i) * a.ldq + static_cast<int64_t>(h * G + r - i * G) * D + 8 * piece;
                copy_async_16(&s_q[buffer][k][8 * piece], real ? src : a.q, real);
            }
            if (threadIdx.x < ROWS) {
                const int k = threadIdx.x, r = stage * ROWS + k, i = r / G;
                s_sees[buffer][k] = r < rows ? visible(a, w, i0 + i) : 0;
                if (r < rows) copy_async_4(&s_lse[buffer][k], a.lse + (static_cast<int64_t>(w.row0) + i0 + i) * a.heads + h * G + r - i * G);
                else s_lse[buffer][k] = INFINITY;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        // codes and scale of a head's keys, fetched a head ahead
        uint4 codes[KC][2] = {};
        float scale = 0.0f;
        auto fetch_keys = [&](int h) {
            if (page < 0) return;
            const uint8_t* kp = a.c.k.codes + (page_codes(a.c, page, h) + (t0 & ((1 << a.c.page_shift) - 1)) + g) * D + 16 * t;
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                codes[c][0] = __ldg(reinterpret_cast<const uint4*>(kp + 64 * c));
                codes[c][1] = __ldg(reinterpret_cast<const uint4*>(kp + 8 * D + 64 * c));
            }
            scale = __ldg(a.c.k.scales + static_cast<int64_t>(page) * a.c.kv_heads + h);
        };
        fetch(h0, stage0, 0);
        fetch_keys(h0);
        int buffer = 0;
        for (int h = h0; h < h1; ++h) {
            uint32_t kf[KC][4][4];
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                const uint4 x = codes[c][0], y = codes[c][1];
                const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    word_to_pairs<T, TYPE>(xs[q], &kf[c][q][0], &kf[c][q][2]);
                    word_to_pairs<T, TYPE>(ys[q], &kf[c][q][1], &kf[c][q][3]);
                }
            }
            const float fac = scale * a.scale_log2;
            if (h + 1 < h1) fetch_keys(h + 1);
            for (int stage = stage0; stage < stages; ++stage, buffer ^= 1) {
                const bool last = stage + 1 == stages;
                if (!last) fetch(h, stage + 1, buffer ^ 1);
                else if (h + 1 < h1) fetch(h + 1, stage0, buffer ^ 1);
                else asm volatile("cp.async.commit_group;" ::: "memory");
                asm volatile("cp.async.wait_group 1;" ::: "memory");
                __syncthreads();
                if (page >= 0) {
                    const int blocks = min(ROWS, rows - stage * ROWS + 7) / 8;
                    for (int n = 0; n < blocks; ++n) {
                        float sc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int c = 0; c < KC; ++c)
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const uint4 q = *reinterpret_cast<const uint4*>(&s_q[buffer][8 * n + g][64 * c + 16 * t + 8 * half]);
                                mma_rows<T>(sc, kf[c][2 * half], q.x, q.y);
                                mma_rows<T>(sc, kf[c][2 * half + 1], q.z, q.w);
                            }
                        const float2 lse = *reinterpret_cast<const float2*>(&s_lse[buffer][8 * n + 2 * t]);
                        const int2 sees = *reinterpret_cast<const int2*>(&s_sees[buffer][8 * n + 2 * t]);
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float l = (e ? lse.y : lse.x) * 1.4426950408889634f;
                            const int n_seen = (fabsf(l) < INFINITY ? (e ? sees.y : sees.x) : 0) - t0;      // rows that saw nothing, or are not numbers
                            if (g < n_seen) sum[0] += fast_exp2(fmaf(sc[e], fac, -l));
                            if (g + 8 < n_seen) sum[1] += fast_exp2(fmaf(sc[e + 2], fac, -l));
                        }
                    }
                }
                __syncthreads();
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 1);
        sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 2);
        const int token = t0 + g + 8 * e;
        if (t != 0 || token >= w.len) continue;
        if (m.parts > 1) m.sums[(static_cast<int64_t>(part) * a.batch + w.b) * (static_cast<int64_t>(m.tiles) * TOKENS) + token] = sum[e];
        else add_to_past(m, w.b, token, w.tokens, w.n_q, sum[e]);
    }
}

// Scores to weights, summed over heads and rows: a lane takes BLOCKS tokens, 32 apart, the warps of a CTA take the heads in turn and meet
// in shared memory. ROWS rows of a key/value head, 0: any number.
constexpr int FOLD_WARPS = 8;
template <int ROWS, int BLOCKS>
__global__ void __launch_bounds__(FOLD_WARPS * 32) kv_mass_fold_kernel(MassArgs m) {
    __shared__ float red[FOLD_WARPS][32 * BLOCKS];
    pdl_launch_dependents();
    pdl_wait();
    const AttnArgs& a = m.a;
    const int b = static_cast<int>(blockIdx.x / m.tiles), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int token0 = static_cast<int>(blockIdx.x % m.tiles) * 32 * BLOCKS;
    Where w = {};
    w.b = b;
    w.row0 = a.cu[b];
    w.n_q = max(a.cu[b + 1] - w.row0, 0);
    w.tokens = max(a.lens[b], 0);
    w.len = min(w.tokens, a.max_len);
    if (token0 >= w.len) return;
    const int nq = min(w.n_q, a.max_q), per_token = ROWS ? ROWS : a.max_q * a.group, first = max(0, w.n_q - m.last_q) * a.group;
    const int rows = nq * a.group;                                 // of the head; `first` and behind count
    const int limit = nq > 0 && a.c.pages > 0 ? visible(a, w, nq - 1) : 0;      // scores of tokens in front of it are there
    float sum[BLOCKS] = {};
    if (first < rows) {
#pragma unroll 2
        for (int h = warp; h < a.c.kv_heads; h += FOLD_WARPS) {
            const float* s = a.scores + ((static_cast<int64_t>(b) * a.c.kv_heads + h) * a.max_len + token0 + lane) * per_token;
            const float* lse = a.lse + static_cast<int64_t>(w.row0) * a.heads + h * a.group;
            // weights of rows r .. r + N - 1 of this head, N consecutive numbers of a token
            auto add = [&](auto n, int r) {
                constexpr int N = decltype(n)::value;
                float x[BLOCKS][N], minus[N];
#pragma unroll
                for (int k = 0; k < BLOCKS; ++k) {
                    const bool there = token0 + 32 * k + lane < limit;
                    if constexpr (N == 4) {
                        const float4 v = there ? __ldg(reinterpret_cast<const float4*>(s + 32 * k * per_token + r)) : make_float4(0, 0, 0, 0);
                        x[k][0] = v.x;
                        x[k][1] = v.y;
                        x[k][2] = v.z;
                        x[k][3] = v.w;
                    } else {
                        x[k][0] = there ? __ldg(s + 32 * k * per_token + r) : 0.0f;
                    }
                }
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const int i = (r + e) / a.group;
                    const float l = r + e >= first && r + e < rows ? -1.4426950408889634f * __ldg(lse + static_cast<int64_t>(i) * a.heads + r + e - i * a.group) : -INFINITY;
                    minus[e] = fabsf(l) < INFINITY ? l : -INFINITY;
                }
#pragma unroll
                for (int k = 0; k < BLOCKS; ++k)
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (minus[e] > -INFINITY && token0 + 32 * k + lane < limit) sum[k] += fast_exp2(x[k][e] + minus[e]);
            };
            if constexpr (ROWS % 4 == 0 && ROWS > 0) {
#pragma unroll
                for (int r = 0; r < ROWS; r += 4) add(std::integral_constant<int, 4>(), r);
            } else if constexpr (ROWS == 1) {
                add(std::integral_constant<int, 1>(), 0);
            } else {
                for (int r = 0; r < per_token; ++r) add(std::integral_constant<int, 1>(), r);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < BLOCKS; ++k) red[warp][32 * k + lane] = sum[k];
    __syncthreads();
    for (int x = threadIdx.x; x < 32 * BLOCKS && token0 + x < w.len; x += FOLD_WARPS * 32) {
        float total = red[0][x];
#pragma unroll
        for (int i = 1; i < FOLD_WARPS; ++i) total += red[i][x];
        add_to_past(m, b, token0 + x, w.tokens, w.n_q, total);
    }
}
template <int BLOCKS>
cudaError_t launch_fold(const MassArgs& m, unsigned grid, cudaStream_t s) {
    const int rows = m.a.max_q * m.a.group;
    const dim3 g(grid), t(FOLD_WARPS * 32);
    if (rows == 1) return launch_dependent(kv_mass_fold_kernel<1, BLOCKS>, g, t, 0, s, m);
    if (rows == 4) return launch_dependent(kv_mass_fold_kernel<4, BLOCKS>, g, t, 0, s, m);
    if (rows == 8) return launch_dependent(kv_mass_fold_kernel<8, BLOCKS>, g, t, 0, s, m);
    return launch_dependent(kv_mass_fold_kernel<0, BLOCKS>, g, t, 0, s, m);
}

constexpr int SUM_THREADS = 128;
__global__ void __launch_bounds__(SUM_THREADS) kv_mass_sum_kernel(MassArgs m, unsigned blocks) {
    pdl_launch_dependents();
    pdl_wait();
    const AttnArgs& a = m.a;
    const int b = static_cast<int>(blockIdx.x / blocks), token = static_cast<int>(blockIdx.x % blocks) * SUM_THREADS + threadIdx.x;
    const int tokens = max(a.lens[b], 0);
    if (token >= min(tokens, a.max_len)) return;
    const int64_t width = static_cast<int64_t>(m.tiles) * TOKENS;
    const float* p = m.sums + b * width + token;
    float sum = 0.0f;
#pragma unroll 8
    for (int i = 0; i < m.parts; ++i) sum += p[i * a.batch * width];
    add_to_past(m, b, token, tokens, max(a.cu[b + 1] - a.cu[b], 0), sum);
}

template <typename T, int TYPE>
cudaError_t mass_dim(const MassArgs& m, unsigned grid, cudaStream_t s) {
    if (m.a.c.head_dim == 64) return launch_dependent(kv_mass_kernel<T, TYPE, 64>, dim3(grid), dim3(WARPS * 32), 0, s, m);
    if (m.a.c.head_dim == 128) return launch_dependent(kv_mass_kernel<T, TYPE, 128>, dim3(grid), dim3(WARPS * 32), 0, s, m);
    return launch_dependent(kv_mass_kernel<T, TYPE, 256>, dim3(grid), dim3(WARPS * 32), 0, s, m);
}
cudaError_t mass_as(const MassArgs& m, int type, int dtype, unsigned grid, cudaStream_t s) {
    if (dtype == SQAP_FP16) return type == SQAP_KV_INT8 ? mass_dim<__half, SQAP_KV_INT8>(m, grid, s) : mass_dim<__half, SQAP_KV_E4M3>(m, grid, s);
    return type == SQAP_KV_INT8 ? mass_dim<__nv_bfloat16, SQAP_KV_INT8>(m, grid, s) : mass_dim<__nv_bfloat16, SQAP_KV_E4M3>(m, grid, s);
}

struct MassPlan {
    bool keep;                     // the scores are kept
    int blocks;                    // then: runs of 32 tokens that a lane of the second kernel takes
    int tiles, parts;
    size_t attention, bytes;       // of the workspace: the attention's part in front, and all
    bool fits;
};
// Scores are kept where the register kernel has at most 8 rows of a head, or at most 15 and either no more heads than the second kernel has
// warps, or long histories: 4 bytes a row and token, written and read, against 2 D of codes. Kept / computed again, us, D = 128: 1 row, 16 x 290
// tokens of 32 heads 14 / 23; 4 rows, 32 x 16384 of 8 heads 149 / 230; 8 rows, 16 x 290 of 32 23 / 22, 16 x 1000 42 / 52, 32 x 12000 of 8
// 117 / 168; 12 rows, 16 x 290 of 32 43 / 30, 16 x 1000 75 / 66, 16 x 4000 156 / 179, of 8 heads 32 x 290 26 / 27, 32 x 1000 41 / 48, 32 x 12000
// 185 / 217; 16 rows, 16 x 290 of 32 51 / 30, 16 x 4000 200 / 182, of 8 heads 32 x 290 29 / 27, 32 x 1000 44 / 49, 32 x 12000 220 / 221.
bool keeps_scores(const sqap_kv_cache* c, int max_q, int max_len, int heads) {
    const int group = heads / c->kv_heads;
    if (!few_rows(max_q, group, c->head_dim)) return false;
    const int rows = max_q * group;
    return rows <= 8 || (rows < 16 && (c->kv_heads <= FOLD_WARPS || max_len > 2048));
}
MassPlan plan_mass(const sqap_kv_cache* c, int batch, int max_q, int max_len, int heads) {
    MassPlan p;
    p.keep = keeps_scores(c, max_q, max_len, heads);
    p.attention = (sqap_kv_attention_workspace_bytes(c, batch, max_q, max_len, heads) + 15) / 16 * 16;
    if (p.keep) {
        const int64_t runs = max_len > 0 ? (max_len - 1) / 32 + 1 : 0;
        p.blocks = size_product(batch, runs) > 8ll * sm_count() ? 4 : 1;
        p.tiles = static_cast<int>((runs + p.blocks - 1) / p.blocks);
        p.parts = 1;
        const int64_t scores = size_product(batch, heads, max_len, max_q);
        p.fits = size_product(batch, p.tiles) <= 0x7FFFFFFF && scores < int64_t{1} << 60;
        p.bytes = p.attention + static_cast<size_t>(scores) * 4;
        return p;
    }
    p.tiles = max_len > 0 ? (max_len - 1) / TOKENS + 1 : 0;
    const int64_t ctas = size_product(batch, p.tiles), want = ctas > 0 ? static_cast<int64_t>(c->head_dim <= 128 ? 5 : 2) * sm_count() / ctas : 1;
    // as many as run at once, each with the same number of heads but the last
    const int64_t heads_each = want > 0 ? (c->kv_heads + want - 1) / want : c->kv_heads;
    p.parts = static_cast<int>((c->kv_heads + heads_each - 1) / heads_each);
    p.fits = size_product(ctas, p.parts) <= 0x7FFFFFFF;
    p.bytes = p.attention + (p.parts > 1 ? static_cast<size_t>(p.parts) * batch * p.tiles * TOKENS * 4 : 0);
    return p;
}

}  // namespace
}  // namespace kv
}  // namespace sqap

extern "C" size_t sqap_kv_attention_mass_workspace_bytes(const sqap_kv_cache* cache, int batch, int max_q, int max_len, int heads, int last_q) {
    using namespace sqap::kv;
    if (check_cache(cache) != SQAP_OK || batch <= 0 || max_q <= 0 || max_len < 0 || max_len > 1 << 30 || heads <= 0 || heads % cache->kv_heads != 0 || last_q < 0)
        return 0;
    const MassPlan p = plan_mass(cache, batch, max_q, max_len, heads);
    return p.fits ? p.bytes : 0;
}

extern "C" sqap_status sqap_kv_attention_mass(const sqap_kv_cache* cache, const int32_t* table, int64_t ldt, int batch, const int32_t* lens,
                                              const int32_t* cu_q, int max_q, int max_len, const void* q, int64_t ldq, int heads, float scale,
                                              uint32_t flags, int last_q, void* out, int64_t ldo, float* lse, const float* past, float* mass,
                                              int64_t ldm, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace sqap;
    using namespace sqap::kv;
    MassArgs m;
    bool work;
    sqap_status st = begin_attention(m.a, work, cache, table, ldt, batch, lens, cu_q, max_q, max_len, q, ldq, heads, scale, flags, out, ldo, lse, dtype);
    if (st != SQAP_OK) return st;
    if (last_q < 0 || ldm < 0) return SQAP_ERR_INVALID;
    if (!work) return SQAP_OK;
    if (!lse || (ldm > 0 && !mass)) return SQAP_ERR_INVALID;
    if ((reinterpret_cast<uintptr_t>(past) & 3u) || (reinterpret_cast<uintptr_t>(mass) & 3u)) return SQAP_ERR_ALIGN;
    const MassPlan p = plan_mass(cache, batch, max_q, max_len, heads);
    if (!p.fits) return SQAP_ERR_UNSUPPORTED;
    if (p.bytes > 0) {
        if (!workspace) return SQAP_ERR_INVALID;
        if (!aligned16(workspace)) return SQAP_ERR_ALIGN;
        if (workspace_bytes < p.bytes) return SQAP_ERR_NOMEM;
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool weigh = ldm > 0 && p.tiles > 0;
    m.a.scores = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.attention);
    st = run_attention(m.a, p.keep && weigh, cache->type, dtype, workspace, p.attention, s);
    if (st != SQAP_OK || !weigh) return st;
    m.last_q = last_q;
    m.past = past;
    m.mass = mass;
    m.ldm = ldm;
    m.tiles = p.tiles;
    m.parts = p.parts;
    if (p.keep) {
        const unsigned grid = static_cast<unsigned>(static_cast<int64_t>(batch) * p.tiles);
        return finish_launch(p.blocks > 1 ? launch_fold<4>(m, grid, s) : launch_fold<1>(m, grid, s));
    }
    m.sums = m.a.scores;
    st = finish_launch(mass_as(m, cache->type, dtype, static_cast<unsigned>(static_cast<int64_t>(batch) * p.tiles * p.parts), s));
    if (st != SQAP_OK || p.parts <= 1) return st;
    const unsigned blocks = static_cast<unsigned>((static_cast<int64_t>(p.tiles) * TOKENS + SUM_THREADS - 1) / SUM_THREADS);
    return finish_launch(launch_dependent(kv_mass_sum_kernel, dim3(blocks * static_cast<unsigned>(batch)), dim3(SUM_THREADS), 0, s, m, blocks));
}
