// Attention over the paged 8-bit cache: checks, the choice of kernel and of the pieces a history is cut into, and the kernel
// that joins the pieces.
#include "kv_attention.cuh"

namespace sqap {
namespace kv {
namespace {

// Pieces from which on four warps join a row (32 heads, 4096 keys in 16 pieces: 10.5 -> 8.7 us with the attention).
constexpr int COMBINE_SPLITS = 8;

// out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s. A row is joined by WARPS warps, which take its pieces in turn and meet in
// shared memory; four rows / WARPS to a CTA.
template <typename T, int D, int WARPS>
__global__ void __launch_bounds__(128) kv_combine_kernel(AttnArgs a) {
    __shared__ float red[WARPS > 1 ? WARPS : 1][WARPS > 1 ? D : 1], red_l[4];
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % WARPS;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * (4 / WARPS) + warp / WARPS;
    const int i = static_cast<int>(id % a.max_q);
    const int64_t bh = id / a.max_q;
    const int head = static_cast<int>(bh % a.heads);
    const int64_t b = bh / a.heads;
    if (b >= a.batch) return;                                    // WARPS == 4: the whole CTA
    const int row0 = a.cu[b];
    if (i >= a.cu[b + 1] - row0) return;
    const int64_t at = part_index(a, static_cast<int>(b), head, i, 0);
    float m = -INFINITY;
    for (int s = lane; s < a.splits; s += 32) m = fmaxf(m, a.part_ml[at + s].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float ref = m == -INFINITY ? 0.0f : m;
    float l = 0.0f, y[D / 32] = {};
#pragma unroll 4
    for (int s = part; s < a.splits; s += WARPS) {
        const float2 ml = a.part_ml[at + s];
        const float f = fast_exp2(ml.x - ref);                   // 0 for a piece without keys, whose output and denominator are 0
        l = fmaf(ml.y, f, l);
        const float2* p = reinterpret_cast<const float2*>(a.part_o + (at + s) * D) + lane;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) {
            const float2 x = p[32 * e];
            y[2 * e] = fmaf(x.x, f, y[2 * e]);
            y[2 * e + 1] = fmaf(x.y, f, y[2 * e + 1]);
        }
    }
    if (WARPS > 1) {
#pragma unroll
        for (int e = 0; e < D / 64; ++e) *reinterpret_cast<float2*>(&red[part][64 * e + 2 * lane]) = make_float2(y[2 * e], y[2 * e + 1]);
        if (lane == 0) red_l[part] = l;
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int w = 1; w < WARPS; ++w) {
            l += red_l[w];
#pragma unroll
            for (int e = 0; e < D / 64; ++e) {
                const float2 x = *reinterpret_cast<const float2*>(&red[w][64 * e + 2 * lane]);
                y[2 * e] += x.x;
                y[2 * e + 1] += x.y;
            }
        }
    }
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;
    const int64_t row = static_cast<int64_t>(row0) + i;
    uint32_t* out = reinterpret_cast<uint32_t*>(static_cast<T*>(a.out) + row * a.ldo + static_cast<int64_t>(head) * D) + lane;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) out[32 * e] = pack2<T>(y[2 * e] * inv, y[2 * e + 1] * inv);
    if (lane == 0 && a.lse) a.lse[row * a.heads + head] = l != 0.0f ? log_sum(m, l) : -INFINITY;
}

template <typename T, int D>
cudaError_t combine_dim(const AttnArgs& a, cudaStream_t s) {
    const int64_t rows = static_cast<int64_t>(a.batch) * a.heads * a.max_q;
    if (a.splits >= COMBINE_SPLITS && rows <= 0x7FFFFFFF) return launch_dependent(kv_combine_kernel<T, D, 4>, dim3(static_cast<unsigned>(rows)), dim3(128), 0, s, a);
    return launch_dependent(kv_combine_kernel<T, D, 1>, dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(128), 0, s, a);
}
template <typename T>
cudaError_t combine_as(const AttnArgs& a, cudaStream_t s) {
    if (a.c.head_dim == 64) return combine_dim<T, 64>(a, s);
    if (a.c.head_dim == 128) return combine_dim<T, 128>(a, s);
    return combine_dim<T, 256>(a, s);
}

struct Plan {
    bool decode;
    int tiles, splits, chunk;
};
// From the sizes (and the device) alone, so that the workspace can be asked for ahead. Decode: up to 1024 keys a history is cut only where there
// are fewer than three CTAs to an SM, beyond that to four, and to sixteen as long as pieces keep 1024 keys (uneven histories then even
// out). Measured, us, with four / eight / sixteen CTAs to an SM, uneven histories of up to so many keys: 32 x 16384, 8 heads 132 / 147 / 127;
// 32 x 8192, 32 heads 258 / 232 / 219; 32 x 4096, 32 heads 147 / 135 / 131, 8 heads 48 / 48 / 48; 16 x 2048, 32 heads 51.5 / 51.1 / 51.3; but
// one of 32768, 32 heads 42 / 57 / 57 (8 heads 21 all three). Three / four up to 1024 keys: 16 x 290, 32 heads 11.7 / 15.2, 16 x 1000 27.0 / 31.5.
// Prompts: two rounds of CTAs where there is less than one, in pieces of 1024 keys at least: cut / whole, us, 256 rows (8 heads, groups of
// 4) behind 3000 keys 44 / 63, behind 8000 76 / 114; 288 rows behind 4096 (32 heads) 59 / 62.
Plan plan_for(int64_t batch, int kv_heads, int group, int head_dim, int64_t max_q, int64_t max_len) {
    Plan p;
    const int64_t rows = max_q * group;
    p.decode = rows <= decode_max_rows(head_dim);
    const int per_tile = head_dim <= 128 ? PREFILL_TC_ROWS : PREFILL_ROWS;
    p.tiles = p.decode ? 1 : static_cast<int>((rows + per_tile - 1) / per_tile);
    const int64_t ctas = size_product(batch, kv_heads, p.tiles);
    const int64_t sms = sm_count();
    auto pieces = [&](int per_sm) { return ctas > 0 ? (sms * per_sm + ctas - 1) / ctas : 1; };
    auto least = [](int64_t x, int64_t y) { return x < y ? x : y; };
    int64_t splits;
    if (p.decode) {
        const int64_t fill = least(pieces(max_len > 1024 ? 4 : 3), (max_len + 255) / 256), even = least(pieces(16), max_len / 1024);
        splits = fill > even ? fill : even;
    } else {
        splits = ctas < sms ? least(pieces(2), max_len / 1024) : 1;
    }
    if (splits < 1) splits = 1;
    const int64_t chunk = ((max_len + splits - 1) / splits + 127) / 128 * 128;
    p.chunk = static_cast<int>(chunk < 128 ? 128 : chunk);
    p.splits = static_cast<int>((max_len + p.chunk - 1) / p.chunk);
    if (p.splits < 1) p.splits = 1;
    return p;
}
// What the kernels' 32-bit indexes hold.
bool sizes_fit(int batch, int kv_heads, int heads, int max_q, int max_len) {
    return size_product(max_q, heads / kv_heads) <= 1 << 30 && max_len <= 1 << 30 && size_product(batch, heads, max_q) <= 4ll * 0x7FFFFFFF;
}
bool grid_fits(int batch, int kv_heads, const Plan& p) { return size_product(batch, kv_heads, p.splits, p.tiles) <= 0x7FFFFFFF; }
size_t part_bytes(int64_t batch, int heads, int64_t max_q, int head_dim, const Plan& p) {
    if (p.splits <= 1) return 0;
    const size_t parts = static_cast<size_t>(batch) * heads * max_q * p.splits;
    return parts * (static_cast<size_t>(head_dim) * 4 + 8);
}

}  // namespace
}  // namespace kv
}  // namespace sqap

extern "C" size_t sqap_kv_attention_workspace_bytes(const sqap_kv_cache* cache, int batch, int max_q, int max_len, int heads) {
    using namespace sqap::kv;
    if (check_cache(cache) != SQAP_OK || batch <= 0 || max_q <= 0 || max_len < 0 || heads <= 0 || heads % cache->kv_heads != 0) return 0;
    if (!sizes_fit(batch, cache->kv_heads, heads, max_q, max_len)) return 0;
    const Plan p = plan_for(batch, cache->kv_heads, heads / cache->kv_heads, cache->head_dim, max_q, max_len);
    return grid_fits(batch, cache->kv_heads, p) ? part_bytes(batch, heads, max_q, cache->head_dim, p) : 0;
}

extern "C" sqap_status sqap_kv_attention(const sqap_kv_cache* cache, const int32_t* table, int64_t ldt, int batch, const int32_t* lens,
                                         const int32_t* cu_q, int max_q, int max_len, const void* q, int64_t ldq, int heads, float scale,
                                         uint32_t flags, void* out, int64_t ldo, float* lse, int dtype, void* workspace,
                                         size_t workspace_bytes, void* stream) {
    using namespace sqap;
    using namespace sqap::kv;
    sqap_status st = check_cache(cache);
    if (st != SQAP_OK) return st;
    if (batch < 0 || max_q < 0 || max_len < 0 || ldt < 0 || ldt > 0x7FFFFFFF || heads <= 0 || !row_type(dtype)) return SQAP_ERR_INVALID;
    if (flags & ~SQAP_KV_CAUSAL) return SQAP_ERR_INVALID;
    if (heads % cache->kv_heads != 0 || !(scale == scale) || scale - scale != 0.0f) return SQAP_ERR_INVALID;
    const int64_t width = static_cast<int64_t>(heads) * cache->head_dim;
    if (ldq < width || ldo < width) return SQAP_ERR_INVALID;
    if (ldq % 8 != 0 || ldo % 8 != 0) return SQAP_ERR_ALIGN;
    if (batch == 0 || max_q == 0) return SQAP_OK;
    if (!lens || !cu_q || !q || !out || (ldt > 0 && !table)) return SQAP_ERR_INVALID;
    if (!aligned16(q) || !aligned16(out) || (reinterpret_cast<uintptr_t>(lse) & 3u)) return SQAP_ERR_ALIGN;
    AttnArgs a;
    a.c = device_view(cache);
    a.group = heads / cache->kv_heads;
    if (!sizes_fit(batch, cache->kv_heads, heads, max_q, max_len)) return SQAP_ERR_UNSUPPORTED;
    const Plan p = plan_for(batch, cache->kv_heads, a.group, cache->head_dim, max_q, max_len);
    if (!grid_fits(batch, cache->kv_heads, p)) return SQAP_ERR_UNSUPPORTED;
    const size_t need = part_bytes(batch, heads, max_q, cache->head_dim, p);
    if (need > 0) {
        if (!workspace) return SQAP_ERR_INVALID;
        if (!aligned16(workspace)) return SQAP_ERR_ALIGN;
        if (workspace_bytes < need) return SQAP_ERR_NOMEM;
    }
    a.table = table;
    a.ldt = ldt;
    a.batch = batch;
    a.lens = lens;
    a.cu = cu_q;
    a.max_q = max_q;
    a.max_len = max_len;
    a.q = q;
    a.ldq = ldq;
    a.heads = heads;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.causal = (flags & SQAP_KV_CAUSAL) ? 1 : 0;
    a.out = out;
    a.ldo = ldo;
    a.lse = lse;
    a.splits = p.splits;
    a.chunk = p.chunk;
    a.tiles = p.tiles;
    const int64_t parts = static_cast<int64_t>(batch) * heads * max_q * p.splits;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = p.splits > 1 ? reinterpret_cast<float2*>(a.part_o + parts * cache->head_dim) : nullptr;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (p.decode) st = launch_kv_decode(a, cache->type, dtype, s);
    else if (cache->head_dim <= 128) st = launch_kv_prefill_tc(a, cache->type, dtype, s);
    else st = launch_kv_prefill(a, cache->type, dtype, s);
    if (st != SQAP_OK || p.splits <= 1) return st;
    return finish_launch(dtype == SQAP_FP16 ? combine_as<__half>(a, s) : combine_as<__nv_bfloat16>(a, s));
}
