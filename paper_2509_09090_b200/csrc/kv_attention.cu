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
    __shared__ alignas(8) float red[WARPS > 1 ? WARPS : 1][WARPS > 1 ? D : 1], red_l[4];
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % WARPS;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * (4 / WARPS) + warp / WARPS;
    const int i = static_cast<int>(id % a.max_q);
    const int64_t bh = id / a.max_q;
    const int head = static_cast<int>(bh % a.heads);
    int64_t b = bh / a.heads;
    if (a.cu_group) {                                            // place of a sequence in a group
        const int64_t group = b / a.max_group;
        if (group >= a.groups) return;
        const int first = a.cu_group[group];
        b = first + b % a.max_group;
        if (first < 0 || b >= a.cu_group[group + 1]) return;
    }
    if (b >= a.batch) return;                                    // WARPS == 4: the whole CTA
    const int row0 = a.cu[b];
    if (i >= a.cu[b + 1] - row0) return;
    const int64_t at = part_index(a, static_cast<int>(b), head, i, 0);
    float m = -INFINITY;
    for (int s = lane; s < a.parts; s += 32) m = fmaxf(m, a.part_ml[at + s].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float ref = m == -INFINITY ? 0.0f : m;
    float l = 0.0f, y[D / 32] = {};
#pragma unroll 4
    for (int s = part; s < a.parts; s += WARPS) {
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
cudaError_t combine_dim(const AttnArgs& a, int64_t units, cudaStream_t s) {
    const int64_t rows = units * a.heads * a.max_q;
    if (a.parts >= COMBINE_SPLITS && rows <= 0x7FFFFFFF) return launch_dependent(kv_combine_kernel<T, D, 4>, dim3(static_cast<unsigned>(rows)), dim3(128), 0, s, a);
    return launch_dependent(kv_combine_kernel<T, D, 1>, dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(128), 0, s, a);
}
template <typename T>
cudaError_t combine_as(const AttnArgs& a, int64_t units, cudaStream_t s) {
    if (a.c.head_dim == 64) return combine_dim<T, 64>(a, units, s);
    if (a.c.head_dim == 128) return combine_dim<T, 128>(a, units, s);
    return combine_dim<T, 256>(a, units, s);
}
sqap_status combine(const AttnArgs& a, int64_t units, int dtype, cudaStream_t s) {
    return finish_launch(dtype == SQAP_FP16 ? combine_as<__half>(a, units, s) : combine_as<__nv_bfloat16>(a, units, s));
}

struct Plan {
    bool decode;
    int row_tile;          // of the register kernel
    int tiles, splits, chunk;
};
// From the sizes (and the device) alone, so that the workspace can be asked for ahead: `units` sequences (or groups) of `rows` rows that look
// at up to max_len keys each. Decode: up to 1024 keys a history is cut only where there
// are fewer than three CTAs to an SM, beyond that to four, and to sixteen as long as pieces keep 1024 keys (uneven histories then even
// out). Measured, us, with four / eight / sixteen CTAs to an SM, uneven histories of up to so many keys: 32 x 16384, 8 heads 132 / 147 / 127;
// 32 x 8192, 32 heads 258 / 232 / 219; 32 x 4096, 32 heads 147 / 135 / 131, 8 heads 48 / 48 / 48; 16 x 2048, 32 heads 51.5 / 51.1 / 51.3; but
// one of 32768, 32 heads 42 / 57 / 57 (8 heads 21 all three). Three / four up to 1024 keys: 16 x 290, 32 heads 11.7 / 15.2, 16 x 1000 27.0 / 31.5.
// ALIKE: all rows look at about as many keys (a window): as many pieces as all run at once. 32 windows of 2048, 8 heads, us: 1 piece 46, 2 33,
// 3 39, 5 37, 9 40.
// Prompts: two rounds of CTAs where there is less than one, in pieces of 1024 keys at least: cut / whole, us, 256 rows (8 heads, groups of
// 4) behind 3000 keys 44 / 63, behind 8000 76 / 114; 288 rows behind 4096 (32 heads) 59 / 62.
int64_t least(int64_t x, int64_t y) { return x < y ? x : y; }
// Histories of uneven lengths, as a rule; of about the same (windows); cut on the device, each into the same number of pieces.
enum Cut { UNEVEN, ALIKE, EVENLY };
Plan plan_rows(int64_t units, int kv_heads, int head_dim, int64_t rows, int64_t max_len, bool decode, Cut cut = UNEVEN, int row_tile = 0) {
    Plan p;
    p.decode = decode;
    p.row_tile = row_tile > 0 ? row_tile : rows <= 8 ? 8 : decode_max_rows(head_dim);
    const int per_tile = p.decode ? p.row_tile : head_dim <= 128 ? PREFILL_TC_ROWS : PREFILL_ROWS;
    p.tiles = static_cast<int>((rows + per_tile - 1) / per_tile);
    const int64_t ctas = size_product(units, kv_heads, p.tiles);
    const int64_t sms = sm_count();
    auto pieces = [&](int per_sm) { return ctas > 0 ? (sms * per_sm + ctas - 1) / ctas : 1; };
    int64_t splits;
    if (p.decode) {
        const int64_t at_once = sms * (p.row_tile <= 8 && head_dim <= 128 ? 4 : 2);
        const int64_t fill = least(cut == ALIKE ? at_once / (ctas > 0 ? ctas : 1) : pieces(max_len > 1024 ? 4 : 3), (max_len + 255) / 256), even = least(pieces(16), max_len / 1024);
        splits = fill > even ? fill : even;
    } else {
        splits = ctas >= sms ? 1 : cut != UNEVEN ? least(sms / (ctas > 0 ? ctas : 1), max_len / 512) : least(pieces(2), max_len / 1024);
    }
    if (splits < 1) splits = 1;
    p.splits = static_cast<int>(splits);
    p.chunk = 0;
    if (cut == EVENLY) return p;
    const int64_t chunk = ((max_len + splits - 1) / splits + 127) / 128 * 128;
    p.chunk = static_cast<int>(chunk < 128 ? 128 : chunk);
    p.splits = static_cast<int>((max_len + p.chunk - 1) / p.chunk);
    if (p.splits < 1) p.splits = 1;
    return p;
}
Plan plan_for(int64_t batch, int kv_heads, int group, int head_dim, int64_t max_q, int64_t max_len) {
    const int64_t rows = max_q * group;
    return plan_rows(batch, kv_heads, head_dim, rows, max_len, rows <= decode_max_rows(head_dim));
}
// What the kernels' 32-bit indexes hold.
bool sizes_fit(int batch, int kv_heads, int heads, int max_q, int max_len) {
    return size_product(max_q, heads / kv_heads) <= 1 << 30 && max_len <= 1 << 30 && size_product(batch, heads, max_q) <= 4ll * 0x7FFFFFFF;
}
bool grid_fits(int64_t units, int kv_heads, const Plan& p) { return size_product(units, kv_heads, p.splits, p.tiles) <= 0x7FFFFFFF; }
size_t part_bytes(int64_t batch, int heads, int64_t max_q, int head_dim, int parts) {
    if (parts <= 1) return 0;
    return static_cast<size_t>(batch) * heads * max_q * parts * (static_cast<size_t>(head_dim) * 4 + 8);
}

// Keys that the rows of a CTA look at, at most: a window for the first of its queries, on to the last, the sinks, and both rounded to tiles.
int64_t window_keys(int64_t max_q, int64_t max_len, int group, int head_dim, int64_t window, int64_t sinks) {
    const int64_t rows = max_q * group, tile = head_dim <= 128 ? PREFILL_TC_ROWS : PREFILL_ROWS;
    const int64_t queries = rows <= decode_max_rows(head_dim) || max_q < tile / group + 2 ? max_q : tile / group + 2;
    const int64_t keys = window + queries + sinks + 128;
    return keys < max_len ? keys : max_len;
}
Plan plan_window(int64_t batch, int kv_heads, int group, int head_dim, int64_t max_q, int64_t max_len, int64_t window, int64_t sinks) {
    const int64_t rows = max_q * group;
    return plan_rows(batch, kv_heads, head_dim, rows, window_keys(max_q, max_len, group, head_dim, window, sinks), rows <= decode_max_rows(head_dim), ALIKE);
}

// Shared prefixes: the rows of a group over its prefix, then those of each sequence over its own tokens. The pieces of both are cut on
// the device, from the lengths that it finds; the plan only says how many there are.
struct SharedPlan {
    bool together;         // one launch of the register kernel over the prefix and the own tokens of a group's sequences
    Plan prefix, own;      // `together`: prefix is its plan
    View own_view;         // the own tokens: a CTA takes a sequence, or a tile of the group's rows
    int64_t own_units;
    int prefix_parts;      // 0: there is no prefix
    bool join;             // the kernel of the own tokens joins the pieces of the prefix
    int parts;             // pieces in the workspace
};
// The register kernel takes a group in tiles of 8 rows, each of which reads the prefix (from L2, but for one) and its own sequences' tokens;
// the kernels for many rows read a prefix once for 256 (128) rows, and then the own tokens want a launch of their own. us, tiles / the
// others, 40 to 100 own tokens: 32 heads, prefix 256, 16 groups of 10, 32, 64 rows 40 / 71, 80 / 107, 143 / 165; 8 heads, prefix 16384,
// 16 and 32 rows 23 / 34, 40 / 32; prefix 1000, 16 groups of 16, 32, 64 rows 31 / 34, 43 / 37, 63 / 49; head_dim 256, prefix 4096, 32
// rows 43 / 63. (Tiles of 16 rows: 45, 108, 188; 28, 37; 39, 53, 82.)
bool in_row_tiles(int head_dim, int64_t rows, int64_t max_group, int64_t max_prefix) {
    if (max_prefix == 0 || rows > decode_max_rows(head_dim)) return false;
    const int64_t tiles = (rows * max_group + 7) / 8;
    return tiles <= (head_dim <= 128 ? 3 : 6) || size_product(tiles - 1, max_prefix) <= (head_dim <= 128 ? 2048 : 8192);
}
SharedPlan plan_shared(int kv_heads, int group, int head_dim, int64_t max_q, int64_t max_len, int64_t groups, int64_t max_group,
                       int64_t max_prefix) {
    SharedPlan p;
    const int64_t rows = max_q * group, together = rows * max_group;
    const int64_t own = max_len > max_prefix ? max_len - max_prefix : 1;        // behind the longest prefix
    const int tile = decode_max_rows(head_dim);
    const int64_t sequences = least(max_group, (rows + 6) / rows + 1);          // that a tile of 8 rows meets, if it begins with a sequence's last row
    const int64_t met = size_product(own, sequences);
    // The register kernel's places in all that a row tile meets are 32-bit numbers; behind a prefix shorter than the longest, own tokens are up to max_len.
    const bool places_fit = size_product(sequences, max_len) + max_prefix <= 1 << 30;
    p.together = places_fit && in_row_tiles(head_dim, rows, max_group, max_prefix);
    if (p.together) {
        p.prefix = p.own = plan_rows(groups, kv_heads, head_dim, together, met + max_prefix, true, EVENLY, 8);
        p.own_view = VIEW_SHARED;
        p.own_units = groups;
        p.prefix_parts = 0;
        p.join = false;
        p.parts = p.prefix.splits;
        return p;
    }
    const int64_t places = size_product(groups, max_group);
    // Short tokens of many sequences: a tile of rows to a CTA (16 x 16 sequences of 4 rows, 8 heads, 64 own tokens: 49 us, a sequence to a CTA 53;
    // 16 x 64 of one row, 32 heads, 40 own tokens: 165 / 311; but 4 x 64 of one row, 8 heads, 1000 own tokens: 157 / 143).
    p.own_view = places_fit && rows <= 4 && own <= 512 && size_product(places, kv_heads) > 8ll * sm_count() ? VIEW_OWN_ROWS : VIEW_OWN;
    p.own_units = p.own_view == VIEW_OWN ? places : groups;
    p.own = p.own_view == VIEW_OWN ? plan_rows(places, kv_heads, head_dim, rows, own, rows <= tile, EVENLY)
                                   : plan_rows(groups, kv_heads, head_dim, together, met, true, EVENLY, 8);
    p.prefix = plan_rows(groups, kv_heads, head_dim, together, max_prefix, false, EVENLY);
    p.prefix_parts = max_prefix > 0 ? p.prefix.splits : 0;
    p.join = p.own.decode && p.own.splits == 1 && p.prefix_parts > 0;
    p.parts = p.prefix_parts + (p.join ? 0 : p.own.splits);
    if (p.join && p.parts < 2) p.parts = 2;      // a single one goes through the workspace too
    return p;
}
bool shared_fits(const sqap_kv_cache* c, int groups, int max_group, int max_q, int heads, const SharedPlan& p) {
    return size_product(max_group, max_q, heads / c->kv_heads) <= 1 << 30 && grid_fits(groups, c->kv_heads, p.prefix) &&
           grid_fits(p.own_units, c->kv_heads, p.own) && size_product(groups, max_group, heads, max_q) <= 4ll * 0x7FFFFFFF;
}

sqap_status take_workspace(AttnArgs& a, int parts, void* workspace, size_t workspace_bytes) {
    a.parts = parts;
    const size_t need = part_bytes(a.batch, a.heads, a.max_q, a.c.head_dim, parts);
    if (need == 0) return SQAP_OK;
    if (!workspace) return SQAP_ERR_INVALID;
    if (!aligned16(workspace)) return SQAP_ERR_ALIGN;
    if (workspace_bytes < need) return SQAP_ERR_NOMEM;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + static_cast<int64_t>(a.batch) * a.heads * a.max_q * parts * a.c.head_dim);
    return SQAP_OK;
}
sqap_status launch(AttnArgs a, const Plan& p, View view, int64_t units, int type, int dtype, cudaStream_t s) {
    a.splits = p.splits;
    a.chunk = p.chunk;
    a.tiles = p.tiles;
    a.row_tile = p.row_tile;
    if (p.decode) return launch_kv_decode(a, view, units, type, dtype, s);
    if (a.c.head_dim <= 128) return launch_kv_prefill_tc(a, view, units, type, dtype, s);
    return launch_kv_prefill(a, view, units, type, dtype, s);
}

}  // namespace

// What the attention calls have in common: checks, and the arguments of the kernels but for the plan. `work`: there is something to do.
sqap_status begin_attention(AttnArgs& a, bool& work, const sqap_kv_cache* cache, const int32_t* table, int64_t ldt, int batch, const int32_t* lens,
                       const int32_t* cu_q, int max_q, int max_len, const void* q, int64_t ldq, int heads, float scale, uint32_t flags,
                       void* out, int64_t ldo, float* lse, int dtype) {
    work = false;
    const sqap_status st = check_cache(cache);
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
    if (!sizes_fit(batch, cache->kv_heads, heads, max_q, max_len)) return SQAP_ERR_UNSUPPORTED;
    a = {};
    a.c = device_view(cache);
    a.group = heads / cache->kv_heads;
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
    work = true;
    return SQAP_OK;
}
bool few_rows(int max_q, int group, int head_dim) { return static_cast<int64_t>(max_q) * group <= decode_max_rows(head_dim); }
sqap_status run_attention(const AttnArgs& args, bool scores, int type, int dtype, void* workspace, size_t workspace_bytes, cudaStream_t s) {
    AttnArgs a = args;
    const Plan p = plan_for(a.batch, a.c.kv_heads, a.group, a.c.head_dim, a.max_q, a.max_len);
    if (!grid_fits(a.batch, a.c.kv_heads, p)) return SQAP_ERR_UNSUPPORTED;
    sqap_status st = take_workspace(a, p.splits, workspace, workspace_bytes);
    if (st != SQAP_OK) return st;
    st = launch(a, p, scores ? VIEW_SCORES : VIEW_ALL, a.batch, type, dtype, s);
    if (st != SQAP_OK || a.parts <= 1) return st;
    return combine(a, a.batch, dtype, s);
}
}  // namespace kv
}  // namespace sqap

extern "C" size_t sqap_kv_attention_workspace_bytes(const sqap_kv_cache* cache, int batch, int max_q, int max_len, int heads) {
    using namespace sqap::kv;
    if (check_cache(cache) != SQAP_OK || batch <= 0 || max_q <= 0 || max_len < 0 || heads <= 0 || heads % cache->kv_heads != 0) return 0;
    if (!sizes_fit(batch, cache->kv_heads, heads, max_q, max_len)) return 0;
    const Plan p = plan_for(batch, cache->kv_heads, heads / cache->kv_heads, cache->head_dim, max_q, max_len);
    return grid_fits(batch, cache->kv_heads, p) ? part_bytes(batch, heads, max_q, cache->head_dim, p.splits) : 0;
}

extern "C" sqap_status sqap_kv_attention(const sqap_kv_cache* cache, const int32_t* table, int64_t ldt, int batch, const int32_t* lens,
                                         const int32_t* cu_q, int max_q, int max_len, const void* q, int64_t ldq, int heads, float scale,
                                         uint32_t flags, void* out, int64_t ldo, float* lse, int dtype, void* workspace,
                                         size_t workspace_bytes, void* stream) {
    using namespace sqap;
    using namespace sqap::kv;
    AttnArgs a;
    bool work;
    const sqap_status st = begin_attention(a, work, cache, table, ldt, batch, lens, cu_q, max_q, max_len, q, ldq, heads, scale, flags, out, ldo, lse, dtype);
    if (st != SQAP_OK || !work) return st;
    return run_attention(a, false, cache->type, dtype, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

extern "C" size_t sqap_kv_attention_window_workspace_bytes(const sqap_kv_cache* cache, int batch, int max_q, int max_len, int heads,
                                                           int window, int sinks) {
    using namespace sqap::kv;
    if (check_cache(cache) != SQAP_OK || batch <= 0 || max_q <= 0 || max_len < 0 || heads <= 0 || heads % cache->kv_heads != 0) return 0;
    if (window <= 0 || sinks < 0 || !sizes_fit(batch, cache->kv_heads, heads, max_q, max_len)) return 0;
    const Plan p = plan_window(batch, cache->kv_heads, heads / cache->kv_heads, cache->head_dim, max_q, max_len, window, sinks);
    return grid_fits(batch, cache->kv_heads, p) ? part_bytes(batch, heads, max_q, cache->head_dim, p.splits) : 0;
}

extern "C" sqap_status sqap_kv_attention_window(const sqap_kv_cache* cache, const int32_t* table, int64_t ldt, int batch, const int32_t* lens,
                                                const int32_t* cu_q, int max_q, int max_len, const void* q, int64_t ldq, int heads,
                                                float scale, int window, int sinks, void* out, int64_t ldo, float* lse, int dtype,
                                                void* workspace, size_t workspace_bytes, void* stream) {
    using namespace sqap;
    using namespace sqap::kv;
    AttnArgs a;
    bool work;
    sqap_status st = begin_attention(a, work, cache, table, ldt, batch, lens, cu_q, max_q, max_len, q, ldq, heads, scale, SQAP_KV_CAUSAL, out, ldo, lse, dtype);
    if (st != SQAP_OK) return st;
    if (window <= 0 || sinks < 0) return SQAP_ERR_INVALID;
    if (!work) return SQAP_OK;
    const Plan p = plan_window(batch, cache->kv_heads, a.group, cache->head_dim, max_q, max_len, window, sinks);
    if (!grid_fits(batch, cache->kv_heads, p)) return SQAP_ERR_UNSUPPORTED;
    st = take_workspace(a, p.splits, workspace, workspace_bytes);
    if (st != SQAP_OK) return st;
    a.window = window;
    a.sinks = sinks < max_len ? sinks : max_len;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    st = launch(a, p, VIEW_WINDOW, batch, cache->type, dtype, s);
    if (st != SQAP_OK || a.parts <= 1) return st;
    return combine(a, batch, dtype, s);
}

extern "C" size_t sqap_kv_attention_shared_workspace_bytes(const sqap_kv_cache* cache, int batch, int max_q, int max_len, int groups,
                                                           int max_group, int max_prefix, int heads) {
    using namespace sqap::kv;
    if (check_cache(cache) != SQAP_OK || batch <= 0 || max_q <= 0 || max_len < 0 || heads <= 0 || heads % cache->kv_heads != 0) return 0;
    if (groups <= 0 || max_group <= 0 || max_prefix < 0 || !sizes_fit(batch, cache->kv_heads, heads, max_q, max_len)) return 0;
    if (size_product(max_group, max_q, heads / cache->kv_heads) > 1 << 30) return 0;
    const SharedPlan p = plan_shared(cache->kv_heads, heads / cache->kv_heads, cache->head_dim, max_q, max_len, groups, max_group,
                                     max_prefix < max_len ? max_prefix : max_len);
    return shared_fits(cache, groups, max_group, max_q, heads, p) ? part_bytes(batch, heads, max_q, cache->head_dim, p.parts) : 0;
}

extern "C" sqap_status sqap_kv_attention_shared(const sqap_kv_cache* cache, const int32_t* table, int64_t ldt, int batch, const int32_t* lens,
                                                const int32_t* cu_q, int max_q, int max_len, const int32_t* cu_group, int groups,
                                                int max_group, const int32_t* prefix, int max_prefix, const void* q, int64_t ldq, int heads,
                                                float scale, uint32_t flags, void* out, int64_t ldo, float* lse, int dtype,
                                                void* workspace, size_t workspace_bytes, void* stream) {
    using namespace sqap;
    using namespace sqap::kv;
    AttnArgs a;
    bool work;
    sqap_status st = begin_attention(a, work, cache, table, ldt, batch, lens, cu_q, max_q, max_len, q, ldq, heads, scale, flags, out, ldo, lse, dtype);
    if (st != SQAP_OK) return st;
    if (groups < 0 || max_group < 0 || max_prefix < 0) return SQAP_ERR_INVALID;
    if (!work || groups == 0 || max_group == 0) return SQAP_OK;
    if (!cu_group || !prefix) return SQAP_ERR_INVALID;
    if ((reinterpret_cast<uintptr_t>(cu_group) & 3u) || (reinterpret_cast<uintptr_t>(prefix) & 3u)) return SQAP_ERR_ALIGN;
    if (size_product(max_group, max_q, a.group) > 1 << 30) return SQAP_ERR_UNSUPPORTED;
    max_prefix = max_prefix < max_len ? max_prefix : max_len;
    const SharedPlan p = plan_shared(cache->kv_heads, a.group, cache->head_dim, max_q, max_len, groups, max_group, max_prefix);
    if (!shared_fits(cache, groups, max_group, max_q, heads, p)) return SQAP_ERR_UNSUPPORTED;
    st = take_workspace(a, p.parts, workspace, workspace_bytes);
    if (st != SQAP_OK) return st;
    a.cu_group = cu_group;
    a.prefix = prefix;
    a.groups = groups;
    a.max_group = max_group;
    a.max_prefix = max_prefix;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int64_t places = static_cast<int64_t>(groups) * max_group;
    if (p.together) {
        st = launch(a, p.prefix, VIEW_SHARED, groups, cache->type, dtype, s);
        if (st != SQAP_OK || a.parts <= 1) return st;
        return combine(a, places, dtype, s);
    }
    if (p.prefix_parts > 0) {
        st = launch(a, p.prefix, VIEW_PREFIX, groups, cache->type, dtype, s);
        if (st != SQAP_OK) return st;
    }
    a.part0 = p.join ? 0 : p.prefix_parts;
    a.join = p.join ? p.prefix_parts : 0;
    st = launch(a, p.own, p.own_view, p.own_units, cache->type, dtype, s);
    if (st != SQAP_OK || a.parts <= 1 || p.join) return st;
    a.part0 = 0;
    return combine(a, places, dtype, s);
}
