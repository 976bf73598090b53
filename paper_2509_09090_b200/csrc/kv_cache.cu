// The paged 8-bit key/value cache: tokens in (append), tokens out (read), pages copied, tokens brought together (compact).
//
// A block is a page of one head: page_tokens x head_dim codes with one scale. All four kernels move every byte once and
// are bounded by HBM; a block is small enough (1 to 32 KB) that its second pass (first the maximum, then the codes)
// finds its input in L1. 16 x 288 tokens, 32 heads of 128: append 21 us, read back 21 (one after the other 38: 5.0 TB/s),
// compaction to 160 19, 128 copies of 16 last pages 15.
#include "kv.cuh"

namespace sqap {
namespace kv {
namespace {

constexpr int THREADS = 128;
constexpr int READ_AHEAD = 8;
constexpr int HELD = 8;      // 16-byte pieces that a thread keeps between the two passes

// Maximum over the block, known to every thread.
__device__ __forceinline__ float block_max(float v, float* red) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < THREADS / 32; ++w) v = fmaxf(v, red[w]);
    return v;
}

struct AppendArgs {
    Cache c;
    const int32_t* table;
    int64_t ldt;
    const int32_t* lens;
    const int32_t* cu;
    int max_new, slots;
    const void* k;
    const void* v;
    int64_t ldk, ldv;
};

// One CTA = one touched page of one sequence, one head, keys or values.
template <typename T, int TYPE>
__global__ void __launch_bounds__(THREADS) kv_append_kernel(AppendArgs a) {
    __shared__ float red[THREADS / 32];
    pdl_launch_dependents();
    pdl_wait();
    const Cache& c = a.c;
    unsigned id = blockIdx.x;
    const int which = id & 1;
    id >>= 1;
    const int h = static_cast<int>(id % c.kv_heads);
    id /= c.kv_heads;
    const int slot = static_cast<int>(id % a.slots), b = static_cast<int>(id / a.slots);
    const int first_row = a.cu[b];
    const int n = max(a.cu[b + 1] - first_row, 0), len = a.lens[b];
    const int start = max(len, 0) - n;                      // position of the first new token; negative positions do not exist
    const int stop = start + min(n, a.max_new);             // behind the last one that is read
    if (stop <= 0) return;
    const int from = max(start, 0);
    const int j = (from >> c.page_shift) + slot;            // page of the sequence
    if (static_cast<int64_t>(j) << c.page_shift >= stop) return;
    const int lo = j << c.page_shift;
    // new tokens of this page
    const int t0 = from > lo ? from : lo;
    const int t1 = static_cast<int>(min(static_cast<int64_t>(stop), static_cast<int64_t>(lo) + (1 << c.page_shift)));
    if (t0 >= t1 || j >= a.ldt) return;
    const int page = checked_page(c, a.table[b * a.ldt + j]);
    if (page < 0) return;
    const Half half = which ? c.v : c.k;
    const int D = c.head_dim, per_row = D / 8, rshift = 31 - __clz(per_row);      // a power of two
    uint8_t* codes = half.codes + page_codes(c, page, h) * D;
    float* scale_at = half.scales + static_cast<int64_t>(page) * c.kv_heads + h;
    const T* src = static_cast<const T*>(which ? a.v : a.k) + static_cast<int64_t>(h) * D;
    const int64_t ld = which ? a.ldv : a.ldk;
    const T* row0 = src + (static_cast<int64_t>(first_row) + (t0 - start)) * ld;
    const int items = (t1 - t0) * per_row;

    // The new tokens' share of a thread: kept in registers where it is small enough (the usual pages), read again otherwise.
    auto source = [&](int i) { return __ldg(reinterpret_cast<const uint4*>(row0 + (i >> rshift) * ld) + (i & (per_row - 1))); };
    uint4 held[HELD];
#pragma unroll
    for (int q = 0; q < HELD; ++q) {
        const int i = threadIdx.x + q * THREADS;
        held[q] = make_uint4(0, 0, 0, 0);
        if (i < items) held[q] = source(i);
    }
    const float before = t0 > lo ? *scale_at : 0.0f;        // tokens in front of the new ones keep their place
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < HELD; ++q) widen8<T>(held[q], &top);
    for (int i = threadIdx.x + HELD * THREADS; i < items; i += THREADS) widen8<T>(source(i), &top);
    // (every thread has read *scale_at before thread 0 writes it; an infinity counts as the largest number: scales are finite)
    const float amax = fminf(block_max(fold_pair<T>(top), red), largest<T>());
    const float scale = fmaxf(before, scale_for<TYPE>(amax));
    if (threadIdx.x == 0) *scale_at = scale;
    if (scale > before && t0 > lo) {                        // they are rounded again to the larger scale
        const float ratio = __fdiv_rn(before, scale);
        for (int i = threadIdx.x; i < (t0 - lo) * per_row; i += THREADS) {
            uint2* p = reinterpret_cast<uint2*>(codes) + i;
            float v[8];
            decode8<TYPE>(*p, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(v[e], ratio);
            *p = encode8<TYPE>(v);
        }
    }
    const float inv = inverse_of(scale);
    uint2* to = reinterpret_cast<uint2*>(codes + static_cast<int64_t>(t0 - lo) * D);
    auto write = [&](int i, uint4 u) {
        float v[8];
        unpack8<T>(u, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(v[e], inv);
        to[i] = finite_codes<TYPE>(encode8<TYPE>(v));
    };
#pragma unroll
    for (int q = 0; q < HELD; ++q)
        if (threadIdx.x + q * THREADS < items) write(threadIdx.x + q * THREADS, held[q]);
    for (int i = threadIdx.x + HELD * THREADS; i < items; i += THREADS) write(i, source(i));
}

struct ReadArgs {
    Cache c;
    const int32_t* table;
    int64_t ldt;
    const int32_t* first;
    const int32_t* cu;
    int max_rows;
    void* k;
    void* v;
    int64_t ldk, ldv;
};

// One warp = 16 consecutive places of a page (a run: contiguous codes) of one sequence and head, keys or values: 8 codes a lane
// and step, 16-byte stores side by side, READ_AHEAD steps' loads in flight. (By tokens instead, all heads of one after the
// other, every 128 bytes come from another page's worth of codes: 31 us where this takes 19, for 16 x 288 tokens, 32 heads.)
template <typename T, int TYPE, int D>
__global__ void __launch_bounds__(THREADS) kv_read_kernel(ReadArgs a, unsigned total, int runs) {
    constexpr int LANES = D / 8, STEPS = 16 * LANES / 32, AHEAD = STEPS < READ_AHEAD ? STEPS : READ_AHEAD;
    pdl_launch_dependents();
    pdl_wait();
    const Cache& c = a.c;
    unsigned id = blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5);
    if (id >= total) return;
    const int lane = threadIdx.x & 31;
    const int h = static_cast<int>(id % c.kv_heads);
    id /= c.kv_heads;
    const int which = id & 1;
    id >>= 1;
    const int run = static_cast<int>(id % runs), b = static_cast<int>(id / runs);
    T* out = static_cast<T*>(which ? a.v : a.k);
    const int r0 = a.cu[b];
    const int n = min(a.cu[b + 1] - r0, a.max_rows);
    const int64_t first = a.first ? a.first[b] : 0;
    const int64_t pos0 = ((first >> 4) + run) << 4, j = pos0 >> c.page_shift;      // first place of the run
    if (!out || pos0 >= first + n) return;
    const int page = pos0 >= 0 && j < a.ldt ? checked_page(c, a.table[b * a.ldt + j]) : -1;
    const Half half = which ? c.v : c.k;
    const int64_t ld = which ? a.ldv : a.ldk;
    const uint2* codes = reinterpret_cast<const uint2*>(half.codes + (page_codes(c, page, h) + (static_cast<int>(pos0) & ((1 << c.page_shift) - 1))) * D);
    const float s = page >= 0 ? __ldg(half.scales + static_cast<int64_t>(page) * c.kv_heads + h) : 0.0f;     // a missing page reads as zero
#pragma unroll
    for (int s0 = 0; s0 < STEPS; s0 += AHEAD) {
        uint2 u[AHEAD];
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) u[q] = page >= 0 ? __ldg(codes + 32 * (s0 + q) + lane) : make_uint2(0, 0);
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            const int piece = 32 * (s0 + q) + lane;
            const int64_t i = pos0 + piece / LANES - first;                        // row of the sequence
            if (i < 0 || i >= n) continue;
            float v[8];
            decode8<TYPE>(u[q], v);
#pragma unroll
            for (int f = 0; f < 8; ++f) v[f] = __fmul_rn(v[f], s);
            *(reinterpret_cast<uint4*>(out + (r0 + i) * ld + h * D) + piece % LANES) = pack8<T>(v);
        }
    }
}

// One CTA = a piece of one page, keys or values.
constexpr int COPY_BYTES = THREADS * 16 * 4;
__global__ void __launch_bounds__(THREADS) kv_copy_pages_kernel(Cache c, const int32_t* pairs, int pieces) {
    pdl_launch_dependents();
    pdl_wait();
    unsigned id = blockIdx.x;
    const int piece = static_cast<int>(id % pieces);
    id /= pieces;
    const int which = id & 1;
    const int2 p = __ldg(reinterpret_cast<const int2*>(pairs) + (id >> 1));
    if (checked_page(c, p.x) < 0 || checked_page(c, p.y) < 0) return;
    const Half half = which ? c.v : c.k;
    const int64_t bytes = (static_cast<int64_t>(c.kv_heads) << c.page_shift) * c.head_dim;
    const uint4* from = reinterpret_cast<const uint4*>(half.codes + p.x * bytes);
    uint4* to = reinterpret_cast<uint4*>(half.codes + p.y * bytes);
    const int64_t base = static_cast<int64_t>(piece) * (COPY_BYTES / 16) + threadIdx.x, end = bytes / 16;
    uint4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (base + i * THREADS < end) v[i] = from[base + i * THREADS];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (base + i * THREADS < end) to[base + i * THREADS] = v[i];
    if (piece == 0)
        for (int h = threadIdx.x; h < c.kv_heads; h += THREADS)
            half.scales[static_cast<int64_t>(p.y) * c.kv_heads + h] = half.scales[static_cast<int64_t>(p.x) * c.kv_heads + h];
}

struct CompactArgs {
    Cache c;
    const int32_t* table;
    int64_t ldt;
    int rows;
    const int32_t* lens;
    const int32_t* src;
    const int32_t* dst;
    const int32_t* kept;
    int64_t ldkept;
    const int32_t* n_kept;
    int max_kept, slots;
};

// One CTA = one page of one destination row, one head, keys or values.
template <int TYPE>
__global__ void __launch_bounds__(THREADS) kv_compact_kernel(CompactArgs a) {
    __shared__ float red[THREADS / 32];
    __shared__ int64_t at[128];     // offset of the token that goes to each place of the page, in tokens; -1: none
    __shared__ float of[128];       // its scale
    pdl_launch_dependents();
    pdl_wait();
    const Cache& c = a.c;
    unsigned id = blockIdx.x;
    const int which = id & 1;
    id >>= 1;
    const int h = static_cast<int>(id % c.kv_heads);
    id /= c.kv_heads;
    const int slot = static_cast<int>(id % a.slots), i = static_cast<int>(id / a.slots);
    const int P = 1 << c.page_shift, D = c.head_dim;
    int n = a.n_kept[i];
    n = n < 0 ? 0 : (n > a.max_kept ? a.max_kept : n);
    const int lo = slot << c.page_shift;
    const int src = a.src[i], dst = a.dst[i];
    if (lo >= n || slot >= a.ldt || src < 0 || src >= a.rows || dst < 0 || dst >= a.rows) return;
    const int page = checked_page(c, a.table[dst * a.ldt + slot]);
    if (page < 0) return;
    const Half half = which ? c.v : c.k;
    if (static_cast<int>(threadIdx.x) < P) {
        const int t = lo + threadIdx.x;
        int64_t where = -1;
        float s = 0.0f;
        if (t < n) {
            const int pos = a.kept[i * a.ldkept + t];
            const int from = pos >= 0 && pos < a.lens[src] && (pos >> c.page_shift) < a.ldt
                                 ? checked_page(c, a.table[src * a.ldt + (pos >> c.page_shift)]) : -1;
            if (from >= 0) {
                where = page_codes(c, from, h) + (pos & (P - 1));
                s = half.scales[static_cast<int64_t>(from) * c.kv_heads + h];
            }
        }
        at[threadIdx.x] = where;
        of[threadIdx.x] = s;
    }
    __syncthreads();
    // 16 codes a piece: at most 16 pieces a thread, of which HELD / 2 stay in registers between the two passes
    const int per16 = D / 16, rshift = 31 - __clz(per16), items = P * per16;
    auto source = [&](int x) {
        const int64_t where = at[x >> rshift];
        return where < 0 ? make_uint4(0, 0, 0, 0) : __ldg(reinterpret_cast<const uint4*>(half.codes + where * D) + (x & (per16 - 1)));
    };
    uint4 held[HELD / 2];
#pragma unroll
    for (int q = 0; q < HELD / 2; ++q) {
        const int x = threadIdx.x + q * THREADS;
        held[q] = make_uint4(0, 0, 0, 0);
        if (x < items) held[q] = source(x);
    }
    float amax = 0.0f;
    auto widen = [&](int x, uint4 u) {
        const float s = of[x >> rshift];
        float v[8];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            decode8<TYPE>(f ? make_uint2(u.z, u.w) : make_uint2(u.x, u.y), v);
#pragma unroll
            for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(__fmul_rn(v[e], s)));
        }
    };
#pragma unroll
    for (int q = 0; q < HELD / 2; ++q)
        if (threadIdx.x + q * THREADS < items) widen(threadIdx.x + q * THREADS, held[q]);
    for (int x = threadIdx.x + HELD / 2 * THREADS; x < items; x += THREADS) widen(x, source(x));
    const float scale = scale_for<TYPE>(block_max(amax, red)), inv = inverse_of(scale);
    if (threadIdx.x == 0) half.scales[static_cast<int64_t>(page) * c.kv_heads + h] = scale;
    uint4* to = reinterpret_cast<uint4*>(half.codes + page_codes(c, page, h) * D);
    auto write = [&](int x, uint4 u) {
        const float s = of[x >> rshift];
        float v[8];
        uint2 r[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            decode8<TYPE>(f ? make_uint2(u.z, u.w) : make_uint2(u.x, u.y), v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(__fmul_rn(v[e], s), inv);
            r[f] = encode8<TYPE>(v);
        }
        to[x] = make_uint4(r[0].x, r[0].y, r[1].x, r[1].y);
    };
#pragma unroll
    for (int q = 0; q < HELD / 2; ++q)
        if (threadIdx.x + q * THREADS < items) write(threadIdx.x + q * THREADS, held[q]);
    for (int x = threadIdx.x + HELD / 2 * THREADS; x < items; x += THREADS) write(x, source(x));
}

constexpr int64_t MAX_GRID = 0x7FFFFFFF;

template <typename T>
cudaError_t append_as(const AppendArgs& a, int type, unsigned grid, cudaStream_t s) {
    if (type == SQAP_KV_INT8) return launch_dependent(kv_append_kernel<T, SQAP_KV_INT8>, dim3(grid), dim3(THREADS), 0, s, a);
    return launch_dependent(kv_append_kernel<T, SQAP_KV_E4M3>, dim3(grid), dim3(THREADS), 0, s, a);
}
template <typename T, int TYPE>
cudaError_t read_dim(const ReadArgs& a, unsigned total, int runs, cudaStream_t s) {
    const dim3 grid((total + THREADS / 32 - 1) / (THREADS / 32));
    if (a.c.head_dim == 64) return launch_dependent(kv_read_kernel<T, TYPE, 64>, grid, dim3(THREADS), 0, s, a, total, runs);
    if (a.c.head_dim == 128) return launch_dependent(kv_read_kernel<T, TYPE, 128>, grid, dim3(THREADS), 0, s, a, total, runs);
    return launch_dependent(kv_read_kernel<T, TYPE, 256>, grid, dim3(THREADS), 0, s, a, total, runs);
}
template <typename T>
cudaError_t read_as(const ReadArgs& a, int type, unsigned total, int runs, cudaStream_t s) {
    return type == SQAP_KV_INT8 ? read_dim<T, SQAP_KV_INT8>(a, total, runs, s) : read_dim<T, SQAP_KV_E4M3>(a, total, runs, s);
}

}  // namespace
}  // namespace kv
}  // namespace sqap

extern "C" sqap_status sqap_kv_append(const sqap_kv_cache* cache, const int32_t* table, int64_t ldt, int batch,
                                      const int32_t* lens, const int32_t* cu_new, int max_new, const void* k, int64_t ldk,
                                      const void* v, int64_t ldv, int dtype, void* stream) {
    using namespace sqap;
    using namespace sqap::kv;
    sqap_status st = check_cache(cache);
    if (st != SQAP_OK) return st;
    const int64_t width = static_cast<int64_t>(cache->kv_heads) * cache->head_dim;
    if (batch < 0 || max_new < 0 || ldt < 0 || ldt > 0x7FFFFFFF || ldk < width || ldv < width || !row_type(dtype)) return SQAP_ERR_INVALID;
    if (ldk % 8 != 0 || ldv % 8 != 0) return SQAP_ERR_ALIGN;
    if (batch == 0 || max_new == 0) return SQAP_OK;
    if (!table || !lens || !cu_new || !k || !v) return SQAP_ERR_INVALID;
    if (!aligned16(k) || !aligned16(v)) return SQAP_ERR_ALIGN;
    if (cache->pages == 0 || ldt == 0) return SQAP_OK;
    AppendArgs a = {device_view(cache), table, ldt, lens, cu_new, max_new, 0, k, v, ldk, ldv};
    // from an offset of page_tokens - 1 on, the tokens touch one page more
    a.slots = static_cast<int>((static_cast<int64_t>(max_new) - 1 + cache->page_tokens - 1) / cache->page_tokens + 1);
    const int64_t grid = size_product(batch, a.slots, cache->kv_heads, 2);
    if (grid > MAX_GRID) return SQAP_ERR_UNSUPPORTED;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return finish_launch(dtype == SQAP_FP16 ? append_as<__half>(a, cache->type, static_cast<unsigned>(grid), s)
                                            : append_as<__nv_bfloat16>(a, cache->type, static_cast<unsigned>(grid), s));
}

extern "C" sqap_status sqap_kv_read(const sqap_kv_cache* cache, const int32_t* table, int64_t ldt, int batch,
                                    const int32_t* first, const int32_t* cu_rows, int max_rows, void* k, int64_t ldk, void* v,
                                    int64_t ldv, int dtype, void* stream) {
    using namespace sqap;
    using namespace sqap::kv;
    sqap_status st = check_cache(cache);
    if (st != SQAP_OK) return st;
    const int64_t width = static_cast<int64_t>(cache->kv_heads) * cache->head_dim;
    if (batch < 0 || max_rows < 0 || ldt < 0 || ldt > 0x7FFFFFFF || !row_type(dtype)) return SQAP_ERR_INVALID;
    if ((k && ldk < width) || (v && ldv < width)) return SQAP_ERR_INVALID;
    if ((k && ldk % 8 != 0) || (v && ldv % 8 != 0) || !aligned16(k) || !aligned16(v)) return SQAP_ERR_ALIGN;
    if (batch == 0 || max_rows == 0 || (!k && !v)) return SQAP_OK;
    if (!cu_rows || (ldt > 0 && !table)) return SQAP_ERR_INVALID;
    // runs of 16 places that max_rows tokens can touch
    const int64_t runs = (static_cast<int64_t>(max_rows) + 14) / 16 + 1, warps = size_product(2, batch, runs, cache->kv_heads);
    if (warps > MAX_GRID) return SQAP_ERR_UNSUPPORTED;
    const ReadArgs a = {device_view(cache), table, ldt, first, cu_rows, max_rows, k, v, ldk, ldv};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return finish_launch(dtype == SQAP_FP16 ? read_as<__half>(a, cache->type, static_cast<unsigned>(warps), static_cast<int>(runs), s)
                                            : read_as<__nv_bfloat16>(a, cache->type, static_cast<unsigned>(warps), static_cast<int>(runs), s));
}

extern "C" sqap_status sqap_kv_copy_pages(const sqap_kv_cache* cache, const int32_t* pairs, int n, void* stream) {
    using namespace sqap;
    using namespace sqap::kv;
    const sqap_status st = check_cache(cache);
    if (st != SQAP_OK) return st;
    if (n < 0) return SQAP_ERR_INVALID;
    if (n == 0) return SQAP_OK;
    if (!pairs) return SQAP_ERR_INVALID;
    if (reinterpret_cast<uintptr_t>(pairs) & 7u) return SQAP_ERR_ALIGN;
    if (cache->pages == 0) return SQAP_OK;
    const int64_t bytes = static_cast<int64_t>(cache->kv_heads) * cache->page_tokens * cache->head_dim;
    const int64_t pieces = (bytes + COPY_BYTES - 1) / COPY_BYTES, grid = size_product(2, n, pieces);
    if (grid > MAX_GRID) return SQAP_ERR_UNSUPPORTED;
    return finish_launch(launch_dependent(kv_copy_pages_kernel, dim3(static_cast<unsigned>(grid)), dim3(THREADS), 0,
                                          static_cast<cudaStream_t>(stream), device_view(cache), pairs, static_cast<int>(pieces)));
}

extern "C" sqap_status sqap_kv_compact(const sqap_kv_cache* cache, const int32_t* table, int64_t ldt, int rows, const int32_t* lens,
                                       const int32_t* src_rows, const int32_t* dst_rows, int n, const int32_t* kept, int64_t ldkept,
                                       const int32_t* n_kept, int max_kept, void* stream) {
    using namespace sqap;
    using namespace sqap::kv;
    const sqap_status st = check_cache(cache);
    if (st != SQAP_OK) return st;
    if (rows < 0 || n < 0 || max_kept < 0 || ldt < 0 || ldt > 0x7FFFFFFF || ldkept < max_kept) return SQAP_ERR_INVALID;
    if (n == 0 || max_kept == 0) return SQAP_OK;
    if (!table || !lens || !src_rows || !dst_rows || !kept || !n_kept) return SQAP_ERR_INVALID;
    if (cache->pages == 0 || rows == 0 || ldt == 0) return SQAP_OK;
    CompactArgs a = {device_view(cache), table, ldt, rows, lens, src_rows, dst_rows, kept, ldkept, n_kept, max_kept, 0};
    a.slots = (max_kept - 1) / cache->page_tokens + 1;
    const int64_t grid = size_product(n, a.slots, cache->kv_heads, 2);
    if (grid > MAX_GRID) return SQAP_ERR_UNSUPPORTED;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (cache->type == SQAP_KV_INT8)
        return finish_launch(launch_dependent(kv_compact_kernel<SQAP_KV_INT8>, dim3(static_cast<unsigned>(grid)), dim3(THREADS), 0, s, a));
    return finish_launch(launch_dependent(kv_compact_kernel<SQAP_KV_E4M3>, dim3(static_cast<unsigned>(grid)), dim3(THREADS), 0, s, a));
}
