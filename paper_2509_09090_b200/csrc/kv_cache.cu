// The paged 8-bit key/value cache: tokens in (append), tokens out (read), pages copied, tokens brought together (compact).
//
// A block is a page of one head: page_tokens x head_dim codes with one scale. All four kernels move every byte once and
// are bounded by HBM; a block is small enough (1 to 32 KB) that its second pass (first the maximum, then the codes)
// finds its input in L1.
#include "kv.cuh"

namespace sqap {
namespace kv {
namespace {

constexpr int THREADS = 128;

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
    int n = a.cu[b + 1] - first_row;
    n = n < 0 ? 0 : (n > a.max_new ? a.max_new : n);
    const int len = a.lens[b];
    const int start = len - n;                              // position of the first new token; negative positions do not exist
    const int from = start < 0 ? 0 : start;
    const int j = (from >> c.page_shift) + slot;            // page of the sequence
    if (static_cast<int64_t>(j) << c.page_shift >= len) return;
    const int lo = j << c.page_shift;
    // new tokens of this page
    const int t0 = from > lo ? from : lo;
    const int t1 = static_cast<int>(min(static_cast<int64_t>(len), static_cast<int64_t>(lo) + (1 << c.page_shift)));
    if (t0 >= t1 || j >= a.ldt) return;
    const int page = checked_page(c, a.table[b * a.ldt + j]);
    if (page < 0) return;
    const Half half = which ? c.v : c.k;
    const int D = c.head_dim, per_row = D / 8;
    uint8_t* codes = half.codes + page_codes(c, page, h) * D;
    float* scale_at = half.scales + static_cast<int64_t>(page) * c.kv_heads + h;
    const T* src = static_cast<const T*>(which ? a.v : a.k) + static_cast<int64_t>(h) * D;
    const int64_t ld = which ? a.ldv : a.ldk;
    const T* row0 = src + (static_cast<int64_t>(first_row) + (t0 - start)) * ld;
    const int items = (t1 - t0) * per_row;

    float amax = 0.0f;
    for (int i = threadIdx.x; i < items; i += THREADS) {
        float v[8];
        unpack8<T>(__ldg(reinterpret_cast<const uint4*>(row0 + (i / per_row) * ld) + i % per_row), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(v[e]));
    }
    const float before = t0 > lo ? *scale_at : 0.0f;        // tokens in front of the new ones keep their place
    amax = block_max(amax, red);                            // (every thread has read *scale_at before thread 0 writes it)
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
    for (int i = threadIdx.x; i < items; i += THREADS) {
        float v[8];
        unpack8<T>(__ldg(reinterpret_cast<const uint4*>(row0 + (i / per_row) * ld) + i % per_row), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(v[e], inv);
        to[i] = encode8<TYPE>(v);
    }
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

// One CTA = one token of one sequence, all heads, keys and values.
template <typename T, int TYPE>
__global__ void __launch_bounds__(THREADS) kv_read_kernel(ReadArgs a) {
    pdl_launch_dependents();
    pdl_wait();
    const Cache& c = a.c;
    const int b = blockIdx.x / a.max_rows, i = blockIdx.x % a.max_rows;
    const int r0 = a.cu[b];
    if (i >= a.cu[b + 1] - r0) return;
    const int64_t pos = static_cast<int64_t>(a.first ? a.first[b] : 0) + i, j = pos >> c.page_shift;
    const int D = c.head_dim, per_row = D / 8;
    const int page = pos >= 0 && j < a.ldt ? checked_page(c, a.table[b * a.ldt + j]) : -1;
    const int t = static_cast<int>(pos) & ((1 << c.page_shift) - 1);
    const int items = c.kv_heads * per_row;
    for (int x = threadIdx.x; x < 2 * items; x += THREADS) {
        const int which = x >= items, y = which ? x - items : x, h = y / per_row, e = y % per_row;
        const Half half = which ? c.v : c.k;
        T* out = static_cast<T*>(which ? a.v : a.k);
        if (!out) continue;
        float v[8] = {};
        if (page >= 0) {
            const float s = __ldg(half.scales + static_cast<int64_t>(page) * c.kv_heads + h);
            decode8<TYPE>(__ldg(reinterpret_cast<const uint2*>(half.codes + (page_codes(c, page, h) + t) * D) + e), v);
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = __fmul_rn(v[q], s);
        }
        *(reinterpret_cast<uint4*>(out + (static_cast<int64_t>(r0) + i) * (which ? a.ldv : a.ldk)) + y) = pack8<T>(v);
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
    const int P = 1 << c.page_shift, D = c.head_dim, per_row = D / 8;
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
    float amax = 0.0f;
    const int items = P * per_row;
    for (int x = threadIdx.x; x < items; x += THREADS) {
        const int t = x / per_row;
        if (at[t] < 0) continue;
        float v[8];
        decode8<TYPE>(__ldg(reinterpret_cast<const uint2*>(half.codes + at[t] * D) + x % per_row), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(__fmul_rn(v[e], of[t])));
    }
    const float scale = scale_for<TYPE>(block_max(amax, red)), inv = inverse_of(scale);
    if (threadIdx.x == 0) half.scales[static_cast<int64_t>(page) * c.kv_heads + h] = scale;
    uint2* to = reinterpret_cast<uint2*>(half.codes + page_codes(c, page, h) * D);
    for (int x = threadIdx.x; x < items; x += THREADS) {
        const int t = x / per_row;
        uint2 r = make_uint2(0, 0);
        if (at[t] >= 0) {
            float v[8];
            decode8<TYPE>(__ldg(reinterpret_cast<const uint2*>(half.codes + at[t] * D) + x % per_row), v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(__fmul_rn(v[e], of[t]), inv);
            r = encode8<TYPE>(v);
        }
        to[x] = r;
    }
}

constexpr int64_t MAX_GRID = 0x7FFFFFFF;

template <typename T>
cudaError_t append_as(const AppendArgs& a, int type, unsigned grid, cudaStream_t s) {
    if (type == SQAP_KV_INT8) return launch_dependent(kv_append_kernel<T, SQAP_KV_INT8>, dim3(grid), dim3(THREADS), 0, s, a);
    return launch_dependent(kv_append_kernel<T, SQAP_KV_E4M3>, dim3(grid), dim3(THREADS), 0, s, a);
}
template <typename T>
cudaError_t read_as(const ReadArgs& a, int type, unsigned grid, cudaStream_t s) {
    if (type == SQAP_KV_INT8) return launch_dependent(kv_read_kernel<T, SQAP_KV_INT8>, dim3(grid), dim3(THREADS), 0, s, a);
    return launch_dependent(kv_read_kernel<T, SQAP_KV_E4M3>, dim3(grid), dim3(THREADS), 0, s, a);
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
    const int64_t grid = static_cast<int64_t>(batch) * a.slots * cache->kv_heads * 2;
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
    const int64_t grid = static_cast<int64_t>(batch) * max_rows;
    if (grid > MAX_GRID) return SQAP_ERR_UNSUPPORTED;
    const ReadArgs a = {device_view(cache), table, ldt, first, cu_rows, max_rows, k, v, ldk, ldv};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return finish_launch(dtype == SQAP_FP16 ? read_as<__half>(a, cache->type, static_cast<unsigned>(grid), s)
                                            : read_as<__nv_bfloat16>(a, cache->type, static_cast<unsigned>(grid), s));
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
    const int64_t pieces = (bytes + COPY_BYTES - 1) / COPY_BYTES, grid = 2 * static_cast<int64_t>(n) * pieces;
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
    const int64_t grid = static_cast<int64_t>(n) * a.slots * cache->kv_heads * 2;
    if (grid > MAX_GRID) return SQAP_ERR_UNSUPPORTED;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (cache->type == SQAP_KV_INT8)
        return finish_launch(launch_dependent(kv_compact_kernel<SQAP_KV_INT8>, dim3(static_cast<unsigned>(grid)), dim3(THREADS), 0, s, a));
    return finish_launch(launch_dependent(kv_compact_kernel<SQAP_KV_E4M3>, dim3(static_cast<unsigned>(grid)), dim3(THREADS), 0, s, a));
}
