// Book-keeping of the cache's pages, on the device: how often each page is used (refs), which pages a sequence has (a row
// of the table) and how many tokens they hold (lens). A page is free while refs is 0; whoever needs pages gets the free
// ones with the lowest numbers, in the order of the list, so that equal states give equal results.
//
// These kernels read a few hundred kilobytes at most and are bounded by latency: reserving is one CTA, because the rank of
// a free page among the free pages and the rank of a request among the requests both come from a scan, and a scan
// inside one CTA needs neither a second launch nor a wait on another CTA. Sharing and releasing pages, where order plays
// no part, takes one CTA per sequence.
#include "kv.cuh"

namespace sqap {
namespace kv {
namespace {

constexpr int THREADS = 1024;
constexpr int MAX_ROWS = 16384;                      // rows of a table, and requests of a call
constexpr int PER_THREAD = 4;                        // pages looked at per thread and step

// Inclusive prefix sum over the CTA; *total gets the sum. red: one word per warp.
__device__ __forceinline__ int64_t scan(int64_t v, int64_t* red, int64_t* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();                                  // red may still be read from the scan before
    if (lane == 31) red[warp] = v;
    __syncthreads();
    int64_t before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        const int64_t x = red[w];
        if (w < warp) before += x;
        sum += x;
    }
    *total = sum;
    return v + before;
}

struct Pool {
    int32_t* refs;
    int pages, page_shift;
    int32_t* table;
    int64_t ldt;
    int rows;
    int32_t* lens;
};

// Shared memory of the reserving kernels: first request of each row, and the requests' pages before and with each.
struct Shared {
    int* first;            // [rows] smallest index of a request for this row
    int* upto;             // [n] pages asked for by requests 0 .. i
    int64_t* red;          // [32]
};

__device__ __forceinline__ int pages_of(int64_t tokens, int shift) { return static_cast<int>((tokens + (1 << shift) - 1) >> shift); }

// Gives the lowest free pages to requests in order: request i wants pages upto[i-1] .. upto[i]-1 of the list of free
// pages, and gets them if the list is that long. give(i, which of its pages, page). Returns the number of free pages
// seen, at least the number asked for if there are that many. Every thread of the CTA calls it.
template <typename Give>
__device__ __forceinline__ int64_t take_pages(const Pool& p, int n, const Shared& sh, Give give) {
    const int wanted = n > 0 ? sh.upto[n - 1] : 0;
    // how many free pages there are decides who is served: counted first, as far as needed
    int64_t found = 0;
    for (int64_t at = 0; at < p.pages && found < wanted; at += THREADS * PER_THREAD) {
        int mine = 0;
#pragma unroll
        for (int e = 0; e < PER_THREAD; ++e) {
            const int64_t page = at + threadIdx.x * PER_THREAD + e;
            mine += page < p.pages && p.refs[page] == 0;
        }
        found += __syncthreads_count(mine & 1) + 2 * static_cast<int64_t>(__syncthreads_count(mine & 2)) + 4 * static_cast<int64_t>(__syncthreads_count(mine & 4));
    }
    int64_t before = 0;
    for (int64_t at = 0; at < p.pages && before < wanted; at += THREADS * PER_THREAD) {
        bool idle[PER_THREAD];
        int mine = 0;
#pragma unroll
        for (int e = 0; e < PER_THREAD; ++e) {
            const int64_t page = at + threadIdx.x * PER_THREAD + e;
            idle[e] = page < p.pages && p.refs[page] == 0;
            mine += idle[e];
        }
        int64_t total;
        int64_t rank = before + scan(mine, sh.red, &total) - mine;
        before += total;
#pragma unroll
        for (int e = 0; e < PER_THREAD; ++e) {
            if (!idle[e]) continue;
            const int64_t r = rank++;
            if (r >= wanted) continue;
            int lo = 0, hi = n - 1;                   // the first request with upto > r
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (sh.upto[mid] > r) hi = mid;
                else lo = mid + 1;
            }
            if (sh.upto[lo] > found) continue;        // not served as a whole: gets nothing
            const int64_t page = at + threadIdx.x * PER_THREAD + e;
            p.refs[page] = 1;
            give(lo, static_cast<int>(r - (lo ? sh.upto[lo - 1] : 0)), static_cast<int>(page));
        }
    }
    return found;
}

// Prefix sums of need(i) into sh.upto. Saturates where the sum passes the number of pages.
template <typename Need>
__device__ __forceinline__ void sum_needs(const Pool& p, int n, const Shared& sh, Need need) {
    int64_t before = 0;
    for (int at = 0; at < n; at += THREADS) {
        const int i = at + threadIdx.x;
        int64_t total;
        const int64_t with = before + scan(i < n ? need(i) : 0, sh.red, &total);
        if (i < n) sh.upto[i] = static_cast<int>(with < p.pages ? with : p.pages + (with > p.pages));
        before += total;
    }
    __syncthreads();
}

extern __shared__ int dyn_smem[];

__device__ __forceinline__ Shared shared_arrays(int rows) {
    __shared__ int64_t red[32];
    return {dyn_smem, dyn_smem + rows, red};
}

// rows[i] grows by add[i] tokens.
__global__ void __launch_bounds__(THREADS) kv_alloc_kernel(Pool p, const int32_t* rows, const int32_t* add, int n, int32_t* granted) {
    pdl_launch_dependents();
    pdl_wait();
    const Shared sh = shared_arrays(p.rows);
    for (int i = threadIdx.x; i < p.rows; i += THREADS) sh.first[i] = n;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS)
        if (rows[i] >= 0 && rows[i] < p.rows) atomicMin(sh.first + rows[i], i);
    __syncthreads();
    auto valid = [&](int i) {
        const int r = rows[i];
        if (r < 0 || r >= p.rows || sh.first[r] != i || add[i] < 0 || p.lens[r] < 0) return false;
        const int64_t to = static_cast<int64_t>(p.lens[r]) + add[i];
        return to <= 0x7FFFFFFF && pages_of(to, p.page_shift) <= p.ldt;
    };
    auto need = [&](int i) {
        return valid(i) ? pages_of(static_cast<int64_t>(p.lens[rows[i]]) + add[i], p.page_shift) - pages_of(p.lens[rows[i]], p.page_shift) : 0;
    };
    sum_needs(p, n, sh, need);
    const int64_t found = take_pages(p, n, sh, [&](int i, int j, int page) {
        const int r = rows[i];
        p.table[r * p.ldt + pages_of(p.lens[r], p.page_shift) + j] = page;
    });
    __syncthreads();                                  // the lengths above are read before they change
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const int own = sh.upto[i] - (i ? sh.upto[i - 1] : 0);
        const bool ok = valid(i) && ((own == 0 && need(i) == 0) || (need(i) > 0 && sh.upto[i] <= found));
        if (ok) p.lens[rows[i]] += add[i];
        if (granted) granted[i] = ok ? 1 : 0;
    }
}

// dst[i] becomes a copy of src[i]: plan and last page.
__global__ void __launch_bounds__(THREADS) kv_fork_kernel(Pool p, const int32_t* src, const int32_t* dst, int n, int2* pairs, int32_t* granted) {
    pdl_launch_dependents();
    pdl_wait();
    const Shared sh = shared_arrays(p.rows);
    for (int i = threadIdx.x; i < p.rows; i += THREADS) sh.first[i] = n;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += THREADS)
        if (dst[i] >= 0 && dst[i] < p.rows) atomicMin(sh.first + dst[i], i);
    __syncthreads();
    // a row that is somebody's source is not written: -1 takes it out
    for (int i = threadIdx.x; i < n; i += THREADS)
        if (src[i] >= 0 && src[i] < p.rows) atomicMin(sh.first + src[i], -1);
    __syncthreads();
    auto valid = [&](int i) {
        const int s = src[i], d = dst[i];
        return s >= 0 && s < p.rows && d >= 0 && d < p.rows && sh.first[d] == i && p.lens[d] == 0 && p.lens[s] >= 0 &&
               pages_of(p.lens[s], p.page_shift) <= p.ldt;
    };
    auto need = [&](int i) { return valid(i) && (p.lens[src[i]] & ((1 << p.page_shift) - 1)) != 0 ? 1 : 0; };
    sum_needs(p, n, sh, need);
    const int64_t found = take_pages(p, n, sh, [&](int i, int, int page) {
        const int j = p.lens[src[i]] >> p.page_shift;
        p.table[dst[i] * p.ldt + j] = page;
        pairs[i] = make_int2(p.table[src[i] * p.ldt + j], page);
    });
    // lens[dst] is 0 for every valid request until here, and no source is a destination
    __syncthreads();
    for (int at = 0; at < n; at += THREADS) {
        const int i = at + threadIdx.x;
        bool ok = false;
        int len = 0;
        if (i < n) {
            const int own = need(i);
            ok = valid(i) && (own == 0 || sh.upto[i] <= found);
            if (!ok || own == 0) pairs[i] = ok ? make_int2(-1, -1) : make_int2(-2, -2);
            if (ok) len = p.lens[src[i]];
        }
        if (ok) p.lens[dst[i]] = len;
        if (i < n && granted) granted[i] = ok ? 1 : 0;
    }
}
// The full pages of the sources are shared. One CTA per request.
__global__ void __launch_bounds__(128) kv_share_kernel(Pool p, const int32_t* src, const int32_t* dst, const int2* pairs) {
    pdl_launch_dependents();
    pdl_wait();
    const int i = blockIdx.x;
    if (pairs[i].x == -2) return;
    const int32_t* from = p.table + src[i] * p.ldt;
    int32_t* to = p.table + dst[i] * p.ldt;
    const int full = p.lens[src[i]] >> p.page_shift, used = pages_of(p.lens[src[i]], p.page_shift);
    for (int64_t j = threadIdx.x; j < p.ldt; j += 128) {
        if (j < full) {
            const int page = from[j];
            to[j] = page;
            if (page >= 0 && page < p.pages) atomicAdd(p.refs + page, 1);
        } else if (j >= used) {
            to[j] = -1;
        }
    }
}

// One CTA per row that is given up. Whoever takes the length takes the pages: a row named twice is freed once.
__global__ void __launch_bounds__(128) kv_free_kernel(Pool p, const int32_t* rows) {
    __shared__ int had;
    pdl_launch_dependents();
    pdl_wait();
    const int r = rows[blockIdx.x];
    if (r < 0 || r >= p.rows) return;
    if (threadIdx.x == 0) had = atomicExch(p.lens + r, 0);
    __syncthreads();
    const int64_t used = had > 0 ? min(static_cast<int64_t>(pages_of(had, p.page_shift)), p.ldt) : 0;
    int32_t* t = p.table + r * p.ldt;
    for (int64_t j = threadIdx.x; j < used; j += 128) {
        const int page = t[j];
        t[j] = -1;
        if (page >= 0 && page < p.pages && atomicSub(p.refs + page, 1) <= 0) atomicAdd(p.refs + page, 1);
    }
}

sqap_status check_pool(const int32_t* refs, int pages, int page_tokens, const int32_t* table, int64_t ldt, int rows, const int32_t* lens) {
    if (pages < 0 || rows < 0 || ldt < 0 || ldt > 0x7FFFFFFF) return SQAP_ERR_INVALID;
    if (page_shift_of(page_tokens) < 0 || rows > MAX_ROWS) return SQAP_ERR_UNSUPPORTED;
    if ((pages > 0 && !refs) || (rows > 0 && (!lens || (ldt > 0 && !table)))) return SQAP_ERR_INVALID;
    return SQAP_OK;
}

template <auto Kernel>
sqap_status smem_limit() {
    static PerDevice<int> setup;
    return setup.run([](int*) { return set_max_dynamic_smem(Kernel, 2 * MAX_ROWS * static_cast<int>(sizeof(int))); });
}

}  // namespace
}  // namespace kv
}  // namespace sqap

extern "C" sqap_status sqap_kv_alloc(int32_t* refs, int pages, int page_tokens, int32_t* table, int64_t ldt, int rows, int32_t* lens,
                                     const int32_t* row_list, const int32_t* add, int n, int32_t* granted, void* stream) {
    using namespace sqap;
    using namespace sqap::kv;
    sqap_status st = check_pool(refs, pages, page_tokens, table, ldt, rows, lens);
    if (st != SQAP_OK) return st;
    if (n < 0) return SQAP_ERR_INVALID;
    if (n > MAX_ROWS) return SQAP_ERR_UNSUPPORTED;
    if (n == 0) return SQAP_OK;
    if (!row_list || !add) return SQAP_ERR_INVALID;
    st = smem_limit<kv_alloc_kernel>();
    if (st != SQAP_OK) return st;
    const Pool p = {refs, pages, page_shift_of(page_tokens), table, ldt, rows, lens};
    return finish_launch(launch_dependent(kv_alloc_kernel, dim3(1), dim3(THREADS), (static_cast<size_t>(rows) + n) * sizeof(int),
                                          static_cast<cudaStream_t>(stream), p, row_list, add, n, granted));
}

extern "C" sqap_status sqap_kv_fork(int32_t* refs, int pages, int page_tokens, int32_t* table, int64_t ldt, int rows, int32_t* lens,
                                    const int32_t* src_rows, const int32_t* dst_rows, int n, int32_t* pairs, int32_t* granted,
                                    void* stream) {
    using namespace sqap;
    using namespace sqap::kv;
    sqap_status st = check_pool(refs, pages, page_tokens, table, ldt, rows, lens);
    if (st != SQAP_OK) return st;
    if (n < 0) return SQAP_ERR_INVALID;
    if (n > MAX_ROWS) return SQAP_ERR_UNSUPPORTED;
    if (n == 0) return SQAP_OK;
    if (!src_rows || !dst_rows || !pairs) return SQAP_ERR_INVALID;
    if (reinterpret_cast<uintptr_t>(pairs) & 7u) return SQAP_ERR_ALIGN;
    st = smem_limit<kv_fork_kernel>();
    if (st != SQAP_OK) return st;
    const Pool p = {refs, pages, page_shift_of(page_tokens), table, ldt, rows, lens};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    st = finish_launch(launch_dependent(kv_fork_kernel, dim3(1), dim3(THREADS), (static_cast<size_t>(rows) + n) * sizeof(int), s, p,
                                        src_rows, dst_rows, n, reinterpret_cast<int2*>(pairs), granted));
    if (st != SQAP_OK) return st;
    return finish_launch(launch_dependent(kv_share_kernel, dim3(n), dim3(128), 0, s, p, src_rows, dst_rows,
                                          reinterpret_cast<const int2*>(pairs)));
}

extern "C" sqap_status sqap_kv_free(int32_t* refs, int pages, int page_tokens, int32_t* table, int64_t ldt, int rows, int32_t* lens,
                                    const int32_t* row_list, int n, void* stream) {
    using namespace sqap;
    using namespace sqap::kv;
    const sqap_status st = check_pool(refs, pages, page_tokens, table, ldt, rows, lens);
    if (st != SQAP_OK) return st;
    if (n < 0) return SQAP_ERR_INVALID;
    if (n > MAX_ROWS) return SQAP_ERR_UNSUPPORTED;
    if (n == 0 || rows == 0) return SQAP_OK;
    if (!row_list) return SQAP_ERR_INVALID;
    const Pool p = {refs, pages, page_shift_of(page_tokens), table, ldt, rows, lens};
    return finish_launch(launch_dependent(kv_free_kernel, dim3(n), dim3(128), 0, static_cast<cudaStream_t>(stream), p, row_list));
}
