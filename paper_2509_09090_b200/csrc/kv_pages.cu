// Book-keeping of the cache's pages, on the device: how often each page is used (refs), which pages a sequence has (a row
// of the table) and how many tokens they hold (lens). A page is free while refs is 0; whoever needs pages gets the free
// ones with the lowest numbers, in the order of the list, so that equal states give equal results.
//
// These kernels read a few hundred kilobytes at most and are bounded by latency: reserving is one CTA, because the rank of
// a free page among the free pages and the rank of a request among the requests both come from a scan, and a scan
// inside one CTA needs neither a second launch nor a wait on another CTA. 256 threads where the pool and the list are small,
// since its barriers are then cheaper (fork of 16 rows to 128 with the copy of their last pages: 17.0 us with 1024, 13.5 with 256; of 1 to 8: 14.6 / 11.2).
// Sharing and releasing pages, where order plays no part, takes one CTA per sequence.
#include "kv.cuh"

namespace sqap {
namespace kv {
namespace {

constexpr int MAX_ROWS = 16384;                      // rows of a table, and requests of a call
constexpr int PER_THREAD = 16;                       // pages looked at per thread and step

// Inclusive prefix sum over the CTA; *total gets the sum. red: one word per warp.
template <int NT>
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
    for (int w = 0; w < NT / 32; ++w) {
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
    int* count;            // [PER_THREAD * NT / 32] free pages of each warp's 32, in page order; then the ones before them
};

__device__ __forceinline__ int pages_of(int64_t tokens, int shift) { return static_cast<int>((tokens + (1 << shift) - 1) >> shift); }

// Gives the lowest free pages to requests in order: request i wants pages upto[i-1] .. upto[i]-1 of the list of free
// pages, and gets them if the list is that long. give(i, which of its pages, page). Returns the number of free pages.
// Every thread of the CTA calls it.
template <int NT, typename Give>
__device__ __forceinline__ int64_t take_pages(const Pool& p, int n, const Shared& sh, Give give) {
    constexpr int STEP = PER_THREAD * NT, CELLS = STEP / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t wanted = n > 0 ? sh.upto[n - 1] : 0;
    uint32_t idle[PER_THREAD];                        // of the warp's 32 pages e NT + 32 warp .. of a step
    auto look = [&](int64_t at) {
        bool is[PER_THREAD];
#pragma unroll
        for (int e = 0; e < PER_THREAD; ++e) {
            const int64_t page = at + e * NT + threadIdx.x;
            is[e] = page < p.pages && p.refs[page] == 0;
        }
#pragma unroll
        for (int e = 0; e < PER_THREAD; ++e) idle[e] = __ballot_sync(0xffffffffu, is[e]);
    };
    // sh.count: free pages of the step in front of each warp's; returns all of them
    auto rank = [&]() {
        __syncthreads();
        if (lane == 0)
#pragma unroll
            for (int e = 0; e < PER_THREAD; ++e) sh.count[e * (NT / 32) + warp] = __popc(idle[e]);
        __syncthreads();
        int sum = 0;
        int64_t total;
        const int c0 = threadIdx.x;
        const bool mine = c0 < CELLS;
        if (mine) sum = sh.count[c0];
        const int64_t with = scan<NT>(sum, sh.red, &total);
        if (mine) sh.count[c0] = static_cast<int>(with - sum);
        __syncthreads();
        return total;
    };
    static_assert(CELLS <= NT, "one cell a thread");
    auto hand_out = [&](int64_t at, int64_t before, int64_t found) {
#pragma unroll
        for (int e = 0; e < PER_THREAD; ++e) {
            if (!((idle[e] >> lane) & 1u)) continue;
            const int64_t r = before + sh.count[e * (NT / 32) + warp] + __popc(idle[e] & ((1u << lane) - 1));
            if (r >= wanted) continue;
            int lo = 0, hi = n - 1;                   // the first request with upto > r
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (sh.upto[mid] > r) hi = mid;
                else lo = mid + 1;
            }
            if (sh.upto[lo] > found) continue;        // not served as a whole: gets nothing
            const int64_t page = at + e * NT + threadIdx.x;
            p.refs[page] = 1;
            give(lo, static_cast<int>(r - (lo ? sh.upto[lo - 1] : 0)), static_cast<int>(page));
        }
    };
    if (wanted == 0) return 0;
    if (p.pages <= STEP) {
        look(0);
        const int64_t found = rank();
        hand_out(0, 0, found);
        return found;
    }
    // how many free pages there are decides who is served: counted first
    int64_t mine = 0, found = 0;
    for (int64_t at = 0; at < p.pages; at += STEP) {
        look(at);
#pragma unroll
        for (int e = 0; e < PER_THREAD; ++e) mine += __popc(idle[e]);
    }
    scan<NT>(lane == 0 ? mine : 0, sh.red, &found);
    int64_t before = 0;
    for (int64_t at = 0; at < p.pages && before < wanted; at += STEP) {
        look(at);
        const int64_t here = rank();
        hand_out(at, before, found);
        before += here;
    }
    return found;
}

// Prefix sums of need(i) into sh.upto. Saturates where the sum passes the number of pages.
template <int NT, typename Need>
__device__ __forceinline__ void sum_needs(const Pool& p, int n, const Shared& sh, Need need) {
    int64_t before = 0;
    for (int at = 0; at < n; at += NT) {
        const int i = at + threadIdx.x;
        int64_t total;
        const int64_t with = before + scan<NT>(i < n ? need(i) : 0, sh.red, &total);
        if (i < n) sh.upto[i] = static_cast<int>(with < p.pages ? with : p.pages + (with > p.pages));
        before += total;
    }
    __syncthreads();
}

extern __shared__ int dyn_smem[];

template <int NT>
__device__ __forceinline__ Shared shared_arrays(int rows) {
    __shared__ int64_t red[32];
    __shared__ int count[PER_THREAD * NT / 32];
    return {dyn_smem, dyn_smem + rows, red, count};
}

// A request as it was found; that of index threadIdx.x is kept, others are looked at again.
struct Request {
    int a, b;              // alloc: row, tokens to add; fork: source, destination
    int len;               // tokens of the row (source)
    int need;              // pages
    bool ok;
};

// rows[i] grows by add[i] tokens.
template <int NT>
__global__ void __launch_bounds__(NT) kv_alloc_kernel(Pool p, const int32_t* rows, const int32_t* add, int n, int32_t* granted) {
    pdl_launch_dependents();
    pdl_wait();
    const Shared sh = shared_arrays<NT>(p.rows);
    for (int i = threadIdx.x; i < p.rows; i += NT) sh.first[i] = n;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT)
        if (rows[i] >= 0 && rows[i] < p.rows) atomicMin(sh.first + rows[i], i);
    __syncthreads();
    auto look = [&](int i) {
        Request q = {rows[i], add[i], 0, 0, false};
        if (q.a < 0 || q.a >= p.rows || sh.first[q.a] != i || q.b < 0) return q;
        q.len = p.lens[q.a];
        const int64_t to = static_cast<int64_t>(q.len) + q.b;
        if (q.len < 0 || to > 0x7FFFFFFF || pages_of(to, p.page_shift) > p.ldt) return q;
        q.need = pages_of(to, p.page_shift) - pages_of(q.len, p.page_shift);
        q.ok = true;
        return q;
    };
    Request mine = {};
    if (static_cast<int>(threadIdx.x) < n) mine = look(threadIdx.x);
    auto request = [&](int i) { return i == static_cast<int>(threadIdx.x) ? mine : look(i); };
    sum_needs<NT>(p, n, sh, [&](int i) { return request(i).need; });
    const int64_t found = take_pages<NT>(p, n, sh, [&](int i, int j, int page) {
        const int r = rows[i];
        p.table[r * p.ldt + pages_of(p.lens[r], p.page_shift) + j] = page;
    });
    __syncthreads();                                  // the lengths above are read before they change
    for (int i = threadIdx.x; i < n; i += NT) {
        const Request q = request(i);
        const bool ok = q.ok && (q.need == 0 || sh.upto[i] <= found);
        if (ok) p.lens[q.a] = q.len + q.b;
        if (granted) granted[i] = ok ? 1 : 0;
    }
}

// dst[i] becomes a copy of src[i]: plan and last page.
template <int NT>
__global__ void __launch_bounds__(NT) kv_fork_kernel(Pool p, const int32_t* src, const int32_t* dst, int n, int2* pairs, int32_t* granted) {
    pdl_launch_dependents();
    pdl_wait();
    const Shared sh = shared_arrays<NT>(p.rows);
    for (int i = threadIdx.x; i < p.rows; i += NT) sh.first[i] = n;
    __syncthreads();
    // a row that is somebody's source is not written: -1 takes it out
    for (int i = threadIdx.x; i < n; i += NT) {
        if (dst[i] >= 0 && dst[i] < p.rows) atomicMin(sh.first + dst[i], i);
        if (src[i] >= 0 && src[i] < p.rows) atomicMin(sh.first + src[i], -1);
    }
    __syncthreads();
    auto look = [&](int i) {
        Request q = {src[i], dst[i], 0, 0, false};
        if (q.a < 0 || q.a >= p.rows || q.b < 0 || q.b >= p.rows || sh.first[q.b] != i) return q;
        q.len = p.lens[q.a];
        if (q.len < 0 || p.lens[q.b] != 0 || pages_of(q.len, p.page_shift) > p.ldt) return q;
        // an unfinished last page is copied, if the source has it
        if ((q.len & ((1 << p.page_shift) - 1)) != 0) {
            const int last = p.table[q.a * p.ldt + (q.len >> p.page_shift)];
            q.need = last >= 0 && last < p.pages ? 1 : 0;
        }
        q.ok = true;
        return q;
    };
    Request mine = {};
    if (static_cast<int>(threadIdx.x) < n) mine = look(threadIdx.x);
    auto request = [&](int i) { return i == static_cast<int>(threadIdx.x) ? mine : look(i); };
    sum_needs<NT>(p, n, sh, [&](int i) { return request(i).need; });
    const int64_t found = take_pages<NT>(p, n, sh, [&](int i, int, int page) {
        const int s = src[i], j = p.lens[s] >> p.page_shift;
        p.table[dst[i] * p.ldt + j] = page;
        pairs[i] = make_int2(p.table[s * p.ldt + j], page);
    });
    // lens of a destination is 0 for every valid request until here, and no source is a destination
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) {
        const Request q = request(i);
        const bool ok = q.ok && (q.need == 0 || sh.upto[i] <= found);
        if (!ok || q.need == 0) pairs[i] = ok ? make_int2(-1, -1) : make_int2(-2, -2);
        if (ok) p.lens[q.b] = q.len;
        if (granted) granted[i] = ok ? 1 : 0;
    }
}
// The full pages of the sources are shared. One CTA per request.
__global__ void __launch_bounds__(128) kv_share_kernel(Pool p, const int32_t* src, const int32_t* dst, const int2* pairs) {
    pdl_launch_dependents();
    pdl_wait();
    const int i = blockIdx.x;
    const int given = pairs[i].y;                     // -2: not met; -1: no page to copy; else the destination's last page, entered already
    if (given == -2) return;
    const int32_t* from = p.table + src[i] * p.ldt;
    int32_t* to = p.table + dst[i] * p.ldt;
    const int full = p.lens[src[i]] >> p.page_shift, used = pages_of(p.lens[src[i]], p.page_shift);
    for (int64_t j = threadIdx.x; j < p.ldt; j += 128) {
        if (j < full) {
            const int page = from[j];
            to[j] = page;
            if (page >= 0 && page < p.pages) atomicAdd(p.refs + page, 1);
        } else if (j >= used || given < 0) {
            to[j] = -1;                               // a last page that the source lacks is lacking here as well
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

// One step over the pool, and one request a thread, with 256 threads.
inline bool few(int pages, int n) { return pages <= 256 * PER_THREAD && n <= 256; }

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
    const bool small = few(pages, n);
    st = small ? smem_limit<kv_alloc_kernel<256>>() : smem_limit<kv_alloc_kernel<1024>>();
    if (st != SQAP_OK) return st;
    const Pool p = {refs, pages, page_shift_of(page_tokens), table, ldt, rows, lens};
    const size_t smem = (static_cast<size_t>(rows) + n) * sizeof(int);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return finish_launch(small ? launch_dependent(kv_alloc_kernel<256>, dim3(1), dim3(256), smem, s, p, row_list, add, n, granted)
                               : launch_dependent(kv_alloc_kernel<1024>, dim3(1), dim3(1024), smem, s, p, row_list, add, n, granted));
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
    const bool small = few(pages, n);
    st = small ? smem_limit<kv_fork_kernel<256>>() : smem_limit<kv_fork_kernel<1024>>();
    if (st != SQAP_OK) return st;
    const Pool p = {refs, pages, page_shift_of(page_tokens), table, ldt, rows, lens};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const size_t smem = (static_cast<size_t>(rows) + n) * sizeof(int);
    int2* const out = reinterpret_cast<int2*>(pairs);
    st = finish_launch(small ? launch_dependent(kv_fork_kernel<256>, dim3(1), dim3(256), smem, s, p, src_rows, dst_rows, n, out, granted)
                             : launch_dependent(kv_fork_kernel<1024>, dim3(1), dim3(1024), smem, s, p, src_rows, dst_rows, n, out, granted));
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
