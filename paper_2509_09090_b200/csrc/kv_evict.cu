// Which tokens of a sequence stay in the cache: the last ones, the first ones, and of the rest those with the largest weight.
//
// A CTA, or a cluster of up to eight, takes one sequence. The weights are ordered as whole numbers; the m-th largest is found by narrowing the interval
// that holds it: a histogram of BINS equal parts of the interval (at first from the smallest to the largest weight), the bin that
// holds the m-th, and again within it: two or three rounds for 32 bits. Equal weights are told apart by their place. A
// warp owns runs of 32 consecutive tokens, a lane one of each: its votes give a token's place within the run, one sum over
// the runs in front of it the rest, and the lanes that write the list write side by side.
// Bounded by latency: 4 bytes a token are read once (up to 16384 tokens a CTA are kept in registers, longer ones read again each
// round), and some seven steps of the whole CTA follow one another, four of them with a cluster's barrier: 16 x 288 tokens 4.2 us,
// 32 uneven sequences of up to 16384 12.2 us, one of 131072 18.9 us (weights from HBM; from L2 4.5, 11.4 and 17.6).
#include "kv.cuh"

namespace sqap {
namespace kv {
namespace {

struct EvictArgs {
    float* mass;
    int64_t ldm;
    int rows;
    const int32_t* lens;
    const int32_t* src;
    const int32_t* dst;
    const int32_t* keep;
    int first, recent, max_len;
    int32_t* kept;
    int64_t ldkept;
    int32_t* n_kept;
};

// Order of the numbers as whole numbers; -0 = 0; 1 for what is not a number, in front of all. None of them is 0 or ALWAYS.
constexpr uint32_t ALWAYS = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t order_of(float f) {
    if (!(f == f)) return 1;
    const uint32_t b = __float_as_uint(f + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Shared memory of another CTA of the cluster: the place of `p` there.
__device__ __forceinline__ uint32_t remote_address(const void* p, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
    return r;
}
__device__ __forceinline__ uint2 remote_load(uint32_t at) {
    uint2 v;
    asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void remote_store(uint32_t at, uint32_t x, uint32_t y) {
    asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(at), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
    cluster_arrive();
    cluster_wait();
}

// CTAS CTAs, a cluster, take a sequence; EACH tokens a thread and round, a CTA's side by side; longer sequences take several rounds. Every
// CTA knows what it needs to find the same border: the histograms of all, and how many stay in front of it.
template <int THREADS, int EACH, int CTAS>
__global__ void __launch_bounds__(THREADS) kv_evict_kernel(EvictArgs a) {
    constexpr int BINS = 2 * THREADS, WARPS = THREADS / 32, RUNS = EACH * WARPS;
    static_assert(THREADS * EACH < 65536 && RUNS % 32 == 0, "two counts to a word, runs shared out to whole warps");
    constexpr int BUFFERS = CTAS > 1 ? 2 : 1;    // another CTA may still be reading the bins of the round before
    // the bins; once the border is known, places of the tokens that stay within the CTA's share of the round
    constexpr int SHARED = BUFFERS * BINS * 4 > THREADS * EACH * 2 ? BUFFERS * BINS * 4 : THREADS * EACH * 2;
    __shared__ alignas(8) uint8_t bins_or_list[SHARED];
    uint32_t (*bins)[BINS] = reinterpret_cast<uint32_t (*)[BINS]>(bins_or_list);
    uint16_t* list = reinterpret_cast<uint16_t*>(bins_or_list);
    __shared__ alignas(8) uint32_t of_all[3][CTAS][2];      // of each CTA: smallest order - 1 and largest + 1; places and ties, by parity of the round
    __shared__ uint32_t part[WARPS], least[WARPS], most[WARPS];
    __shared__ uint32_t found[3];        // the bin, how many are above it, how many in it
    __shared__ uint32_t front[RUNS];     // of each run of 32 tokens: those in front of it that stay, and (upper half) that are at the border
    pdl_launch_dependents();
    if (CTAS > 1) cluster_arrive();
    pdl_wait();
    const int i = blockIdx.x / CTAS, rank = blockIdx.x % CTAS, row = a.src[i], dst = a.dst ? a.dst[i] : -1, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool there = row >= 0 && row < a.rows;
    const int64_t held = a.ldm < a.max_len ? a.ldm : a.max_len;
    int len = there ? a.lens[row] : 0;
    len = len < 0 ? 0 : static_cast<int>(len < held ? len : held);
    const int64_t room = a.ldkept;
    int keep = a.keep[i];
    keep = keep < 0 ? 0 : static_cast<int>(keep < room ? keep : room);
    keep = min(keep, len);
    const int recent = min(a.recent, keep), first = min(min(a.first, keep - recent), len - recent);
    const int to = len - recent;         // tokens first .. to - 1 are chosen from
    const uint32_t wanted = static_cast<uint32_t>(keep - recent - first);
    const float* mass = a.mass + (there ? row : 0) * a.ldm;
    const int rounds = (len + CTAS * THREADS * EACH - 1) / (CTAS * THREADS * EACH);
    auto token_of = [&](int r, int e) { return ((r * CTAS + rank) * EACH + e) * THREADS + tid; };
    uint32_t order[EACH];                // 0: no token; ALWAYS: stays whatever its weight is
    auto load = [&](int r) {
        float x[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) x[e] = token_of(r, e) < len ? mass[token_of(r, e)] : 0.0f;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int t = token_of(r, e);
            order[e] = t >= first && t < to ? order_of(x[e]) : t < len ? ALWAYS : 0;
        }
    };
    auto each = [&](auto f) {
        for (int r = 0; r < rounds; ++r) {
            if (rounds > 1) load(r);
#pragma unroll
            for (int e = 0; e < EACH; ++e) f(order[e]);
        }
    };
    if (rounds == 1) load(0);
    if (CTAS > 1) cluster_wait();        // all CTAs have started: their shared memory may be written

    // border: orders above it stay, of those equal to it the first `ties` in their places
    uint32_t border = ALWAYS - 1, ties = 0;
    if (wanted > 0) {
        // The smallest order less 1 and the largest plus 1: 0 then comes out on top of all and ALWAYS at the bottom. They are taken back only
        // once all CTAs' are known: one without a token to choose from has none to take back, the sequence has `wanted` or more.
        uint32_t lo = 0xFFFFFFFFu, hi = 0;
        each([&](uint32_t k) {
            lo = min(lo, k - 1);
            hi = max(hi, k + 1);
        });
        lo = __reduce_min_sync(0xffffffffu, lo);
        hi = __reduce_max_sync(0xffffffffu, hi);
        if (lane == 0) {
            least[warp] = lo;
            most[warp] = hi;
        }
        __syncthreads();
        lo = __reduce_min_sync(0xffffffffu, least[lane < WARPS ? lane : 0]);
        hi = __reduce_max_sync(0xffffffffu, most[lane < WARPS ? lane : 0]);
        if (CTAS > 1) {
            if (tid < CTAS) remote_store(remote_address(&of_all[2][rank], tid), lo, hi);
            cluster_sync();
#pragma unroll
            for (int q = 0; q < CTAS; ++q) {
                lo = min(lo, of_all[2][q][0]);
                hi = max(hi, of_all[2][q][1]);
            }
        }
        ++lo;
        --hi;
        int buffer = 0;
        uint32_t left = wanted;          // of the orders in lo .. hi, the left-th largest is the border
        for (;;) {
            // parts of 2^shift orders, at most BINS of them (shift 0 once the interval is that short)
            const int width = 32 - __clz(hi - lo), shift = max(0, width - (31 - __clz(BINS)));
            for (int b = tid; b < BINS; b += THREADS) bins[buffer][b] = 0;
            __syncthreads();
            each([&](uint32_t k) {
                if (k - lo <= hi - lo) atomicAdd(&bins[buffer][(k - lo) >> shift], 1u);
            });
            // thread t looks at bins BINS - 1 - 2t and the one below it: the sums run from the largest orders down
            uint32_t up, down;
            if (CTAS > 1) {
                cluster_sync();
                uint2 two[CTAS];
#pragma unroll
                for (int q = 0; q < CTAS; ++q) two[q] = remote_load(remote_address(&bins[buffer][BINS - 2 - 2 * tid], q));
                up = down = 0;
#pragma unroll
                for (int q = 0; q < CTAS; ++q) {
                    up += two[q].y;
                    down += two[q].x;
                }
                buffer ^= 1;
            } else {
                __syncthreads();
                up = bins[0][BINS - 1 - 2 * tid];
                down = bins[0][BINS - 2 - 2 * tid];
            }
            uint32_t y = up + down;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t z = __shfl_up_sync(0xffffffffu, y, o);
                if (lane >= o) y += z;
            }
            if (lane == 31) part[warp] = y;
            __syncthreads();
            const uint32_t above = __reduce_add_sync(0xffffffffu, lane < warp ? part[lane] : 0u) + y - up - down;
            if (above < left && left <= above + up) {
                found[0] = BINS - 1 - 2 * tid;
                found[1] = above;
                found[2] = up;
            } else if (above + up < left && left <= above + up + down) {
                found[0] = BINS - 2 - 2 * tid;
                found[1] = above + up;
                found[2] = down;
            }
            __syncthreads();
            const uint32_t in_bin = found[2];
            left -= found[1];
            lo += found[0] << shift;
            hi = min(hi, lo + ((1u << shift) - 1u));
            if (left == in_bin) {        // all of the bin stay: from lo >= 1 on
                border = lo - 1;
                break;
            }
            if (shift == 0) {
                border = lo;
                ties = left;
                break;
            }
        }
    }

    int32_t* kept = a.kept + i * a.ldkept;
    float* carry = dst >= 0 && dst < a.rows && dst != row ? a.mass + dst * a.ldm : nullptr;
    uint32_t sure_before = 0, ties_before = 0;               // of earlier rounds, and of CTAs in front
    for (int r = 0; r < rounds; ++r) {
        if (rounds > 1) load(r);
        uint32_t votes[EACH];                    // of the run: who stays, ties apart
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            votes[e] = __ballot_sync(0xffffffffu, order[e] > border);
            if (lane == 0) front[e * WARPS + warp] = __popc(votes[e]);
        }
        if (ties > 0) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const uint32_t equal = __ballot_sync(0xffffffffu, order[e] == border);
                if (lane == 0) front[e * WARPS + warp] += __popc(equal) << 16;
            }
        }
        __syncthreads();
        // sums in front of each run: RUNS / THREADS of them a thread, or one for some of the threads
        constexpr int SUMMING = RUNS < THREADS ? RUNS : THREADS, MINE = RUNS / SUMMING;
        uint32_t mine[MINE], sum = 0, y = 0;
        if (tid < SUMMING) {
#pragma unroll
            for (int x = 0; x < MINE; ++x) {
                mine[x] = front[tid * MINE + x];
                sum += mine[x];
            }
            y = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t z = __shfl_up_sync(0xffffffffu, y, o);
                if (lane >= o) y += z;
            }
            if (lane == 31) part[warp] = y;
        }
        __syncthreads();
        const uint32_t in_part = lane < SUMMING / 32 ? part[lane] : 0u;
        const uint32_t all = __reduce_add_sync(0xffffffffu, in_part);
        uint32_t at = __reduce_add_sync(0xffffffffu, lane < warp ? in_part : 0u) + y - sum;
        if (tid < SUMMING) {
#pragma unroll
            for (int x = 0; x < MINE; ++x) {
                front[tid * MINE + x] = at;
                at += mine[x];
            }
        }
        __syncthreads();
        uint32_t sure_all = all & 0xFFFFu, ties_all = all >> 16;
        if (CTAS > 1) {
            if (tid < CTAS) remote_store(remote_address(&of_all[r & 1][rank], tid), sure_all, ties_all);
            cluster_sync();
            sure_all = ties_all = 0;
#pragma unroll
            for (int q = 0; q < CTAS; ++q) {
                if (q == rank) {
                    sure_before += sure_all;
                    ties_before += ties_all;
                    sure_all = ties_all = 0;
                }
                sure_all += of_all[r & 1][q][0];
                ties_all += of_all[r & 1][q][1];
            }
        }
        const uint32_t under = (1u << lane) - 1u;
        const uint32_t ties_left = ties - min(ties_before, ties), placed = sure_before + min(ties_before, ties);
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const uint32_t f = front[e * WARPS + warp];
            bool stay = votes[e] >> lane & 1u;
            uint32_t ties_mine = 0;
            if (ties > 0) {
                const uint32_t equal = __ballot_sync(0xffffffffu, order[e] == border);
                ties_mine = min((f >> 16) + __popc(equal & under), ties_left);
                stay = stay || (order[e] == border && ties_mine < ties_left);
            }
            if (stay) list[(f & 0xFFFFu) + __popc(votes[e] & under) + ties_mine] = static_cast<uint16_t>(e * THREADS + tid);
        }
        __syncthreads();
        const int n = static_cast<int>((all & 0xFFFFu) + min(all >> 16, ties_left));
        for (int p = tid; p < n; p += THREADS) {
            const int t = (r * CTAS + rank) * THREADS * EACH + list[p];
            kept[placed + p] = t;
            if (carry) carry[placed + p] = __ldg(mass + t);      // no row is both read and written
        }
        sure_before += sure_all;
        ties_before += ties_all;
        __syncthreads();                         // `front` and `list` are written again
    }
    if (tid == 0 && rank == 0) a.n_kept[i] = keep;
    for (int64_t p = keep + rank * THREADS + tid; p < a.ldkept; p += CTAS * THREADS) kept[p] = -1;
}

template <int THREADS, int EACH, int CTAS>
cudaError_t launch_evict(const EvictArgs& a, int n, cudaStream_t s) {
    if (CTAS == 1) return launch_dependent(kv_evict_kernel<THREADS, EACH, CTAS>, dim3(static_cast<unsigned>(n)), dim3(THREADS), 0, s, a);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(n) * CTAS);
    cfg.blockDim = dim3(THREADS);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CTAS;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kv_evict_kernel<THREADS, EACH, CTAS>, a);
}

}  // namespace
}  // namespace kv
}  // namespace sqap

extern "C" sqap_status sqap_kv_evict(float* mass, int64_t ldm, int rows, const int32_t* lens, const int32_t* src_rows,
                                     const int32_t* dst_rows, int n, const int32_t* keep, int first, int recent, int max_len,
                                     int32_t* kept, int64_t ldkept, int32_t* n_kept, void* stream) {
    using namespace sqap;
    using namespace sqap::kv;
    if (rows < 0 || n < 0 || first < 0 || recent < 0 || max_len < 0 || ldm < 0 || ldkept < 0) return SQAP_ERR_INVALID;
    if (n == 0) return SQAP_OK;
    if (!lens || !src_rows || !keep || !n_kept || (ldm > 0 && !mass) || (ldkept > 0 && !kept)) return SQAP_ERR_INVALID;
    for (const void* p : {static_cast<const void*>(mass), static_cast<const void*>(lens), static_cast<const void*>(src_rows),
                          static_cast<const void*>(dst_rows), static_cast<const void*>(keep), static_cast<const void*>(kept),
                          static_cast<const void*>(n_kept)})
        if (reinterpret_cast<uintptr_t>(p) & 3u) return SQAP_ERR_ALIGN;
    if (ldkept > 0x7FFFFFFF || max_len > 1 << 30) return SQAP_ERR_UNSUPPORTED;
    const EvictArgs a = {mass, ldm, rows, lens, src_rows, dst_rows, keep, first, recent, max_len, kept, ldkept, n_kept};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (max_len <= 1024) return finish_launch(launch_evict<256, 4, 1>(a, n, s));
    if (max_len <= 4096) return finish_launch(launch_evict<1024, 4, 1>(a, n, s));
    // As many CTAs to a sequence as the device has SMs for, as long as each has 4096 tokens or more, and two only where they save a round (us, weights in L2,
    // one CTA / as many as here: 32 x 16384 13.0 / 11.4; one / two: 64 x 16384 13.5 / 16.7). Up to 16 tokens a thread rather than
    // a second round (131072 tokens in eight CTAs, 4 / 16: 31.9 / 17.6).
    const int64_t ctas = sm_count() / (n < sm_count() ? n : sm_count());
    if (ctas >= 8 && max_len > 16384) return finish_launch(max_len <= 32768 ? launch_evict<1024, 4, 8>(a, n, s) : launch_evict<1024, 16, 8>(a, n, s));
    if (ctas >= 4 && max_len > 8192) return finish_launch(max_len <= 16384 ? launch_evict<1024, 4, 4>(a, n, s) : launch_evict<1024, 16, 4>(a, n, s));
    if (ctas >= 2 && max_len <= 8192) return finish_launch(launch_evict<1024, 4, 2>(a, n, s));
    if (ctas >= 2 && max_len > 16384) return finish_launch(launch_evict<1024, 16, 2>(a, n, s));
    return finish_launch(launch_evict<1024, 16, 1>(a, n, s));
}
