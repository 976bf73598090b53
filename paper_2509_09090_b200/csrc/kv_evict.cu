// Which tokens of a sequence stay in the cache: the last ones, the first ones, and of the rest those with the largest weight.
//
// One CTA takes one sequence. The weights are ordered as whole numbers; the m-th largest is found by narrowing the interval
// that holds it: a histogram of BINS equal parts of the interval (at first from the smallest to the largest weight, so that neither
// zeros nor a narrow spread crowd a bin), the bin that holds the m-th, and again within it: two or three rounds for
// 32 bits. Equal weights are told apart by their place. A thread owns consecutive tokens, so that one sum over the CTA in the
// order of the threads gives the places in the list.
// Bounded by latency: 4 bytes a token are read once (up to 16384 tokens are kept in registers, longer ones read again each
// round), and some eight sums over the CTA follow one another.
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

// Order of the numbers as whole numbers from 1 on; -0 = 0; what is not a number comes in front of all.
__device__ __forceinline__ uint32_t order_of(float f) {
    if (!(f == f)) return 0;
    const uint32_t b = __float_as_uint(f + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Sum of x over the threads in front of this one, and over all; a call uses the other half of `part` than the one before.
template <int THREADS>
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t (&part)[2][THREADS / 32], int& turn, uint32_t* all) {
    constexpr int WARPS = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t y = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t z = __shfl_up_sync(0xffffffffu, y, o);
        if (lane >= o) y += z;
    }
    if (lane == 31) part[turn][warp] = y;
    __syncthreads();
    uint32_t w = lane < WARPS ? part[turn][lane] : 0;
    turn ^= 1;
#pragma unroll
    for (int o = 1; o < WARPS; o <<= 1) {
        const uint32_t z = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += z;
    }
    *all = __shfl_sync(0xffffffffu, w, WARPS - 1);
    const uint32_t front = __shfl_sync(0xffffffffu, w, warp > 0 ? warp - 1 : 0);
    return y - x + (warp > 0 ? front : 0);
}

// EACH consecutive tokens a thread and round; longer sequences than THREADS x EACH take several rounds.
template <int THREADS, int EACH>
__global__ void __launch_bounds__(THREADS) kv_evict_kernel(EvictArgs a) {
    constexpr int BINS = 2 * THREADS, WARPS = THREADS / 32;
    __shared__ uint32_t bins[BINS];
    __shared__ uint32_t part[2][WARPS], least[WARPS], most[WARPS];
    __shared__ uint32_t found[3];        // the bin, how many are above it, how many in it
    pdl_launch_dependents();
    pdl_wait();
    const int i = blockIdx.x, row = a.src[i], tid = threadIdx.x, lane = tid & 31;
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
    const int rounds = (len + THREADS * EACH - 1) / (THREADS * EACH);
    float x[EACH];
    auto load = [&](int r) {
        const int t0 = (r * THREADS + tid) * EACH;
#pragma unroll
        for (int e = 0; e < EACH; ++e) x[e] = t0 + e < len ? mass[t0 + e] : 0.0f;
    };
    // f(token, order) for the tokens that are chosen from
    auto each = [&](auto f) {
        for (int r = 0; r < rounds; ++r) {
            if (rounds > 1) load(r);
            const int t0 = (r * THREADS + tid) * EACH;
#pragma unroll
            for (int e = 0; e < EACH; ++e)
                if (t0 + e >= first && t0 + e < to) f(t0 + e, order_of(x[e]));
        }
    };
    if (rounds == 1) load(0);

    // border: orders above it stay, of those equal to it the first `ties` in their places
    uint32_t border = 0, ties = 0;
    if (wanted == static_cast<uint32_t>(to - first)) {
        ties = wanted;                   // all of them: no order is below 0
    } else if (wanted == 0) {
        border = 0xFFFFFFFFu;
    } else {
        uint32_t lo = 0xFFFFFFFFu, hi = 0;
        each([&](int, uint32_t k) {
            lo = min(lo, k);
            hi = max(hi, k);
        });
        lo = __reduce_min_sync(0xffffffffu, lo);
        hi = __reduce_max_sync(0xffffffffu, hi);
        if (lane == 0) {
            least[tid >> 5] = lo;
            most[tid >> 5] = hi;
        }
        __syncthreads();
        lo = least[lane < WARPS ? lane : 0];
        hi = most[lane < WARPS ? lane : 0];
        lo = __reduce_min_sync(0xffffffffu, lo);
        hi = __reduce_max_sync(0xffffffffu, hi);
        uint32_t left = wanted;          // of the orders in lo .. hi, the left-th largest is the border
        for (;;) {
            // parts of 2^shift orders, fewer than BINS of them (shift 0 once the interval is that short)
            const int width = 32 - __clz(hi - lo), shift = max(0, width - (31 - __clz(BINS)));
            for (int b = tid; b < BINS; b += THREADS) bins[b] = 0;
            __syncthreads();
            each([&](int, uint32_t k) {
                if (k >= lo && k <= hi) atomicAdd(&bins[(k - lo) >> shift], 1u);
            });
            __syncthreads();
            // thread t looks at bins BINS - 1 - 2t and the one below it: the sums run from the largest orders down
            const uint32_t up = bins[BINS - 1 - 2 * tid], down = bins[BINS - 2 - 2 * tid];
            const int lane_warp = tid >> 5;
            uint32_t y = up + down;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t z = __shfl_up_sync(0xffffffffu, y, o);
                if (lane >= o) y += z;
            }
            if (lane == 31) part[0][lane_warp] = y;
            __syncthreads();
            uint32_t w = lane < WARPS ? part[0][lane] : 0;
            w = __reduce_add_sync(0xffffffffu, lane < lane_warp ? w : 0u);
            const uint32_t above = w + y - up - down;
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
            if (left == in_bin) {        // all of the bin stay
                border = lo;
                ties = 0xFFFFFFFFu;
                break;
            }
            if (shift == 0) {
                border = lo;
                ties = left;
                break;
            }
        }
        if (ties == 0xFFFFFFFFu) {       // from `border` on: everything above border - 1 (orders of numbers that are chosen from start at 0)
            if (border > 0) {
                --border;
                ties = 0;
            }
        }
    }

    int32_t* kept = a.kept + i * a.ldkept;
    const int dst = a.dst ? a.dst[i] : -1;
    float* carry = dst >= 0 && dst < a.rows ? a.mass + dst * a.ldm : nullptr;
    uint32_t ties_before = 0, kept_before = 0;
    int turn = 1;                        // part[0] was read last
    for (int r = 0; r < rounds; ++r) {
        if (rounds > 1) load(r);
        const int t0 = (r * THREADS + tid) * EACH;
        uint32_t equal = 0, stays = 0;   // bits
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int t = t0 + e;
            if (t >= len) continue;
            if (t < first || t >= to) {
                stays |= 1u << e;
                continue;
            }
            const uint32_t k = order_of(x[e]);
            if (k > border) stays |= 1u << e;
            if (k == border) equal |= 1u << e;
        }
        uint32_t all;
        if (ties > 0) {
            uint32_t place = ties_before + sum_before<THREADS>(__popc(equal), part, turn, &all);
            ties_before += all;
#pragma unroll
            for (int e = 0; e < EACH; ++e)
                if (equal >> e & 1u && place++ < ties) stays |= 1u << e;
        }
        uint32_t place = kept_before + sum_before<THREADS>(__popc(stays), part, turn, &all);
        kept_before += all;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            if (!(stays >> e & 1u)) continue;
            kept[place] = t0 + e;
            if (carry) carry[place] = x[e];
            ++place;
        }
    }
    if (tid == 0) a.n_kept[i] = keep;
    for (int64_t p = keep + tid; p < a.ldkept; p += THREADS) kept[p] = -1;
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
    const dim3 grid(static_cast<unsigned>(n));
    if (max_len <= 1024) return finish_launch(launch_dependent(kv_evict_kernel<256, 4>, grid, dim3(256), 0, s, a));
    if (max_len <= 4096) return finish_launch(launch_dependent(kv_evict_kernel<1024, 4>, grid, dim3(1024), 0, s, a));
    return finish_launch(launch_dependent(kv_evict_kernel<1024, 16>, grid, dim3(1024), 0, s, a));
}
