// Attention of many query rows (prompts) over the paged 8-bit cache on tcgen05, head_dim 64 and 128.
//
// An item is 256 rows (query x head of the group, packed: the heads that share a key/value head share its tiles) of one
// sequence and key/value head, in two halves of 128; its keys are walked 64 at a time. Per tile and half: S = Q K^T into tensor
// memory, the softmax's weights back into tensor memory as the A operand, O += W V.
//   warps 0-3, 4-7  softmax of the two halves: thread = row. Rescale the output where a maximum has grown, and store it.
//   warps 8-15      codes from global memory (one tile ahead, in registers) to fp16 in shared memory, 128B-swizzled; the next
//                   item's queries
//   warp  16        issues the MMAs: the scores of a tile before the output of the tile in front of it, half by half, so that
//                   the tensor core works on one half while the softmax of the other is busy
// Work per 64 keys and half, and what it costs an SM: MMAs 2 x 128 x 64 x D (640 cycles at D = 128: the scores read both
// operands from shared memory), 8192 exponentials (512 cycles), some 3 instructions per weight; and per 64 keys 1.3 per code. It
// is the instructions and the round trips between the roles that bound it (two prompts of 4099 tokens behind 1000, 32 heads in
// groups of 4: 501 us, 818 TFLOP/s, 510 us in a region of seconds; 16 of 288 tokens, 32 heads: 60 us): an earlier form with 128 rows an item and two CTAs to an SM, which converted every tile
// for 128 rows only, issued 8200 warp instructions per 128 x 128 scores, 5000 of them for the conversion, at 64 % of
// the issue slots. Persistent CTAs, one to an SM; 512 columns of tensor memory: two tiles of scores and one output for
// each half.
//
// The running maximum is raised only when a row's maximum has grown by more than 2^8 (the weights then stay within fp16, at
// the same relative precision): rescaling the output in tensor memory is rare after the first tiles. Weights and sums:
// kv_attention.cuh.
//
// Every wait is bounded; on expiry the kernel records SQAP_ERR_TIMEOUT in the device status word and ends.
#include <type_traits>

#include "kv_attention.cuh"
#include "tc_common.cuh"

namespace sqap {
namespace kv {
namespace {

using namespace tc;

constexpr int KEYS = 64;                    // keys per tile
constexpr int GROUPS = KEYS / 16;           // runs of 16 keys: a page never ends inside one
constexpr int CONV_WARPS = 8;
constexpr int CONV_WARP0 = 8, MMA_WARP = CONV_WARP0 + CONV_WARPS;
constexpr int THREADS = 32 * (MMA_WARP + 1);
constexpr int ROWS = PREFILL_TC_ROWS;       // of an item
// Registers: LAUNCH_REGS a thread at launch, of which the converting warps give up what the softmax takes on.
constexpr int LAUNCH_REGS = 96, SOFTMAX_REGS = 120, CONV_REGS = 64;
static_assert(CONV_WARP0 * SOFTMAX_REGS + CONV_WARPS * CONV_REGS <= MMA_WARP * LAUNCH_REGS, "register split");
constexpr int RING = 4;                     // tiles of keys and values in shared memory
constexpr int Q_BLOCK = 128 * 128;          // 128 rows of 64 halves
constexpr int KV_BLOCK = KEYS * 128;        // a tile's keys or values, 64 elements of each
constexpr int TMEM_COLS = 512;              // half g: scores (and weights) of two tiles from 128 g, output from 256 + 128 g
constexpr int O_COL = 256;
constexpr float RAISE = 8.0f;

template <int D>
struct Smem {
    static constexpr int BLOCKS = D / 64, TILE = BLOCKS * KV_BLOCK, HALF_Q = BLOCKS * Q_BLOCK;
    static constexpr int Q = 0, K = 2 * HALF_Q, V = K + RING * TILE, TAIL = V + RING * TILE;
    static constexpr int OFF_FAC = 256, OFF_BAR = OFF_FAC + 2 * ROWS * 4, OFF_WORDS = OFF_BAR + 256;
    static constexpr int BYTES = TAIL + OFF_WORDS + 64 + 1024;      // slack for the alignment
};
// Scales of the tiles in the ring, by run of 16 keys.
struct Scales {
    float ks[RING][GROUPS], lv[RING][GROUPS], iv[RING][GROUPS];
};

__device__ __forceinline__ void tc_mma_f16(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate, uint32_t issue) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(issue)
        : "memory");
}
__device__ __forceinline__ void tc_mma_f16_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate, uint32_t issue) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(issue)
        : "memory");
}
__device__ __forceinline__ void tc_ld32(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// Values [key][element], elements contiguous (the operand's N dimension): 128B-swizzled blocks of 64 elements; 8 keys are 1024
// bytes apart, blocks KV_BLOCK.
__device__ __forceinline__ uint64_t smem_desc_values(uint32_t addr) {
    return static_cast<uint64_t>((addr >> 4) & 0x3FFFu) | (static_cast<uint64_t>(KV_BLOCK >> 4) << 16) | (64ull << 32) | (1ull << 46) |
           (2ull << 61);
}

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, bool real) {   // zeros where there is nothing to copy
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// a * b + c of two pairs at once.
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ void unpair(uint64_t d, float* lo, float* hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(*lo), "=f"(*hi) : "l"(d)); }

__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// One item: 256 rows of a sequence and key/value head (and one piece of its history, where those are cut).
struct Item {
    Where w;
    int rows, r_first, key0, end, steps;
    int steps_lo;     // tiles that the lower half of the rows looks at (the upper half: all, or there is no upper half)
};
__device__ __forceinline__ Item item_of(const AttnArgs& a, unsigned id) {
    Item x;
    // tiles outermost, the rows that see the most first
    const unsigned per_tile = static_cast<unsigned>(a.batch) * a.c.kv_heads * a.splits;
    const unsigned tile = id / per_tile;
    x.w = locate(a, id - tile * per_tile, 1);
    x.w.tile = a.tiles - 1 - static_cast<int>(tile);
    x.rows = (x.w.n_q < a.max_q ? x.w.n_q : a.max_q) * a.group;
    x.r_first = x.w.tile * ROWS;
    x.key0 = x.w.split * a.chunk;
    x.end = 0;
    x.steps = x.steps_lo = 0;
    if (x.r_first < x.rows && a.c.pages > 0) {
        const int key1 = a.splits > 1 ? min(x.key0 + a.chunk, x.w.len) : x.w.len;
        const int last = min(x.rows, x.r_first + ROWS) - 1, last_lo = min(x.rows, x.r_first + ROWS / 2) - 1;
        x.end = min(key1, visible(a, x.w, last / a.group));
        const int end_lo = min(key1, visible(a, x.w, last_lo / a.group));
        x.steps = x.end > x.key0 ? (x.end - x.key0 + KEYS - 1) / KEYS : 0;
        x.steps_lo = end_lo > x.key0 ? (end_lo - x.key0 + KEYS - 1) / KEYS : 0;
    }
    return x;
}
// Tiles of half g, 0 where it has no rows.
__device__ __forceinline__ int half_steps(const Item& x, int g) {
    if (g == 0) return x.steps_lo;
    return x.r_first + ROWS / 2 < x.rows ? x.steps : 0;
}

template <typename T, int TYPE, int D>
__global__ void __launch_bounds__(THREADS, 1) kv_prefill_tc_kernel(AttnArgs a, unsigned items, int* status) {
    using S = Smem<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* sm = smem_raw + (base - smem_u32(smem_raw));
    Scales* scales = reinterpret_cast<Scales*>(sm + S::TAIL);
    float* row_fac = reinterpret_cast<float*>(sm + S::TAIL + S::OFF_FAC);       // [2][ROWS]: by parity of the item
    static_assert(sizeof(Scales) <= S::OFF_FAC, "tail layout");
    const uint32_t bar0 = base + S::TAIL + S::OFF_BAR;
    // Tile n of the CTA lies in slot n % RING, in that barrier's phase n / RING. Tile c of a half (its own count) uses the
    // half's barriers of parity c & 1, in their phase c >> 1.
    auto kv_full = [&](uint32_t slot) { return bar0 + 8u * slot; };                                // keys, values, scales (and row factors)
    auto kv_free = [&](uint32_t slot) { return bar0 + 8u * (RING + slot); };
    auto s_full = [&](int g, uint32_t c) { return bar0 + 8u * (2 * RING + 2 * g + (c & 1)); };     // scores are there
    auto p_full = [&](int g, uint32_t c) { return bar0 + 8u * (2 * RING + 4 + 2 * g + (c & 1)); }; // weights are there
    auto o_done = [&](int g, uint32_t c) { return bar0 + 8u * (2 * RING + 8 + 2 * g + (c & 1)); }; // the output has taken them
    const uint32_t q_full = bar0 + 8u * (2 * RING + 12), q_free = q_full + 8u;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(sm + S::TAIL + S::OFF_WORDS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + S::TAIL + S::OFF_WORDS + 8);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (uint32_t b = 0; b < RING; ++b) {
            mbar_init(kv_full(b), CONV_WARPS);
            mbar_init(kv_free(b), 1);
        }
        for (uint32_t b = 0; b < 4; ++b) {
            mbar_init(s_full(b >> 1, b), 1);
            mbar_init(p_full(b >> 1, b), 4);
            mbar_init(o_done(b >> 1, b), 1);
        }
        mbar_init(q_full, CONV_WARPS);
        mbar_init(q_free, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(const_cast<uint32_t*>(tmem_slot))), "n"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t tmem = *tmem_slot;
    const int G = a.group;
    bool failed = false;
    auto wait_phase = [&](uint32_t bar, uint32_t phase) { return __all_sync(0xffffffffu, mbar_wait(bar, phase & 1u, abort_flag)) != 0; };
    // the place of the CTA's next tile in the ring, and how often the ring has been walked
    uint32_t slot = 0, walk = 0;
    auto next_slot = [&]() {
        if (++slot == RING) {
            slot = 0;
            ++walk;
        }
    };

    if (warp < CONV_WARP0) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFTMAX_REGS));
        const int half = warp >> 2;
        const uint32_t t_lane = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + 128 * half, t_o = t_lane + O_COL;
        uint32_t n = 0;             // tiles of this half so far
        uint32_t full_items = 0;
        Item next = item_of(a, blockIdx.x);
        for (unsigned id = blockIdx.x; id < items; id += gridDim.x) {
            const Item x = next;
            const int r = x.r_first + static_cast<int>(threadIdx.x);
            const bool real = r < x.rows;
            const int qi = real ? r / G : 0, head = x.w.h * G + (real ? r - qi * G : 0);
            const int lim = real ? min(visible(a, x.w, qi), x.end) : 0;
            const bool idle = x.r_first + warp * 32 >= x.rows;          // no rows: whatever these lanes hold goes nowhere
            const int steps = half_steps(x, half);
            float m = -INFINITY, l = 0.0f, fac = 0.0f;
            for (int j = 0; j < steps; ++j, ++n, next_slot()) {
                // (the tile's scales and the rows' factors are written before kv_full)
                if (!wait_phase(kv_full(slot), walk) || !wait_phase(s_full(half, n), n >> 1)) { failed = true; break; }
                if (!idle) {
                    tc_fence_after();
                    if (j == 0) fac = row_fac[(full_items & 1) * ROWS + threadIdx.x];
                    const float* ks = scales->ks[slot];
                    const float* lv = scales->lv[slot];
                    const float* iv = scales->iv[slot];
                    const int seen = lim - (x.key0 + j * KEYS);         // this row sees the first `seen` keys of the tile
                    const uint32_t t_s = t_lane + KEYS * (n & 1);
                    uint32_t v[KEYS];
                    tc_ld32(t_s, v);
                    tc_ld32(t_s + 32, v + 32);
                    tc_wait_ld();
                    if (!__all_sync(0xffffffffu, seen >= KEYS)) {
#pragma unroll
                        for (int i = 0; i < KEYS; ++i)
                            if (i >= seen) v[i] = 0xFF800000u;
                    }
                    // of a run's scores; never 0, so that what is masked stays at -inf
                    auto factor = [&](int run) { return fmaxf(fac * ks[run], 1e-37f); };
                    // the maximum of the scores of a run of 16, then one scaling
                    float top = -INFINITY;
#pragma unroll
                    for (int run = 0; run < GROUPS; ++run) {
                        float y = __uint_as_float(v[16 * run]);
#pragma unroll
                        for (int i = 1; i < 15; i += 2)
                            y = fmaxf(fmaxf(y, __uint_as_float(v[16 * run + i])), __uint_as_float(v[16 * run + i + 1]));
                        y = fmaxf(y, __uint_as_float(v[16 * run + 15]));
                        // a missing page has lv = -inf, and scores of zero
                        top = fmaxf(top, fmaf(y, factor(run), lv[run]));
                    }
                    const bool raise = m == -INFINITY ? top != -INFINITY : top > m + RAISE;
                    if (__any_sync(0xffffffffu, raise)) {
                        const float f = raise ? fast_exp2(m - top) : 1.0f;      // m = -inf: 0
                        if (raise) m = top;
                        l *= f;
                        if (j > 0) {
                            if (!wait_phase(o_done(half, n - 1), (n - 1) >> 1)) { failed = true; break; }
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < D / 16; ++c) {
                                uint32_t u[16];
                                tc_ld16(t_o + 16 * c, u);
                                tc_wait_ld();
#pragma unroll
                                for (int i = 0; i < 16; ++i) u[i] = __float_as_uint(__uint_as_float(u[i]) * f);
                                tc_st16(t_o + 16 * c, u);
                            }
                        }
                    }
                    const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
                    for (int run = 0; run < GROUPS; ++run) {
                        const float f = factor(run), z = lv[run] - ref;
                        const uint64_t f2 = pair_of(f, f), z2 = pair_of(z, z);
                        uint32_t p[8];
                        uint64_t sum = 0;
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            float w0, w1;
                            unpair(fma_pair(pair_of(__uint_as_float(v[16 * run + i]), __uint_as_float(v[16 * run + i + 1])), f2, z2), &w0, &w1);
                            w0 = fast_exp2(w0);
                            w1 = fast_exp2(w1);
                            sum = add_pair(sum, pair_of(w0, w1));
                            p[i / 2] = half2_of(w0, w1);
                        }
                        float s0, s1;
                        unpair(sum, &s0, &s1);
                        l = fmaf(s0 + s1, iv[run], l);
                        tc_st8(t_s + 8 * run, p);                       // the scores are in registers
                    }
                    tc_wait_st();
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(half, n));
            }
            if (failed) break;
            if (id + gridDim.x < items) next = item_of(a, id + gridDim.x);      // while the last output product runs
            for (int j = steps; j < x.steps; ++j) next_slot();          // tiles that the other half alone looks at
            if (x.steps > 0) ++full_items;
            if (steps > 0) {
                if (!wait_phase(o_done(half, n - 1), (n - 1) >> 1)) { failed = true; break; }
                tc_fence_after();
            }
            if (idle) continue;
            const float inv = l != 0.0f ? 1.0f / l : 0.0f;
            const int64_t row = static_cast<int64_t>(x.w.row0) + qi;
            const int64_t at = a.splits > 1 && real ? part_index(a, x.w.b, head, qi, x.w.split) : 0;
            T* out = static_cast<T*>(a.out) + row * a.ldo + static_cast<int64_t>(head) * D;
            float* po = a.part_o + at * D;
#pragma unroll
            for (int c = 0; c < D / 64; ++c) {
                uint32_t v[64];
                if (steps > 0) {
                    tc_ld32(t_o + 64 * c, v);
                    tc_ld32(t_o + 64 * c + 32, v + 32);
                    tc_wait_ld();
                } else {
#pragma unroll
                    for (int i = 0; i < 64; ++i) v[i] = 0;
                }
                if (!real) continue;
                if (a.splits > 1) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) reinterpret_cast<uint4*>(po + 64 * c)[i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float z[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[e] = __uint_as_float(v[8 * i + e]) * inv;
                        reinterpret_cast<uint4*>(out + 64 * c)[i] = pack8<T>(z);
                    }
                }
            }
            if (real) {
                if (a.splits > 1) a.part_ml[at] = make_float2(m, l);
                else if (a.lse) a.lse[row * a.heads + head] = l != 0.0f ? log_sum(m, l) : -INFINITY;
            }
            tc_fence_before();
        }
    } else if (warp < MMA_WARP) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(CONV_REGS));
        const int tid = threadIdx.x - 32 * CONV_WARP0;
        const int shift = a.c.page_shift, mask = (1 << shift) - 1;
        // A thread's pieces of a tile: 16 codes of key tid / 4, elements 64 b + 16 (tid % 4) on. Eight lanes then write eight
        // different 16-byte units.
        constexpr int BLOCKS = S::BLOCKS;
        static_assert(CONV_WARPS * 8 == KEYS, "one key for four threads");
        uint4 kc[BLOCKS], vc[BLOCKS];
        const int row = tid >> 2;
        // The tiles of this CTA's items, one after another.
        struct Tile {
            const int32_t* table;
            int h, k0, end;            // keys k0 .. of a sequence of `end` keys that count; end = 0: no more tiles
            int row0, r_first, rows;   // rows > 0: the first tile of an item, whose queries are wanted
        };
        unsigned id = blockIdx.x;
        Tile then = {};
        int left = 0;                  // tiles of the item behind `then`
        auto open_item = [&]() {
            then.end = 0;
            while (id < items) {
                const Item x = item_of(a, id);
                id += gridDim.x;
                if (x.steps == 0) continue;
                then.table = a.table + x.w.b * a.ldt;
                then.h = x.w.h;
                then.k0 = x.key0;
                then.end = x.end;
                then.row0 = x.w.row0;
                then.r_first = x.r_first;
                then.rows = x.rows;
                left = x.steps - 1;
                break;
            }
        };
        auto advance = [&]() {
            if (left > 0) {
                --left;
                then.k0 += KEYS;
                then.rows = 0;
            } else {
                open_item();
            }
        };
        // The table entry as it is; checked when it is used, so that nothing waits for it here.
        auto entry_of = [&](const Tile& t) {
            const int key = t.k0 + row, j = key >> shift;
            return key < t.end && j < a.ldt ? __ldg(t.table + j) : -1;
        };
        // Place of this thread's codes in the cache; -1 behind the end or where there is no page.
        const uint32_t page_bytes = static_cast<uint32_t>(a.c.kv_heads * D) << shift;      // 2^31 at most
        auto place_of = [&](const Tile& t, int entry) {
            const int64_t at = static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(entry)) * page_bytes) +
                               (((static_cast<uint32_t>(t.h) << shift) + ((t.k0 + row) & mask)) * D + (tid & 3) * 16);
            return checked_page(a.c, entry) < 0 ? -1 : at;
        };
        auto fetch = [&](const uint8_t* codes, int64_t place, uint4 (&to)[BLOCKS]) {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                to[b] = make_uint4(0, 0, 0, 0);                // zero codes, whatever lies there
                if (place >= 0) to[b] = __ldg(reinterpret_cast<const uint4*>(codes + place + 64 * b));
            }
        };
        // Scales: one thread of each run of 16 keys.
        float ks = 0.0f, vs = -1.0f;                           // vs < 0: no page
        const bool scaler = (tid & 63) == 0;
        auto fetch_scales = [&](const Tile& t, int entry) {
            ks = 0.0f;
            vs = -1.0f;
            if (scaler && checked_page(a.c, entry) >= 0) {
                const int64_t s = static_cast<int64_t>(entry) * a.c.kv_heads + t.h;
                ks = __ldg(a.c.k.scales + s);
                vs = __ldg(a.c.v.scales + s);
            }
        };
        const int unit = (tid & 3) * 2;
        const uint32_t to0 = row * 128 + ((unit ^ (row & 7)) << 4), to1 = row * 128 + (((unit + 1) ^ (row & 7)) << 4);
        auto put = [&](int region, const uint4 (&from)[BLOCKS]) {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const uint32_t in[4] = {from[b].x, from[b].y, from[b].z, from[b].w};
                uint32_t out[8];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (TYPE == SQAP_KV_INT8) {
                        out[2 * q] = biased_to_half2<0>(in[q] ^ 0x80808080u);
                        out[2 * q + 1] = biased_to_half2<1>(in[q] ^ 0x80808080u);
                    } else {
                        out[2 * q] = e4m3x2_to_half2(in[q] & 0xFFFFu);
                        out[2 * q + 1] = e4m3x2_to_half2(in[q] >> 16);
                    }
                }
                uint8_t* to = sm + region + b * KV_BLOCK;
                *reinterpret_cast<uint4*>(to + to0) = make_uint4(out[0], out[1], out[2], out[3]);
                *reinterpret_cast<uint4*>(to + to1) = make_uint4(out[4], out[5], out[6], out[7]);
            }
        };
        // Queries: a warp brings Q_ROWS rows, LPR lanes to a row.
        constexpr int Q_ROWS = ROWS / CONV_WARPS, LPR = D / 8, RPI = 32 / LPR, Q_STEPS = Q_ROWS / RPI;
        static_assert(Q_ROWS == 32, "the lanes of a warp write its rows' factors");
        const int qc = lane % LPR, q_row0 = (warp - CONV_WARP0) * Q_ROWS + lane / LPR;
        auto q_at = [&](int i) {
            const int rr = q_row0 + i * RPI;
            return static_cast<uint32_t>(S::Q + (rr >> 7) * S::HALF_Q + (qc >> 3) * Q_BLOCK + (rr & 127) * 128 + (((qc & 7) ^ (rr & 7)) << 4));
        };
        auto begin_queries = [&](const Tile& t) {
            const int first = t.r_first + q_row0;
            const T* q = static_cast<const T*>(a.q) + static_cast<int64_t>(t.row0) * a.ldq + static_cast<int64_t>(t.h) * G * D + 8 * qc;
            if (G == 1) {
                const T* p = q + first * a.ldq;
#pragma unroll
                for (int i = 0; i < Q_STEPS; ++i, p += RPI * a.ldq) {
                    const bool there = first + i * RPI < t.rows;
                    cp_async_16(base + q_at(i), there ? p : q, there);
                }
            } else {
                int qi = first / G, g = first - qi * G;
#pragma unroll 4
                for (int i = 0; i < Q_STEPS; ++i) {
                    const bool there = first + i * RPI < t.rows;
                    cp_async_16(base + q_at(i), there ? q + qi * a.ldq + g * D : q, there);
                    g += RPI;
                    while (g >= G) {
                        g -= G;
                        ++qi;
                    }
                }
            }
        };
        auto finish_queries = [&](float* fac) {
            cp_async_wait();
            // bf16 rows are scaled one by one to fit fp16; a negative scale goes into the queries, so that no factor is negative
            if (std::is_same<T, __half>::value) {
                if (a.scale_log2 < 0.0f)
                    for (int i = 0; i < Q_STEPS; ++i) {
                        uint4* u = reinterpret_cast<uint4*>(sm + q_at(i));
                        *u = make_uint4(u->x ^ 0x80008000u, u->y ^ 0x80008000u, u->z ^ 0x80008000u, u->w ^ 0x80008000u);
                    }
                fac[tid] = fabsf(a.scale_log2);
            } else {
#pragma unroll 4
                for (int i = 0; i < Q_STEPS; ++i) {
                    uint4* u = reinterpret_cast<uint4*>(sm + q_at(i));
                    float v[8];
                    unpack8<T>(*u, v);
                    float amax = 0.0f, back;
#pragma unroll
                    for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(v[e]));
#pragma unroll
                    for (int o = 1; o < LPR; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
                    float up = fit_exponent(amax, &back);
                    if (a.scale_log2 < 0.0f) up = -up;
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] *= up;
                    *u = pack8<__half>(v);
                    if (qc == 0) fac[q_row0 + i * RPI] = back * fabsf(a.scale_log2);
                }
            }
        };

        // The tile being written, its codes in registers; and the one after, its table entry on its way.
        open_item();
        Tile now = then;
        int entry = entry_of(now);
        int64_t place = place_of(now, entry);
        fetch(a.c.k.codes, place, kc);
        fetch(a.c.v.codes, place, vc);
        fetch_scales(now, entry);
        advance();
        entry = entry_of(then);
        uint32_t full_items = 0;
        for (; now.end > 0; next_slot()) {
            const bool opens = now.rows > 0;
            if (opens) {
                // the last scores of the item before have been taken
                if (full_items > 0 && !wait_phase(q_free, full_items - 1)) { failed = true; break; }
                begin_queries(now);
            }
            // whoever was in this slot has been used up
            if (walk > 0 && !wait_phase(kv_free(slot), walk - 1)) { failed = true; break; }
            put(S::K + slot * S::TILE, kc);
            if (scaler) {
                const float lv = __log2f(vs > 0.0f ? vs : ZERO_PAGE_SCALE);
                scales->ks[slot][tid >> 6] = ks;
                scales->lv[slot][tid >> 6] = vs < 0.0f ? -INFINITY : lv;
                scales->iv[slot][tid >> 6] = fast_exp2(-lv);
            }
            place = place_of(then, entry);
            fetch(a.c.k.codes, place, kc);
            fetch_scales(then, entry);
            put(S::V + slot * S::TILE, vc);
            fetch(a.c.v.codes, place, vc);
            if (opens) {
                finish_queries(row_fac + (full_items & 1) * ROWS);
                ++full_items;
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(kv_full(slot));
                if (opens) mbar_arrive(q_full);
            }
            now = then;
            if (now.end > 0) {
                advance();
                entry = entry_of(then);
            }
        }
    } else {
        const uint32_t issue = elect_one();
        const uint32_t idesc_s = (1u << 4) | (static_cast<uint32_t>(KEYS >> 3) << 17) | (128u >> 4 << 24);
        const uint32_t idesc_o = (1u << 4) | (1u << 16) | (static_cast<uint32_t>(D >> 3) << 17) | (128u >> 4 << 24);
        uint32_t full_items = 0;
        uint32_t n[2] = {0, 0};                 // tiles of either half so far, and up to which the scores have been issued
        uint32_t s_slot = 0, s_walk = 0;        // place of the tile whose scores are issued next
        // Scores of half g's tile c, from slot s_slot.
        auto scores = [&](int g, uint32_t c) {
            // two tiles earlier these columns held weights: they have been read
            if (c > 1 && !wait_phase(o_done(g, c), (c - 2) >> 1)) return false;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                tc_mma_f16(tmem + 128 * g + KEYS * (c & 1), smem_desc_sw128(base + S::Q + g * S::HALF_Q + (k >> 2) * Q_BLOCK) + 2u * (k & 3),
                           smem_desc_sw128(base + S::K + s_slot * S::TILE + (k >> 2) * KV_BLOCK) + 2u * (k & 3), idesc_s, k != 0 ? 1u : 0u, issue);
            tc_commit_if(s_full(g, c), issue);
            return true;
        };
        auto output = [&](int g, uint32_t c, bool first) {
            if (!wait_phase(p_full(g, c), c >> 1)) return false;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < KEYS / 16; ++k)
                tc_mma_f16_ts(tmem + O_COL + 128 * g, tmem + 128 * g + KEYS * (c & 1) + 8u * k, smem_desc_values(base + S::V + slot * S::TILE) + 128u * k,
                              idesc_o, first && k == 0 ? 0u : 1u, issue);
            tc_commit_if(o_done(g, c), issue);
            return true;
        };
        for (unsigned id = blockIdx.x; id < items && !failed; id += gridDim.x) {
            const Item x = item_of(a, id);
            if (x.steps == 0) continue;
            const int steps[2] = {half_steps(x, 0), half_steps(x, 1)};
            if (!wait_phase(q_full, full_items)) { failed = true; break; }
            ++full_items;
            // tile j of the item: its scores first, then the output of the tile before
            for (int j = 0; j <= x.steps && !failed; ++j) {
                if (j < x.steps && !wait_phase(kv_full(s_slot), s_walk)) { failed = true; break; }
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    if (j < steps[g] && !scores(g, n[g])) { failed = true; break; }
                    if (j > 0 && j <= steps[g] && !output(g, n[g] - 1, j == 1)) { failed = true; break; }
                    if (j < steps[g]) ++n[g];
                }
                if (failed) break;
                if (j + 1 == x.steps) tc_commit_if(q_free, issue);
                if (j > 0) {
                    tc_commit_if(kv_free(slot), issue);
                    next_slot();
                }
                if (j < x.steps && ++s_slot == RING) {
                    s_slot = 0;
                    ++s_walk;
                }
            }
        }
    }

    if (failed) {
        *abort_flag = 1;
        atomicOr(status, SQAP_ERR_TIMEOUT);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(TMEM_COLS) : "memory");
}

template <typename T, int TYPE, int D>
sqap_status launch_as(const AttnArgs& a, unsigned items, int* status, cudaStream_t s) {
    static PerDevice<int> setup;
    const sqap_status st = setup.run([](int*) {
        // the softmax's registers come out of those that the kernel is launched with: with fewer, it would wait for them for ever
        cudaFuncAttributes f;
        const cudaError_t e = cudaFuncGetAttributes(&f, kv_prefill_tc_kernel<T, TYPE, D>);
        if (e != cudaSuccess) {
            note_cuda_error(e);
            cudaGetLastError();
            return SQAP_ERR_CUDA;
        }
        if (f.numRegs < LAUNCH_REGS) return SQAP_ERR_UNSUPPORTED;
        return set_max_dynamic_smem(kv_prefill_tc_kernel<T, TYPE, D>, Smem<D>::BYTES);
    });
    if (st != SQAP_OK) return st;
    const unsigned slots = static_cast<unsigned>(sm_count());
    return finish_launch(launch_dependent(kv_prefill_tc_kernel<T, TYPE, D>, dim3(items < slots ? items : slots), dim3(THREADS),
                                          Smem<D>::BYTES, s, a, items, status));
}
template <typename T>
sqap_status launch_type(const AttnArgs& a, int type, unsigned items, int* status, cudaStream_t s) {
    if (a.c.head_dim == 64)
        return type == SQAP_KV_INT8 ? launch_as<T, SQAP_KV_INT8, 64>(a, items, status, s) : launch_as<T, SQAP_KV_E4M3, 64>(a, items, status, s);
    return type == SQAP_KV_INT8 ? launch_as<T, SQAP_KV_INT8, 128>(a, items, status, s) : launch_as<T, SQAP_KV_E4M3, 128>(a, items, status, s);
}

}  // namespace

sqap_status launch_kv_prefill_tc(const AttnArgs& a, int type, int dtype, cudaStream_t s) {
    int* status = device_status_word();
    if (!status) return SQAP_ERR_CUDA;
    if (!device_is_sm100()) return SQAP_ERR_UNSUPPORTED;
    const unsigned items = static_cast<unsigned>(static_cast<int64_t>(a.batch) * a.c.kv_heads * a.splits * a.tiles);
    return dtype == SQAP_FP16 ? launch_type<__half>(a, type, items, status, s) : launch_type<__nv_bfloat16>(a, type, items, status, s);
}

}  // namespace kv
}  // namespace sqap
