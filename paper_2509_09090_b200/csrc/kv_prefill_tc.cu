// Attention of many query rows (prompts) over the paged 8-bit cache on tcgen05, head_dim 64 and 128.
//
// One CTA takes 128 rows (query x head of the group, packed: the heads that share a key/value head share its tiles) of
// one sequence and key/value head and walks the keys 128 at a time. Per tile: S = Q K^T into tensor memory, the softmax's
// weights back into tensor memory as the A operand, O += W V.
//   warps 0-3  softmax: thread = row. Also load the queries at the start and store the output at the end.
//   warps 4-7  codes from global memory (one tile ahead, in registers) to fp16 in shared memory, 128B-swizzled
//   warp  8    issues the MMAs
// Work per tile and what it costs an SM: MMAs 2 x 128 x 128 x D (1024 cycles at D = 128), 16384 exponentials (1024 cycles),
// some 3 instructions per weight and 1.3 per code besides. None of it is far ahead of the others, so they have to
// overlap: a CTA runs score - softmax - output in turn in 256 columns of tensor memory and half an SM's shared memory, and
// two CTAs on an SM fill each other's gaps. Shared memory is single-buffered: the keys of the next tile are written during
// the softmax of this one, its values during the next scores.
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

constexpr int KEYS = 128;                   // keys per tile
constexpr int GROUPS = KEYS / 16;           // runs of 16 keys: a page never ends inside one
constexpr int THREADS = 288;
constexpr int BLOCK_BYTES = 128 * 128;      // 128 rows of 64 halves
constexpr int TMEM_COLS = 256;              // scores (and weights) 0 .. 127, output from 128
constexpr int O_COL = 128;
constexpr float RAISE = 8.0f;

template <int D>
struct Smem {
    static constexpr int BLOCKS = D / 64;
    static constexpr int Q = 0, K = BLOCKS * BLOCK_BYTES, V = 2 * K, TAIL = 3 * K;
    static constexpr int BYTES = TAIL + 512 + 1024;      // scales, barriers, flags; slack for the alignment
};
// scales of the two tiles in flight, by run of 16 keys
struct Scales {
    float ks[2][GROUPS], lv[2][GROUPS], iv[2][GROUPS];
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
__device__ __forceinline__ void tc_st32_f(uint32_t taddr, const uint32_t* r) {
    tc_st16(taddr, r);
    tc_st16(taddr + 16, r + 16);
}
__device__ __forceinline__ void tc_wait_st_f() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Values [key][element], elements contiguous (the operand's N dimension): 128B-swizzled blocks of 64 elements; 8 keys are 1024
// bytes apart, blocks BLOCK_BYTES.
__device__ __forceinline__ uint64_t smem_desc_values(uint32_t addr) {
    return static_cast<uint64_t>((addr >> 4) & 0x3FFFu) | (static_cast<uint64_t>(BLOCK_BYTES >> 4) << 16) | (64ull << 32) | (1ull << 46) |
           (2ull << 61);
}

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

// One item: 128 rows of a sequence and key/value head (and one piece of its history, where those are cut).
struct Item {
    Where w;
    int rows, r_first, key0, end, steps;
};
__device__ __forceinline__ Item item_of(const AttnArgs& a, unsigned id) {
    Item x;
    // tiles outermost, the rows that see the most first
    const unsigned per_tile = static_cast<unsigned>(a.batch) * a.c.kv_heads * a.splits;
    const unsigned tile = id / per_tile;
    x.w = locate(a, (id - tile * per_tile) * a.tiles);
    x.w.tile = a.tiles - 1 - static_cast<int>(tile);
    x.rows = (x.w.n_q < a.max_q ? x.w.n_q : a.max_q) * a.group;
    x.r_first = x.w.tile * PREFILL_ROWS;
    x.key0 = x.w.split * a.chunk;
    x.end = 0;
    if (x.r_first < x.rows && a.c.pages > 0) {
        const int last = min(x.rows, x.r_first + PREFILL_ROWS) - 1;
        const int key1 = a.splits > 1 ? min(x.key0 + a.chunk, x.w.len) : x.w.len;
        x.end = min(key1, visible(a, x.w, last / a.group));
    }
    x.steps = x.end > x.key0 ? (x.end - x.key0 + KEYS - 1) / KEYS : 0;
    return x;
}

template <typename T, int TYPE, int D>
__global__ void __launch_bounds__(THREADS, 2) kv_prefill_tc_kernel(AttnArgs a, unsigned items, int* status) {
    using S = Smem<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* sm = smem_raw + (base - smem_u32(smem_raw));
    Scales* scales = reinterpret_cast<Scales*>(sm + S::TAIL);
    static_assert(sizeof(Scales) <= 256, "tail layout");
    const uint32_t bar0 = base + S::TAIL + 256;
    const uint32_t k_full = bar0, s_full = bar0 + 8, p_full = bar0 + 16, v_full = bar0 + 24, o_done = bar0 + 32, q_full = bar0 + 40;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(sm + S::TAIL + 256 + 56);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + S::TAIL + 256 + 64);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        mbar_init(k_full, 4);
        mbar_init(s_full, 5);       // the MMAs, and the four warps that wrote the tile's scales
        mbar_init(p_full, 4);
        mbar_init(v_full, 4);
        mbar_init(o_done, 1);
        mbar_init(q_full, 4);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) {
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
    uint32_t n = 0;                 // tiles so far, over all items: the barriers' phases

    if (warp < 4) {
        const uint32_t t_s = tmem + (static_cast<uint32_t>(warp * 32) << 16), t_o = t_s + O_COL;
        const float sign = a.scale_log2 < 0.0f ? -1.0f : 1.0f;     // goes into the queries: no factor of a score is negative
        // The warp's 32 rows of queries, scaled row by row to fit fp16, to shared memory; returns the factor of this lane's row.
        auto load_queries = [&](const Item& x) {
            constexpr int LPR = D / 8, RPI = 32 / LPR;             // lanes per row, rows per step
            uint4 u[LPR];
#pragma unroll
            for (int i = 0; i < LPR; ++i) {
                const int r = x.r_first + warp * 32 + i * RPI + lane / LPR;
                u[i] = make_uint4(0, 0, 0, 0);
                if (r < x.rows)
                    u[i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + (static_cast<int64_t>(x.w.row0) + r / G) * a.ldq +
                                                                static_cast<int64_t>(x.w.h * G + r % G) * D) + lane % LPR);
            }
            float mine = 0.0f;
#pragma unroll
            for (int i = 0; i < LPR; ++i) {
                float v[8];
                unpack8<T>(u[i], v);
                float amax = 0.0f, back;
#pragma unroll
                for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(v[e]));
#pragma unroll
                for (int o = 1; o < LPR; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
                const float up = fit_exponent(amax, &back) * sign;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= up;
                const int row = warp * 32 + i * RPI + lane / LPR, c = lane % LPR;
                *reinterpret_cast<uint4*>(sm + S::Q + (c >> 3) * BLOCK_BYTES + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = pack8<__half>(v);
                back = __shfl_sync(0xffffffffu, back, (lane % RPI) * LPR);
                if (lane / RPI == i) mine = back;
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full);
            return mine * fabsf(a.scale_log2);
        };
        // Maximum of the tile's exponents for this row: first the scores of a run of 16, then one scaling (the factors are >= 0).
        auto tile_max = [&](auto masked, float fac, int seen, const float* ks, const float* lv) {
            constexpr bool MASKED = decltype(masked)::value;
            float top = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t v[32];
                tc_ld32(t_s + 32 * c, v);
                tc_wait_ld();
                if (MASKED) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (32 * c + i >= seen) v[i] = 0xFF800000u;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float x = __uint_as_float(v[16 * h]);
#pragma unroll
                    for (int i = 1; i < 15; i += 2) x = fmaxf(fmaxf(x, __uint_as_float(v[16 * h + i])), __uint_as_float(v[16 * h + i + 1]));
                    x = fmaxf(x, __uint_as_float(v[16 * h + 15]));
                    // a missing page has lv = -inf (and scores of zero); a masked run stays -inf whatever the factor
                    const float y = fmaf(x, fac * ks[2 * c + h], lv[2 * c + h]);
                    top = fmaxf(top, MASKED && x == -INFINITY ? x : y);
                }
            }
            return top;
        };
        // The weights of the tile, into the columns that its scores leave; returns the growth of the denominator.
        auto tile_weights = [&](auto masked, float fac, float ref, int seen, const float* ks, const float* lv, const float* iv) {
            constexpr bool MASKED = decltype(masked)::value;
            float grow = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t v[32], p[16];
                tc_ld32(t_s + 32 * c, v);
                tc_wait_ld();
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float f = fac * ks[2 * c + h], z = lv[2 * c + h] - ref;
                    const uint64_t f2 = pair_of(f, f), z2 = pair_of(z, z);
                    uint64_t sum = 0;
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        float x0, x1;
                        unpair(fma_pair(pair_of(__uint_as_float(v[16 * h + i]), __uint_as_float(v[16 * h + i + 1])), f2, z2), &x0, &x1);
                        x0 = fast_exp2(x0);
                        x1 = fast_exp2(x1);
                        if (MASKED) {
                            if (32 * c + 16 * h + i >= seen) x0 = 0.0f;
                            if (32 * c + 16 * h + i + 1 >= seen) x1 = 0.0f;
                        }
                        sum = add_pair(sum, pair_of(x0, x1));
                        p[8 * h + i / 2] = half2_of(x0, x1);
                    }
                    float s0, s1;
                    unpair(sum, &s0, &s1);
                    grow = fmaf(s0 + s1, iv[2 * c + h], grow);
                }
                tc_st16(t_s + 16 * c, p);                // columns already read
            }
            return grow;
        };

        unsigned id = blockIdx.x;
        Item x = item_of(a, id);
        float fac = x.steps > 0 ? load_queries(x) : 0.0f;
        for (;;) {
            const int r = x.r_first + static_cast<int>(threadIdx.x);
            const bool real = r < x.rows;
            const int qi = real ? r / G : 0, head = x.w.h * G + (real ? r % G : 0);
            const int lim = real ? min(visible(a, x.w, qi), x.end) : 0;
            float m = -INFINITY, l = 0.0f;
            for (int j = 0; j < x.steps; ++j, ++n) {
                if (!__all_sync(0xffffffffu, mbar_wait(s_full, n & 1, abort_flag))) { failed = true; break; }
                tc_fence_after();
                const float* ks = scales->ks[n & 1];
                const float* lv = scales->lv[n & 1];
                const float* iv = scales->iv[n & 1];
                const int seen = lim - (x.key0 + j * KEYS);    // this row sees the first `seen` keys of the tile
                const bool whole = __all_sync(0xffffffffu, seen >= KEYS);
                const float top = whole ? tile_max(std::false_type(), fac, seen, ks, lv) : tile_max(std::true_type(), fac, seen, ks, lv);
                const bool raise = m == -INFINITY ? top != -INFINITY : top > m + RAISE;
                if (__any_sync(0xffffffffu, raise)) {
                    const float f = raise ? fast_exp2(m - top) : 1.0f;      // m = -inf: 0
                    if (raise) m = top;
                    l *= f;
                    if (j > 0) {
#pragma unroll 1
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t v[32];
                            tc_ld32(t_o + 32 * c, v);
                            tc_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
                            tc_st32_f(t_o + 32 * c, v);
                        }
                    }
                }
                const float ref = m == -INFINITY ? 0.0f : m;
                l += whole ? tile_weights(std::false_type(), fac, ref, seen, ks, lv, iv) : tile_weights(std::true_type(), fac, ref, seen, ks, lv, iv);
                tc_wait_st_f();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full);
            }
            if (failed) break;
            // the next item's queries while the last output product runs (the last scores have been taken: s_full)
            const Item y = x;
            id += gridDim.x;
            const bool more = id < items;
            if (more) {
                x = item_of(a, id);
                if (x.steps > 0) fac = load_queries(x);
            }
            if (y.steps > 0) {
                if (!__all_sync(0xffffffffu, mbar_wait(o_done, (n - 1) & 1, abort_flag))) { failed = true; break; }
                tc_fence_after();
            }
            const float inv = l > 0.0f ? 1.0f / l : 0.0f;
            const int64_t row = static_cast<int64_t>(y.w.row0) + qi;
            const int64_t at = a.splits > 1 && real ? part_index(a, y.w.b, head, qi, y.w.split) : 0;
#pragma unroll 1
            for (int c = 0; c < (y.r_first < y.rows ? D / 32 : 0); ++c) {
                uint32_t v[32];
                if (y.steps > 0) {
                    tc_ld32(t_o + 32 * c, v);
                    tc_wait_ld();
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = 0;
                }
                if (!real) continue;
                if (a.splits > 1) {
                    uint4* po = reinterpret_cast<uint4*>(a.part_o + at * D + 32 * c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) po[i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                } else {
                    uint4* out = reinterpret_cast<uint4*>(static_cast<T*>(a.out) + row * a.ldo + static_cast<int64_t>(head) * D + 32 * c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float z[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[e] = __uint_as_float(v[8 * i + e]) * inv;
                        out[i] = pack8<T>(z);
                    }
                }
            }
            if (real) {
                if (a.splits > 1) a.part_ml[at] = make_float2(m, l);
                else if (a.lse) a.lse[row * a.heads + head] = l > 0.0f ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
            }
            if (!more) break;
        }
    } else if (warp < 8) {
        const int tid = threadIdx.x - 128;
        const int shift = a.c.page_shift, mask = (1 << shift) - 1;
        // A thread's pieces of a tile: 16 codes of keys tid / 4 + 32 i, elements 64 b + 16 (tid % 4) on. Eight lanes then
        // write eight different 16-byte units, and a thread's place in the swizzle never changes.
        constexpr int BLOCKS = S::BLOCKS;
        uint4 held[4][BLOCKS];      // keys and values in turn: either is fetched while the other's place is still in use
        const int32_t* table = nullptr;
        int h = 0, end = 0;
        auto page_at = [&](int key) {
            const int j = key >> shift;
            return key < end && j < a.ldt ? checked_page(a.c, __ldg(table + j)) : -1;
        };
        auto fetch = [&](const Half& half, int k0) {
            int page[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) page[i] = page_at(k0 + (tid >> 2) + 32 * i);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint8_t* p = half.codes + (page_codes(a.c, page[i], h) + ((k0 + (tid >> 2) + 32 * i) & mask)) * D + (tid & 3) * 16;
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    held[i][b] = make_uint4(0, 0, 0, 0);       // behind the end: zero codes, whatever lies there
                    if (page[i] >= 0) held[i][b] = __ldg(reinterpret_cast<const uint4*>(p + 64 * b));
                }
            }
        };
        const int row = tid >> 2, unit = (tid & 3) * 2;
        uint8_t* const to0 = sm + row * 128 + ((unit ^ (row & 7)) << 4);
        uint8_t* const to1 = sm + row * 128 + (((unit + 1) ^ (row & 7)) << 4);
        auto put = [&](int region) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    const uint32_t in[4] = {held[i][b].x, held[i][b].y, held[i][b].z, held[i][b].w};
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
                    *reinterpret_cast<uint4*>(to0 + region + b * BLOCK_BYTES + i * 32 * 128) = make_uint4(out[0], out[1], out[2], out[3]);
                    *reinterpret_cast<uint4*>(to1 + region + b * BLOCK_BYTES + i * 32 * 128) = make_uint4(out[4], out[5], out[6], out[7]);
                }
        };
        for (unsigned id = blockIdx.x; id < items && !failed; id += gridDim.x) {
            const Item x = item_of(a, id);
            table = a.table + x.w.b * a.ldt;
            h = x.w.h;
            end = x.end;
            if (x.steps > 0) fetch(a.c.k, x.key0);
            for (int j = 0; j < x.steps; ++j, ++n) {
                const int k0 = x.key0 + j * KEYS;
                float ks = 0.0f, vs = 0.0f;
                int page = -1;
                if (tid < GROUPS) {
                    page = page_at(k0 + 16 * tid);
                    if (page >= 0) {
                        const int64_t s = static_cast<int64_t>(page) * a.c.kv_heads + h;
                        ks = __ldg(a.c.k.scales + s);
                        vs = __ldg(a.c.v.scales + s);
                    }
                }
                // keys: the scores of the tile before have been taken
                if (n > 0 && !__all_sync(0xffffffffu, mbar_wait(s_full, (n - 1) & 1, abort_flag))) { failed = true; break; }
                put(S::K);
                if (tid < GROUPS) {
                    const float lv = __log2f(vs > 0.0f ? vs : ZERO_PAGE_SCALE);
                    scales->ks[n & 1][tid] = ks;
                    scales->lv[n & 1][tid] = page >= 0 ? lv : -INFINITY;
                    scales->iv[n & 1][tid] = fast_exp2(-lv);
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(s_full);
                    mbar_arrive(k_full);
                }
                fetch(a.c.v, k0);
                // values: the output of the tile before has taken them
                if (n > 0 && !__all_sync(0xffffffffu, mbar_wait(o_done, (n - 1) & 1, abort_flag))) { failed = true; break; }
                put(S::V);
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(v_full);
                if (j + 1 < x.steps) fetch(a.c.k, k0 + KEYS);
            }
        }
    } else {
        const uint32_t issue = elect_one();
        const uint32_t idesc_s = (1u << 4) | (static_cast<uint32_t>(KEYS >> 3) << 17) | (128u >> 4 << 24);
        const uint32_t idesc_o = (1u << 4) | (1u << 16) | (static_cast<uint32_t>(D >> 3) << 17) | (128u >> 4 << 24);
        uint32_t full_items = 0;
        for (unsigned id = blockIdx.x; id < items && !failed; id += gridDim.x) {
            const Item x = item_of(a, id);
            if (x.steps == 0) continue;
            if (!__all_sync(0xffffffffu, mbar_wait(q_full, full_items & 1, abort_flag))) { failed = true; break; }
            ++full_items;
            for (int j = 0; j < x.steps; ++j, ++n) {
                bool ok = mbar_wait(k_full, n & 1, abort_flag);
                if (ok && n > 0) ok = mbar_wait(o_done, (n - 1) & 1, abort_flag);     // the weights in the score columns have been read
                if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    tc_mma_f16(tmem, smem_desc_sw128(base + S::Q + (k >> 2) * BLOCK_BYTES) + 2u * (k & 3),
                               smem_desc_sw128(base + S::K + (k >> 2) * BLOCK_BYTES) + 2u * (k & 3), idesc_s, k != 0 ? 1u : 0u, issue);
                tc_commit_if(s_full, issue);
                ok = mbar_wait(v_full, n & 1, abort_flag) && mbar_wait(p_full, n & 1, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < KEYS / 16; ++k)
                    tc_mma_f16_ts(tmem + O_COL, tmem + 8u * k, smem_desc_values(base + S::V) + 128u * k, idesc_o, (j | k) != 0 ? 1u : 0u, issue);
                tc_commit_if(o_done, issue);
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
    if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(TMEM_COLS) : "memory");
}

template <typename T, int TYPE, int D>
sqap_status launch_as(const AttnArgs& a, unsigned items, int* status, cudaStream_t s) {
    static PerDevice<int> setup;
    const sqap_status st = setup.run([](int*) { return set_max_dynamic_smem(kv_prefill_tc_kernel<T, TYPE, D>, Smem<D>::BYTES); });
    if (st != SQAP_OK) return st;
    const unsigned slots = 2u * static_cast<unsigned>(sm_count());
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
