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

template <typename T, int TYPE, int D>
__global__ void __launch_bounds__(THREADS, 2) kv_prefill_tc_kernel(AttnArgs a, int* status) {
    using S = Smem<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* sm = smem_raw + (base - smem_u32(smem_raw));
    Scales* scales = reinterpret_cast<Scales*>(sm + S::TAIL);
    static_assert(sizeof(Scales) <= 256, "tail layout");
    const uint32_t bar0 = base + S::TAIL + 256;
    const uint32_t k_full = bar0, s_full = bar0 + 8, p_full = bar0 + 16, v_full = bar0 + 24, o_done = bar0 + 32;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(sm + S::TAIL + 256 + 48);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + S::TAIL + 256 + 56);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        mbar_init(k_full, 4);
        mbar_init(s_full, 5);       // the MMAs, and the four warps that wrote the tile's scales
        mbar_init(p_full, 4);
        mbar_init(v_full, 4);
        mbar_init(o_done, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(const_cast<uint32_t*>(tmem_slot))), "n"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_launch_dependents();
    pdl_wait();

    Where w = locate(a, blockIdx.x);
    w.tile = a.tiles - 1 - w.tile;                       // the rows that see the most first
    const int G = a.group;
    const int nq = w.n_q < a.max_q ? w.n_q : a.max_q;
    const int rows = nq * G;
    const int r_first = w.tile * PREFILL_ROWS;
    const bool any = r_first < rows;
    const int key0 = w.split * a.chunk;
    const int key1 = a.splits > 1 ? min(key0 + a.chunk, w.len) : w.len;
    const int last_row = min(rows, r_first + PREFILL_ROWS) - 1;
    const int end = any && a.c.pages > 0 ? min(key1, visible(a, w, last_row / G)) : 0;
    const int steps = end > key0 ? (end - key0 + KEYS - 1) / KEYS : 0;

    // the softmax's thread for row r: query, its factor, the keys that it may see
    const int r = r_first + static_cast<int>(threadIdx.x);
    const bool real = warp < 4 && r < rows;
    const int qi = real ? r / G : 0, head = w.h * G + (real ? r % G : 0);
    float fac = 0.0f;
    int lim = 0;
    if (warp < 4 && steps > 0) {
        const T* src = static_cast<const T*>(a.q) + (static_cast<int64_t>(w.row0) + qi) * a.ldq + static_cast<int64_t>(head) * D;
        float amax = 0.0f;
        if (real)
#pragma unroll 4
            for (int c = 0; c < D / 8; ++c) {
                float v[8];
                unpack8<T>(__ldg(reinterpret_cast<const uint4*>(src) + c), v);
#pragma unroll
                for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(v[e]));
            }
        float back;
        float up = fit_exponent(amax, &back);
        if (a.scale_log2 < 0.0f) up = -up;               // so that the factor of a score is never negative
        fac = back * fabsf(a.scale_log2);
#pragma unroll 4
        for (int c = 0; c < D / 8; ++c) {
            float v[8] = {};
            if (real) {
                unpack8<T>(__ldg(reinterpret_cast<const uint4*>(src) + c), v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= up;
            }
            const int row = threadIdx.x;
            *reinterpret_cast<uint4*>(sm + S::Q + (c >> 3) * BLOCK_BYTES + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = pack8<__half>(v);
        }
        lim = real ? min(visible(a, w, qi), end) : 0;
        fence_proxy_async();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    bool failed = false;

    if (warp < 4) {
        const uint32_t t_s = tmem + (static_cast<uint32_t>(warp * 32) << 16), t_o = t_s + O_COL;
        float m = -INFINITY, l = 0.0f;
        for (int j = 0; j < steps; ++j) {
            if (!__all_sync(0xffffffffu, mbar_wait(s_full, j & 1, abort_flag))) { failed = true; break; }
            tc_fence_after();
            const float* ks = scales->ks[j & 1];
            const float* lv = scales->lv[j & 1];
            const float* iv = scales->iv[j & 1];
            const int seen = lim - (key0 + j * KEYS);    // this row sees the first `seen` keys of the tile
            const bool whole = __all_sync(0xffffffffu, seen >= KEYS);
            float top = -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t v[32];
                tc_ld32(t_s + 32 * c, v);
                tc_wait_ld();
                if (!whole) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (32 * c + i >= seen) v[i] = 0xFF800000u;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float x = __uint_as_float(v[16 * h]);
#pragma unroll
                    for (int i = 1; i < 16; ++i) x = fmaxf(x, __uint_as_float(v[16 * h + i]));
                    // a missing page has lv = -inf (and scores of zero); -inf stays -inf unless the factor is zero
                    const float f = fac * ks[2 * c + h];
                    x = x == -INFINITY ? x : fmaf(x, f, lv[2 * c + h]);
                    top = fmaxf(top, x);
                }
            }
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
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t v[32], p[16];
                tc_ld32(t_s + 32 * c, v);
                tc_wait_ld();
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float f = fac * ks[2 * c + h], z = lv[2 * c + h] - ref;
                    const uint64_t f2 = pair_of(f, f), z2 = pair_of(z, z);
                    float sum0 = 0.0f, sum1 = 0.0f;
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        float x0, x1;
                        unpair(fma_pair(pair_of(__uint_as_float(v[16 * h + i]), __uint_as_float(v[16 * h + i + 1])), f2, z2), &x0, &x1);
                        x0 = fast_exp2(x0);
                        x1 = fast_exp2(x1);
                        if (!whole) {
                            if (32 * c + 16 * h + i >= seen) x0 = 0.0f;
                            if (32 * c + 16 * h + i + 1 >= seen) x1 = 0.0f;
                        }
                        sum0 += x0;
                        sum1 += x1;
                        p[8 * h + i / 2] = half2_of(x0, x1);
                    }
                    l = fmaf(sum0 + sum1, iv[2 * c + h], l);
                }
                tc_st16(t_s + 16 * c, p);                // columns already read
            }
            tc_wait_st_f();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full);
        }
        if (steps > 0 && !failed) {
            if (!__all_sync(0xffffffffu, mbar_wait(o_done, (steps - 1) & 1, abort_flag))) failed = true;
            tc_fence_after();
        }
        if (any && !failed) {
            const float inv = l > 0.0f ? 1.0f / l : 0.0f;
            const int64_t row = static_cast<int64_t>(w.row0) + qi;
            const int64_t at = a.splits > 1 && real ? part_index(a, w.b, head, qi, w.split) : 0;
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                uint32_t v[32];
                if (steps > 0) {
                    tc_ld32(t_o + 32 * c, v);
                    tc_wait_ld();
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = 0;
                }
                if (!real) continue;
                const float* y = reinterpret_cast<const float*>(v);
                if (a.splits > 1) {
                    float4* po = reinterpret_cast<float4*>(a.part_o + at * D + 32 * c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) po[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
                } else {
                    uint4* out = reinterpret_cast<uint4*>(static_cast<T*>(a.out) + row * a.ldo + static_cast<int64_t>(head) * D + 32 * c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float z[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[e] = y[8 * i + e] * inv;
                        out[i] = pack8<T>(z);
                    }
                }
            }
            if (real) {
                if (a.splits > 1) a.part_ml[at] = make_float2(m, l);
                else if (a.lse) a.lse[row * a.heads + head] = l > 0.0f ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
            }
        }
    } else if (warp < 8) {
        const int tid = threadIdx.x - 128;
        const int32_t* table = a.table + w.b * a.ldt;
        const int shift = a.c.page_shift, mask = (1 << shift) - 1;
        auto page_at = [&](int key) {
            const int j = key >> shift;
            return key < end && j < a.ldt ? checked_page(a.c, __ldg(table + j)) : -1;
        };
        constexpr int CHUNKS = KEYS * D / 16 / 128;      // 16-byte pieces of codes per thread and tile
        // piece x: 16 elements x % 4 of block x / 512, key x / 4 % 128: eight lanes then write eight different 16-byte units
        uint4 held[CHUNKS];     // keys and values in turn: either is fetched while the other's place is still in use
        auto fetch = [&](const Half& half, int k0) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const int x = tid + 128 * i, key = k0 + ((x >> 2) & 127), col = (x >> 9) * 64 + (x & 3) * 16;
                const int page = page_at(key);
                held[i] = make_uint4(0, 0, 0, 0);        // behind the end: zero codes, whatever lies there
                if (page >= 0) held[i] = __ldg(reinterpret_cast<const uint4*>(half.codes + (page_codes(a.c, page, w.h) + (key & mask)) * D + col));
            }
        };
        auto put = [&](int region) {
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const int x = tid + 128 * i, row = (x >> 2) & 127, unit = (x & 3) * 2;
                uint8_t* to = sm + region + (x >> 9) * BLOCK_BYTES + row * 128;
                const uint32_t in[4] = {held[i].x, held[i].y, held[i].z, held[i].w};
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
                *reinterpret_cast<uint4*>(to + ((unit ^ (row & 7)) << 4)) = make_uint4(out[0], out[1], out[2], out[3]);
                *reinterpret_cast<uint4*>(to + (((unit + 1) ^ (row & 7)) << 4)) = make_uint4(out[4], out[5], out[6], out[7]);
            }
        };
        if (steps > 0) fetch(a.c.k, key0);
        for (int j = 0; j < steps; ++j) {
            const int k0 = key0 + j * KEYS;
            // keys: the scores of the tile before have been taken
            if (j > 0 && !__all_sync(0xffffffffu, mbar_wait(s_full, (j - 1) & 1, abort_flag))) { failed = true; break; }
            put(S::K);
            if (tid < GROUPS) {
                const int page = page_at(k0 + 16 * tid);
                float ks = 0.0f, vs = 0.0f;
                if (page >= 0) {
                    const int64_t s = static_cast<int64_t>(page) * a.c.kv_heads + w.h;
                    ks = __ldg(a.c.k.scales + s);
                    vs = __ldg(a.c.v.scales + s);
                }
                const float lv = __log2f(vs > 0.0f ? vs : ZERO_PAGE_SCALE);
                scales->ks[j & 1][tid] = ks;
                scales->lv[j & 1][tid] = page >= 0 ? lv : -INFINITY;
                scales->iv[j & 1][tid] = fast_exp2(-lv);
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(s_full);
                mbar_arrive(k_full);
            }
            fetch(a.c.v, k0);
            // values: the output of the tile before has taken them
            if (j > 0 && !__all_sync(0xffffffffu, mbar_wait(o_done, (j - 1) & 1, abort_flag))) { failed = true; break; }
            put(S::V);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(v_full);
            if (j + 1 < steps) fetch(a.c.k, k0 + KEYS);
        }
    } else {
        const uint32_t issue = elect_one();
        const uint32_t idesc_s = (1u << 4) | (static_cast<uint32_t>(KEYS >> 3) << 17) | (128u >> 4 << 24);
        const uint32_t idesc_o = (1u << 4) | (1u << 16) | (static_cast<uint32_t>(D >> 3) << 17) | (128u >> 4 << 24);
        for (int j = 0; j < steps; ++j) {
            bool ok = mbar_wait(k_full, j & 1, abort_flag);
            if (ok && j > 0) ok = mbar_wait(o_done, (j - 1) & 1, abort_flag);     // the weights in the score columns have been read
            if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                tc_mma_f16(tmem, smem_desc_sw128(base + S::Q + (k >> 2) * BLOCK_BYTES) + 2u * (k & 3),
                           smem_desc_sw128(base + S::K + (k >> 2) * BLOCK_BYTES) + 2u * (k & 3), idesc_s, k != 0 ? 1u : 0u, issue);
            tc_commit_if(s_full, issue);
            ok = mbar_wait(v_full, j & 1, abort_flag) && mbar_wait(p_full, j & 1, abort_flag);
            if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < KEYS / 16; ++k)
                tc_mma_f16_ts(tmem + O_COL, tmem + 8u * k, smem_desc_values(base + S::V) + 128u * k, idesc_o, (j | k) != 0 ? 1u : 0u, issue);
            tc_commit_if(o_done, issue);
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
sqap_status launch_as(const AttnArgs& a, unsigned grid, int* status, cudaStream_t s) {
    static PerDevice<int> setup;
    const sqap_status st = setup.run([](int*) { return set_max_dynamic_smem(kv_prefill_tc_kernel<T, TYPE, D>, Smem<D>::BYTES); });
    if (st != SQAP_OK) return st;
    return finish_launch(launch_dependent(kv_prefill_tc_kernel<T, TYPE, D>, dim3(grid), dim3(THREADS), Smem<D>::BYTES, s, a, status));
}
template <typename T>
sqap_status launch_type(const AttnArgs& a, int type, unsigned grid, int* status, cudaStream_t s) {
    if (a.c.head_dim == 64)
        return type == SQAP_KV_INT8 ? launch_as<T, SQAP_KV_INT8, 64>(a, grid, status, s) : launch_as<T, SQAP_KV_E4M3, 64>(a, grid, status, s);
    return type == SQAP_KV_INT8 ? launch_as<T, SQAP_KV_INT8, 128>(a, grid, status, s) : launch_as<T, SQAP_KV_E4M3, 128>(a, grid, status, s);
}

}  // namespace

sqap_status launch_kv_prefill_tc(const AttnArgs& a, int type, int dtype, cudaStream_t s) {
    int* status = device_status_word();
    if (!status) return SQAP_ERR_CUDA;
    if (!device_is_sm100()) return SQAP_ERR_UNSUPPORTED;
    const unsigned grid = static_cast<unsigned>(static_cast<int64_t>(a.batch) * a.c.kv_heads * a.splits * a.tiles);
    return dtype == SQAP_FP16 ? launch_type<__half>(a, type, grid, status, s) : launch_type<__nv_bfloat16>(a, type, grid, status, s);
}

}  // namespace kv
}  // namespace sqap
