// Product of two microscaled 4-bit matrices on the block-scaled tensor cores:
//   out[m][n] = round( (sum_k x[m][k] w[n][k]) * gx * gw ),   x, w = e2m1 code * block scale
// tcgen05.mma kind::mxf4nvf4 / mxf4 with .block_scale: the tensor core multiplies the 4-bit codes, applies both block
// scales and accumulates in fp32; nothing is unpacked on the way. Weights are the MMA-M operand (128 rows of a tile),
// tokens the MMA-N operand (BN columns), so that a handful of tokens costs a narrow tile and not a mostly empty one.
//
// This kernel is for few tokens, few weight rows and long K (use_clusters()); many tokens or rows: mx4_pair.cu. What bounds it: the
// weight stream (0.5625 or 0.53 bytes per weight, 3.7 us of HBM for 4096 x 11008), and around it the set-up (some 2400 cycles)
// and the exchange of partial sums (3000 to 4000 at 160 tokens). 160 x 4096 x 11008 in MXFP4 with the quantizer: 16.1 us, the
// product alone 13.4.
//
// A stage of the shared-memory ring holds 256 elements of K: 128 bytes per row of either operand (one 128B-swizzled
// TMA box each) and the scale tiles that belong to them, copied as they lie in memory (512 bytes per 128 rows and
// four blocks). Per stage the issuing warp copies the scale tiles to tensor memory (tcgen05.cp 32x128b.warpx4: 32 rows
// of 16 bytes, repeated for the four lane quadrants; column c of a tile then holds the scales of rows 32c .. 32c+31)
// and issues one MMA per 64 elements. Copies and MMAs of one thread execute in issue order; two sets of scale columns
// take turns all the same, so a copy never has to follow the MMAs that read what it overwrites.
//
// One cluster of `ksplit` CTAs per tile, each with its slice of the K stages. The partial sums meet in shared memory
// (distributed stores), are added in rank order (the result does not depend on timing), scaled, rounded once and
// stored 16 bytes per thread. Every wait on a barrier is bounded; on expiry the kernel records SQAP_ERR_TIMEOUT in the
// device status word and runs on to the cluster barriers, which every thread of every CTA reaches on every path.
#include "mx4.cuh"
#include "tc_common.cuh"

namespace sqap {
namespace mx4 {

using namespace tc;

constexpr int BM = 128;                   // weight rows per tile
constexpr int BK = 256;                   // elements of K per stage
constexpr int BN_MAX = 256;
constexpr int S_MAX = 10;
constexpr int KSPLIT_MAX = 8;
constexpr int A_BYTES = BM * BK / 2;      // 16 KB
constexpr int SF_TILE = 512;              // scales of 128 rows x 4 blocks
constexpr int THREADS = 256;              // warp 0: TMA, warp 1: MMA, all: exchange and epilogue, in two groups of four
constexpr int CHUNK_BYTES = BM * 16 * 4;  // 16 tokens of a partial sum: four planes [128 rows][4 tokens] fp32
constexpr int STAGE_BYTES = BM * 16 * 2;  // a chunk of 16-bit outputs on its way out
constexpr int TAIL_BYTES = 512;           // barriers and flags behind the ring

struct MxArgs {
    const uint8_t* x_sf;
    const uint8_t* w_sf;
    const float* gx;
    const float* gw;
    void* out;
    int64_t ldo;
    int M, N, K;
    int BN;
    int out_dtype;
    int stages, stage_bytes;
    int k_tiles;       // scale tiles along K
    int tmem_cols;
    int ksplit;
    int early;         // the weights may be fetched before the dependency wait (see launch())
    int* status;
};

__device__ __forceinline__ void st_cluster_v4(uint32_t cluster_addr, const uint32_t* v) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(cluster_addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
// Untiled bulk copy global -> this CTA's shared memory (both addresses and the size are multiples of 16).
__device__ __forceinline__ void bulk_load_if(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar, uint32_t issue) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %4, 0;\n\t"
        "@q cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n\t}"
        ::"r"(dst), "l"(src), "r"(bytes), "r"(bar), "r"(issue)
        : "memory");
}
// Scale tile in shared memory: 32 rows of 16 bytes, unswizzled; the 8-row groups are 128 bytes apart.
__device__ __forceinline__ uint64_t smem_desc_scales(uint32_t addr) {
    return static_cast<uint64_t>((addr >> 4) & 0x3FFFu) | (8ull << 32) | (1ull << 46);
}
__device__ __forceinline__ void tc_copy_scales(uint32_t taddr, uint64_t desc, uint32_t issue) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %2, 0;\n\t"
        "@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}"
        ::"r"(taddr), "l"(desc), "r"(issue)
        : "memory");
}
template <int FMT>
__device__ __forceinline__ void tc_mma_mx4(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                           uint32_t accumulate, uint32_t issue) {
    if (FMT == SQAP_MX_NVFP4)
        asm volatile(
            "{\n\t.reg .pred p, q;\n\t"
            "setp.ne.b32 p, %6, 0;\n\t"
            "setp.ne.b32 q, %7, 0;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate), "r"(issue)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p, q;\n\t"
            "setp.ne.b32 p, %6, 0;\n\t"
            "setp.ne.b32 q, %7, 0;\n\t"
            "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate), "r"(issue)
            : "memory");
}

// Instruction descriptor: e2m1 x e2m1, fp32 sums, scale type e4m3 (nvfp4) or power of two (mxfp4).
__host__ __device__ inline uint32_t instr_desc(int format, int M, int BN) {
    return (1u << 7) | (1u << 10) | (static_cast<uint32_t>(BN >> 3) << 17) | (format == SQAP_MX_MXFP4 ? 1u << 23 : 0u) |
           (static_cast<uint32_t>(M >> 4) << 24);
}

template <int FMT>
__global__ void __launch_bounds__(THREADS)
mx4_linear_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, MxArgs a) {
    constexpr int TILES = FMT == SQAP_MX_NVFP4 ? 4 : 2;     // scale tiles along K per stage
    constexpr int PER_TILE = 4 / TILES;                     // MMAs (64 elements of K) per scale tile
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;   // identical in every CTA of the cluster
    uint8_t* sm = smem_raw + (base - smem_u32(smem_raw));
    const int S = a.stages;
    const uint32_t bar0 = base + static_cast<uint32_t>(S * a.stage_bytes);
    auto full = [&](int s) { return bar0 + 8u * s; };
    auto done = [&](int s) { return bar0 + 8u * (S_MAX + s); };
    const uint32_t acc_full = bar0 + 8u * (2 * S_MAX);
    uint8_t* tail = sm + S * a.stage_bytes + 8 * (2 * S_MAX + 1);
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(tail);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + 8);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = static_cast<int>(cluster_ctarank());
    const int nt = static_cast<int>(blockIdx.x) / a.ksplit, n0 = nt * BM;
    const int k_steps = (a.K + BK - 1) / BK;
    const int ks_begin = rank * k_steps / a.ksplit, ks_end = (rank + 1) * k_steps / a.ksplit;
    const int my_steps = ks_end - ks_begin;
    const int sfb_rows = (a.BN + 127) / 128;                 // scale tiles across a token tile
    const int m_sf_tiles = (a.M + 127) / 128;
    const int sfb_here = m_sf_tiles < sfb_rows ? m_sf_tiles : sfb_rows;   // those that exist
    auto a_addr = [&](int s) { return base + static_cast<uint32_t>(s * a.stage_bytes); };
    auto b_addr = [&](int s) { return a_addr(s) + A_BYTES; };
    auto sfa_addr = [&](int s) { return b_addr(s) + static_cast<uint32_t>(a.BN * 128); };
    auto sfb_addr = [&](int s, int r) { return sfa_addr(s) + TILES * SF_TILE * (1 + r); };
    // scale tiles that stage ks of the matrix really has (the last stage may be short)
    auto sf_tiles = [&](int ks) { return a.k_tiles - ks * TILES < TILES ? a.k_tiles - ks * TILES : TILES; };

    auto issue_weights = [&](int ks, int s, uint32_t issue) {
        const uint32_t sf = static_cast<uint32_t>(sf_tiles(ks) * SF_TILE);
        mbar_expect_tx_if(full(s), static_cast<uint32_t>(A_BYTES + a.BN * 128) + sf * (1 + sfb_here), issue);
        tma_load_2d_if(a_addr(s), &tm_w, ks * (BK / 2), n0, full(s), issue);
        bulk_load_if(sfa_addr(s), a.w_sf + (static_cast<size_t>(nt) * a.k_tiles + ks * TILES) * SF_TILE, sf, full(s), issue);
    };
    auto issue_tokens = [&](int ks, int s, uint32_t issue) {
        const uint32_t sf = static_cast<uint32_t>(sf_tiles(ks) * SF_TILE);
        tma_load_2d_if(b_addr(s), &tm_x, ks * (BK / 2), 0, full(s), issue);
        for (int r = 0; r < sfb_here; ++r)
            bulk_load_if(sfb_addr(s, r), a.x_sf + (static_cast<size_t>(r) * a.k_tiles + ks * TILES) * SF_TILE, sf, full(s), issue);
    };
    const int pre = my_steps < S ? my_steps : S;   // stages issued before the main loop
    if (warp == 0) {
        if (lane == 0) {
            for (int s = 0; s < S; ++s) {
                mbar_init(full(s), 1);
                mbar_init(done(s), 1);
            }
            mbar_init(acc_full, 1);
            abort_flag[0] = 0;
            abort_flag[1] = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        const uint32_t issue = elect_one();
        if (a.early)
            for (int it = 0; it < pre; ++it) issue_weights(ks_begin + it, it, issue);
    }
    pdl_launch_dependents();
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(const_cast<uint32_t*>(tmem_slot))), "r"(a.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    bool failed = false;
    pdl_wait();

    if (warp == 0) {
        const uint32_t issue = elect_one();
        for (int it = 0; it < pre; ++it) {
            if (!a.early) issue_weights(ks_begin + it, it, issue);
            issue_tokens(ks_begin + it, it, issue);
        }
        int s = pre == S ? 0 : pre;
        uint32_t ph = pre == S ? 1u : 0u;
        int it = pre;
        for (; it < my_steps; ++it) {
            if (!__all_sync(0xffffffffu, mbar_wait(done(s), ph ^ 1u, abort_flag))) { failed = true; break; }
            issue_weights(ks_begin + it, s, issue);
            issue_tokens(ks_begin + it, s, issue);
            if (++s == S) { s = 0; ph ^= 1u; }
        }
        if (failed && issue) {
            // give every armed stage a bounded chance to land before shared memory is reused or released
            for (int back = 0; back < S; ++back) {
                const int last = it - 1 - back;
                if (last >= 0) mbar_wait(full(last % S), static_cast<uint32_t>(last / S) & 1u, abort_flag + 1);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        const uint32_t issue = elect_one();
        const uint32_t idesc = instr_desc(FMT, BM, a.BN);
        const uint32_t acc_cols = static_cast<uint32_t>(a.BN < 32 ? 32 : a.BN);
        const uint32_t set_cols = TILES * 4u * (1u + sfb_rows);   // scale columns of one stage
        int s = 0;
        uint32_t ph = 0;
        for (int it = 0; it < my_steps; ++it) {
            if (!__all_sync(0xffffffffu, mbar_wait(full(s), ph, abort_flag))) { failed = true; break; }
            tc_fence_after();
            const int ks = ks_begin + it;
            const int mmas = a.K - ks * BK >= BK ? 4 : (a.K - ks * BK + 63) / 64;
            const uint32_t sfa = tmem_base + acc_cols + (it & 1) * set_cols, sfb = sfa + TILES * 4u;
            const int tiles = sf_tiles(ks);
            for (int t = 0; t < tiles; ++t) {
                tc_copy_scales(sfa + 4u * t, smem_desc_scales(sfa_addr(s) + t * SF_TILE), issue);
                for (int r = 0; r < sfb_here; ++r)
                    tc_copy_scales(sfb + 4u * (t * sfb_rows + r), smem_desc_scales(sfb_addr(s, r) + t * SF_TILE), issue);
            }
            const uint64_t adesc = smem_desc_sw128(a_addr(s)), bdesc = smem_desc_sw128(b_addr(s));
            for (int k = 0; k < mmas; ++k) {
                const int t = k / PER_TILE;
                // with two MMAs to a tile the second takes the upper two bytes of each scale word
                const uint32_t id = FMT == SQAP_MX_MXFP4 ? ((k & 1) ? (2u << 4) | (2u << 29) : 0u) : 0u;
                tc_mma_mx4<FMT>(tmem_base, adesc + 2u * k, bdesc + 2u * k, idesc | id, sfa + 4u * t, sfb + 4u * t * sfb_rows,
                                (it | k) != 0 ? 1u : 0u, issue);
            }
            tc_commit_if(done(s), issue);
            if (++s == S) { s = 0; ph ^= 1u; }
        }
        if (!failed) tc_commit_if(acc_full, issue);
    }

    // ---------------- partial sums -> the CTA that owns their tokens. 16-token chunk c belongs to rank c % ksplit,
    // which keeps the part of source r at (r * own_max + c / ksplit) * CHUNK_BYTES: thread = weight row, 16 bytes to a plane.
    const int chunks = a.BN >> 4;
    const int own_max = (chunks + a.ksplit - 1) / a.ksplit;
    if (!failed && !mbar_wait(acc_full, 0u, abort_flag)) failed = true;
    if (failed) {
        *abort_flag = 1;
        atomicOr(a.status, SQAP_ERR_TIMEOUT);
    }
    failed = __syncthreads_or(failed ? 1 : 0) != 0;
    tc_fence_after();
    cluster_sync_all();   // every CTA's MMAs are done (or given up): the rings are idle
    const int quad = warp & 3, group = warp >> 2, row = quad * 32 + lane;
    if (!failed) {
        const uint32_t taddr = tmem_base + (static_cast<uint32_t>(quad * 32) << 16);
        for (int c = group; c < chunks; c += 2) {
            uint32_t v[16];
            tc_ld16(taddr + 16 * c, v);
            const uint32_t dst = map_to_cta(base + static_cast<uint32_t>((rank * own_max + c / a.ksplit) * CHUNK_BYTES + row * 16),
                                            static_cast<uint32_t>(c % a.ksplit));
            tc_wait_ld();
#pragma unroll
            for (int q = 0; q < 4; ++q) st_cluster_v4(dst + q * (BM * 16), v + 4 * q);
        }
    }
    tc_fence_before();
    __syncwarp();
    cluster_sync_all();   // all parts have arrived; nobody touches another CTA's shared memory from here on
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(a.tmem_cols) : "memory");
    }
    if (failed) return;
    const float alpha = __fmul_rn(a.gx ? __ldg(a.gx) : 1.0f, a.gw ? __ldg(a.gw) : 1.0f);
    const int own = (chunks - rank + a.ksplit - 1) / a.ksplit;
    // 16-bit outputs go through shared memory ([token][channel], behind the exchange) so that a thread stores 16 bytes: two
    // buffers a group in turn, one barrier of the group a chunk.
    uint8_t* const stage0 = sm + own_max * a.ksplit * CHUNK_BYTES + group * 2 * STAGE_BYTES;
    for (int lc = group, turn = 0; lc < own; lc += 2, turn ^= 1) {
        const int m_first = 16 * (lc * a.ksplit + rank);
        float y[16];
        const uint8_t* part = sm + lc * CHUNK_BYTES + row * 16;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 f = *reinterpret_cast<const float4*>(part + q * (BM * 16));
            y[4 * q] = f.x; y[4 * q + 1] = f.y; y[4 * q + 2] = f.z; y[4 * q + 3] = f.w;
        }
        for (int r = 1; r < a.ksplit; ++r) {
            part += own_max * CHUNK_BYTES;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 f = *reinterpret_cast<const float4*>(part + q * (BM * 16));
                y[4 * q] += f.x; y[4 * q + 1] += f.y; y[4 * q + 2] += f.z; y[4 * q + 3] += f.w;
            }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] *= alpha;
        if (a.out_dtype == SQAP_FP32) {                              // a warp's 32 channels of a token are 128 bytes
            float* o = static_cast<float*>(a.out) + static_cast<int64_t>(m_first) * a.ldo + n0 + row;
            if (n0 + row < a.N)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (m_first + e < a.M) o[e * a.ldo] = y[e];
            continue;
        }
        uint8_t* stage = stage0 + turn * STAGE_BYTES;
#pragma unroll
        for (int e = 0; e < 16; ++e)
            *reinterpret_cast<uint16_t*>(stage + e * (BM * 2) + row * 2) = a.out_dtype == SQAP_FP16 ? bits16<SQAP_FP16>(y[e]) : bits16<SQAP_BF16>(y[e]);
        bar_sync_named(1 + group, 128);
#pragma unroll
        for (int p = row; p < 16 * (BM / 8); p += 128) {
            const int token = p / (BM / 8), piece = p % (BM / 8), m = m_first + token, n = n0 + 8 * piece;
            if (m >= a.M || n >= a.N) continue;
            const uint16_t* src = reinterpret_cast<const uint16_t*>(stage + token * (BM * 2) + piece * 16);
            uint16_t* o = static_cast<uint16_t*>(a.out) + static_cast<int64_t>(m) * a.ldo + n;
            if (n + 8 <= a.N) {
                *reinterpret_cast<uint4*>(o) = *reinterpret_cast<const uint4*>(src);
            } else {
                for (int e = 0; e < a.N - n; ++e) o[e] = src[e];
            }
        }
    }
}

// Which kernel. The pairs (mx4_pair.cu) take 256 weight rows and up to 192 tokens each and walk K alone: some 5 us and 0.25 us
// per 256 elements of K and round. The clusters here split K where there are few tiles, but then exchange 4 bytes per token and
// weight row of every slice. So they are for long K, few weight rows and few tokens. Measured with the quantizer, clusters / pairs,
// us, NVFP4, operands from HBM: 4096 x 11008 (rows x K): 13.9 / 15.9 for 16 tokens, 15.5 / 16.4 for 64, 16.5 / 17.0 for 128, 17.9 / 18.1
// for 160, 20.0 / 18.4 for 256; 1024 x 16384: 11.7 / 20.9 for 16, 19.1 / 23.3 for 256; 1024 x 4096: 7.7 / 9.3 for 16, 8.6 / 9.5 for 64,
// 10.1 / 9.5 for 128; 4096 x 4096: 10.4 / 9.8 for 16, 14.4 / 10.6 for 256; 12288 x 4096: 17.2 / 11.8 for 16, 21.6 / 17.3 for 256.
// MXFP4 differs by up to 2 us on both sides and by the same sign.
static bool use_clusters(int M, int N, int K) {
    const int64_t steps = (K + BK - 1) / BK, weight_tiles = (N + 2 * BM - 1) / (2 * BM);
    return M <= BN_MAX && 64ll * M <= K && steps * (sm_count() / 2) > 128 * weight_tiles;
}

static sqap_status launch(const Mx4Product& q, cudaStream_t s) {
    const int M = q.M, N = q.N, K = q.K, format = q.format;
    if (mx4_gemv_takes(M, N, K, format)) return launch_mx4_gemv(q, nullptr, 0, 0, nullptr, s);
    if (!use_clusters(M, N, K)) return launch_mx4_pair(q, s);
    MxArgs k;
    k.early = q.early ? 1 : 0;
    k.x_sf = q.x_scales;
    k.w_sf = q.w_scales;
    k.gx = q.gx;
    k.gw = q.gw;
    k.out = q.out;
    k.ldo = q.ldo;
    k.M = M;
    k.N = N;
    k.K = K;
    k.out_dtype = q.out_dtype;
    k.status = device_status_word();
    if (!k.status) return SQAP_ERR_CUDA;
    if (!device_is_sm100()) return SQAP_ERR_UNSUPPORTED;
    k.k_tiles = mx4_k_tiles(K, format);
    k.BN = (M + 15) / 16 * 16;   // one token tile: use_clusters()
    const int tiles_k = format == SQAP_MX_NVFP4 ? 4 : 2, sfb_rows = (k.BN + 127) / 128;
    k.stage_bytes = (A_BYTES + k.BN * 128 + tiles_k * SF_TILE * (1 + sfb_rows) + 1023) / 1024 * 1024;
    // Narrow tiles: two CTAs to an SM, so that one streams while the other exchanges and stores.
    const int per_sm = k.BN <= 64 ? 2 : 1;
    const int ring = (per_sm == 2 ? 108 : 222) * 1024;
    const int k_steps = (K + BK - 1) / BK;
    k.stages = ring / k.stage_bytes;
    if (k.stages > S_MAX) k.stages = S_MAX;
    const int acc = k.BN < 32 ? 32 : k.BN, cols = acc + 2 * tiles_k * 4 * (1 + sfb_rows);
    k.tmem_cols = 32;
    while (k.tmem_cols < cols) k.tmem_cols *= 2;

    // K split: rounds of clusters over the device x (stages of a CTA + its fixed cost), in units of a stage
    const int slots = sm_count() * per_sm;
    const long tiles = (N + BM - 1) / BM;
    double best = -1.0;
    k.ksplit = 1;
    for (int c = 1; c <= KSPLIT_MAX && c <= k_steps; ++c) {
        const long rounds = (tiles * c + slots - 1) / slots;
        const double cost = static_cast<double>(rounds) * ((k_steps + c - 1) / c + 5.0) + (c > 1 ? 1.0 + 0.25 * c : 0.0);
        if (best < 0 || cost < best) {
            best = cost;
            k.ksplit = c;
        }
    }
    // The exchange and the staging, own_max * ksplit * CHUNK_BYTES + 4 * STAGE_BYTES, lie in the idle ring: it is 4 KB larger at least,
    // over all BN, formats and splits.
    const int smem = k.stages * k.stage_bytes + TAIL_BYTES + 1024;

    CUtensorMap tm_w, tm_x;
    if (!make_map(&tm_w, q.w_codes, N, K / 2, BM, 128, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_map(&tm_x, q.x_codes, M, K / 2, k.BN, 128, CU_TENSOR_MAP_SWIZZLE_128B))
        return SQAP_ERR_CUDA;
    static PerDevice<int> setup;
    const sqap_status st = setup.run([](int*) {
        const sqap_status s0 = set_max_dynamic_smem(mx4_linear_kernel<SQAP_MX_NVFP4>, 227 * 1024);
        return s0 != SQAP_OK ? s0 : set_max_dynamic_smem(mx4_linear_kernel<SQAP_MX_MXFP4>, 227 * 1024);
    });
    if (st != SQAP_OK) return st;

    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(tiles * k.ksplit));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(k.ksplit);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = format == SQAP_MX_NVFP4 ? cudaLaunchKernelEx(&cfg, mx4_linear_kernel<SQAP_MX_NVFP4>, tm_w, tm_x, k)
                                                  : cudaLaunchKernelEx(&cfg, mx4_linear_kernel<SQAP_MX_MXFP4>, tm_w, tm_x, k);
    if (e != cudaSuccess) {
        note_cuda_error(e);
        cudaGetLastError();
        return SQAP_ERR_CUDA;
    }
    count_launch();
    return check_launch();
}

static sqap_status check(int M, const void* wc, const void* ws, int N, int K, int format, const void* out, int64_t ldo,
                         int out_dtype) {
    if (M < 0 || N <= 0 || K <= 0 || ldo < N) return SQAP_ERR_INVALID;
    if (format != SQAP_MX_NVFP4 && format != SQAP_MX_MXFP4) return SQAP_ERR_INVALID;
    if (out_dtype != SQAP_FP16 && out_dtype != SQAP_BF16 && out_dtype != SQAP_FP32) return SQAP_ERR_INVALID;
    if (K % 32 != 0 || (ldo * type_bytes(out_dtype)) % 16 != 0) return SQAP_ERR_ALIGN;
    if (M == 0) return SQAP_OK;
    if (!wc || !ws || !out) return SQAP_ERR_INVALID;
    if (!aligned16(wc) || !aligned16(ws) || !aligned16(out)) return SQAP_ERR_ALIGN;
    return SQAP_OK;
}

static Mx4Product product(const uint8_t* xc, const uint8_t* xs, const float* gx, int M, const uint8_t* wc, const uint8_t* ws, const float* gw,
                          int N, int K, int format, void* out, int64_t ldo, int out_dtype, bool early) {
    const bool g = format == SQAP_MX_NVFP4;   // MXFP4 has no scale of the tensor
    return {xc, xs, wc, ws, g ? gx : nullptr, g ? gw : nullptr, out, ldo, M, N, K, format, out_dtype, early};
}

static size_t codes_bytes(int M, int K) { return (static_cast<size_t>(M) * (K / 2) + 255) / 256 * 256; }

}  // namespace mx4
}  // namespace sqap

extern "C" size_t sqap_mx4_workspace_bytes(int M, int N, int K, int format) {
    (void)N;
    if (M <= 0 || K <= 0) return 256;
    const size_t n = sqap::mx4::codes_bytes(M, K) + sqap_mx4_scale_bytes(M, K, format);
    return (n + 255) / 256 * 256;
}

extern "C" sqap_status sqap_mx4_linear(const uint8_t* x_codes, const uint8_t* x_scales, const float* x_tensor_scale, int M,
                                       const uint8_t* w_codes, const uint8_t* w_scales, const float* w_tensor_scale, int N, int K,
                                       int format, void* out, int64_t ldo, int out_dtype, void* stream) {
    using namespace sqap;
    const sqap_status st = mx4::check(M, w_codes, w_scales, N, K, format, out, ldo, out_dtype);
    if (st != SQAP_OK || M == 0) return st;
    if (!x_codes || !x_scales) return SQAP_ERR_INVALID;
    if (!aligned16(x_codes) || !aligned16(x_scales)) return SQAP_ERR_ALIGN;
    return mx4::launch(mx4::product(x_codes, x_scales, x_tensor_scale, M, w_codes, w_scales, w_tensor_scale, N, K, format, out, ldo, out_dtype, false),
                       static_cast<cudaStream_t>(stream));
}

extern "C" sqap_status sqap_mx4_quantize_linear(const void* x, int x_dtype, int M, int64_t ldx, const int32_t* row_index,
                                                const float* x_tensor_scale, const uint8_t* w_codes, const uint8_t* w_scales,
                                                const float* w_tensor_scale, int N, int K, int format, void* out, int64_t ldo,
                                                int out_dtype, void* workspace, size_t workspace_bytes, void* stream) {
    using namespace sqap;
    sqap_status st = mx4::check(M, w_codes, w_scales, N, K, format, out, ldo, out_dtype);
    if (st != SQAP_OK) return st;
    uint8_t* codes = static_cast<uint8_t*>(workspace);
    uint8_t* scales = codes + mx4::codes_bytes(M, K);
    st = check_mx4_quantize(x, x_dtype, M, K, ldx, format, workspace, workspace);
    if (st != SQAP_OK || M == 0) return st;
    if (workspace_bytes < sqap_mx4_workspace_bytes(M, N, K, format)) return SQAP_ERR_NOMEM;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (mx4_gemv_takes(M, N, K, format))   // quantizes its few rows itself
        return launch_mx4_gemv(mx4::product(nullptr, nullptr, x_tensor_scale, M, w_codes, w_scales, w_tensor_scale, N, K, format, out, ldo, out_dtype, false),
                               x, x_dtype, ldx, row_index, s);
    st = launch_mx4_quantize(x, x_dtype, M, K, ldx, row_index, format, x_tensor_scale, codes, scales, s);
    if (st != SQAP_OK) return st;
    return mx4::launch(mx4::product(codes, scales, x_tensor_scale, M, w_codes, w_scales, w_tensor_scale, N, K, format, out, ldo, out_dtype, true), s);
}
