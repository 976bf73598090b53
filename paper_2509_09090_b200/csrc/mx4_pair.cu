// Product of two microscaled 4-bit matrices for many tokens, on CTA pairs (tcgen05 cta_group::2). Mathematics, operands and scale
// layout: mx4_linear.cu.
//
// A cluster of two CTAs computes 256 x BN tiles (BN 64, 128 or 192 tokens): each CTA holds 128 weight rows and half of the
// token rows, and the pair's tensor cores share both halves, so an SM fetches 28 KB of codes instead of 40 per 256
// elements of K at BN = 192. The scales of the tokens are wanted in full by both CTAs (4 KB), those of the weights by their own
// (2 KB). The codes' bytes are counted on the leader's barrier, where the MMAs are issued.
// What bounds it: the four-bit MMAs of a stage (256 elements of K) take 384 cycles at BN = 192. 4608 x 12288 x 4096 in NVFP4 with
// the quantizer takes 112 us in bursts of a millisecond, of it the product 98 to 103 (4.5 PFLOP/s, tensor pipe 68 %), and 132 us (product
// 117) in a region of seconds, where the power limit holds the SM clock at 1.4 GHz. A stage costs 0.32 us there; with one MMA of four issued it is 0.23, with no loads
// 0.22, with neither 0.21: the round trip of a stage's signals (done -> scales written again -> issued) and the SM clock, which
// the full load brings down to 1.55 GHz in a burst already, share the rest. A tile's results cost 1.6 us of issue slots beside it.
// The scales go to tensor memory through registers (four warps: shared memory -> tcgen05.st, one lane quadrant each): a
// tcgen05.cp of a scale tile holds up the tensor pipe for some 24 cycles, and a stage has twelve of them beside 374 cycles of
// MMAs (measured: pipe busy 78 %, with MMAs 44 %; 15 us more for 4608 x 12288 x 4096).
// Tensor memory (512 columns): two accumulators of BN columns, so that a tile is stored while the next is computed, and three to six
// sets of scale columns. A scale tile's place in shared memory is free as soon as it has been read, so the scales run ahead of
// the codes and have a loading warp of their own; two groups of four warps copy them, a stage each in turn.
//   warp 0     TMA      warp 1  MMA (one thread of the leader)      warps 2-9  epilogue: four lane quadrants x two halves of the tokens
//   warps 10-17  scales to tensor memory      warp 18  scales' TMA
// A token tile may start in the middle of a 128-row scale tile (BN = 64, 192): 64 rows are two columns of a tile, so its scales
// are taken from two columns further on.
// Every wait on a barrier is bounded; on expiry the kernel records SQAP_ERR_TIMEOUT in the device status word, drains, and
// returns through the cluster barrier.
#include "mx4.cuh"
#include "tc_common.cuh"

namespace sqap {
namespace mx4p {

using namespace tc;

constexpr int BM = 128;                   // weight rows per CTA
constexpr int BK = 256;                   // elements of K per stage
constexpr int BN_MAX = 192;
constexpr int S = 6;
constexpr int A_BYTES = BM * BK / 2;      // 16 KB
constexpr int B_BYTES = BN_MAX / 2 * BK / 2;   // 12 KB: this CTA's half of the tokens
constexpr int SF_TILE = 512;
constexpr int SFB_TILES = 2;              // row tiles that a token tile can reach into
constexpr int OFF_A = 0, OFF_B = OFF_A + S * A_BYTES;
constexpr int OFF_SFA = OFF_B + S * B_BYTES, SF_BYTES = 4 * SF_TILE;
constexpr int OFF_SFB = OFF_SFA + S * SF_BYTES;
constexpr int OFF_STAGE = OFF_SFB + S * SFB_TILES * SF_BYTES;   // staging of the coalesced stores: two halves x two buffers
constexpr int OFF_BAR = OFF_STAGE + EPI_STAGE_TOTAL;
constexpr int SMEM_BYTES = OFF_BAR + 256 + 1024;
constexpr int EPI_WARPS = 8;
constexpr int SF_WARP0 = 2 + EPI_WARPS;
constexpr int SF_GROUPS = 2;              // of four scale warps; they take the stages in turn
constexpr int SF_LOADER = SF_WARP0 + 4 * SF_GROUPS;
constexpr int THREADS = 32 * (SF_LOADER + 1);
// Scale columns: a stage's set has, for each scale tile along K, 4 columns of weight scales and 6 of token scales (192 rows,
// from where the token tile starts). As many sets as the accumulators leave room for, a stage of the ring each at most:
// from the end of a stage's MMAs to the set written again and signalled takes some 1000 cycles, the MMAs of a stage 2 BN.
constexpr int SFB_COLS = BN_MAX / 32, SET_COLS = 4 * (4 + SFB_COLS);
__host__ __device__ constexpr int sets_for(int bn) { return (512 - 2 * bn) / SET_COLS < S ? (512 - 2 * bn) / SET_COLS : S; }
static_assert(SMEM_BYTES <= 227 * 1024 && sets_for(BN_MAX) >= 2, "budgets");
static_assert(8 * (4 * S + 4) + 16 <= 256, "barrier block");

struct PairArgs {
    const float* gx;
    const float* gw;
    void* out;
    int64_t ldo;
    int M, N, K;
    int BN, m_tiles, n_tiles;
    int out_dtype;
    int k_tiles;
    int early;
    int* status;
};

// Into this CTA's shared memory; the bytes are counted on a barrier that may live in the peer CTA.
__device__ __forceinline__ void tma_pair_if(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar_cluster, uint32_t issue) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar_cluster), "r"(issue)
        : "memory");
}
__device__ __forceinline__ void tc_commit_pair(uint32_t bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
        ::"r"(bar), "h"(static_cast<uint16_t>(3))
        : "memory");
}
// 16 lanes x 32 columns as fragments of 8 x 8: r[4 u + 2 h + e] is row 8 h + lane / 4, column 8 u + 2 (lane % 4) + e.
__device__ __forceinline__ void tc_ld_fragments(uint32_t taddr, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr));
}
// Four 8 x 8 fragments of 16-bit values, turned, to the rows of 16 bytes that lanes 0-7, 8-15, ... address.
__device__ __forceinline__ void store_turned(uint32_t row, const uint32_t* p) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(row), "r"(p[0]), "r"(p[1]), "r"(p[2]), "r"(p[3]) : "memory");
}
template <int OUT>
__device__ __forceinline__ uint32_t bits16x2(float lo, float hi) {
    if (OUT == SQAP_FP16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <int FMT>
__device__ __forceinline__ void tc_mma_mx4(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                           uint32_t accumulate) {
    if (FMT == SQAP_MX_NVFP4)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
            : "memory");
}

template <int FMT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
mx4_pair_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_wsf,
                const __grid_constant__ CUtensorMap tm_xsf, PairArgs a) {
    constexpr int TILES = FMT == SQAP_MX_NVFP4 ? 4 : 2;     // scale tiles along K per stage
    constexpr int PER_TILE = 4 / TILES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;   // identical in both CTAs of the pair
    uint8_t* sm = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t bar0 = base + OFF_BAR;
    auto full = [&](int s) { return bar0 + 8u * s; };                  // leader's: the stage's codes have landed and its scales are in
                                                                       // tensor memory, in both CTAs
    auto done = [&](int s) { return bar0 + 8u * (S + s); };            // the MMAs of the stage in slot s are done (both CTAs)
    auto acc_full = [&](int b) { return bar0 + 8u * (2 * S + b); };
    auto acc_empty = [&](int b) { return bar0 + 8u * (2 * S + 2 + b); };   // leader's
    auto sf_full = [&](int s) { return bar0 + 8u * (2 * S + 4 + s); };     // this CTA's scale tiles of the stage have landed
    auto sf_empty = [&](int s) { return bar0 + 8u * (3 * S + 4 + s); };    // ... and have been read
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(sm + OFF_BAR + 8 * (4 * S + 4));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + OFF_BAR + 8 * (4 * S + 4) + 8);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();          // 0 = leader
    const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const int half_bn = a.BN >> 1;
    const int k_steps = (a.K + BK - 1) / BK;
    const int total_tiles = a.m_tiles * a.n_tiles;
    const uint32_t sets = sets_for(a.BN);
    const uint32_t stage_tx = 2u * static_cast<uint32_t>(A_BYTES + half_bn * (BK / 2)), sf_tx = TILES * SF_TILE * (1 + SFB_TILES);

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full(s), 1 + 8);   // the loads; four scale warps of either CTA
            mbar_init(done(s), 1);
            mbar_init(sf_full(s), 1);
            mbar_init(sf_empty(s), 4);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full(b), 1);
            mbar_init(acc_empty(b), 2 * EPI_WARPS);
        }
        abort_flag[0] = 0;
        abort_flag[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(const_cast<uint32_t*>(tmem_slot))) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    pdl_launch_dependents();
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();   // the peer's barriers exist before anything signals them
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    bool failed = false;

    if (warp == 0) {
        const uint32_t issue = elect_one();
        auto weights = [&](int s, int ks, int n_tile, uint32_t bar) {
            const int nt = 2 * n_tile + static_cast<int>(rank);        // 128-row tile of the weights
            tma_pair_if(base + OFF_A + s * A_BYTES, &tm_w, ks * (BK / 2), nt * BM, bar, issue);
        };
        uint32_t early = 0;
        if (a.early && pair < total_tiles) {
            early = static_cast<uint32_t>(k_steps < S ? k_steps : S);
            for (uint32_t ks = 0; ks < early; ++ks) weights(static_cast<int>(ks), static_cast<int>(ks), pair % a.n_tiles, map_to_cta(full(ks), 0));
        }
        pdl_wait();
        uint32_t it = 0;
        for (int tile = pair; tile < total_tiles && !failed; tile += n_pairs) {
            const int n_tile = tile % a.n_tiles, m_tile = tile / a.n_tiles;
            for (int ks = 0; ks < k_steps; ++ks, ++it) {
                const int s = it % S;
                if (it >= S && !__all_sync(0xffffffffu, mbar_wait(done(s), (it / S - 1) & 1u, abort_flag))) { failed = true; break; }
                if (rank == 0) mbar_expect_tx_if(full(s), stage_tx, issue);
                const uint32_t bar = map_to_cta(full(s), 0);
                if (it >= early) weights(s, ks, n_tile, bar);
                tma_pair_if(base + OFF_B + s * B_BYTES, &tm_x, ks * (BK / 2), m_tile * a.BN + static_cast<int>(rank) * half_bn, bar, issue);
            }
        }
    } else if (warp == SF_LOADER) {
        const uint32_t issue = elect_one();
        auto weights = [&](int s, int ks, int n_tile) {
            mbar_expect_tx_if(sf_full(s), sf_tx, issue);
            tma_load_2d_if(base + OFF_SFA + s * SF_BYTES, &tm_wsf, 0, (2 * n_tile + static_cast<int>(rank)) * a.k_tiles + ks * TILES, sf_full(s), issue);
        };
        uint32_t early = 0;
        if (a.early && pair < total_tiles) {
            early = static_cast<uint32_t>(k_steps < S ? k_steps : S);
            for (uint32_t ks = 0; ks < early; ++ks) weights(static_cast<int>(ks), static_cast<int>(ks), pair % a.n_tiles);
        }
        pdl_wait();
        uint32_t it = 0;
        for (int tile = pair; tile < total_tiles && !failed; tile += n_pairs) {
            const int n_tile = tile % a.n_tiles, row_tile = tile / a.n_tiles * a.BN / 128;
            for (int ks = 0; ks < k_steps; ++ks, ++it) {
                const int s = it % S;
                if (it >= S && !__all_sync(0xffffffffu, mbar_wait(sf_empty(s), (it / S - 1) & 1u, abort_flag))) { failed = true; break; }
                if (it >= early) weights(s, ks, n_tile);
#pragma unroll
                for (int r = 0; r < SFB_TILES; ++r)
                    tma_load_2d_if(base + OFF_SFB + (s * SFB_TILES + r) * SF_BYTES, &tm_xsf, 0, (row_tile + r) * a.k_tiles + ks * TILES, sf_full(s), issue);
            }
        }
    } else if (warp == 1) {
        pdl_wait();
        if (rank == 0 && elect_one()) {
            // One thread alone: its instructions are what the tensor core waits for, so no votes, and the barrier of the next stage is
            // looked at before this stage's products are issued.
            const uint32_t idesc = (1u << 7) | (1u << 10) | (static_cast<uint32_t>(a.BN >> 3) << 17) | (FMT == SQAP_MX_MXFP4 ? 1u << 23 : 0u) |
                                   (static_cast<uint32_t>((2 * BM) >> 4) << 24);
            const uint64_t adesc0 = smem_desc_sw128(base + OFF_A), bdesc0 = smem_desc_sw128(base + OFF_B);
            uint32_t lt = 0, ph = 0;
            const uint32_t set0 = tmem_base + 2u * a.BN, last_set = set0 + (sets - 1) * SET_COLS;
            uint32_t set = set0;
            int s = 0;
            bool ready = false;
            for (int tile = pair; tile < total_tiles && !failed; tile += n_pairs, ++lt) {
                const int b = lt & 1;
                if (!mbar_wait(acc_empty(b), ((lt >> 1) & 1u) ^ 1u, abort_flag)) { failed = true; break; }
                tc_fence_after();
                const uint32_t d = tmem_base + static_cast<uint32_t>(b * a.BN);
                for (int ks = 0; ks < k_steps; ++ks) {
                    if (!ready && !mbar_wait(full(s), ph, abort_flag)) { failed = true; break; }
                    tc_fence_after();
                    const int next = s + 1 == S ? 0 : s + 1;
                    const uint32_t next_ph = s + 1 == S ? ph ^ 1u : ph;
                    ready = mbar_test_wait(full(next), next_ph);
                    const uint32_t sfa = set, sfb = sfa + 4 * TILES;
                    const uint64_t adesc = adesc0 + static_cast<uint32_t>(s * (A_BYTES / 16)), bdesc = bdesc0 + static_cast<uint32_t>(s * (B_BYTES / 16));
                    const int mmas = a.K - ks * BK >= BK ? 4 : (a.K - ks * BK + 63) / 64;
                    auto mma = [&](int k) {
                        const int t = k / PER_TILE;
                        const uint32_t id = FMT == SQAP_MX_MXFP4 && (k & 1) ? (2u << 4) | (2u << 29) : 0u;
                        tc_mma_mx4<FMT>(d, adesc + 2u * k, bdesc + 2u * k, idesc | id, sfa + 4u * t, sfb + SFB_COLS * t, k != 0 || ks != 0 ? 1u : 0u);
                    };
                    if (mmas == 4) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) mma(k);
                    } else {
                        for (int k = 0; k < mmas; ++k) mma(k);
                    }
                    tc_commit_pair(done(s));
                    s = next;
                    ph = next_ph;
                    set = set == last_set ? set0 : set + SET_COLS;
                }
                if (failed) break;
                tc_commit_pair(acc_full(b));
            }
        }
        __syncwarp();
    } else if (warp >= SF_WARP0) {
        // ---------------- scales: lane i of every quadrant holds rows i, 32 + i, 64 + i, 96 + i of a tile, a column each
        pdl_wait();   // the waits below are bounded, and the loads that they wait for may not start before the kernel in front is done
        const int quad = warp & 3;
        const uint32_t mine = tmem_base + (static_cast<uint32_t>(quad * 32) << 16) + 2u * a.BN;
        const uint32_t my_tiles = pair < total_tiles ? (total_tiles - 1 - pair) / n_pairs + 1 : 0, stages = my_tiles * k_steps;
        int tile = pair, ks = (warp - SF_WARP0) >> 2;
        uint32_t set = ks;
        for (uint32_t it = ks; it < stages; it += SF_GROUPS, ks += SF_GROUPS, set += SF_GROUPS) {
            if (set >= sets) set -= sets;
            while (ks >= k_steps) {
                ks -= k_steps;
                tile += n_pairs;
            }
            const bool middle = (tile / a.n_tiles) * a.BN % 128 != 0;          // the token tile starts 64 rows into a scale tile
            const int s = it % S;
            if (!__all_sync(0xffffffffu, mbar_wait(sf_full(s), (it / S) & 1u, abort_flag))) { failed = true; break; }
            constexpr int COLS = TILES * (4 + SFB_COLS);
            uint32_t r[(COLS + 7) / 8 * 8] = {};
            auto get = [&](int off) { return *reinterpret_cast<const uint4*>(sm + off + lane * 16); };
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                const uint4 w = get(OFF_SFA + s * SF_BYTES + t * SF_TILE);
                const uint4 x = get(OFF_SFB + s * SFB_TILES * SF_BYTES + t * SF_TILE), y = get(OFF_SFB + (s * SFB_TILES + 1) * SF_BYTES + t * SF_TILE);
                r[4 * t] = w.x; r[4 * t + 1] = w.y; r[4 * t + 2] = w.z; r[4 * t + 3] = w.w;
                uint32_t* b = r + 4 * TILES + SFB_COLS * t;
                b[0] = middle ? x.z : x.x;
                b[1] = middle ? x.w : x.y;
                b[2] = middle ? y.x : x.z;
                b[3] = middle ? y.y : x.w;
                b[4] = middle ? y.z : y.x;
                b[5] = middle ? y.w : y.y;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(sf_empty(s));
            // the MMAs that read this set `sets` stages ago are done
            if (it >= sets && !__all_sync(0xffffffffu, mbar_wait(done((it - sets) % S), ((it - sets) / S) & 1u, abort_flag))) { failed = true; break; }
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < COLS; c += 8) tc_st8(mine + set * SET_COLS + c, r + c);
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_cta(full(s), 0));
        }
    } else {
        pdl_wait();
        const float alpha = __fmul_rn(a.gx ? __ldg(a.gx) : 1.0f, a.gw ? __ldg(a.gw) : 1.0f);
        const int quad = warp & 3, row = quad * 32 + lane;
        const int hf = (warp - 2) >> 2, tid_half = static_cast<int>(threadIdx.x) - (2 + 4 * hf) * 32;
        const int split = ((a.BN / 16 + 1) / 2) * 16;
        const int c_begin = hf == 0 ? 0 : split, c_end = hf == 0 ? split : a.BN;
        uint8_t* stage_half = sm + OFF_STAGE + hf * 2 * EPI_STAGE_BYTES;
        // 32 tokens at a time in the layout of 8 x 8 fragments (channel lane / 4, tokens 2 (lane % 4) and the next), turned on the way
        // to shared memory; the 16-byte pieces of a token's row there are permuted by the token against bank conflicts. A thread
        // copies out piece tid_half % 16 of tokens tid_half / 16 and 8 further on.
        const int out_token = tid_half >> 4, out_piece = tid_half & 15;
        const uint32_t put = smem_u32(stage_half) + (lane & 7) * (BM * 2) + ((quad * 4 + (lane >> 3)) ^ (lane & 7)) * 16;
        const uint8_t* take = stage_half + out_token * (BM * 2) + (out_piece ^ out_token) * 16;
        auto store_tile = [&](auto out_type, uint32_t taddr, int m0, int n0) {
            constexpr int OUT = decltype(out_type)::value;
            const int n = n0 + out_piece * 8, n_left = a.N - n;
            int m = m0 + c_begin + out_token;
            uint16_t* dst = static_cast<uint16_t*>(a.out) + static_cast<int64_t>(m) * a.ldo + n;
            for (int c = c_begin; c < c_end; c += 32) {
                uint32_t v[2][16];
                tc_ld_fragments(taddr + c, v[0]);
                tc_ld_fragments(taddr + c + (16u << 16), v[1]);
                tc_wait_ld();
#pragma unroll
                for (int part = 0; part < 2; ++part) {             // 16 tokens each, into two buffers in turn
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        uint32_t p[4];
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const uint32_t* x = v[g >> 1] + 8 * part + 4 * u + 2 * (g & 1);
                            p[g] = bits16x2<OUT>(__uint_as_float(x[0]) * alpha, __uint_as_float(x[1]) * alpha);
                        }
                        store_turned(put + part * EPI_STAGE_BYTES + u * 8 * (BM * 2), p);
                    }
                    // A thread can only be two buffers ahead of the slowest after passing the barrier in between
                    bar_sync_named(2 + hf, 128);
#pragma unroll
                    for (int i = 0; i < 2; ++i, m += 8, dst += 8 * a.ldo) {
                        if (m >= a.M || n_left <= 0) continue;
                        const uint4 y = *reinterpret_cast<const uint4*>(take + part * EPI_STAGE_BYTES + i * 8 * (BM * 2));
                        if (n_left >= 8) {
                            *reinterpret_cast<uint4*>(dst) = y;
                        } else {
                            const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                            for (int e = 0; e < 7; ++e)
                                if (e < n_left) dst[e] = static_cast<uint16_t>(w[e >> 1] >> (16 * (e & 1)));
                        }
                    }
                }
            }
        };
        uint32_t lt = 0;
        for (int tile = pair; tile < total_tiles && !failed; tile += n_pairs, ++lt) {
            const int b = lt & 1;
            const int n0 = (tile % a.n_tiles) * (2 * BM) + static_cast<int>(rank) * BM, m0 = (tile / a.n_tiles) * a.BN;
            // all epilogue warps leave the loop together if any wait ran out, so the barriers below never hang
            if (bar_or(1, 32 * EPI_WARPS, !mbar_wait(acc_full(b), (lt >> 1) & 1u, abort_flag))) { failed = true; break; }
            tc_fence_after();
            const uint32_t taddr = tmem_base + (static_cast<uint32_t>(quad * 32) << 16) + static_cast<uint32_t>(b * a.BN);
            if (a.out_dtype == SQAP_FP32) {                            // a warp's 32 channels of a token are 128 bytes
                for (int c = c_begin; c < c_end; c += 16) {
                    uint32_t v[16];
                    tc_ld16(taddr + c, v);
                    tc_wait_ld();
                    float* o = static_cast<float*>(a.out) + static_cast<int64_t>(m0 + c) * a.ldo + n0 + row;
                    if (n0 + row < a.N)
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (m0 + c + j < a.M) o[j * a.ldo] = __uint_as_float(v[j]) * alpha;
                }
            } else if (a.out_dtype == SQAP_FP16) {
                store_tile(std::integral_constant<int, SQAP_FP16>{}, taddr, m0, n0);
            } else {
                store_tile(std::integral_constant<int, SQAP_BF16>{}, taddr, m0, n0);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_cta(acc_empty(b), 0));
        }
    }

    if (failed) {
        *abort_flag = 1;
        atomicOr(a.status, SQAP_ERR_TIMEOUT);
    }
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        // the loads in flight are counted on barriers that no one waits for any more: give them a fixed while to land
        const long long t0 = clock64();
        while (clock64() - t0 < 200000) {}
    }
    cluster_sync_all();   // neither CTA leaves (or frees tensor memory) while the other may still signal it
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem_base) : "memory");
}

// Scale tiles as a matrix of 512-byte rows, boxes of `box_rows` of them.
static bool make_scale_map(CUtensorMap* m, const void* ptr, uint64_t tiles, uint32_t box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {SF_TILE / 4, tiles};
    const cuuint64_t strides[1] = {SF_TILE};
    const cuuint32_t box[2] = {SF_TILE / 4, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int FMT>
static sqap_status resident_pairs(int* pairs) {
    static PerDevice<int> setup;
    const int* p = nullptr;
    const sqap_status st = setup.run(
        [](int* out) {
            const sqap_status s0 = set_max_dynamic_smem(mx4_pair_kernel<FMT>, SMEM_BYTES);
            if (s0 != SQAP_OK) return s0;
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(static_cast<unsigned>(sm_count() / 2 * 2));
            cfg.blockDim = dim3(THREADS);
            cfg.dynamicSmemBytes = SMEM_BYTES;
            cudaLaunchAttribute attr;
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = 2;
            attr.val.clusterDim.y = 1;
            attr.val.clusterDim.z = 1;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            int n = 0;
            if (cudaOccupancyMaxActiveClusters(&n, mx4_pair_kernel<FMT>, &cfg) != cudaSuccess || n <= 0) {
                cudaGetLastError();
                n = sm_count() / 2;
            }
            *out = n;
            return SQAP_OK;
        },
        &p);
    if (st == SQAP_OK) *pairs = *p;
    return st;
}

}  // namespace mx4p

sqap_status launch_mx4_pair(const Mx4Product& q, cudaStream_t s) {
    using namespace mx4p;
    PairArgs k;
    k.gx = q.gx;
    k.gw = q.gw;
    k.out = q.out;
    k.ldo = q.ldo;
    k.M = q.M;
    k.N = q.N;
    k.K = q.K;
    k.out_dtype = q.out_dtype;
    k.early = q.early ? 1 : 0;
    k.k_tiles = mx4_k_tiles(q.K, q.format);
    k.status = device_status_word();
    if (!k.status) return SQAP_ERR_CUDA;
    if (!device_is_sm100()) return SQAP_ERR_UNSUPPORTED;
    int pairs = 0;
    const sqap_status st = q.format == SQAP_MX_NVFP4 ? resident_pairs<SQAP_MX_NVFP4>(&pairs) : resident_pairs<SQAP_MX_MXFP4>(&pairs);
    if (st != SQAP_OK) return st;
    k.n_tiles = (q.N + 2 * BM - 1) / (2 * BM);
    // Tokens per tile: rounds of tiles over the pairs x bytes per stage, to which its time is nearly proportional (0.25 us at 64 tokens,
    // 0.32 at 192).
    double best = -1.0;
    for (int bn = 64; bn <= BN_MAX; bn += 64) {
        const int mt = (q.M + bn - 1) / bn;
        const long tiles = static_cast<long>(mt) * k.n_tiles;
        const double cost = static_cast<double>((tiles + pairs - 1) / pairs) * (A_BYTES + bn * 64 + 6144);
        if (best < 0 || cost < best) {
            best = cost;
            k.BN = bn;
            k.m_tiles = mt;
        }
    }
    const uint32_t stage_tiles = q.format == SQAP_MX_NVFP4 ? 4 : 2;
    CUtensorMap tm_w, tm_x, tm_wsf, tm_xsf;
    if (!make_map(&tm_w, q.w_codes, q.N, q.K / 2, BM, 128, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_map(&tm_x, q.x_codes, q.M, q.K / 2, k.BN / 2, 128, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_scale_map(&tm_wsf, q.w_scales, static_cast<uint64_t>((q.N + 127) / 128) * k.k_tiles, stage_tiles) ||
        !make_scale_map(&tm_xsf, q.x_scales, static_cast<uint64_t>((q.M + 127) / 128) * k.k_tiles, stage_tiles))
        return SQAP_ERR_CUDA;
    const int tiles = k.m_tiles * k.n_tiles;
    if (tiles < pairs) pairs = tiles;
    const cudaError_t e = q.format == SQAP_MX_NVFP4
                              ? launch_dependent(mx4_pair_kernel<SQAP_MX_NVFP4>, dim3(2 * pairs), dim3(THREADS), SMEM_BYTES, s, tm_w, tm_x, tm_wsf, tm_xsf, k)
                              : launch_dependent(mx4_pair_kernel<SQAP_MX_MXFP4>, dim3(2 * pairs), dim3(THREADS), SMEM_BYTES, s, tm_w, tm_x, tm_wsf, tm_xsf, k);
    if (e != cudaSuccess) {
        note_cuda_error(e);
        cudaGetLastError();
        return SQAP_ERR_CUDA;
    }
    count_launch();
    return check_launch();
}

}  // namespace sqap
