// Rotary positions with one or several axes: pairs of elements of every head, turned by position x frequency.
//
// Bounded by HBM: two bytes in and two out per element. The angles belong to the row and not to its heads, so a CTA makes
// the sines and cosines of a block's rows once, in shared memory, while its elements are on their way; a thread then turns the same
// run of pairs in several heads. The angle is formed in 64 bits, as a part of a turn: the frequency in 2^-64 of a turn times the position,
// of which whole turns overflow; a position of a million loses nothing (in fp32 its angle would be off by 0.06). 4608 rows of
// 64 heads of 128, bf16, three axes: 28.1 us, 5.4 TB/s (a plain copy of as many bytes 24.5); 9710 rows of 3 heads of 256, where the sines
// count, 11.7 us; 16 rows of 64 heads 2.2 us. Four units a thread in flight instead of two: 30.9 us; sines and cosines in the order of the
// pairs, so that the lanes of different units meet in the banks: 35.5.
#include <type_traits>

#include "kv.cuh"

namespace sqap {
namespace {

constexpr int THREADS = 128;
constexpr int CTAS = 10;                 // of an SM
constexpr int MOST = 2;                  // units that a thread has in flight
constexpr int MAX_HEAD = 256, MAX_AXES = 8;
constexpr int TABLE_BYTES = 16384;       // sines and cosines of a block's rows, at most, where it has several units a thread

struct RotaryArgs {
    const void* x;
    int64_t ldx;
    void* out;
    int64_t ldo;
    int64_t units;                       // rows x heads
    int heads, head_dim, half;           // half: pairs of a head
    int turning, per_head;               // units of a head that hold pairs, and with those that are only copied
    int by_row, by_head;                 // at_once, in rows and heads
    uint32_t by_per_head, by_half;       // 2^16 / per_head and 2^16 / half, rounded up: quotients of numbers below THREADS without a division
    int touched, table_pairs;            // rows that a block's units can lie in (times the heads 31 bits), and the pairs of these
    int rows_at_once;                    // rows whose pairs the CTA's threads take at once
    int at_once, slots;                  // heads that the CTA's threads take at once, and how often
    const int32_t* positions;
    int64_t ldp;
    const float* freq;
    uint8_t axis[MAX_HEAD / 2];
};

template <int BYTES>
struct Word;
template <>
struct Word<8> { using type = uint2; };
template <>
struct Word<16> { using type = uint4; };

// VEC elements of a run of pairs. Neighbours: a unit is one run of VEC elements (VEC / 2 pairs); otherwise two, half a turning part apart.
template <typename T, int VEC, bool NEIGHBOURS>
__global__ void __launch_bounds__(THREADS, CTAS) rotary_kernel(const __grid_constant__ RotaryArgs a) {
    using W = typename Word<2 * VEC>::type;
    // [row][pair of pairs of a unit][unit]: cosines and sines of two pairs, side by side for the lanes of different units
    extern __shared__ float4 turn[];
    constexpr int PAIRS = NEIGHBOURS ? VEC / 2 : VEC;        // of a unit
    pdl_launch_dependents();
    pdl_wait();
    const int lane_head = threadIdx.x * a.by_per_head >> 16, unit = threadIdx.x - lane_head * a.per_head;
    const bool turns = unit < a.turning;
    const T* x = static_cast<const T*>(a.x);
    T* out = static_cast<T*>(a.out);
    // elements of the unit within its head; units behind the turning ones are copied, eight elements each
    const int e0 = turns ? unit * VEC : 2 * a.half + (unit - a.turning) * 8;
    // A thread keeps to one pair, whose frequency it holds in 2^-64 of a turn: times a position, what passes 64 bits are whole turns.
    const int turn_row = threadIdx.x * a.by_half >> 16, pair = threadIdx.x - turn_row * a.half;
    const int slot = ((pair % PAIRS / 2) * a.turning + pair / PAIRS) * 2 + (pair & 1);
    uint64_t part = 0;
    if (turn_row < a.rows_at_once) {
        const double turns_each = static_cast<double>(__ldg(a.freq + pair)) * 0.15915494309189533577;      // 1 / (2 pi)
        part = __double2ull_rz((turns_each - floor(turns_each)) * 18446744073709551616.0);
    }
    const int32_t* position = a.positions + a.axis[pair] * a.ldp;
    const int per_block = a.at_once * a.slots;

    // A block of (row, head) pairs: its elements on their way, then the angles of its rows, then the turning.
    int64_t row0;
    int head0;
    W u[MOST], v[MOST];
    uint4 same[MOST];
    int row_of[MOST];                    // of the block's rows; -1: no unit
    int64_t to[MOST];
    auto fetch = [&](int64_t first) {
        row0 = first >> 32 ? first / a.heads : static_cast<uint32_t>(first) / static_cast<uint32_t>(a.heads);
        head0 = static_cast<int>(first - row0 * a.heads);
        // rows and heads of the units: by_row rows and by_head heads from one to the next
        int row = (head0 + lane_head) / a.heads, head = head0 + lane_head - row * a.heads;
        const T* from = x + row0 * a.ldx + e0;
#pragma unroll
        for (int k = 0; k < MOST; ++k) {
            const bool there = k < a.slots && lane_head < a.at_once && first + k * a.at_once + lane_head < a.units;
            row_of[k] = there ? row : -1;
            to[k] = (row0 + row) * a.ldo + head * a.head_dim + e0;
            if (there) {
                const T* p = from + row * a.ldx + head * a.head_dim;
                if (turns) {
                    u[k] = *reinterpret_cast<const W*>(p);
                    if (!NEIGHBOURS) v[k] = *reinterpret_cast<const W*>(p + a.half);
                } else if (out != x) {
                    same[k] = *reinterpret_cast<const uint4*>(p);
                }
            }
            row += a.by_row;
            head += a.by_head;
            if (head >= a.heads) {
                head -= a.heads;
                ++row;
            }
        }
    };
    int64_t first = static_cast<int64_t>(blockIdx.x) * per_block;
    fetch(first);
    float4* table = turn;
    while (true) {
        const int64_t left = a.units - first;
        const int last = head0 + static_cast<int>(left < per_block ? left : per_block);
        if (turn_row < a.rows_at_once)
            for (int r = turn_row; r < a.touched && r * a.heads < last; r += a.rows_at_once) {
                const uint64_t at = part * static_cast<uint64_t>(static_cast<int64_t>(__ldg(position + row0 + r)));
                float s, c;
                sincospif(static_cast<float>(static_cast<int32_t>(at >> 32)) * 4.656612873077393e-10f, &s, &c);     // half turns
                reinterpret_cast<float2*>(table)[r * a.half + slot] = make_float2(c, s);
            }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < MOST; ++k) {
            if (row_of[k] < 0) continue;
            T* p = out + to[k];
            if (!turns) {
                if (out != x) *reinterpret_cast<uint4*>(p) = same[k];
                continue;
            }
            const float4* t = table + row_of[k] * (a.half / 2) + unit;
            uint32_t* lo = reinterpret_cast<uint32_t*>(&u[k]);
            uint32_t* hi = reinterpret_cast<uint32_t*>(&v[k]);
            auto wide = [](uint32_t w) {
                if (std::is_same<T, __half>::value) return __half22float2(*reinterpret_cast<const __half2*>(&w));
                return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
            };
#pragma unroll
            for (int i = 0; i < PAIRS / 2; ++i) {
                const float4 cs = t[i * a.turning];
                if (NEIGHBOURS) {
                    const float2 p0 = wide(lo[2 * i]), p1 = wide(lo[2 * i + 1]);
                    lo[2 * i] = kv::pack2<T>(fmaf(p0.x, cs.x, -(p0.y * cs.y)), fmaf(p0.y, cs.x, p0.x * cs.y));
                    lo[2 * i + 1] = kv::pack2<T>(fmaf(p1.x, cs.z, -(p1.y * cs.w)), fmaf(p1.y, cs.z, p1.x * cs.w));
                } else {
                    const float2 p0 = wide(lo[i]), p1 = wide(hi[i]);
                    lo[i] = kv::pack2<T>(fmaf(p0.x, cs.x, -(p1.x * cs.y)), fmaf(p0.y, cs.z, -(p1.y * cs.w)));
                    hi[i] = kv::pack2<T>(fmaf(p1.x, cs.x, p0.x * cs.y), fmaf(p1.y, cs.z, p0.y * cs.w));
                }
            }
            *reinterpret_cast<W*>(p) = u[k];
            if (!NEIGHBOURS) *reinterpret_cast<W*>(p + a.half) = v[k];
        }
        first += static_cast<int64_t>(gridDim.x) * per_block;
        if (first >= a.units) return;
        fetch(first);
        table = table == turn ? turn + a.table_pairs / 2 : turn;         // the other one may still be read
    }
}

template <typename T>
cudaError_t launch_as(const RotaryArgs& a, bool neighbours, unsigned grid, size_t table, cudaStream_t s) {
    if (neighbours) return launch_dependent(rotary_kernel<T, 8, true>, dim3(grid), dim3(THREADS), table, s, a);
    if (a.half % 8 == 0) return launch_dependent(rotary_kernel<T, 8, false>, dim3(grid), dim3(THREADS), table, s, a);
    return launch_dependent(rotary_kernel<T, 4, false>, dim3(grid), dim3(THREADS), table, s, a);
}

}  // namespace
}  // namespace sqap

extern "C" sqap_status sqap_rotary(const void* x, int64_t ldx, int rows, int heads, int head_dim, int rot_dim, const int32_t* positions,
                                   int64_t ldp, int axes, const uint8_t* axis_of, const float* freq, uint32_t flags, void* out,
                                   int64_t ldo, int dtype, void* stream) {
    using namespace sqap;
    if (rows < 0 || heads <= 0 || head_dim <= 0 || rot_dim <= 0 || rot_dim > head_dim || axes <= 0) return SQAP_ERR_INVALID;
    if ((flags & ~SQAP_ROTARY_NEIGHBOURS) || !kv::row_type(dtype)) return SQAP_ERR_INVALID;
    if (head_dim > MAX_HEAD || axes > MAX_AXES) return SQAP_ERR_UNSUPPORTED;
    if (head_dim % 8 != 0 || rot_dim % 8 != 0) return SQAP_ERR_ALIGN;
    const int64_t width = static_cast<int64_t>(heads) * head_dim;
    if (width > 0x7FFFFFFF) return SQAP_ERR_UNSUPPORTED;
    if (ldx < width || ldo < width || ldp < rows) return SQAP_ERR_INVALID;
    if (ldx % 8 != 0 || ldo % 8 != 0) return SQAP_ERR_ALIGN;
    RotaryArgs a;
    for (int i = 0; i < rot_dim / 2; ++i) {
        a.axis[i] = axis_of ? axis_of[i] : 0;
        if (a.axis[i] >= axes) return SQAP_ERR_INVALID;
    }
    if (rows == 0) return SQAP_OK;
    if (!x || !out || !positions || !freq) return SQAP_ERR_INVALID;
    if (!aligned16(x) || !aligned16(out) || (reinterpret_cast<uintptr_t>(positions) & 3u) || (reinterpret_cast<uintptr_t>(freq) & 3u))
        return SQAP_ERR_ALIGN;
    if (x == out && ldx != ldo) return SQAP_ERR_INVALID;
    const bool neighbours = flags & SQAP_ROTARY_NEIGHBOURS;
    a.x = x;
    a.ldx = ldx;
    a.out = out;
    a.ldo = ldo;
    a.units = static_cast<int64_t>(rows) * heads;
    a.heads = heads;
    a.head_dim = head_dim;
    a.half = rot_dim / 2;
    a.turning = neighbours ? rot_dim / 8 : a.half / (a.half % 8 == 0 ? 8 : 4);
    a.per_head = a.turning + (x == out ? 0 : (head_dim - rot_dim) / 8);
    a.at_once = THREADS / a.per_head;
    a.by_per_head = (65536u + a.per_head - 1) / a.per_head;
    a.by_half = (65536u + a.half - 1) / a.half;
    a.rows_at_once = THREADS / a.half;
    a.by_row = a.at_once / heads;
    a.by_head = a.at_once % heads;
    a.positions = positions;
    a.ldp = ldp;
    a.freq = freq;
    // As many units in flight as leave every SM some CTAs, and as the table of the rows that they can touch allows.
    const int64_t waves = a.units / (static_cast<int64_t>(a.at_once) * sm_count() * CTAS);
    a.slots = static_cast<int>(waves < 1 ? 1 : waves < MOST ? waves : MOST);
    auto touched = [&](int slots) {
        const int64_t n = (static_cast<int64_t>(a.at_once) * slots + heads - 2) / heads + 1;
        return static_cast<int>(n < rows ? n : rows);
    };
    while (a.slots > 1 && static_cast<int64_t>(touched(a.slots)) * a.half * 8 > TABLE_BYTES) --a.slots;
    a.touched = touched(a.slots);
    a.table_pairs = a.touched * a.half;
    const int64_t per_block = static_cast<int64_t>(a.at_once) * a.slots, blocks = (a.units + per_block - 1) / per_block;
    const int64_t at_once = static_cast<int64_t>(sm_count()) * CTAS, grid = blocks < at_once ? blocks : at_once;
    const size_t table = static_cast<size_t>(a.table_pairs) * 8 * (blocks > grid ? 2 : 1);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return kv::finish_launch(dtype == SQAP_FP16 ? launch_as<__half>(a, neighbours, static_cast<unsigned>(grid), table, s)
                                                : launch_as<__nv_bfloat16>(a, neighbours, static_cast<unsigned>(grid), table, s));
}
