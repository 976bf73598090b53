// Rotary positions with one or several axes: pairs of elements of every head, turned by position x frequency.
//
// Bounded by HBM: two bytes in and two out per element. The angles belong to the row and not to its heads, so a CTA makes
// the sines and cosines of its rows once, in shared memory, while its elements are on their way; a thread then turns the same
// run of pairs in several heads. The angle is formed in 64 bits, in turns, and only what is left of the whole turns goes to fp32: a
// position of a million loses nothing (in fp32 its angle would be off by 0.06).
#include <type_traits>

#include "kv.cuh"

namespace sqap {
namespace {

constexpr int THREADS = 128;
constexpr int MOST = 4;                  // units that a thread has in flight
constexpr int MAX_HEAD = 256, MAX_AXES = 8;
constexpr int TABLE_BYTES = 32768;       // sines and cosines of a CTA's rows, at most

struct RotaryArgs {
    const void* x;
    int64_t ldx;
    void* out;
    int64_t ldo;
    int64_t units;                       // rows x heads
    int heads, head_dim, half;           // half: pairs of a head
    int turning, per_head;               // units of a head that hold pairs, and with those that are only copied
    int at_once, slots, table_rows;      // heads that the CTA's threads take at once, how often, and the rows they can touch
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
__global__ void __launch_bounds__(THREADS) rotary_kernel(const __grid_constant__ RotaryArgs a) {
    using W = typename Word<2 * VEC>::type;
    extern __shared__ float2 turn[];     // [row][pair]: cosine, sine
    pdl_launch_dependents();
    pdl_wait();
    const int64_t first = static_cast<int64_t>(blockIdx.x) * a.at_once * a.slots;     // (row, head) pairs of this CTA
    const int64_t row0 = first / a.heads;
    const int head0 = static_cast<int>(first - row0 * a.heads);
    const int unit = static_cast<int>(threadIdx.x) % a.per_head, lane_head = static_cast<int>(threadIdx.x) / a.per_head;
    const bool turns = unit < a.turning;
    const T* x = static_cast<const T*>(a.x);
    T* out = static_cast<T*>(a.out);
    // elements of the unit within its head; units behind the turning ones are copied, eight elements each
    const int e0 = turns ? unit * VEC : 2 * a.half + (unit - a.turning) * 8;
    W u[MOST], v[MOST];
    uint4 same[MOST];
    int row_of[MOST], head_of[MOST];
#pragma unroll
    for (int k = 0; k < MOST; ++k) {
        const int h = head0 + k * a.at_once + lane_head;
        row_of[k] = h / a.heads;
        head_of[k] = h - row_of[k] * a.heads;
        if (k >= a.slots || lane_head >= a.at_once || first + k * a.at_once + lane_head >= a.units) row_of[k] = -1;
        if (row_of[k] < 0) continue;
        const T* p = x + (row0 + row_of[k]) * a.ldx + head_of[k] * a.head_dim + e0;
        if (turns) {
            u[k] = *reinterpret_cast<const W*>(p);
            if (!NEIGHBOURS) v[k] = *reinterpret_cast<const W*>(p + a.half);
        } else if (out != x) {
            same[k] = *reinterpret_cast<const uint4*>(p);
        }
    }
    const int64_t rows = a.units / a.heads;
    const int here = static_cast<int>(rows - row0 < a.table_rows ? rows - row0 : a.table_rows);
    for (int i = threadIdx.x; i < here * a.half; i += THREADS) {
        const int r = i / a.half, p = i - r * a.half;
        const double turns_of = static_cast<double>(__ldg(a.positions + a.axis[p] * a.ldp + row0 + r)) * static_cast<double>(__ldg(a.freq + p)) *
                                0.15915494309189533577;                       // 1 / (2 pi)
        float s, c;
        sincospif(static_cast<float>(2.0 * (turns_of - rint(turns_of))), &s, &c);
        turn[i] = make_float2(c, s);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < MOST; ++k) {
        if (row_of[k] < 0) continue;
        T* p = out + (row0 + row_of[k]) * a.ldo + head_of[k] * a.head_dim + e0;
        if (!turns) {
            if (out != x) *reinterpret_cast<uint4*>(p) = same[k];
            continue;
        }
        const float2* t = turn + row_of[k] * a.half + (NEIGHBOURS ? e0 / 2 : e0);
        uint32_t* lo = reinterpret_cast<uint32_t*>(&u[k]);
        uint32_t* hi = reinterpret_cast<uint32_t*>(&v[k]);
        auto wide = [](uint32_t w) {
            if (std::is_same<T, __half>::value) return __half22float2(*reinterpret_cast<const __half2*>(&w));
            return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
        };
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            const float2 p0 = wide(lo[i]);
            if (NEIGHBOURS) {
                const float2 cs = t[i];
                lo[i] = kv::pack2<T>(fmaf(p0.x, cs.x, -(p0.y * cs.y)), fmaf(p0.y, cs.x, p0.x * cs.y));
            } else {
                const float2 p1 = wide(hi[i]), c0 = t[2 * i], c1 = t[2 * i + 1];
                lo[i] = kv::pack2<T>(fmaf(p0.x, c0.x, -(p1.x * c0.y)), fmaf(p0.y, c1.x, -(p1.y * c1.y)));
                hi[i] = kv::pack2<T>(fmaf(p1.x, c0.x, p0.x * c0.y), fmaf(p1.y, c1.x, p0.y * c1.y));
            }
        }
        *reinterpret_cast<W*>(p) = u[k];
        if (!NEIGHBOURS) *reinterpret_cast<W*>(p + a.half) = v[k];
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
    a.positions = positions;
    a.ldp = ldp;
    a.freq = freq;
    // As many units in flight as leave every SM some CTAs, and as the table of the rows that they can touch allows.
    const int64_t waves = a.units / (static_cast<int64_t>(a.at_once) * sm_count() * 8);
    a.slots = static_cast<int>(waves < 1 ? 1 : waves < MOST ? waves : MOST);
    auto touched = [&](int slots) {
        const int64_t n = (static_cast<int64_t>(a.at_once) * slots + heads - 2) / heads + 1;
        return static_cast<int>(n < rows ? n : rows);
    };
    while (a.slots > 1 && static_cast<int64_t>(touched(a.slots)) * a.half * 8 > TABLE_BYTES) --a.slots;
    a.table_rows = touched(a.slots);
    const int64_t per_cta = static_cast<int64_t>(a.at_once) * a.slots, grid = (a.units + per_cta - 1) / per_cta;
    if (grid > 0x7FFFFFFF) return SQAP_ERR_UNSUPPORTED;
    const size_t table = static_cast<size_t>(a.table_rows) * a.half * 8;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return kv::finish_launch(dtype == SQAP_FP16 ? launch_as<__half>(a, neighbours, static_cast<unsigned>(grid), table, s)
                                                : launch_as<__nv_bfloat16>(a, neighbours, static_cast<unsigned>(grid), table, s));
}
