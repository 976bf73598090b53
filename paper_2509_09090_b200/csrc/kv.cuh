// Internal: the paged 8-bit key/value cache as the kernels see it, conversions and checks.
#pragma once

#include <type_traits>

#include "common.cuh"

namespace sqap {
namespace kv {

// One of the two halves of the cache (keys or values): codes [pages][kv_heads][page_tokens][head_dim], scales [pages][kv_heads].
struct Half {
    uint8_t* codes;
    float* scales;
};
struct Cache {
    Half k, v;
    int pages, kv_heads, page_shift, head_dim;
};

// Scales smaller than this are stored as 0 (int8) or as this (e4m3): the reciprocals that the kernels form stay normal.
constexpr float MIN_SCALE = 7.888609052210118e-31f;   // 2^-100
constexpr int MIN_EXP = -100;

inline int page_shift_of(int page_tokens) {
    switch (page_tokens) {
        case 16: return 4;
        case 32: return 5;
        case 64: return 6;
        case 128: return 7;
    }
    return -1;
}

inline sqap_status check_cache(const sqap_kv_cache* c) {
    if (!c || c->pages < 0 || c->kv_heads <= 0 || c->head_dim <= 0) return SQAP_ERR_INVALID;
    if (c->type != SQAP_KV_INT8 && c->type != SQAP_KV_E4M3) return SQAP_ERR_INVALID;
    if (page_shift_of(c->page_tokens) < 0) return SQAP_ERR_UNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return SQAP_ERR_UNSUPPORTED;
    if (c->kv_heads > 65535 || static_cast<int64_t>(c->kv_heads) * c->head_dim > (1 << 24)) return SQAP_ERR_UNSUPPORTED;
    if (c->pages == 0) return SQAP_OK;
    if (!c->k || !c->v || !c->k_scale || !c->v_scale) return SQAP_ERR_INVALID;
    if (!aligned16(c->k) || !aligned16(c->v)) return SQAP_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(c->k_scale) & 3u) || (reinterpret_cast<uintptr_t>(c->v_scale) & 3u)) return SQAP_ERR_ALIGN;
    return SQAP_OK;
}
inline Cache device_view(const sqap_kv_cache* c) {
    Cache d;
    d.k = {static_cast<uint8_t*>(c->k), c->k_scale};
    d.v = {static_cast<uint8_t*>(c->v), c->v_scale};
    d.pages = c->pages;
    d.kv_heads = c->kv_heads;
    d.page_shift = page_shift_of(c->page_tokens);
    d.head_dim = c->head_dim;
    return d;
}
// Product of sizes (none negative), at most 2^62: where 64 bits do not hold it, it is too large for every limit that it is held against.
template <typename... I>
inline int64_t size_product(I... sizes) {
    constexpr int64_t TOP = int64_t{1} << 62;
    int64_t p = 1;
    for (const int64_t s : {static_cast<int64_t>(sizes)...})
        if (__builtin_mul_overflow(p, s, &p) || p > TOP) p = TOP;
    return p;
}
inline bool row_type(int t) { return t == SQAP_FP16 || t == SQAP_BF16; }
inline sqap_status finish_launch(cudaError_t e) {
    if (e != cudaSuccess) {
        note_cuda_error(e);
        cudaGetLastError();
        return SQAP_ERR_CUDA;
    }
    count_launch();
    return check_launch();
}

#ifdef __CUDACC__
// Codes of head h of a page (64-bit offsets: a cache easily passes 2^32 bytes).
__device__ __forceinline__ int64_t page_codes(const Cache& c, int page, int h) {
    return (static_cast<int64_t>(page) * c.kv_heads + h) << c.page_shift;   // in tokens; times head_dim bytes
}
// A page number out of the table; -1 for anything that is not a page of the cache.
__device__ __forceinline__ int checked_page(const Cache& c, int page) { return page >= 0 && page < c.pages ? page : -1; }

// fp16x2 of two e4m3 codes in the low 16 bits.
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(two)));
    return h;
}
// fp16x2 of bytes 0 and 1 (or 2 and 3) of a word of int8 codes with their sign bits flipped (code + 128): the byte becomes
// the low mantissa bits of 1024 + 128 + code, exactly; then 1152 is taken off.
template <int HI>
__device__ __forceinline__ uint32_t biased_to_half2(uint32_t w) {
    const uint32_t h = __byte_perm(w, 0x64646464u, HI ? 0x4342 : 0x4140);
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&h), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// Eight codes -> eight numbers (without the scale).
template <int TYPE>
__device__ __forceinline__ void decode8(uint2 w, float* v) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t u = i ? w.y : w.x;
        uint32_t a, b;
        if (TYPE == SQAP_KV_INT8) {
            a = biased_to_half2<0>(u ^ 0x80808080u);
            b = biased_to_half2<1>(u ^ 0x80808080u);
        } else {
            a = e4m3x2_to_half2(u & 0xFFFFu);
            b = e4m3x2_to_half2(u >> 16);
        }
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&a)), g = __half22float2(*reinterpret_cast<const __half2*>(&b));
        v[4 * i] = f.x;
        v[4 * i + 1] = f.y;
        v[4 * i + 2] = g.x;
        v[4 * i + 3] = g.y;
    }
}
// Largest magnitude of eight 16-bit floats, as a pair to be folded by the caller; exact, a NaN loses.
template <typename T>
__device__ __forceinline__ void widen8(uint4 u, uint32_t* top) {
    const uint32_t w[4] = {u.x & 0x7FFF7FFFu, u.y & 0x7FFF7FFFu, u.z & 0x7FFF7FFFu, u.w & 0x7FFF7FFFu};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (std::is_same<T, __half>::value) asm("max.f16x2 %0, %0, %1;" : "+r"(*top) : "r"(w[i]));
        else asm("max.bf16x2 %0, %0, %1;" : "+r"(*top) : "r"(w[i]));
    }
}
template <typename T>
__device__ __forceinline__ float fold_pair(uint32_t top) {
    if (std::is_same<T, __half>::value) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&top));
        return fmaxf(f.x, f.y);
    }
    return fmaxf(__uint_as_float(top << 16), __uint_as_float(top & 0xFFFF0000u));
}
// Eight numbers, already divided by the scale (magnitude 127 or 448 at most, by a rounding or two) -> eight codes.
// int8: adding 1.5 * 2^23 leaves the nearest whole number, ties to even, in the low bits; its low byte is the code.
template <int TYPE>
__device__ __forceinline__ uint2 encode8(const float* y) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (TYPE == SQAP_KV_INT8) {
            uint32_t b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = __float_as_uint(__fadd_rn(y[4 * i + j], 12582912.0f));
            w[i] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
        } else {
            uint16_t a, b;
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(a) : "f"(y[4 * i]), "f"(y[4 * i + 1]));
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(b) : "f"(y[4 * i + 2]), "f"(y[4 * i + 3]));
            w[i] = a | (static_cast<uint32_t>(b) << 16);
        }
    }
    return make_uint2(w[0], w[1]);
}
// Eight codes without not-a-numbers (e4m3 has them, 0x7F and 0xFF; they become zeros): a weight of 0 times one would reach rows that do
// not see it. A byte's low seven bits plus one carry into its top bit for 0x7F alone.
template <int TYPE>
__device__ __forceinline__ uint2 finite_codes(uint2 w) {
    if (TYPE == SQAP_KV_INT8) return w;
    const uint32_t x = ((w.x & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u, y = ((w.y & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
    if (x | y) {
        w.x &= ~((x >> 7) * 0x7Fu);
        w.y &= ~((y >> 7) * 0x7Fu);
    }
    return w;
}
template <typename T>
__device__ __forceinline__ float largest();
template <>
__device__ __forceinline__ float largest<__half>() { return 65504.0f; }
template <>
__device__ __forceinline__ float largest<__nv_bfloat16>() { return __uint_as_float(0x7F7F0000u); }
// Scale of a block whose largest magnitude is amax.
template <int TYPE>
__device__ __forceinline__ float scale_for(float amax) {
    if (TYPE == SQAP_KV_INT8) {
        const float s = __fdiv_rn(amax, 127.0f);
        return s < MIN_SCALE ? 0.0f : s;
    }
    if (!(amax > 0.0f)) return 0.0f;
    // the smallest power of two that brings amax to 448 = 0.875 * 2^9 or below
    const uint32_t b = __float_as_uint(amax);
    const int e = static_cast<int>(b >> 23) - 126;                 // amax = m 2^e, 0.5 <= m < 1 (normal amax)
    int x = e - 9 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);         // m > 0.875
    x = x < MIN_EXP ? MIN_EXP : x;
    return __uint_as_float(static_cast<uint32_t>(x + 127) << 23);
}
__device__ __forceinline__ float inverse_of(float scale) { return scale > 0.0f ? __frcp_rn(scale) : 0.0f; }

template <typename T>
__device__ __forceinline__ void unpack8(uint4 u, float* v);
template <>
__device__ __forceinline__ void unpack8<__half>(uint4 u, float* v) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
template <>
__device__ __forceinline__ void unpack8<__nv_bfloat16>(uint4 u, float* v) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename T>
__device__ __forceinline__ uint4 pack8(const float* v) {
    return make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
}
#endif

}  // namespace kv
}  // namespace sqap
