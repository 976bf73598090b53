// Device routines of the microscaled 4-bit operators: sixteen elements to codes and scale, and the scales' layout.
#pragma once

#include "mx4.cuh"

namespace sqap {

// Sixteen consecutive elements, and the largest magnitude among them (two at a time where they have 16 bits).
template <typename T>
__device__ __forceinline__ float load16(const T* p, float* v);
template <>
__device__ __forceinline__ float load16<__half>(const __half* p, float* v) {
    uint32_t top = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint4 u = __ldg(reinterpret_cast<const uint4*>(p) + h);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            v[8 * h + 2 * i] = f.x;
            v[8 * h + 2 * i + 1] = f.y;
            asm("max.f16x2 %0, %0, %1;" : "+r"(top) : "r"(w[i] & 0x7FFF7FFFu));
        }
    }
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&top));
    return fmaxf(f.x, f.y);
}
template <>
__device__ __forceinline__ float load16<__nv_bfloat16>(const __nv_bfloat16* p, float* v) {
    uint32_t top = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint4 u = __ldg(reinterpret_cast<const uint4*>(p) + h);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[8 * h + 2 * i] = __uint_as_float(w[i] << 16);
            v[8 * h + 2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            asm("max.bf16x2 %0, %0, %1;" : "+r"(top) : "r"(w[i] & 0x7FFF7FFFu));
        }
    }
    return fmaxf(__uint_as_float(top << 16), __uint_as_float(top & 0xFFFF0000u));
}
template <>
__device__ __forceinline__ float load16<float>(const float* p, float* v) {
    float top = 0.0f;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const float4 f = __ldg(reinterpret_cast<const float4*>(p) + h);
        v[4 * h] = f.x;
        v[4 * h + 1] = f.y;
        v[4 * h + 2] = f.z;
        v[4 * h + 3] = f.w;
        top = fmaxf(fmaxf(fmaxf(top, fabsf(f.x)), fmaxf(fabsf(f.y), fabsf(f.z))), fabsf(f.w));
    }
    return top;
}

// Eight numbers -> eight e2m1 codes (round to nearest, ties to even, at most 6), element 0 in the lowest nibble.
__device__ __forceinline__ uint32_t to_e2m1x8(const float* y) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
    return r;
}
// Two e4m3 numbers, `lo` in the low byte (round to nearest even, at most 448).
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float e4m3_to_float(uint32_t b) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(b & 0xFFu)));
    return __half2float(__ushort_as_half(static_cast<unsigned short>(h & 0xFFFFu)));
}

// Byte of (row, block) in the scale array: tiles of 128 rows x 4 blocks, 512 bytes each, row tile major.
__device__ __forceinline__ size_t scale_offset(int row, int block, int k_tiles) {
    return (static_cast<size_t>(row >> 7) * k_tiles + (block >> 2)) * 512u + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

// Sixteen consecutive elements of a row and their largest magnitude: returns the scale byte of their block, and in v what
// their codes are rounded from.
// MXFP4: the block's other half is in the neighbouring lane (lane ^ 1); every lane of the warp calls it.
template <int FMT>
__device__ __forceinline__ uint32_t quantize16(float* v, float amax, float gs) {
    if (FMT == SQAP_MX_NVFP4) {
        // scale = e4m3(amax / 6 / g); the codes are those of x / (scale g)
        const uint32_t sbyte = to_e4m3x2(__fdiv_rn(__fdiv_rn(amax, 6.0f), gs), 0.0f) & 0xFFu;
        const float sc = e4m3_to_float(sbyte);
        const float inv = sc > 0.0f ? __frcp_rn(__fmul_rn(sc, gs)) : 0.0f;
        // Adding and taking away 24 rounds to a multiple of 2^-19: a quotient that lies exactly halfway between two codes,
        // which the rounded reciprocal may miss by an ulp, comes out halfway again.
        // (The additions two at a time; a multiplication in the same form would be contracted with them.)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            float2 y = make_float2(__fmul_rn(v[i], inv), __fmul_rn(v[i + 1], inv));
            asm("{\n\t.reg .b64 y, c;\n\t"
                "mov.b64 y, {%0, %1};\n\t"
                "mov.b64 c, {%2, %2};\n\t"
                "add.rn.f32x2 y, y, c;\n\t"
                "mov.b64 c, {%3, %3};\n\t"
                "add.rn.f32x2 y, y, c;\n\t"
                "mov.b64 {%0, %1}, y;\n\t}"
                : "+f"(y.x), "+f"(y.y) : "f"(24.0f), "f"(-24.0f));
            v[i] = y.x;
            v[i + 1] = y.y;
        }
        return sbyte;
    }
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    // exponent of the scale: floor(log2 amax) - 2, at least -127 (0 as well); 2^-e is then a normal number
    int e = static_cast<int>(__float_as_uint(amax) >> 23) - 127;
    if (e == -127 && amax > 0.0f) e = 31 - __clz(static_cast<int>(__float_as_uint(amax))) - 149;   // subnormal
    e = amax > 0.0f ? max(e - 2, -127) : -127;
    const float inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __fmul_rn(v[i], inv);
    return static_cast<uint32_t>(e + 127);
}
// A scale byte as a number.
template <int FMT>
__device__ __forceinline__ float scale_value(uint32_t b) {
    if (FMT == SQAP_MX_NVFP4) return e4m3_to_float(b);
    return b ? __uint_as_float(b << 23) : __uint_as_float(0x00400000u);   // 2^(b - 127); 255 (not a number) gives infinity
}

}  // namespace sqap
