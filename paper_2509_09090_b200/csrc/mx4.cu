// Microscaled 4-bit floating point: the quantizer of a row-major matrix and its inverse.
//
// A number is (e2m1 code) x (scale of its block of 16 or 32 consecutive elements of a row) x (scale of the tensor).
// Both kernels move each element once and do a dozen instructions on it: they are bounded by HBM (2 bytes in and 0.56
// out per fp16 element). One thread owns 16 consecutive elements: two 16-byte loads and one 8-byte store, and the
// maximum of a block of 16 never leaves the thread (a block of 32 takes one shuffle).
#include "mx4.cuh"

namespace sqap {
namespace {

constexpr int THREADS = 256;

template <typename T>
__device__ __forceinline__ void load16(const T* p, float* v);
template <>
__device__ __forceinline__ void load16<__half>(const __half* p, float* v) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint4 u = __ldg(reinterpret_cast<const uint4*>(p) + h);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            v[8 * h + 2 * i] = f.x;
            v[8 * h + 2 * i + 1] = f.y;
        }
    }
}
template <>
__device__ __forceinline__ void load16<__nv_bfloat16>(const __nv_bfloat16* p, float* v) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint4 u = __ldg(reinterpret_cast<const uint4*>(p) + h);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[8 * h + 2 * i] = __uint_as_float(w[i] << 16);
            v[8 * h + 2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}
template <>
__device__ __forceinline__ void load16<float>(const float* p, float* v) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        const float4 f = __ldg(reinterpret_cast<const float4*>(p) + h);
        v[4 * h] = f.x;
        v[4 * h + 1] = f.y;
        v[4 * h + 2] = f.z;
        v[4 * h + 3] = f.w;
    }
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

// One thread = 16 elements. The threads of a row are padded to whole words of four scales, so that the padding
// behind the last block of a row is written as zero.
template <typename T, int FMT>
__global__ void __launch_bounds__(THREADS)
mx4_quantize_kernel(const T* __restrict__ x, int M, int K, int64_t ldx, const int32_t* __restrict__ row_index,
                    const float* __restrict__ tensor_scale, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    constexpr int PER_WORD = FMT == SQAP_MX_NVFP4 ? 4 : 8;   // threads that fill one word of four scales
    const int groups = K / 16, k_tiles = mx4_k_tiles(K, FMT);
    const int g = blockIdx.x * THREADS + threadIdx.x;
    // The wait comes first: the product that follows fetches its weights as soon as it may start, and they can be
    // the output of a kernel in front of this one.
    pdl_wait();
    pdl_launch_dependents();
    const float gs = tensor_scale ? __ldg(tensor_scale) : 1.0f;
    for (int row = blockIdx.y; row < M; row += gridDim.y) {
        const int src = row_index ? __ldg(row_index + row) : row;
        float v[16];
        if (g < groups) load16<T>(x + static_cast<int64_t>(src) * ldx + 16 * g, v);
        else {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = 0.0f;
        }
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) amax = fmaxf(amax, fabsf(v[i]));
        uint32_t sbyte;
        if (FMT == SQAP_MX_NVFP4) {
            // scale = e4m3(amax / 6 / g); the codes are those of x / (scale g)
            sbyte = to_e4m3x2(__fdiv_rn(__fdiv_rn(amax, 6.0f), gs), 0.0f) & 0xFFu;
            const float sc = e4m3_to_float(sbyte);
            const float inv = sc > 0.0f ? __fdiv_rn(1.0f, __fmul_rn(sc, gs)) : 0.0f;
            // Adding and taking away 24 rounds to a multiple of 2^-19: a quotient that lies exactly halfway between
            // two codes, which the rounded reciprocal may miss by an ulp, comes out halfway again.
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = __fadd_rn(__fadd_rn(__fmul_rn(v[i], inv), 24.0f), -24.0f);
        } else {
            amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            // exponent of the scale: floor(log2 amax) - 2, at least -127 (0 as well); 2^-e is then a normal number
            int e = static_cast<int>(__float_as_uint(amax) >> 23) - 127;
            if (e == -127 && amax > 0.0f) e = 31 - __clz(static_cast<int>(__float_as_uint(amax))) - 149;   // subnormal
            e = amax > 0.0f ? max(e - 2, -127) : -127;
            sbyte = static_cast<uint32_t>(e + 127);
            const float inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = __fmul_rn(v[i], inv);
        }
        if (g < groups) {
            const uint2 c = make_uint2(to_e2m1x8(v), to_e2m1x8(v + 8));
            *reinterpret_cast<uint2*>(codes + static_cast<size_t>(row) * (K / 2) + 8 * static_cast<size_t>(g)) = c;
        } else {
            sbyte = 0;
        }
        // four scales of consecutive blocks -> one word
        uint32_t word;
        if (FMT == SQAP_MX_NVFP4) {
            word = sbyte << (8 * (threadIdx.x & 3));
            word |= __shfl_xor_sync(0xffffffffu, word, 1);
            word |= __shfl_xor_sync(0xffffffffu, word, 2);
        } else {
            word = sbyte << (8 * ((threadIdx.x >> 1) & 3));
            word |= __shfl_xor_sync(0xffffffffu, word, 2);
            word |= __shfl_xor_sync(0xffffffffu, word, 4);
        }
        const int kt = g / PER_WORD;
        if (threadIdx.x % PER_WORD == 0 && kt < k_tiles)
            *reinterpret_cast<uint32_t*>(scales + scale_offset(row, 4 * kt, k_tiles)) = word;
    }
}

template <typename T>
__device__ __forceinline__ T from_float(float f);
template <>
__device__ __forceinline__ __half from_float<__half>(float f) { return __float2half_rn(f); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float f) { return __float2bfloat16_rn(f); }
template <>
__device__ __forceinline__ float from_float<float>(float f) { return f; }

// One thread = 8 codes (one 4-byte load) -> 8 numbers (one or two 16-byte stores).
template <typename T, int FMT>
__global__ void __launch_bounds__(THREADS)
mx4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int M, int K,
                      const float* __restrict__ tensor_scale, T* __restrict__ out, int64_t ldo) {
    const int g = blockIdx.x * THREADS + threadIdx.x, k_tiles = mx4_k_tiles(K, FMT);
    pdl_launch_dependents();
    pdl_wait();
    if (8 * g >= K) return;
    const float gs = tensor_scale ? __ldg(tensor_scale) : 1.0f;
    for (int row = blockIdx.y; row < M; row += gridDim.y) {
        const uint32_t c = __ldg(reinterpret_cast<const uint32_t*>(codes + static_cast<size_t>(row) * (K / 2)) + g);
        const uint32_t b = __ldg(scales + scale_offset(row, 8 * g / mx4_block(FMT), k_tiles));
        float sc;
        if (FMT == SQAP_MX_NVFP4) sc = __fmul_rn(e4m3_to_float(b), gs);
        else sc = b ? __uint_as_float(b << 23) : __uint_as_float(0x00400000u);   // 2^(b - 127); 255 (not a number) gives infinity
        alignas(16) T y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t n = (c >> (4 * i)) & 15u, e = (n >> 1) & 3u, m = n & 1u;
            // code magnitude: m/2 for e = 0, else (1 + m/2) 2^(e-1)
            const float mag = e ? __uint_as_float(((126u + e) << 23) | (m << 22)) : 0.5f * static_cast<float>(m);
            y[i] = from_float<T>(__fmul_rn((n & 8u) ? -mag : mag, sc));
        }
        uint4* o = reinterpret_cast<uint4*>(out + static_cast<int64_t>(row) * ldo + 8 * g);
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) o[i] = reinterpret_cast<const uint4*>(y)[i];
    }
}

inline unsigned rows_y(int M) { return static_cast<unsigned>(M < 65535 ? M : 65535); }

template <typename T>
cudaError_t quantize_as(const void* x, int M, int K, int64_t ldx, const int32_t* row_index, int format, const float* tensor_scale,
                        uint8_t* codes, uint8_t* scales, cudaStream_t s) {
    const int per_word = format == SQAP_MX_NVFP4 ? 4 : 8;
    const int lanes = mx4_k_tiles(K, format) * per_word;
    const dim3 grid((lanes + THREADS - 1) / THREADS, rows_y(M));
    if (format == SQAP_MX_NVFP4)
        return launch_dependent(mx4_quantize_kernel<T, SQAP_MX_NVFP4>, grid, dim3(THREADS), 0, s, static_cast<const T*>(x), M, K,
                                ldx, row_index, tensor_scale, codes, scales);
    return launch_dependent(mx4_quantize_kernel<T, SQAP_MX_MXFP4>, grid, dim3(THREADS), 0, s, static_cast<const T*>(x), M, K, ldx,
                            row_index, tensor_scale, codes, scales);
}

template <typename T>
cudaError_t dequantize_as(const uint8_t* codes, const uint8_t* scales, int M, int K, int format, const float* tensor_scale,
                          void* out, int64_t ldo, cudaStream_t s) {
    const dim3 grid((K / 8 + THREADS - 1) / THREADS, rows_y(M));
    if (format == SQAP_MX_NVFP4)
        return launch_dependent(mx4_dequantize_kernel<T, SQAP_MX_NVFP4>, grid, dim3(THREADS), 0, s, codes, scales, M, K,
                                tensor_scale, static_cast<T*>(out), ldo);
    return launch_dependent(mx4_dequantize_kernel<T, SQAP_MX_MXFP4>, grid, dim3(THREADS), 0, s, codes, scales, M, K, tensor_scale,
                            static_cast<T*>(out), ldo);
}

sqap_status finish(cudaError_t e) {
    if (e != cudaSuccess) {
        note_cuda_error(e);
        cudaGetLastError();
        return SQAP_ERR_CUDA;
    }
    count_launch();
    return check_launch();
}

inline bool float_type(int t) { return t == SQAP_FP16 || t == SQAP_BF16 || t == SQAP_FP32; }
inline bool mx4_format(int f) { return f == SQAP_MX_NVFP4 || f == SQAP_MX_MXFP4; }

}  // namespace

sqap_status check_mx4_quantize(const void* x, int x_dtype, int M, int K, int64_t ldx, int format, const void* codes,
                               const void* scales) {
    if (M < 0 || K <= 0 || ldx < K || !float_type(x_dtype) || !mx4_format(format)) return SQAP_ERR_INVALID;
    if (K % 32 != 0 || (ldx * type_bytes(x_dtype)) % 16 != 0) return SQAP_ERR_ALIGN;
    if (M == 0) return SQAP_OK;
    if (!x || !codes || !scales) return SQAP_ERR_INVALID;
    if (!aligned16(x) || !aligned16(codes) || !aligned16(scales)) return SQAP_ERR_ALIGN;
    return SQAP_OK;
}

sqap_status launch_mx4_quantize(const void* x, int x_dtype, int M, int K, int64_t ldx, const int32_t* row_index, int format,
                                const float* tensor_scale, uint8_t* codes, uint8_t* scales, cudaStream_t s) {
    if (x_dtype == SQAP_FP16) return finish(quantize_as<__half>(x, M, K, ldx, row_index, format, tensor_scale, codes, scales, s));
    if (x_dtype == SQAP_BF16) return finish(quantize_as<__nv_bfloat16>(x, M, K, ldx, row_index, format, tensor_scale, codes, scales, s));
    return finish(quantize_as<float>(x, M, K, ldx, row_index, format, tensor_scale, codes, scales, s));
}

}  // namespace sqap

extern "C" size_t sqap_mx4_scale_bytes(int rows, int K, int format) {
    using namespace sqap;
    if (rows <= 0 || K <= 0 || !mx4_format(format)) return 0;
    return (static_cast<size_t>(rows) + 127) / 128 * mx4_k_tiles(K, format) * 512u;
}

extern "C" sqap_status sqap_mx4_quantize(const void* x, int x_dtype, int M, int K, int64_t ldx, const int32_t* row_index,
                                         int format, const float* tensor_scale, uint8_t* codes, uint8_t* scales, void* stream) {
    using namespace sqap;
    const sqap_status st = check_mx4_quantize(x, x_dtype, M, K, ldx, format, codes, scales);
    if (st != SQAP_OK || M == 0) return st;
    return launch_mx4_quantize(x, x_dtype, M, K, ldx, row_index, format, tensor_scale, codes, scales,
                               static_cast<cudaStream_t>(stream));
}

extern "C" sqap_status sqap_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int M, int K, int format,
                                           const float* tensor_scale, void* out, int64_t ldo, int out_dtype, void* stream) {
    using namespace sqap;
    if (M < 0 || K <= 0 || ldo < K || !float_type(out_dtype) || !mx4_format(format)) return SQAP_ERR_INVALID;
    if (K % 32 != 0 || (ldo * type_bytes(out_dtype)) % 16 != 0) return SQAP_ERR_ALIGN;
    if (M == 0) return SQAP_OK;
    if (!codes || !scales || !out) return SQAP_ERR_INVALID;
    if (!aligned16(codes) || !aligned16(scales) || !aligned16(out)) return SQAP_ERR_ALIGN;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (out_dtype == SQAP_FP16) return finish(dequantize_as<__half>(codes, scales, M, K, format, tensor_scale, out, ldo, s));
    if (out_dtype == SQAP_BF16) return finish(dequantize_as<__nv_bfloat16>(codes, scales, M, K, format, tensor_scale, out, ldo, s));
    return finish(dequantize_as<float>(codes, scales, M, K, format, tensor_scale, out, ldo, s));
}
