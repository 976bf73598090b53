// Microscaled 4-bit floating point: the quantizer of a row-major matrix and its inverse.
//
// A number is (e2m1 code) x (scale of its block of 16 or 32 consecutive elements of a row) x (scale of the tensor).
// Both kernels move each element once and do a dozen instructions on it: they are bounded by HBM (2 bytes in and 0.56
// out per fp16 element). One thread owns 16 consecutive elements: two 16-byte loads and one 8-byte store, and the
// maximum of a block of 16 never leaves the thread (a block of 32 takes one shuffle). 4608 x 4096 in NVFP4: 12.1 us
// (48 MB, 4.0 TB/s), back 12.5; the two launches in turn 23.1, since the inverse needs the last codes.
#include "mx4_device.cuh"

namespace sqap {
namespace {

constexpr int THREADS = 256;

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
        float v[16], amax = 0.0f;
        if (g < groups) amax = load16<T>(x + static_cast<int64_t>(src) * ldx + 16 * g, v);
        else {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = 0.0f;
        }
        uint32_t sbyte = quantize16<FMT>(v, amax, gs);
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
        const float sc = FMT == SQAP_MX_NVFP4 ? __fmul_rn(scale_value<FMT>(b), gs) : scale_value<FMT>(b);
        alignas(16) T y[8];
        uint32_t h[4];                                // pairs of codes as fp16, exactly
        asm("{\n\t.reg .b8 a, b, c, d;\n\t"
            "mov.b32 {a, b, c, d}, %4;\n\t"
            "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
            "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
            "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
            "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
            : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(c));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
            y[2 * i] = from_float<T>(__fmul_rn(f.x, sc));
            y[2 * i + 1] = from_float<T>(__fmul_rn(f.y, sc));
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
