// Internal interface of the microscaled 4-bit operators (mx4.cu: quantizer and its inverse; mx4_linear.cu: product).
#pragma once

#include "common.cuh"

namespace sqap {

// Elements that share a scale.
inline __host__ __device__ int mx4_block(int format) { return format == SQAP_MX_NVFP4 ? 16 : 32; }
// 512-byte scale tiles (128 rows x 4 blocks) along K.
inline __host__ __device__ int mx4_k_tiles(int K, int format) { return (K / mx4_block(format) + 3) / 4; }

// Rows of any of the accepted input types -> codes and scales (arguments checked by the caller).
sqap_status launch_mx4_quantize(const void* x, int x_dtype, int M, int K, int64_t ldx, const int32_t* row_index, int format,
                                const float* tensor_scale, uint8_t* codes, uint8_t* scales, cudaStream_t s);
sqap_status check_mx4_quantize(const void* x, int x_dtype, int M, int K, int64_t ldx, int format, const void* codes,
                               const void* scales);

// One product (arguments checked by the caller). early: the kernel in front of it in the stream is this library's activation
// quantizer, which lets its dependents start only after its own dependency wait. Whatever wrote the weights has then
// completed, and they may be fetched while the quantizer still runs. Without it the weights may be the output of the kernel
// right in front.
struct Mx4Product {
    const uint8_t *x_codes, *x_scales, *w_codes, *w_scales;
    const float *gx, *gw;
    void* out;
    int64_t ldo;
    int M, N, K, format, out_dtype;
    bool early;
};
// The weight stream for a handful of tokens (mx4_gemv.cu). x: rows that it quantizes itself (x_codes and x_scales are then not
// read), or null.
constexpr int MX4_GEMV_MAX_ROWS = 4;
bool mx4_gemv_takes(int M, int N, int K, int format);
sqap_status launch_mx4_gemv(const Mx4Product& q, const void* x, int x_dtype, int64_t ldx, const int32_t* row_index, cudaStream_t s);
// The kernel for many tokens (mx4_pair.cu).
sqap_status launch_mx4_pair(const Mx4Product& q, cudaStream_t s);

inline int type_bytes(int dtype) { return dtype == SQAP_FP32 ? 4 : 2; }

}  // namespace sqap
