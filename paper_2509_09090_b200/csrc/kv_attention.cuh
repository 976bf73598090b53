// Internal: what the attention kernels over the 8-bit cache share.
#pragma once

#include "kv.cuh"

namespace sqap {
namespace kv {

// For one query row and its keys t:   s_t = (q . k_t) * scale,   out = sum_t 2^(s_t log2 e) v_t / sum_t 2^(s_t log2 e).
// The codes enter the matrix instructions as they are (exact in fp16); the scale of a page's keys multiplies its scores, and
// the scale of its values goes into the exponent:  w_t = 2^(s_t log2 e + log2 vs - m) is the weight of the value CODES, with m
// the running maximum of the whole exponent, so w_t <= 1 whatever the scales are and fp16 holds it to 11 bits; the
// denominator adds w_t / vs. A page of zero values adds to the denominator alone, and must not raise m: that would push the other
// pages' weights into the subnormals of fp16. It is given a scale below all others: values of fp16 rows have scales of 2^-32 to
// 2^9, and 2^-60 leaves 28 binary orders in which its own probability may be the larger one. Smaller still, and fp32 would lose
// its w_t (which ends at 2^-126) where the denominator needs it: with 2^-60, next to scales of 2^9, below 2^-57 of the others.
constexpr float ZERO_PAGE_SCALE = 8.673617379884035e-19f;   // 2^-60

struct AttnArgs {
    Cache c;
    const int32_t* table;
    int64_t ldt;
    int batch;
    const int32_t* lens;
    const int32_t* cu;
    int max_q, max_len;
    const void* q;
    int64_t ldq;
    int heads, group;      // query heads, and how many of them share a key/value head
    float scale_log2;      // scale * log2 e
    int causal;
    void* out;
    int64_t ldo;
    float* lse;            // [rows][heads] or null
    int splits, chunk;     // a history is cut into `splits` pieces of `chunk` keys, or one
    float* part_o;         // [batch][heads][max_q][splits][D]
    float2* part_ml;       // the same without D: maximum and denominator
    int tiles;             // row tiles per (sequence, key/value head)
};

// Work of a CTA, from its index.
struct Where {
    int b, h, split, tile;
    int row0, n_q;         // first row of the sequence, its query rows
    int tokens, len;       // its tokens, and how many of them are looked at (max_len at most)
};
__device__ __forceinline__ Where locate(const AttnArgs& a, unsigned id, int tiles) {
    Where w;
    w.tile = w.split = 0;
    if (tiles > 1) {
        w.tile = static_cast<int>(id % tiles);
        id /= tiles;
    }
    if (a.splits > 1) {
        w.split = static_cast<int>(id % a.splits);
        id /= a.splits;
    }
    w.h = static_cast<int>(id % a.c.kv_heads);
    w.b = static_cast<int>(id / a.c.kv_heads);
    w.row0 = a.cu[w.b];
    const int n = a.cu[w.b + 1] - w.row0;
    w.n_q = n < 0 ? 0 : n;
    const int len = a.lens[w.b];
    w.tokens = len < 0 ? 0 : len;
    w.len = min(w.tokens, a.max_len);
    return w;
}
// Keys that query i of the sequence may look at (the first so many).
__device__ __forceinline__ int visible(const AttnArgs& a, const Where& w, int i) {
    if (!a.causal) return w.len;
    const int64_t n = static_cast<int64_t>(w.tokens) - w.n_q + i + 1;
    return n < 0 ? 0 : static_cast<int>(min(n, static_cast<int64_t>(w.len)));
}
__device__ __forceinline__ int64_t part_index(const AttnArgs& a, int b, int head, int i, int split) {
    return ((static_cast<int64_t>(b) * a.heads + head) * a.max_q + i) * a.splits + split;
}
// Largest power of two not above 2^9 / amax, so that amax lands in [2^8, 2^9): rows of bf16 then fit fp16 with 22 binary
// orders below their largest element, more than an fp32 sum resolves.
__device__ __forceinline__ float fit_exponent(float amax, float* back) {
    int e = static_cast<int>(__float_as_uint(amax) >> 23) - 127;
    if (!(amax > 0.0f) || e > 127) e = 8;
    e = max(e, -110);
    *back = __uint_as_float(static_cast<uint32_t>(127 + e - 8) << 23);
    return __uint_as_float(static_cast<uint32_t>(127 - e + 8) << 23);
}

__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// ln of 2^m l, l > 0. The exponent of l meets m before the logarithm of its mantissa does: the exponents of the pages' scales, which
// both contain, then cancel without a rounding at their size. An l that is not finite is the answer.
__device__ __forceinline__ float log_sum(float m, float l) {
    if (!(l < INFINITY)) return l;
    const uint32_t b = __float_as_uint(l);
    return (m + static_cast<float>(static_cast<int>(b >> 23) - 127) + log2f(__uint_as_float((b & 0x7FFFFFu) | 0x3F800000u))) * 0.69314718055994531f;
}
__device__ __forceinline__ void mma_16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

template <typename T>
__device__ __forceinline__ float to_f(T x);
template <>
__device__ __forceinline__ float to_f<__half>(__half x) { return __half2float(x); }
template <>
__device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

// Few query rows per key/value head (kv_decode.cu) and many: head_dim 64 and 128 (kv_prefill_tc.cu), 256 (kv_prefill.cu).
// With 256 elements a lane cannot hold the output of more than 8 rows in registers.
// Rows per key/value head up to which the register kernel takes the call. That / the prompt kernel, us, 16 sequences: 4 rows, 32 heads
// of 64, 290 keys 9.1 / 26, 4096 keys 53 / 245; 8 rows, 32 heads of 128, 290 keys 12.5 / 30.6; 8 rows, 32 heads of 256, 290 keys 20 / 69.
// 9 to 16 rows, 8 heads of 128: 100 keys 8.3 / 9.4, 500 keys 14.7 / 16.1, 2048 keys 31 / 44, 32 sequences of 16384 182 / 526, 64 of 290
// 21 / 34. The other sign only where 128 CTAs walk some 290 keys in one round, 14.2 / 12.6, which no rule of its own was made for.
inline int decode_max_rows(int head_dim) { return head_dim == 256 ? 8 : 16; }
constexpr int PREFILL_ROWS = 128, PREFILL_TC_ROWS = 256;   // query rows of a CTA's item
sqap_status launch_kv_decode(const AttnArgs& a, int type, int dtype, cudaStream_t s);
sqap_status launch_kv_prefill_tc(const AttnArgs& a, int type, int dtype, cudaStream_t s);
sqap_status launch_kv_prefill(const AttnArgs& a, int type, int dtype, cudaStream_t s);

}  // namespace kv
}  // namespace sqap
