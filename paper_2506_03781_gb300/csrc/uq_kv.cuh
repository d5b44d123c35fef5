// The paged key-value cache: its layout on the device and the arithmetic of
// its rows (see uq_api.h), shared by the kernels that write, read and attend
// over it.
#pragma once

#include "uq_common.cuh"

namespace uq {

constexpr int kKvGroup = 64;                       // channels of an int4 group
constexpr float kKvTiny = 7.888609052210118e-31f;  // 2^-100: smaller ranges are kept as zeros
#define kKvNan __uint_as_float(0x7fffffffu)
constexpr uint32_t kKvNanPair = 0x7fff7fffu;

template <int FMT, int HD>
struct KvRow {
    static constexpr int kBytes = FMT == UQ_KV_BF16 ? 2 * HD : FMT == UQ_KV_INT8 ? HD : HD / 2;
    static constexpr int kWords = FMT == UQ_KV_BF16 ? 0 : FMT == UQ_KV_INT8 ? 1 : HD / kKvGroup;   // 32-bit scale words
};

// 32-bit pairs of bf16, the low half first.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float bf16_low(uint32_t p) { return __uint_as_float(p << 16); }
__device__ __forceinline__ float bf16_high(uint32_t p) { return __uint_as_float(p & 0xffff0000u); }

// max and min that keep a NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float min_nan(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// (x & MASK) | pattern
template <uint32_t MASK>
__device__ __forceinline__ uint32_t masked(uint32_t x, uint32_t pattern) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(x), "n"(MASK), "r"(pattern));
    return r;
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
constexpr uint32_t kKvBf16_128 = 0x43004300u;      // 128 twice: the lowest seven bits count ones
// Two int8 codes in the low bytes of x's halves (the high bytes are ignored) as
// bf16: 128 + the low seven bits, less 128, or 256 where the sign bit is set.
__device__ __forceinline__ uint32_t bf16_of_int8(uint32_t x, uint32_t bf16_128) {
    return sub_bf16x2(masked<0x007f007fu>(x, bf16_128), masked<0x00800080u>(x, bf16_128));
}
// Two int4 codes in the low bits of x's halves as bf16: 128 + code, less `bias`.
__device__ __forceinline__ uint32_t bf16_of_int4(uint32_t x, uint32_t bf16_128, uint32_t bias) {
    return sub_bf16x2(masked<0x000f000fu>(x, bf16_128), bias);
}

}  // namespace uq
