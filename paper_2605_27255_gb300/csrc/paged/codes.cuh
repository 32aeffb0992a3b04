// 8-bit cache entries: e4m3 codes and the scale that a block of a kv head has.
//
// The append's scales are powers of two between 2^-100 and 2^7, so that multiplying by one rounds
// nothing: codes move to a larger scale exactly, but for those that become
// subnormal, and a code times its scale is a bf16 number.  (A scale from the block's
// maximum over 448 would fit a little tighter, gain nothing for a floating-point code, and
// round every held entry again whenever a later one is larger.)
#pragma once

#include <cuda_fp16.h>

#include "paged.cuh"

namespace pipo {

constexpr int kScaleLow = -100, kScaleHigh = 7;  // exponents
constexpr float kCodeMax = 448.f;                // largest e4m3 value

// The scale of a block whose largest magnitude is `most`: it is left in [32, 64), so that entries
// up to seven times as large can follow without a new scale, and those down to 2^-11 of it
// keep all four digits.
__device__ __forceinline__ float scale_of(float most) {
    const int e = (int)(__float_as_uint(most) >> 23 & 255u) - 127 - 5;  // (0 and subnormals: below kScaleLow)
    return __uint_as_float((uint32_t)(min(max(e, kScaleLow), kScaleHigh) + 127) << 23);
}

// the magnitude that counts for the scale: that of finite values
__device__ __forceinline__ float finite_abs(float x) { return fabsf(x) <= 3.402823466e38f ? fabsf(x) : 0.f; }

// four values as codes, the first one in the low byte; beyond 448 they saturate, NaN stays NaN
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)hi << 16 | lo;
}

// two codes as fp16 (exact)
__device__ __forceinline__ uint32_t decode2(uint16_t x) {
    uint32_t y;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y) : "h"(x));
    return y;
}
__device__ __forceinline__ uint32_t decode_lo(uint32_t w) { return decode2((uint16_t)w); }
__device__ __forceinline__ uint32_t decode_hi(uint32_t w) { return decode2((uint16_t)(w >> 16)); }

// two values as fp16, the first one in the low half
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// four values as e5m2, the first one in the low byte, and two of them back
__device__ __forceinline__ uint32_t encode4_e5m2(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)hi << 16 | lo;
}
__device__ __forceinline__ float2 decode2_e5m2(uint16_t x) {
    uint32_t y;
    asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(y) : "h"(x));
    return __half22float2(*reinterpret_cast<const __half2*>(&y));
}

// 2^e, -126 <= e <= 127
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// The exponent of the power of two that queries of largest magnitude `most` are divided by on their way to formats with
// 5 exponent bits: the largest ends in [2^14, 2^15), a row of tiny ones (below 2^-112) lower, but no further than that
// a bf16 number's last digit, 2^-133, is still 2^-7 (0 for zeros)
__device__ __forceinline__ int query_exponent(float most) {
    return most > 0.f ? max((int)(__float_as_uint(most) >> 23) - 127, -112) - 14 : 0;
}

}  // namespace pipo
