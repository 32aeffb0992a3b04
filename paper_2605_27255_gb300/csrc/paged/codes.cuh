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

// The power of two that queries of largest magnitude `most` are divided by on their way to fp16: they end below
// 2 and above 2^-126 of themselves (1 for zeros)
__device__ __forceinline__ float query_scale(float most) {
    return most > 0.f ? __uint_as_float(max(__float_as_uint(most) & 0x7f800000u, 0x00800000u)) : 1.f;
}

}  // namespace pipo
