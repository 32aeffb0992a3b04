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

// The logarithm of a values' scale: that of a power of two is exact (its fraction's is that of 1).
constexpr float kNoScale = -110.f;  // of zero: below every scale, and the sums below stay in fp32
__device__ __forceinline__ float log2_scale(float x) {
    const uint32_t u = __float_as_uint(x);
    float y;
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(__uint_as_float((u & 0x007fffffu) | 0x3f800000u)));
    return x > 0.f ? (float)((int)(u >> 23) - 127) + y : kNoScale;
}

// Weights and the values' scales.  With a row's scores s as exponents of two and v = log2 of the scale of an entry's
// block, the output is sum 2^(s + v) code / sum 2^s.  Both sums are taken against one reference R, the largest s + v
// that the row itself sees (moved once it has been passed by 2^8): a block beside its window, or one without weight,
// takes no digits from the others, however large its scale.  sum 2^(s - R) stays within 2^110 either way, since
// scales lie between 2^-110 and 2^100.
// The weights that meet the codes, 2^(s + v - R), are held 2^7 times as large: fp16 has them between 2^15 and 2^-24, so
// that what is lost is below 2^-32 of the row's largest (weight times scale), and 11 digits are kept down to 2^-21.
// sum 2^(s - R) is their sum times 2^-v, a block at a time, but where a block's scale lies so far below another one's that
// they would leave fp32 while its scores matter: then it comes from exponentials of its own.
// R is kept as a score and the logarithm of a scale: beside large scores (from 2^14 on, where a sum has 10 digits
// left behind the point) their difference is taken before the scales are added.
// A part of an item is left as its own output with the logarithm of its sum, R + log2 sum 2^(s - R), rounded, and what
// the rounding took, so that parts whose references lie far apart can be joined.
constexpr float kWeightUp = 7.f;
constexpr float kWeightTop = 8.f + kWeightUp;  // an exponent above it moves the reference
constexpr float kFarScale = 60.f;              // exponents between scales
constexpr float kLargeScore = 4194304.f;
constexpr float kNoScore = -3e38f;             // a reference before the first entry

__device__ __forceinline__ float code_ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 2^x for a sum that may lie up to 2^110 from one, so that 2^x itself may not be a fp32 number: twice its half
__device__ __forceinline__ float times_ex2(float sum, float x) {
    const float y = code_ex2(0.5f * x);
    return sum * y * y;
}
// What a part is left as: (m, l) for the reference m + v and the sum, `by` for its output
struct PartRef {
    float m, l, by;
};
__device__ __forceinline__ PartRef part_ref(float m, float v, float sum) {
    if (sum == 0.f) return {-INFINITY, 0.f, 0.f};  // (nothing seen)
    float y;
    asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(sum));
    const float a = v + y, all = m + a, l = code_ex2((m - all) + a);
    return {all, l, l / sum * (1.f / (1 << (int)kWeightUp))};
}

}  // namespace pipo
