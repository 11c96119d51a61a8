// Elementwise arithmetic of the dense products: operand types, the activations of the gated block
// and their slopes, all in fp32.
#pragma once

#include "device_common.h"

namespace bsr {

struct bf16 {
    unsigned short bits;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16 x) { return bf16_bits_to_float(x.bits); }

// fp32 -> bf16, nearest with ties to even (the compiler's conversion: v_cvt_pk_bf16_f32).
__device__ __forceinline__ bf16 to_bf16(float x) {
    const __bf16 h = static_cast<__bf16>(x);
    bf16 r;
    __builtin_memcpy(&r, &h, 2);
    return r;
}
template <class T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float x) { return to_bf16(x); }

// exp(x) for -88 <= x <= 88 (its correction would make a NaN of an infinity), to about 2 ulp: 2^p with
// p = x log2(e) rounded, times 1 + ln(2) r for the part r of the product that the rounding dropped
// (log2(e) in two parts).
__device__ __forceinline__ float fast_exp(float x) {
    constexpr float kLog2e = 1.44269502162933349609f, kLog2eLow = 1.92596299112661746887e-8f;
    const float p = x * kLog2e;
    const float r = fmaf(x, kLog2eLow, fmaf(x, kLog2e, -p));
    const float e = __builtin_amdgcn_exp2f(p);
    return fmaf(e, r * 0.693147182464599609375f, e);
}

// 1 / (1 + exp(-z)), to about 4 ulp for z > -87.3, where it is 2^-126, and 0 below: the reciprocal gives
// nothing smaller, so that the largest -g times it is 0 too.  The hardware's exponential and reciprocal (1
// ulp each): with expf and a division the epilogue of a 256 x 256 tile took a tenth of the tile's time.
__device__ __forceinline__ float sigmoid(float z) {
    return __builtin_amdgcn_rcpf(1.0f + fast_exp(__builtin_amdgcn_fmed3f(-z, -88.0f, 88.0f)));
}

constexpr float kSqrtHalf = 0.70710678118654752f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;
constexpr float kTwoSqrt2OverPi = 1.5957691216057308f;   // 2 sqrt(2 / pi)
constexpr float kGeluCubic = 0.044715f;

// act(g).  GELU's normal distribution function is erfc(-g / sqrt 2) / 2, which keeps its relative
// accuracy for negative g where 1 + erf cancels; its tanh form is g sigmoid(2 z) with
// 1 + tanh z = 2 sigmoid(2 z), which does not cancel either.
template <int ACT> __device__ __forceinline__ float activate(float g) {
    if constexpr (ACT == BSR_ACT_SILU) return g * sigmoid(g);
    if constexpr (ACT == BSR_ACT_GELU) return 0.5f * g * erfcf(-kSqrtHalf * g);
    if constexpr (ACT == BSR_ACT_GELU_TANH)
        return g * sigmoid(kTwoSqrt2OverPi * g * (1.0f + kGeluCubic * g * g));
    return g <= 0.0f ? 0.0f : g;   // a NaN stays one
}

// act(g) and its slope.
template <int ACT> __device__ __forceinline__ void activate_slope(float g, float &a, float &da) {
    if constexpr (ACT == BSR_ACT_SILU) {
        const float p = sigmoid(g);
        a = g * p;
        da = p * (1.0f + g * (1.0f - p));
    } else if constexpr (ACT == BSR_ACT_GELU) {
        const float p = 0.5f * erfcf(-kSqrtHalf * g);
        a = g * p;
        da = p + g * kInvSqrt2Pi * expf(-0.5f * g * g);
    } else if constexpr (ACT == BSR_ACT_GELU_TANH) {
        const float p = sigmoid(kTwoSqrt2OverPi * g * (1.0f + kGeluCubic * g * g));
        a = g * p;
        // g^2 held below 10^4, where p (1 - p) is 0 from |g| = 11 on: 0 times an infinite square is NaN
        const float gg = fminf(g * g, 1e4f);
        da = p + g * p * (1.0f - p) * kTwoSqrt2OverPi * (1.0f + 3.0f * kGeluCubic * gg);
    } else {
        a = g <= 0.0f ? 0.0f : g;
        da = g > 0.0f ? 1.0f : (g <= 0.0f ? 0.0f : g);
    }
}

}  // namespace bsr
