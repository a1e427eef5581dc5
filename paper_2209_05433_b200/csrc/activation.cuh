// Activation functions of the fused epilogues and their derivatives, in binary32.
//   relu       max(z, 0)
//   gelu       z Phi(z),  Phi(z) = (1 + erf(z / sqrt 2)) / 2
//   gelu_tanh  z (1 + tanh t) / 2 = z s(2t),  t = sqrt(2/pi) (z + 0.044715 z^3),  s(x) = 1 / (1 + exp(-x))
//   silu       z s(z)
// The logistic form of the tanh approximation needs no subtraction of nearly equal numbers.  At -inf the functions
// give their limit 0 (not 0 * inf); NaN stays NaN.
#pragma once

#include <cuda_runtime.h>

#include "../../include/fp8_b200.h"

namespace fp8b200 {

// 2^x and 1/x by the hardware's approximations (2 and 1 ulp).  Results below the normal range become 0, which is what the
// callers want of a vanishing weight; the library forms that keep subnormals cost four more instructions each.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float reciprocal_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 1 / (1 + 2^y); 2^y overflows to infinity, where the quotient is 0 and so is the limit.
__device__ __forceinline__ float logistic2(float y) { return reciprocal_fast(1.0f + exp2_fast(y)); }

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kGeluTwoC = 1.5957691216057308f;      // 2 sqrt(2/pi)
constexpr float kGeluCubic = 0.044715f;
constexpr float kInvSqrtTwoPi = 0.39894228040143268f;

// Phi(z), the normal distribution function, and bell = exp(-z^2/2).  Rational approximation 7.1.26 of Abramowitz and
// Stegun, Handbook of Mathematical Functions (absolute error of erf below 1.5e-7, half of that for Phi):
//   erfc(x) = t (a1 + t (a2 + t (a3 + t (a4 + t a5)))) exp(-x^2),  t = 1 / (1 + 0.3275911 x),  x = |z| / sqrt 2.
// No branches, one exponential that the derivative uses too (the library's erff takes two paths of a dozen terms).
__device__ __forceinline__ float normal_cdf(float z, float& bell) {
    const float t = reciprocal_fast(fmaf(0.3275911f * 0.70710678118654752f, fabsf(z), 1.0f));
    bell = exp2_fast(-0.5f * kLog2e * z * z);
    float q = fmaf(0.5f * 1.061405429f, t, -0.5f * 1.453152027f);
    q = fmaf(q, t, 0.5f * 1.421413741f);
    q = fmaf(q, t, -0.5f * 0.284496736f);
    q = fmaf(q, t, 0.5f * 0.254829592f);
    const float tail = q * t * bell;                              // Phi(-|z|)
    return z < 0.0f ? tail : 1.0f - tail;                         // NaN: tail is NaN
}

// Weight of the smooth activations, act(z) = z * weight(z), at any z.  FAR: where the weight has reached 0 (below -FAR)
// or 1 (above FAR) in binary32, and its derivative 0.
template <int ACT> struct Far { static constexpr float value = ACT == FP8_ACT_SILU ? 100.0f : 16.0f; };

template <int ACT>
__device__ __forceinline__ float activate(float z) {
    if (ACT == FP8_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == FP8_ACT_NONE) return z;
    float w, bell;
    if (ACT == FP8_ACT_GELU) w = normal_cdf(z, bell);
    else if (ACT == FP8_ACT_GELU_TANH) w = logistic2(z * fmaf(-kLog2e * kGeluTwoC * kGeluCubic * z, z, -kLog2e * kGeluTwoC));
    else w = logistic2(-kLog2e * z);
    return fmaxf(z, -Far<ACT>::value) * w;                        // -inf: finite times 0; NaN: the weight is NaN
}

// act(z) and act'(z) = weight + z * weight'.  The second term is evaluated at z held within +-FAR, where it has vanished,
// so that it never multiplies an infinity by a zero.
template <int ACT>
__device__ __forceinline__ void activate_with_slope(float z, float& value, float& slope) {
    if (ACT == FP8_ACT_RELU) {
        value = z < 0.0f ? 0.0f : z;
        slope = z > 0.0f ? 1.0f : 0.0f;
        return;
    }
    if (ACT == FP8_ACT_NONE) {
        value = z;
        slope = 1.0f;
        return;
    }
    const float above = fmaxf(z, -Far<ACT>::value), c = fminf(above, Far<ACT>::value);
    if (ACT == FP8_ACT_GELU) {
        float bell;
        const float w = normal_cdf(z, bell);
        value = above * w;
        slope = fmaf(c * kInvSqrtTwoPi, bell, w);
    } else if (ACT == FP8_ACT_GELU_TANH) {
        const float w = logistic2(z * fmaf(-kLog2e * kGeluTwoC * kGeluCubic * z, z, -kLog2e * kGeluTwoC));
        value = above * w;
        slope = fmaf(c * w * (1.0f - w), fmaf(3.0f * kGeluTwoC * kGeluCubic * c, c, kGeluTwoC), w);
    } else {
        const float w = logistic2(-kLog2e * z);
        value = above * w;
        slope = fmaf(c * w, 1.0f - w, w);
    }
}

// Calls f with the activation as a compile-time constant: f(std::integral_constant-like tag).  `act` is uniform over
// the grid, so the branch costs one comparison per call.
template <int V> struct ActTag { static constexpr int value = V; };
template <typename F>
__device__ __forceinline__ void with_activation(int act, F&& f) {
    switch (act) {
        case FP8_ACT_RELU: f(ActTag<FP8_ACT_RELU>{}); break;
        case FP8_ACT_GELU: f(ActTag<FP8_ACT_GELU>{}); break;
        case FP8_ACT_GELU_TANH: f(ActTag<FP8_ACT_GELU_TANH>{}); break;
        case FP8_ACT_SILU: f(ActTag<FP8_ACT_SILU>{}); break;
        default: f(ActTag<FP8_ACT_NONE>{}); break;
    }
}

}  // namespace fp8b200
