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

// 1 / (1 + exp(-x)): exp overflows to infinity below -88, where the quotient is 0 and so is the limit.
__device__ __forceinline__ float logistic(float x) { return __fdividef(1.0f, 1.0f + __expf(-x)); }

// z times a weight that vanishes towards -inf
__device__ __forceinline__ float gated_by(float z, float weight) { return weight == 0.0f ? 0.0f : z * weight; }

constexpr float kGeluTwoC = 1.5957691216057308f;      // 2 sqrt(2/pi)
constexpr float kGeluCubic = 0.044715f;
constexpr float kInvSqrtTwoPi = 0.39894228040143268f;

// Phi(z), the normal distribution function, and density_scaled = exp(-z^2/2).  Rational approximation 7.1.26 of Abramowitz
// and Stegun, Handbook of Mathematical Functions (absolute error of erf below 1.5e-7, half of that for Phi):
//   erfc(x) = t (a1 + t (a2 + t (a3 + t (a4 + t a5)))) exp(-x^2),  t = 1 / (1 + 0.3275911 x),  x = |z| / sqrt 2.
// No branches, one exponential that the derivative uses too (the library's erff takes two paths of a dozen terms).
__device__ __forceinline__ float normal_cdf(float z, float& density_scaled) {
    const float t = __fdividef(1.0f, fmaf(0.3275911f * 0.70710678118654752f, fabsf(z), 1.0f));
    density_scaled = __expf(-0.5f * z * z);
    float q = fmaf(1.061405429f, t, -1.453152027f);
    q = fmaf(q, t, 1.421413741f);
    q = fmaf(q, t, -0.284496736f);
    q = fmaf(q, t, 0.254829592f);
    const float tail = 0.5f * q * t * density_scaled;             // Phi(-|z|)
    return z < 0.0f ? tail : 1.0f - tail;                         // NaN: tail is NaN
}

template <int ACT>
__device__ __forceinline__ float activate(float z) {
    if (ACT == FP8_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == FP8_ACT_GELU) {
        float e;
        return gated_by(z, normal_cdf(z, e));
    }
    if (ACT == FP8_ACT_GELU_TANH) return gated_by(z, logistic(kGeluTwoC * z * fmaf(kGeluCubic * z, z, 1.0f)));
    if (ACT == FP8_ACT_SILU) return gated_by(z, logistic(z));
    return z;
}

// act(z) and act'(z).  The second term of the derivative is evaluated at z held within +-LIMIT, where it has long
// vanished, so that it never multiplies an infinity by a zero.
template <int ACT>
__device__ __forceinline__ void activate_with_slope(float z, float& value, float& slope) {
    if (ACT == FP8_ACT_RELU) {
        value = z < 0.0f ? 0.0f : z;
        slope = z > 0.0f ? 1.0f : 0.0f;
    } else if (ACT == FP8_ACT_GELU) {
        const float c = fminf(fmaxf(z, -16.0f), 16.0f);           // the density has long vanished there
        float e;
        const float w = normal_cdf(z, e);
        value = gated_by(z, w);
        slope = fmaf(c * kInvSqrtTwoPi, e, w);
    } else if (ACT == FP8_ACT_GELU_TANH) {
        const float c = fminf(fmaxf(z, -16.0f), 16.0f);
        const float w = logistic(kGeluTwoC * z * fmaf(kGeluCubic * z, z, 1.0f));
        value = gated_by(z, w);
        slope = fmaf(c * w * (1.0f - w), kGeluTwoC * fmaf(3.0f * kGeluCubic * c, c, 1.0f), w);
    } else if (ACT == FP8_ACT_SILU) {
        const float c = fminf(fmaxf(z, -100.0f), 100.0f);
        const float w = logistic(z);
        value = gated_by(z, w);
        slope = fmaf(c * w, 1.0f - w, w);
    } else {
        value = z;
        slope = 1.0f;
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
