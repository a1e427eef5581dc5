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

// Two binary32 values in one 64-bit register: the arithmetic below runs on pairs, one instruction for both (mul, add and
// fma on pairs round each half like their scalar forms).
struct Pair {
    unsigned long long v;
    __device__ __forceinline__ Pair() {}
    __device__ __forceinline__ Pair(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi)); }
    __device__ __forceinline__ explicit Pair(float both) : Pair(both, both) {}
    __device__ __forceinline__ void split(float& lo, float& hi) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
};
__device__ __forceinline__ Pair operator*(Pair a, Pair b) {
    Pair d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
    return d;
}
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
    return d;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return d;
}

// 1 / (1 + 2^y) and, as `rest`, one minus that: 2^y / (1 + 2^y), not a difference, which would lose the slope's second term
// where the weight is near 1.  2^y overflows to infinity, where the quotient is 0 and so is the limit; `rest` is then the
// largest number times 0, not infinity times 0.
__device__ __forceinline__ Pair logistic2(Pair y, Pair& rest) {
    float a, b, u, v;
    y.split(a, b);
    const float ea = exp2_fast(a), eb = exp2_fast(b);
    (Pair(ea, eb) + Pair(1.0f)).split(u, v);
    const Pair w(reciprocal_fast(u), reciprocal_fast(v));
    rest = Pair(fminf(ea, 3.402823466e38f), fminf(eb, 3.402823466e38f)) * w;      // NaN: w is NaN
    return w;
}

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kGeluTwoC = 1.5957691216057308f;      // 2 sqrt(2/pi)
constexpr float kGeluCubic = 0.044715f;
constexpr float kInvSqrtTwoPi = 0.39894228040143268f;

// Phi(z), the normal distribution function, and bell = exp(-z^2/2):
//   Phi(-x) = bell * t q(t),  t = 1 / (1 + 0.3 x),  x = |z|,
// q the polynomial of degree 7 in t of least relative error on 0 <= x <= 16, fitted to exp(x^2/2) erfc(x / sqrt 2) / 2 in 40
// digits: 4e-8 up to x = 2.5, rising to 8e-7 (of a value below 1e-9) at x = 6.  The sum is about 2.7 times as sensitive to t as
// t is, so the hardware's reciprocal gets a Newton step.  In binary32 the tail is good to some (24 + 2 z^2) 2^-24 of itself,
// gelu and its slope to the rounding of the plain form (0.5 z (1 + erf)) around 0 and far better below -2, without the
// one-signed error that a shorter polynomial leaves in a column sum.  No branches, one exponential that the slope uses too.
__device__ __forceinline__ Pair normal_cdf(float z0, float z1, Pair& bell) {
    float a, b;
    const Pair z(z0, z1);
    // held at 16, where bell is 0: an infinity would make the Newton step 0 * inf (NaN: bell is NaN)
    const Pair d = fma2(Pair(fminf(fabsf(z0), 16.0f), fminf(fabsf(z1), 16.0f)), Pair(0.3f), Pair(1.0f));
    d.split(a, b);
    Pair t(reciprocal_fast(a), reciprocal_fast(b));
    t = fma2(t, fma2(d * Pair(-1.0f), t, Pair(1.0f)), t);
    (z * z * Pair(-0.5f * kLog2e)).split(a, b);
    bell = Pair(exp2_fast(a), exp2_fast(b));
    Pair q = fma2(Pair(0.0366736986f), t, Pair(-0.161047950f));
    q = fma2(q, t, Pair(0.212333053f));
    q = fma2(q, t, Pair(-0.0584820472f));
    q = fma2(q, t, Pair(0.130657554f));
    q = fma2(q, t, Pair(0.0994357392f));
    q = fma2(q, t, Pair(0.120801814f));
    q = fma2(q, t, Pair(0.119628169f));
    const Pair tail = q * t * bell;                               // Phi(-|z|)
    float t0, t1, u0, u1;
    tail.split(t0, t1);
    fma2(tail, Pair(-1.0f), Pair(1.0f)).split(u0, u1);
    return Pair(z0 < 0.0f ? t0 : u0, z1 < 0.0f ? t1 : u1);        // NaN: tail is NaN
}

// Where the weight of a smooth activation, act(z) = z * weight(z), has reached 0 (below -FAR) or 1 (above FAR) in binary32,
// and its derivative 0.
template <int ACT> struct Far { static constexpr float value = ACT == FP8_ACT_SILU ? 100.0f : 16.0f; };

// The weight, and what its derivative takes beside it: gelu the bell, the others one minus the weight.
template <int ACT>
__device__ __forceinline__ Pair weight(float z0, float z1, Pair& other) {
    if (ACT == FP8_ACT_GELU) return normal_cdf(z0, z1, other);
    const Pair z(z0, z1);
    if (ACT == FP8_ACT_GELU_TANH) return logistic2(z * fma2(z * z, Pair(-kLog2e * kGeluTwoC * kGeluCubic), Pair(-kLog2e * kGeluTwoC)), other);
    return logistic2(z * Pair(-kLog2e), other);
}

// weight + z * weight', of a weight and its `other`
template <int ACT>
__device__ __forceinline__ Pair slope_of(Pair z, Pair w, Pair other) {
    if (ACT == FP8_ACT_GELU) return fma2(z * Pair(kInvSqrtTwoPi), other, w);
    const Pair bend = z * w * other;
    if (ACT == FP8_ACT_SILU) return bend + w;
    return fma2(bend, fma2(z * z, Pair(3.0f * kGeluTwoC * kGeluCubic), Pair(kGeluTwoC)), w);
}

// act of two values in place
template <int ACT>
__device__ __forceinline__ void activate(float& z0, float& z1) {
    if (ACT == FP8_ACT_RELU) {
        z0 = z0 < 0.0f ? 0.0f : z0;
        z1 = z1 < 0.0f ? 0.0f : z1;
    } else if (ACT != FP8_ACT_NONE) {
        Pair other;
        const Pair w = weight<ACT>(z0, z1, other);
        // -inf: finite times 0; NaN: the weight is NaN
        (Pair(fmaxf(z0, -Far<ACT>::value), fmaxf(z1, -Far<ACT>::value)) * w).split(z0, z1);
    }
}

// act'(z) alone, of values that are within +-FAR or NaN (relu and none: any values).
template <int ACT>
__device__ __forceinline__ Pair slope_within(float z0, float z1) {
    if (ACT == FP8_ACT_NONE) return Pair(1.0f);
    if (ACT == FP8_ACT_RELU) return Pair(z0 > 0.0f ? 1.0f : 0.0f, z1 > 0.0f ? 1.0f : 0.0f);
    Pair other;
    const Pair w = weight<ACT>(z0, z1, other);
    return slope_of<ACT>(Pair(z0, z1), w, other);
}

// act(z) and act'(z) = weight + z * weight' of two values.  The second term is evaluated at z held within +-FAR, where it
// has vanished, so that it never multiplies an infinity by a zero.
template <int ACT>
__device__ __forceinline__ void activate_with_slope(float z0, float z1, Pair& value, Pair& slope) {
    if (ACT == FP8_ACT_RELU) {
        value = Pair(z0 < 0.0f ? 0.0f : z0, z1 < 0.0f ? 0.0f : z1);
        slope = Pair(z0 > 0.0f ? 1.0f : 0.0f, z1 > 0.0f ? 1.0f : 0.0f);
        return;
    }
    if (ACT == FP8_ACT_NONE) {
        value = Pair(z0, z1);
        slope = Pair(1.0f);
        return;
    }
    constexpr float FAR = Far<ACT>::value;
    const float a0 = fmaxf(z0, -FAR), a1 = fmaxf(z1, -FAR);
    const Pair c(fminf(a0, FAR), fminf(a1, FAR));
    Pair other;
    const Pair w = weight<ACT>(z0, z1, other);
    value = Pair(a0, a1) * w;
    slope = slope_of<ACT>(c, w, other);
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
