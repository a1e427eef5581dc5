// Eight consecutive values at a time: magnitudes and FP8 conversion, shared by the fused epilogues and the backward pass.
#pragma once

#include <stdint.h>

#include "activation.cuh"
#include "codec.cuh"

namespace fp8b200 {

__device__ __forceinline__ float max_nan(float a, float b) {      // NaN if either operand is NaN
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// max(|a|, |b|, |c|), NaN if any is NaN
__device__ __forceinline__ float most3(float a, float b, float c) {
    float d;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Largest magnitude, NaN once any value is NaN.
__device__ __forceinline__ float most8(const float (&v)[8]) {
    return most3(most3(v[0], v[1], v[2]), most3(v[3], v[4], v[5]), most3(v[6], v[7], 0.0f));
}

// FP8 codes of eight values of which one is special (or, non-saturating, too large): one at a time, kept small.
__device__ __forceinline__ uint2 encode8_special(const float (&v)[8], float scale_d, bool e4m3, bool nosat) {
    uint64_t codes = 0;
#pragma unroll 1
    for (int i = 7; i >= 0; --i) {
        float x = v[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) x = i == j ? v[j] : x;
        const float y = x * scale_d;
        uint32_t code;
        if (y != y) code = ((__float_as_uint(x) >> 24) & 0x80u) | 0x7Fu;
        else if (e4m3) code = nosat ? encode_scalar<kE4M3, true>(y) : encode_scalar<kE4M3, false>(y);
        else code = nosat ? encode_scalar<kE5M2, true>(y) : encode_scalar<kE5M2, false>(y);
        codes = codes << 8 | code;
    }
    return make_uint2((uint32_t)codes, (uint32_t)(codes >> 32));
}

// Whether the packed hardware convert may be used for values of which `most` is the largest magnitude: all finite and,
// non-saturating, in range.  Scaling is monotonic, so the largest decides for all.
__device__ __forceinline__ bool converts_packed(float most, float scale_d, bool e4m3, bool nosat) {
    const float far = most * fabsf(scale_d);
    const bool over = e4m3 ? far > Fmt<kE4M3>::nosat_limit : far >= Fmt<kE5M2>::nosat_limit;
    return far <= 3.402823466e38f && !(nosat && over);
}

// Codes of v * scale_d; `most` is most8(v).
template <int FMT>
__device__ __forceinline__ uint2 encode8_as(const float (&v)[8], float most, float scale_d, bool nosat) {
    if (__builtin_expect(!converts_packed(most, scale_d, FMT == kE4M3, nosat), 0)) return encode8_special(v, scale_d, FMT == kE4M3, nosat);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; i += 2) (Pair(v[i], v[i + 1]) * Pair(scale_d)).split(y[i], y[i + 1]);
    return make_uint2(cvt_quad<FMT>(y[0], y[1], y[2], y[3]), cvt_quad<FMT>(y[4], y[5], y[6], y[7]));
}

}  // namespace fp8b200
