// AdamW over many tensors in one launch (sm_100a): clipping by a norm that is on the device, decoupled weight decay, moments in
// binary32 or in 8 bits, and the new parameters once more as bf16 or as FP8 codes with their amax.
//
//   g' = g * coef,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// 8-bit moments are E4M3 codes in blocks of 256 with a binary32 scale each, so that a block's largest magnitude is 448: m
// rounded to nearest, and r = sqrt(v) (twice the range of v in the same exponents) rounded up or down with the probability of
// its distance.  To nearest, r would stand still: with b2 near 1 it moves by less than half a step at a time.  An r that is
// not zero keeps at least the smallest code: a divisor must not vanish beside an m that did not.
//
// The arithmetic is rounded operation by operation, in the order written above: a rounding up or down hangs on the last bit, and
// whoever follows the formula in binary32 gets the same moments, scales and codes, and the same parameters but for the few
// quotients that come out a last bit off (none of 8 million; more where the numerator is below 2^-100).
//
// Bound by HBM: every element is read and written once.  A warp takes a block of 256, a lane eight neighbours of it.  268M
// binary32 parameters with bf16 gradients and E4M3 copies: 1124 us with 32-bit moments (6.5 TB/s), 778 us with 8-bit ones (5.2 TB/s:
// 57 instructions per element take half of the issue slots).  288 small tensors, 3M elements: 14.6 us.  With the rate and the step
// count on the device every thread works out the two factors in binary64: a tensor of 77777 elements 5.4 us in a graph, 3.0 without.
#include <cuda_runtime.h>
#include <stdint.h>

#include <cmath>

#include "activation.cuh"
#include "codec.cuh"
#include "common.cuh"
#include "octet.cuh"

namespace fp8b200 {
namespace adamw {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int BLOCK = 256;                                 // elements that share a scale: 8 per lane
constexpr int64_t LEAST_CHUNK = 2048;                      // elements of a tensor handled by one CTA: at least,
constexpr int64_t MOST_CHUNK = 65536;                      // at most, and
constexpr int64_t MOST_CHUNK_32 = 8192;                    // in lists without 8-bit moments (268M parameters 1095 us; 1113 with 16384)
// 80 registers a thread, of which some spill (72 bytes of stores); 2 CTAs would spill nothing, 4 eight times as much (268M parameters
// with 8-bit moments: 704 us with 3 CTAs, 823 with 2, 784 with 4).
constexpr int CTAS_PER_SM = 3;
static_assert(MOST_CHUNK <= 32 * WARPS * BLOCK, "a lane for the scales of each of a warp's blocks");

struct Entry {
    const void* g;
    void* p;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    void* copy;
    const float* copy_scale;
    float* amax;
    int64_t n;
    int64_t first_chunk;
    int64_t number;                                        // of its first element among all: where its random numbers start
    float decay;
    uint8_t g_bf16, p_bf16, state, copy_t;
    uint8_t vectors, has_copy, reserved[2];                // vectors: every address suits the widest access
    uint32_t pad[5];
};
static_assert(sizeof(Entry) == 128, "table layout");

struct Params {
    const Entry* entries;
    const int32_t* chunk_entry;
    int64_t count, chunks, chunk;
    unsigned int* counter;                                 // workspace: [0] CTAs that are done, [4..] amax of each entry
    unsigned int* amax;
    double ln_beta1, ln_beta2, lr;
    float beta1, beta2, rest1, rest2, eps;                 // rest: 1 - beta
    float rate, root2;                                     // lr / (1 - b1^t), 1 / sqrt(1 - b2^t); not used where lr or t is on the device
    float max_norm;
    uint64_t seed;
    int64_t step;
    const float* norm;
    const float* lr_dev;
    int64_t* step_dev;
    int finish;                                            // the last CTA has something to do
};

__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x846CA68Bu;
    return x ^ (x >> 16);
}

// 32 bytes of a lane in one access
__device__ __forceinline__ void ld8(const void* p, uint32_t (&w)[8]) {
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ void st8(void* p, const uint32_t (&w)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
__device__ __forceinline__ uint4 ld4(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint2 ld2(const void* p) {
    uint2 v;
    asm volatile("ld.global.L1::no_allocate.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
    return v;
}

// A lane's share of a block as it lies in memory.
template <bool G_BF16, bool P_BF16, bool CODES> struct Raw {
    static constexpr int STATE = CODES ? 2 : 8;
    uint32_t g[8], p[8], m[STATE], v[STATE];
    float ms, vs;                                           // the block's scales

    // i: the lane's first element
    __device__ __forceinline__ void fetch(const Entry& e, int64_t i) {
        fetch_wide<P_BF16>(e.p, i, p);
        fetch_wide<G_BF16>(e.g, i, g);
        if (CODES) {
            const uint2 a = ld2(reinterpret_cast<const uint8_t*>(e.m) + i), b = ld2(reinterpret_cast<const uint8_t*>(e.v) + i);
            m[0] = a.x; m[1] = a.y; v[0] = b.x; v[1] = b.y;
        } else {
            fetch_wide<false>(e.m, i, *reinterpret_cast<uint32_t(*)[8]>(m));
            fetch_wide<false>(e.v, i, *reinterpret_cast<uint32_t(*)[8]>(v));
        }
    }
    // element by element; `count` of them exist, the others read as 0
    __device__ __forceinline__ void fetch_some(const Entry& e, int64_t i, int count) {
        some_wide<P_BF16>(e.p, i, count, p);
        some_wide<G_BF16>(e.g, i, count, g);
        if (CODES) {
            some_codes(e.m, i, count, m);
            some_codes(e.v, i, count, v);
        } else {
            some_wide<false>(e.m, i, count, *reinterpret_cast<uint32_t(*)[8]>(m));
            some_wide<false>(e.v, i, count, *reinterpret_cast<uint32_t(*)[8]>(v));
        }
    }
    template <bool BF16> static __device__ __forceinline__ void fetch_wide(const void* base, int64_t i, uint32_t (&w)[8]) {
        if (BF16) {
            const uint4 q = ld4(reinterpret_cast<const uint16_t*>(base) + i);
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        } else {
            ld8(reinterpret_cast<const float*>(base) + i, w);
        }
    }
    template <bool BF16> static __device__ __forceinline__ void some_wide(const void* base, int64_t i, int count, uint32_t (&w)[8]) {
#pragma unroll
        for (int j = 0; j < (BF16 ? 4 : 8); ++j) {
            if (BF16) {
                const uint16_t* h = reinterpret_cast<const uint16_t*>(base) + i + 2 * j;
                w[j] = (2 * j < count ? (uint32_t)h[0] : 0u) | (2 * j + 1 < count ? (uint32_t)h[1] << 16 : 0u);
            } else {
                w[j] = j < count ? reinterpret_cast<const uint32_t*>(base)[i + j] : 0u;
            }
        }
    }
    static __device__ __forceinline__ void some_codes(const void* base, int64_t i, int count, uint32_t (&w)[STATE]) {
        const uint8_t* at = reinterpret_cast<const uint8_t*>(base) + i;
        w[0] = w[1] = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j >> 2] |= j < count ? (uint32_t)at[j] << (8 * (j & 3)) : 0u;
    }
};

template <bool BF16>
__device__ __forceinline__ void values(const uint32_t (&w)[8], Pair (&v)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
        v[j] = BF16 ? Pair(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xFFFF0000u)) : Pair(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
}
template <bool BF16>
__device__ __forceinline__ void store_wide(void* base, int64_t i, int count, const uint32_t (&w)[8]) {
    if (count == 8) {
        if (BF16) *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(base) + i) = make_uint4(w[0], w[1], w[2], w[3]);
        else      st8(reinterpret_cast<float*>(base) + i, w);
    } else {                                                // one by one
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j >= (count & 15)) continue;
            if (BF16) reinterpret_cast<uint16_t*>(base)[i + j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
            else      reinterpret_cast<uint32_t*>(base)[i + j] = w[j];
        }
    }
}
__device__ __forceinline__ void store_codes(void* base, int64_t i, int count, uint2 c) {
    uint8_t* at = reinterpret_cast<uint8_t*>(base) + i;
    if (count == 8) {
        *reinterpret_cast<uint2*>(at) = c;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < (count & 15)) at[j] = (uint8_t)((j < 4 ? c.x : c.y) >> (8 * (j & 3)));
    }
}
__device__ __forceinline__ void decode8(const uint32_t* c, Pair scale, Pair (&v)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 a = decode_pair<kE4M3>(j & 1 ? c[j >> 1] >> 16 : c[j >> 1] & 0xFFFFu);
        v[j] = Pair(a.x, a.y) * scale;
    }
}
__device__ __forceinline__ float inverse_root(float x) {     // 2 ulp, of normal numbers
    float y;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Square roots rounded to nearest, of numbers below 2^77: the product x / sqrt(x) of the approximation is corrected by its residual over
// twice the root.  The residual is exact where x is above 2^-101, so it is taken of 2^50 x, which the smallest x brings there; factors of two
// round nothing.  NaN for larger or infinite x.
__device__ __forceinline__ Pair root_nearest(Pair x) {
    float a, b;
    const Pair big = x * Pair(0x1p50f);
    (big + Pair(0x1p-126f)).split(a, b);                    // zero has a root too; every other `big` stays as it is
    const Pair q(inverse_root(a), inverse_root(b));
    const Pair r = x * (q * Pair(0x1p25f));
    return fma2(fma2(r, r * Pair(-0x1p50f), big), q * Pair(0x1p-26f), r);
}
constexpr float MOST_ROOT = 0x1p38f;                        // of what root_nearest is asked for
// Quotients of numbers far from the end of the range, rounded to nearest but for a few: the product with the approximate reciprocal is
// corrected by its residual, which the fused operation gives without error where a is above 2^-100 (Markstein's correction; that the
// reciprocal is not the correctly rounded one leaves a rare last bit).
__device__ __forceinline__ Pair quotient_nearest(Pair a, Pair b) {
    float x, y;
    b.split(x, y);
    const Pair minus(-x, -y);
    const Pair q(reciprocal_fast(x), reciprocal_fast(y));
    const Pair r = a * q;
    return fma2(fma2(minus, r, a), q, r);
}
// The halves added one by one: as an addition of pairs it came out fused with the product before it.
__device__ __forceinline__ Pair sum(Pair a, Pair b) {
    float x, y, z, w;
    a.split(x, y);
    b.split(z, w);
    return Pair(__fadd_rn(x, z), __fadd_rn(y, w));
}
__device__ __forceinline__ void split8(const Pair (&p)[4], float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j].split(v[2 * j], v[2 * j + 1]);
}
// what brings a block's largest magnitude, of 0 or from SMALL on, to 448; 0 for a block of zeros
constexpr float SMALL = 0x1p-119f;
__device__ __forceinline__ float to_448(float most) { return most == 0.0f ? 0.0f : __frcp_rn(most) * 448.0f; }

// Code of y in [0, 448] rounded up with the probability of its distance from the code below: floor(y / step + u), u = chance / 65536.
// Above the smallest normal value (2^-6) the step is an eighth of the power of two below y, and 8 .. 16 steps make up y, so the
// number of steps and the exponent add up to the code; below, the steps themselves are the code.  A y that is not zero gets at
// least code 1.
__device__ __forceinline__ uint32_t encode_chance(float y, uint32_t chance) {
    const uint32_t bits = __float_as_uint(y), e = max(bits & 0x7F800000u, 121u << 23);          // the power of two below y
    const float u = (float)chance * (1.0f / 65536.0f);
    const float steps = fmaf(y, __uint_as_float((257u << 23) - e), u);
    return max((e >> 20) + (uint32_t)steps - 121u * 8u, min(bits, 1u));
}
// Codes of eight at once, words[j] holding the chances of 2j and 2j + 1.  Of normal values the code is what stands above bit 20
// once the chance has been added below it: shifted left by 4 (the exponent's offset of 120 goes as 0x40 on top), the highest byte.
__device__ __forceinline__ uint2 encode8_chance(const float (&y)[8], const uint32_t (&words)[4]) {
    uint32_t c[8];
    const float least = fminf(fminf(fminf(y[0], y[1]), fminf(y[2], y[3])), fminf(fminf(y[4], y[5]), fminf(y[6], y[7])));
    if (least >= 0.015625f) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            c[j] = (__float_as_uint(y[j]) << 4) + __byte_perm(words[j >> 1], 0x40000000u, j & 1 ? 0x7324 : 0x7104);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] = encode_chance(y[j], j & 1 ? words[j >> 1] >> 16 : words[j >> 1] & 0xFFFFu) << 24;
    }
    auto pack = [](uint32_t q, uint32_t t, uint32_t u, uint32_t o) { return __byte_perm(__byte_perm(q, t, 0x0073), __byte_perm(u, o, 0x0073), 0x5410); };
    return make_uint2(pack(c[0], c[1], c[2], c[3]), pack(c[4], c[5], c[6], c[7]));
}

struct Step {
    float coef, rate, root2, lr;                            // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    uint32_t key;
    int skip;
    bool plainly;                                           // the library's root and quotient for all
};

// One block of 256 that is in registers: moments, parameters and what is stored.  i: the lane's first element; count: 8, or what
// the element-wise stores take (16 more for eight of them).  Leaves the new scales in w; returns the largest magnitude among the
// parameters, where there is a copy.
template <bool G_BF16, bool P_BF16, bool CODES>
__device__ __forceinline__ float update_block(const Params& a, const Entry& e, const Step& s, Raw<G_BF16, P_BF16, CODES>& w, int64_t i, int count, float keep,
                                              float copy_scale) {
    Pair p[4], g[4], m[4], v[4], r[4];
    if (!s.skip) {
        values<P_BF16>(w.p, p);
        values<G_BF16>(w.g, g);
        bool fits;                                          // the first moment beside a second one that does; the gradient's share is in s.plainly
        if (CODES) {
            fits = fabsf(w.ms * s.rate) <= 1e14f;           // a code is 448 at most
            decode8(w.m, Pair(w.ms), m);
            decode8(w.v, Pair(w.vs), r);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = r[j] * r[j];
        } else {
            values<false>(*reinterpret_cast<uint32_t(*)[8]>(w.m), m);
            values<false>(*reinterpret_cast<uint32_t(*)[8]>(w.v), v);
            float old[8];
            split8(m, old);
            fits = most8(old) * fabsf(s.rate) <= 1e17f;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const Pair gj = g[j] * Pair(s.coef);
            m[j] = sum(Pair(a.beta1) * m[j], Pair(a.rest1) * gj);
            v[j] = sum(Pair(a.beta2) * v[j], Pair(a.rest2) * gj * gj);
        }
        float f[8], y[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = root_nearest(v[j]);
        split8(r, f);
        float r_top = most8(f);
        // moments or an eps that bring the steps of the root or the quotient near the end of the range, or past it: the library's
        const bool plainly = !(r_top <= MOST_ROOT) || s.plainly || !fits;
        if (plainly) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float x, z;
                v[j].split(x, z);
                r[j] = Pair(__fsqrt_rn(x), __fsqrt_rn(z));
            }
            split8(r, f);
            r_top = most8(f);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const Pair up = Pair(-s.rate) * m[j], down = sum(r[j] * Pair(s.root2), Pair(a.eps));
            Pair change;
            if (plainly) {
                float x, z, b, d;
                up.split(x, z);
                down.split(b, d);
                change = Pair(__fdiv_rn(x, b), __fdiv_rn(z, d));
            } else {
                change = quotient_nearest(up, down);
            }
            p[j] = sum(p[j] * Pair(keep), change);
        }
        if (CODES) {
            split8(m, y);
            // largest magnitudes of the block (a NaN is larger than any number), and each half of the warp one factor
            const float m_most = __uint_as_float(warp_max_u32(__float_as_uint(most8(y)))), r_most = __uint_as_float(warp_max_u32(__float_as_uint(r_top)));
            w.ms = m_most * (1.0f / 448.0f);
            w.vs = r_most * (1.0f / 448.0f);
            float up = to_448((threadIdx.x & 16) ? r_most : m_most);
            if (m_most < SMALL) {
                // The factor would overflow, and the scale is subnormal: codes of m over the scale as it is stored, both brought up by
                // a power of two.  A scale of 0 makes them 0.  (No root of a second moment is that small.)
#pragma unroll
                for (int j = 0; j < 4; ++j) m[j] = m[j] * Pair(0x1p100f);
                if (!(threadIdx.x & 16)) up = w.ms == 0.0f ? 0.0f : __frcp_rn(w.ms * 0x1p100f);
            }
            const Pair m_up(__shfl_sync(0xFFFFFFFFu, up, 0)), r_up(__shfl_sync(0xFFFFFFFFu, up, 16));
#pragma unroll
            for (int j = 0; j < 4; ++j) (m[j] * m_up).split(y[2 * j], y[2 * j + 1]);
            store_codes(e.m, i, count, make_uint2(cvt_quad<kE4M3>(y[0], y[1], y[2], y[3]), cvt_quad<kE4M3>(y[4], y[5], y[6], y[7])));
            uint32_t words[4];
            const uint32_t pair = (uint32_t)((uint64_t)(e.number + i) >> 1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                words[j] = mix((pair + j) * 0x9E3779B1u + s.key);
                (r[j] * r_up).split(y[2 * j], y[2 * j + 1]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = fminf(y[j], 448.0f);
            store_codes(e.v, i, count, encode8_chance(y, words));
        } else {
            uint32_t t[8];
            split8(m, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = __float_as_uint(f[j]);
            store_wide<false>(e.m, i, count, t);
            split8(v, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = __float_as_uint(f[j]);
            store_wide<false>(e.v, i, count, t);
        }
        split8(p, f);
        if (count < 8) {                                    // what is not there stays out of the amax, whatever eps is
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = j < count ? f[j] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (!P_BF16) w.p[j] = __float_as_uint(f[j]);
            else if ((j & 1) == 0) w.p[j >> 1] = pack_bf16(f[j], f[j + 1]);
        }
        store_wide<P_BF16>(e.p, i, count, w.p);
    }
    if (!e.has_copy) return 0.0f;
    float f[8];                                             // of the parameters as stored
    values<P_BF16>(w.p, p);
    split8(p, f);
    if (e.copy_t == FP8_STORE_BF16) {
        uint32_t t[8];
#pragma unroll
        for (int j = 0; j < 8; j += 2) t[j >> 1] = pack_bf16(f[j], f[j + 1]);
        store_wide<true>(e.copy, i, count, t);
        return 0.0f;
    }
    const float top = most8(f);
    store_codes(e.copy, i, count, e.copy_t == FP8_STORE_E4M3 ? encode8_as<kE4M3>(f, top, copy_scale, false) : encode8_as<kE5M2>(f, top, copy_scale, false));
    return top;
}

template <bool G_BF16, bool P_BF16, bool CODES>
__device__ __forceinline__ float update_chunk(const Params& a, const Entry& e, const Step& s, int64_t lo, int64_t n) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float keep = __fsub_rn(1.0f, __fmul_rn(s.lr, e.decay));
    const float copy_scale = e.copy_t >= FP8_STORE_E4M3 && e.has_copy ? __ldg(e.copy_scale) : 1.0f;
    const int whole = e.vectors ? (int)(n / BLOCK) : 0, blocks = (int)((n + BLOCK - 1) / BLOCK);
    using Block = Raw<G_BF16, P_BF16, CODES>;
    auto fetch = [&](Block& w, int b) { w.fetch(e, lo + (int64_t)b * BLOCK + lane * 8); };
    float most = 0.0f;
    auto update = [&](Block& w, int b) {
        most = max_nan(most, update_block<G_BF16, P_BF16, CODES>(a, e, s, w, lo + (int64_t)b * BLOCK + lane * 8, 8, keep, copy_scale));
    };
    // element by element: the last block of a tensor, and all of one whose addresses do not suit vectors
    auto some = [&](Block& w, int b) {
        const int64_t i = lo + (int64_t)b * BLOCK + lane * 8;
        const int count = (int)max((int64_t)0, min((int64_t)8, lo + n - i));
        w.fetch_some(e, i, count);
        most = max_nan(most, update_block<G_BF16, P_BF16, CODES>(a, e, s, w, i, count == 8 ? 16 + 8 : count, keep, copy_scale));
    };
    Block now;
    if (!CODES) {                                           // the warps side by side
        int b = warp;
        for (; b < whole; b += WARPS) {
            fetch(now, b);
            update(now, b);
        }
#pragma unroll 1
        for (; b < blocks; b += WARPS) some(now, b);
        return most;
    }
    // 8-bit moments: a warp has blocks that follow one another, so that their scales are one access, a lane each (one scale at a
    // time, four bytes from and to lines that eight warps shared, cost a quarter of the time: 268M parameters 884 us instead of
    // 663).  The next block is on its way while one is worked on, in the other of two sets of registers; the last turn fetches its
    // own block once more and drops it, as a fetch that may not happen would be waited for at once.
    const int each = (blocks + WARPS - 1) / WARPS, b0 = warp * each, b1 = min(b0 + each, blocks), fast = min(b1, whole);
    if (b0 >= b1) return most;
    float* const ms_at = e.m_scale + lo / BLOCK + b0 + lane;      // chunks are whole blocks
    float* const vs_at = e.v_scale + lo / BLOCK + b0 + lane;
    const bool mine = b0 + lane < b1;
    float ms = mine ? *ms_at : 0.0f, vs = mine ? *vs_at : 0.0f;
    auto scales = [&](Block& w, int b) {
        w.ms = __shfl_sync(0xFFFFFFFFu, ms, b - b0);
        w.vs = __shfl_sync(0xFFFFFFFFu, vs, b - b0);
    };
    auto keep_scales = [&](const Block& w, int b) {
        if (lane == b - b0) { ms = w.ms; vs = w.vs; }
    };
    int b = b0;
    if (b < fast) {
        Block next;
        fetch(now, b);
        while (b < fast) {
            fetch(next, min(b + 1, fast - 1));
            scales(now, b);
            update(now, b);
            keep_scales(now, b);
            if (++b >= fast) break;
            fetch(now, min(b + 1, fast - 1));
            scales(next, b);
            update(next, b);
            keep_scales(next, b);
            ++b;
        }
    }
#pragma unroll 1
    for (; b < b1; ++b) {
        scales(now, b);
        some(now, b);
        keep_scales(now, b);
    }
    if (mine) { *ms_at = ms; *vs_at = vs; }
    return most;
}

// One CTA per chunk.  Its warps go their own ways: each reads the table entry and the step's numbers for itself, and the one
// that is done last counts the CTA.  (With barriers in the place of that a fifth of the warps' time went by waiting at them.)
__global__ void __launch_bounds__(THREADS, CTAS_PER_SM) k_adamw(const Params a) {
    __shared__ Entry entries[WARPS];
    __shared__ unsigned int done, top;
    const int lane = threadIdx.x & 31;
    if (threadIdx.x == 0) done = top = 0u;
    __syncthreads();
    Entry& e = entries[threadIdx.x >> 5];
    // The table is the plan's own: copied to the device before the first call, written by no kernel.
    int entry = -1;
    if ((int64_t)blockIdx.x < a.chunks) {
        entry = a.chunk_entry[blockIdx.x];
        reinterpret_cast<uint32_t*>(&e)[lane] = reinterpret_cast<const uint32_t*>(a.entries + entry)[lane];
        __syncwarp();
    }
    grid_launch_dependents();
    grid_dependency_wait();
    Step s;
    {
        const int64_t t = a.step_dev ? *a.step_dev + 1 : a.step;
        const float norm = a.norm ? *a.norm : 0.0f;
        s.lr = a.lr_dev ? *a.lr_dev : (float)a.lr;
        s.rate = a.rate;
        s.root2 = a.root2;
        s.skip = a.norm && !(fabsf(norm) <= 3.402823466e38f);
        s.coef = !a.norm || norm <= a.max_norm ? 1.0f : a.max_norm / norm;
        if (a.step_dev || a.lr_dev) {
            s.rate = (float)((a.lr_dev ? (double)s.lr : a.lr) / -expm1((double)t * a.ln_beta1));
            s.root2 = (float)(1.0 / sqrt(-expm1((double)t * a.ln_beta2)));
        }
        // a root of MOST_ROOT at most leaves g' at most MOST_ROOT / sqrt(rest2): times the rate, below 1e17 too
        s.plainly = a.eps < 1e-18f || a.eps > 1e18f || !(fabsf(s.rate) * MOST_ROOT <= 1e17f * sqrtf(a.rest2));
        s.key = mix((uint32_t)a.seed ^ mix((uint32_t)(a.seed >> 32) ^ mix((uint32_t)t)));
    }
    float most = 0.0f;
    if (entry >= 0) {
        const int64_t lo = ((int64_t)blockIdx.x - e.first_chunk) * a.chunk, n = min(a.chunk, e.n - lo);
        switch (e.g_bf16 * 4 + e.p_bf16 * 2 + (e.state == FP8_STATE_E4M3 ? 1 : 0)) {
            case 0: most = update_chunk<false, false, false>(a, e, s, lo, n); break;
            case 1: most = update_chunk<false, false, true>(a, e, s, lo, n); break;
            case 2: most = update_chunk<false, true, false>(a, e, s, lo, n); break;
            case 3: most = update_chunk<false, true, true>(a, e, s, lo, n); break;
            case 4: most = update_chunk<true, false, false>(a, e, s, lo, n); break;
            case 5: most = update_chunk<true, false, true>(a, e, s, lo, n); break;
            case 6: most = update_chunk<true, true, false>(a, e, s, lo, n); break;
            default: most = update_chunk<true, true, true>(a, e, s, lo, n); break;
        }
    }
    if (!a.finish) return;
    const uint32_t bits = warp_max_u32(canonical_nan_bits(__float_as_uint(most) & 0x7FFFFFFFu));
    unsigned int last = 0u;
    if (lane == 0) {
        if (bits != 0u) atomicMax(&top, bits);
        __threadfence_block();
        if (atomicAdd(&done, 1u) == WARPS - 1) {
            __threadfence_block();
            const unsigned int all = atomicMax(&top, 0u);
            if (all != 0u && e.amax) atomicMax(a.amax + entry, all);
            __threadfence();
            last = atomicAdd(a.counter, 1u) == gridDim.x - 1 ? 1u : 0u;
        }
    }
    if (!__shfl_sync(0xFFFFFFFFu, last, 0)) return;
    __threadfence();
    for (int64_t i = lane; i < a.count; i += 32) {
        float* out = a.entries[i].amax;
        if (out) *out = __uint_as_float(atomicExch(a.amax + i, 0u));
    }
    if (lane == 0) {
        *a.counter = 0u;
        if (a.step_dev && !s.skip) *a.step_dev += 1;
    }
}

}  // namespace adamw
}  // namespace fp8b200

using namespace fp8b200;

extern "C" {

static bool beta_ok(double b) { return b >= 0.0 && b < 1.0; }
static bool chunk_ok(int64_t n) { return n >= adamw::LEAST_CHUNK && n <= adamw::MOST_CHUNK && n % adamw::LEAST_CHUNK == 0; }

fp8_status fp8_adamw_plan_size(const fp8_adamw_item* items, int64_t count, fp8_adamw_plan* plan) {
    using namespace fp8b200::adamw;
    if (!plan || (count > 0 && !items)) return FP8_ERR_NULL;
    if (count < 0) return FP8_ERR_SHAPE;
    if (count > 0x7FFFFFFF) return FP8_ERR_UNSUPPORTED;
    int64_t total = 0, amaxes = 0, most_chunk = MOST_CHUNK_32;
    for (int64_t i = 0; i < count; ++i) {
        const fp8_adamw_item& it = items[i];
        const bool codes = it.state == FP8_STATE_E4M3;
        if (codes) most_chunk = MOST_CHUNK;
        if ((it.g_t != FP8_F32 && it.g_t != FP8_BF16) || (it.p_t != FP8_F32 && it.p_t != FP8_BF16) || (it.state != FP8_STATE_F32 && !codes) ||
            (it.copy && (it.copy_t < FP8_STORE_BF16 || it.copy_t > FP8_STORE_E5M2)))
            return FP8_ERR_ENUM;
        if (it.n < 0) return FP8_ERR_SHAPE;
        const bool coded = it.copy && it.copy_t >= FP8_STORE_E4M3;
        if (it.n > 0 && (!it.g || !it.p || !it.m || !it.v || (codes && (!it.m_scale || !it.v_scale)))) return FP8_ERR_NULL;
        if ((coded && !it.copy_scale_dev) || (it.copy_amax_dev && !coded && it.n > 0)) return FP8_ERR_NULL;      // an empty copy has no address, but an amax of 0
        const uintptr_t fours = reinterpret_cast<uintptr_t>(it.m_scale) | reinterpret_cast<uintptr_t>(it.v_scale) | reinterpret_cast<uintptr_t>(it.copy_scale_dev) |
                                reinterpret_cast<uintptr_t>(it.copy_amax_dev) |
                                (codes ? 0 : reinterpret_cast<uintptr_t>(it.m) | reinterpret_cast<uintptr_t>(it.v)) |
                                (it.g_t == FP8_F32 ? reinterpret_cast<uintptr_t>(it.g) : 0) | (it.p_t == FP8_F32 ? reinterpret_cast<uintptr_t>(it.p) : 0);
        const uintptr_t twos = reinterpret_cast<uintptr_t>(it.g) | reinterpret_cast<uintptr_t>(it.p) | (it.copy && !coded ? reinterpret_cast<uintptr_t>(it.copy) : 0);
        if ((fours & 3u) || (twos & 1u)) return FP8_ERR_ALIGN;
        if (!(it.weight_decay >= 0.0f && it.weight_decay <= 3.402823466e38f)) return FP8_ERR_UNSUPPORTED;
        if (it.n > (int64_t)1 << 46 || total > (int64_t)1 << 46) return FP8_ERR_UNSUPPORTED;
        total += (it.n + BLOCK - 1) / BLOCK * BLOCK;
        amaxes += it.copy_amax_dev ? 1 : 0;
    }
    // The chunk is the smallest with which the CTAs fill whole rounds of what the GPU holds at a time, as few rounds as there can
    // be: CTAs start together and end together.  The largest chunk says how few: no chunk needs fewer.
    const int64_t at_a_time = (int64_t)sm_count() * CTAS_PER_SM;
    auto chunks_of = [&](int64_t chunk) {
        int64_t n = 0;
        for (int64_t i = 0; i < count; ++i) n += (items[i].n + chunk - 1) / chunk;
        return n;
    };
    const int64_t fewest = chunks_of(most_chunk), rounds = fewest > 0 ? (fewest + at_a_time - 1) / at_a_time : 1;
    int64_t chunk = total / (rounds * at_a_time) / LEAST_CHUNK * LEAST_CHUNK, chunks;
    if (chunk < LEAST_CHUNK) chunk = LEAST_CHUNK;
    while ((chunks = chunks_of(chunk)) > rounds * at_a_time) chunk += LEAST_CHUNK;
    if (chunks > 0x7FFFFFFF) return FP8_ERR_UNSUPPORTED;
    plan->count = count;
    plan->chunks = chunks;
    plan->chunk = chunk;
    plan->amaxes = amaxes;
    plan->table_bytes = (size_t)count * sizeof(Entry) + (size_t)(chunks + 3) / 4 * 16;
    plan->workspace_bytes = 16 + (size_t)count * 4;
    return FP8_OK;
}

fp8_status fp8_adamw_plan_fill(const fp8_adamw_item* items, const fp8_adamw_plan* plan, void* table_host) {
    using namespace fp8b200::adamw;
    if (!plan || (plan->table_bytes > 0 && !table_host) || (plan->count > 0 && !items)) return FP8_ERR_NULL;
    if (!chunk_ok(plan->chunk)) return FP8_ERR_SHAPE;
    Entry* e = reinterpret_cast<Entry*>(table_host);
    int32_t* map = reinterpret_cast<int32_t*>(reinterpret_cast<uint8_t*>(table_host) + plan->count * (int64_t)sizeof(Entry));
    int64_t chunk = 0, number = 0;
    for (int64_t i = 0; i < plan->count; ++i) {
        const fp8_adamw_item& it = items[i];
        const int64_t n = (it.n + plan->chunk - 1) / plan->chunk;
        if (it.n < 0 || chunk + n > plan->chunks) return FP8_ERR_SHAPE;      // not the items the plan was sized for
        Entry& t = e[i];
        t = Entry{};
        t.g = it.g; t.p = it.p; t.m = it.m; t.v = it.v; t.m_scale = it.m_scale; t.v_scale = it.v_scale;
        t.copy = it.copy; t.copy_scale = it.copy_scale_dev; t.amax = it.copy_amax_dev;
        t.n = it.n; t.first_chunk = chunk; t.number = number; t.decay = it.weight_decay;
        t.g_bf16 = it.g_t == FP8_BF16; t.p_bf16 = it.p_t == FP8_BF16;
        t.state = (uint8_t)it.state; t.copy_t = (uint8_t)(it.copy ? it.copy_t : 0); t.has_copy = it.copy ? 1 : 0;
        const bool codes = it.state == FP8_STATE_E4M3, coded = it.copy && it.copy_t >= FP8_STORE_E4M3;
        auto suits = [](const void* p, int eight_bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(eight_bytes - 1)) == 0; };
        t.vectors = suits(it.g, it.g_t == FP8_BF16 ? 16 : 32) && suits(it.p, it.p_t == FP8_BF16 ? 16 : 32) && suits(it.m, codes ? 8 : 32) &&
                    suits(it.v, codes ? 8 : 32) && (!it.copy || suits(it.copy, coded ? 8 : 16));
        for (int64_t j = 0; j < n; ++j) map[chunk + j] = (int32_t)i;
        chunk += n;
        number += (it.n + BLOCK - 1) / BLOCK * BLOCK;
    }
    return chunk == plan->chunks ? FP8_OK : FP8_ERR_SHAPE;
}

fp8_status fp8_adamw_step(const fp8_adamw_plan* plan, const void* table_dev, void* workspace_dev, const fp8_adamw_options* o, void* stream) {
    using namespace fp8b200::adamw;
    if (!plan || !o) return FP8_ERR_NULL;
    if (plan->count < 0 || plan->chunks < 0 || plan->chunks > 0x7FFFFFFF || !chunk_ok(plan->chunk)) return FP8_ERR_SHAPE;
    if (!workspace_dev || (plan->count > 0 && !table_dev)) return FP8_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(table_dev) & 15u) || (reinterpret_cast<uintptr_t>(workspace_dev) & 15u) || (reinterpret_cast<uintptr_t>(o->norm_dev) & 3u) ||
        (reinterpret_cast<uintptr_t>(o->lr_dev) & 3u) || (reinterpret_cast<uintptr_t>(o->step_dev) & 7u))
        return FP8_ERR_ALIGN;
    if (!beta_ok(o->beta1) || !beta_ok(o->beta2) || !(o->eps >= 0.0) || !std::isfinite(o->eps) || (!o->lr_dev && !std::isfinite(o->lr)) ||
        (!o->step_dev && o->step < 1) || (o->norm_dev && !(o->max_norm >= 0.0f)))
        return FP8_ERR_UNSUPPORTED;
    Params a = {};
    a.entries = reinterpret_cast<const Entry*>(table_dev);
    a.chunk_entry = reinterpret_cast<const int32_t*>(reinterpret_cast<const uint8_t*>(table_dev) + plan->count * (int64_t)sizeof(Entry));
    a.count = plan->count; a.chunks = plan->chunks; a.chunk = plan->chunk;
    a.counter = reinterpret_cast<unsigned int*>(workspace_dev);
    a.amax = a.counter + 4;
    a.ln_beta1 = std::log(o->beta1); a.ln_beta2 = std::log(o->beta2); a.lr = o->lr;
    a.beta1 = (float)o->beta1; a.beta2 = (float)o->beta2; a.rest1 = (float)(1.0 - o->beta1); a.rest2 = (float)(1.0 - o->beta2); a.eps = (float)o->eps;
    if (!o->step_dev && !o->lr_dev) {
        a.rate = (float)(o->lr / (1.0 - std::pow(o->beta1, (double)o->step)));
        a.root2 = (float)(1.0 / std::sqrt(1.0 - std::pow(o->beta2, (double)o->step)));
    }
    a.max_norm = o->max_norm; a.seed = o->seed; a.step = o->step;
    a.norm = o->norm_dev; a.lr_dev = o->lr_dev; a.step_dev = o->step_dev;
    a.finish = plan->amaxes > 0 || o->step_dev ? 1 : 0;
    if (plan->chunks == 0 && !a.finish) return FP8_OK;
    const unsigned grid = plan->chunks > 0 ? (unsigned)plan->chunks : 1u;
    if (launch_programmatic(k_adamw, dim3(grid), dim3(THREADS), (cudaStream_t)stream, a) != cudaSuccess) {
        (void)cudaGetLastError();
        return FP8_ERR_CUDA;
    }
    count_launches(1);
    return launch_status();
}

}  // extern "C"
