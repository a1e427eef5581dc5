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
// The moments' arithmetic is rounded operation by operation, in the order written above, and the root of an 8-bit one
// correctly: a rounding up or down hangs on the last bit, and whoever follows the formula gets the same codes.
//
// Bound by HBM: every element is read and written once.  A warp takes a block of 256, a lane eight neighbours of it.
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
constexpr int64_t MOST_CHUNK = 32768, LEAST_CHUNK = 2048;  // elements of a tensor handled by one CTA

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

// Eight values from element i on; `count` of them exist (the others read as 0).
template <bool BF16>
__device__ __forceinline__ void load_wide(const void* base, int64_t i, int count, bool vectors, uint32_t (&w)[8]) {
    if (vectors && count == 8) {
        if (BF16) {
            const uint4 q = ld4(reinterpret_cast<const uint16_t*>(base) + i);
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        } else {
            ld8(reinterpret_cast<const float*>(base) + i, w);
        }
    } else {
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
}
template <bool BF16>
__device__ __forceinline__ void values(const uint32_t (&w)[8], float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = BF16 ? __uint_as_float(j & 1 ? w[j >> 1] & 0xFFFF0000u : w[j >> 1] << 16) : __uint_as_float(w[j]);
}
template <bool BF16>
__device__ __forceinline__ void store_wide(void* base, int64_t i, int count, bool vectors, const uint32_t (&w)[8]) {
    if (vectors && count == 8) {
        if (BF16) *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(base) + i) = make_uint4(w[0], w[1], w[2], w[3]);
        else      st8(reinterpret_cast<float*>(base) + i, w);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j >= count) continue;
            if (BF16) reinterpret_cast<uint16_t*>(base)[i + j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
            else      reinterpret_cast<uint32_t*>(base)[i + j] = w[j];
        }
    }
}
__device__ __forceinline__ uint2 load_codes(const void* base, int64_t i, int count, bool vectors) {
    const uint8_t* at = reinterpret_cast<const uint8_t*>(base) + i;
    if (vectors && count == 8) return ld2(at);
    uint64_t c = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) c |= j < count ? (uint64_t)at[j] << (8 * j) : 0ull;
    return make_uint2((uint32_t)c, (uint32_t)(c >> 32));
}
__device__ __forceinline__ void store_codes(void* base, int64_t i, int count, bool vectors, uint2 c) {
    uint8_t* at = reinterpret_cast<uint8_t*>(base) + i;
    if (vectors && count == 8) {
        *reinterpret_cast<uint2*>(at) = c;
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < count) at[j] = (uint8_t)((j < 4 ? c.x : c.y) >> (8 * (j & 3)));
}
__device__ __forceinline__ void decode8(uint2 c, float scale, float (&v)[8]) {
    const float2 a = decode_pair<kE4M3>(c.x & 0xFFFFu), b = decode_pair<kE4M3>(c.x >> 16), d = decode_pair<kE4M3>(c.y & 0xFFFFu), e = decode_pair<kE4M3>(c.y >> 16);
    v[0] = a.x * scale; v[1] = a.y * scale; v[2] = b.x * scale; v[3] = b.y * scale;
    v[4] = d.x * scale; v[5] = d.y * scale; v[6] = e.x * scale; v[7] = e.y * scale;
}
__device__ __forceinline__ float root(float x) {             // 1 ulp
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// largest magnitude of the warp's eight values each; NaN if any is NaN
__device__ __forceinline__ float warp_most(const float (&v)[8]) {
    return __uint_as_float(warp_max_u32(canonical_nan_bits(__float_as_uint(most8(v)) & 0x7FFFFFFFu)));
}
// what brings a block's largest magnitude to 448; 0 for a block of zeros
__device__ __forceinline__ float to_448(float most) { return most == 0.0f ? 0.0f : fminf(__frcp_rn(most) * 448.0f, 3.402823466e38f); }

// Code of y in [0, 448] rounded up with the probability of its distance from the code below: floor(y / step + u) for 0 <= u < 1.
// Above the smallest normal value (2^-6) the step is an eighth of the power of two below y, and 8 .. 16 steps make up y, so the
// number of steps and the exponent add up to the code; below, the steps themselves are the code.
__device__ __forceinline__ uint32_t encode_chance(float y, float u) {
    const uint32_t e = max(__float_as_uint(y) >> 23, 121u);
    const float steps = fmaf(y, __uint_as_float((257u - e) << 23), u);
    return ((e - 121u) << 3) + (uint32_t)steps;
}

struct Step {
    float coef, rate, root2, lr;                            // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    uint32_t key;
    int skip;
};

template <bool G_BF16, bool P_BF16, bool CODES>
__device__ __forceinline__ float update_chunk(const Params& a, const Entry& e, const Step& s, int64_t lo, int64_t n) {
    const int lane = threadIdx.x & 31;
    const bool vectors = e.vectors != 0;
    const float keep = fmaf(-s.lr, e.decay, 1.0f);
    const float copy_scale = e.copy_t >= FP8_STORE_E4M3 && e.has_copy ? __ldg(e.copy_scale) : 1.0f;
    float most = 0.0f;
    for (int64_t b = (int64_t)(threadIdx.x >> 5) * BLOCK; b < n; b += WARPS * BLOCK) {
        const int64_t i = lo + b + lane * 8;
        const int count = (int)max((int64_t)0, min((int64_t)8, n - b - lane * 8));
        uint32_t wg[8], wp[8], wm[8], wv[8];
        uint2 cm, cv;
        float ms = 0.0f, vs = 0.0f;
        load_wide<P_BF16>(e.p, i, count, vectors, wp);
        float p[8];
        if (!s.skip) {
            load_wide<G_BF16>(e.g, i, count, vectors, wg);
            if (CODES) {
                cm = load_codes(e.m, i, count, vectors);
                cv = load_codes(e.v, i, count, vectors);
                ms = e.m_scale[(lo + b) / BLOCK];
                vs = e.v_scale[(lo + b) / BLOCK];
            } else {
                load_wide<false>(e.m, i, count, vectors, wm);
                load_wide<false>(e.v, i, count, vectors, wv);
            }
            float g[8], m[8], v[8], r[8];
            values<P_BF16>(wp, p);
            values<G_BF16>(wg, g);
            if (CODES) {
                decode8(cm, ms, m);
                decode8(cv, vs, r);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = r[j] * r[j];
            } else {
                values<false>(wm, m);
                values<false>(wv, v);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float gj = g[j] * s.coef;
                m[j] = __fadd_rn(__fmul_rn(a.beta1, m[j]), __fmul_rn(a.rest1, gj));
                v[j] = __fadd_rn(__fmul_rn(a.beta2, v[j]), __fmul_rn(__fmul_rn(a.rest2, gj), gj));
                r[j] = CODES ? __fsqrt_rn(v[j]) : root(v[j]);
                p[j] = fmaf(p[j], keep, -s.rate * m[j] * reciprocal_fast(fmaf(r[j], s.root2, a.eps)));
            }
            if (count < 8) {                                // what is not there stays out of the amax, whatever eps is
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] = j < count ? p[j] : 0.0f;
            }
            if (CODES) {
                const float m_most = warp_most(m), r_most = warp_most(r);
                const float m_up = to_448(m_most), r_up = to_448(r_most);
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = m[j] * m_up;
                store_codes(e.m, i, count, vectors, make_uint2(cvt_quad<kE4M3>(y[0], y[1], y[2], y[3]), cvt_quad<kE4M3>(y[4], y[5], y[6], y[7])));
                uint32_t c[2] = {0u, 0u};
                const uint32_t pair = (uint32_t)((uint64_t)(e.number + i) >> 1);
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const uint32_t word = mix((pair + j / 2) * 0x9E3779B1u + s.key);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float u = __uint_as_float(0x3F800000u | (h ? word >> 16 << 7 : (word & 0xFFFFu) << 7)) - 1.0f;
                        const uint32_t code = max(encode_chance(fminf(r[j + h] * r_up, 448.0f), u), r[j + h] > 0.0f ? 1u : 0u);
                        c[j >> 2] |= code << (8 * ((j + h) & 3));
                    }
                }
                store_codes(e.v, i, count, vectors, make_uint2(c[0], c[1]));
                if (lane == 0) {
                    e.m_scale[(lo + b) / BLOCK] = m_most * (1.0f / 448.0f);
                    e.v_scale[(lo + b) / BLOCK] = r_most * (1.0f / 448.0f);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) { wm[j] = __float_as_uint(m[j]); wv[j] = __float_as_uint(v[j]); }
                store_wide<false>(e.m, i, count, vectors, wm);
                store_wide<false>(e.v, i, count, vectors, wv);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (!P_BF16) wp[j] = __float_as_uint(p[j]);
                else if ((j & 1) == 0) wp[j >> 1] = pack_bf16(p[j], p[j + 1]);
            }
            store_wide<P_BF16>(e.p, i, count, vectors, wp);
        }
        if (e.has_copy) {                                   // of the parameters as stored
            values<P_BF16>(wp, p);
            if (e.copy_t == FP8_STORE_BF16) {
                uint32_t w[8];
#pragma unroll
                for (int j = 0; j < 8; j += 2) w[j >> 1] = pack_bf16(p[j], p[j + 1]);
                store_wide<true>(e.copy, i, count, vectors, w);
            } else {
                const float top = most8(p);
                most = max_nan(most, top);
                store_codes(e.copy, i, count, vectors, e.copy_t == FP8_STORE_E4M3 ? encode8_as<kE4M3>(p, top, copy_scale, false)
                                                                                   : encode8_as<kE5M2>(p, top, copy_scale, false));
            }
        }
    }
    return most;
}

__global__ void __launch_bounds__(THREADS, 3) k_adamw(const Params a) {
    __shared__ Entry e;
    __shared__ Step s;
    __shared__ uint32_t red[WARPS];
    __shared__ unsigned int last;
    // The table is the plan's own: copied to the device before the first call, written by no kernel.
    int entry = -1;
    if ((int64_t)blockIdx.x < a.chunks) {
        entry = a.chunk_entry[blockIdx.x];
        if (threadIdx.x < 32) reinterpret_cast<uint32_t*>(&e)[threadIdx.x] = reinterpret_cast<const uint32_t*>(a.entries + entry)[threadIdx.x];
    }
    grid_launch_dependents();
    grid_dependency_wait();
    if (threadIdx.x == 0) {
        const int64_t t = a.step_dev ? *a.step_dev + 1 : a.step;
        const float lr = a.lr_dev ? *a.lr_dev : (float)a.lr;
        const float norm = a.norm ? *a.norm : 0.0f;
        s.skip = a.norm && !(fabsf(norm) <= 3.402823466e38f);
        s.coef = !a.norm || norm <= a.max_norm ? 1.0f : a.max_norm / norm;
        // 1 - b^t without cancellation
        const float c1 = -expm1f((float)((double)t * a.ln_beta1)), c2 = -expm1f((float)((double)t * a.ln_beta2));
        s.lr = lr;
        s.rate = lr / c1;
        s.root2 = 1.0f / sqrtf(c2);
        s.key = mix((uint32_t)a.seed ^ mix((uint32_t)(a.seed >> 32) ^ mix((uint32_t)t)));
    }
    __syncthreads();
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
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = bits;
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t top = 0u;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) top = max(top, red[w]);
        if (top != 0u && e.amax) atomicMax(a.amax + entry, top);
        __threadfence();
        last = atomicAdd(a.counter, 1u) == gridDim.x - 1 ? 1u : 0u;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    for (int64_t i = threadIdx.x; i < a.count; i += THREADS) {
        float* out = a.entries[i].amax;
        if (out) *out = __uint_as_float(atomicExch(a.amax + i, 0u));
    }
    if (threadIdx.x == 0) {
        *a.counter = 0u;
        if (a.step_dev && !s.skip) *a.step_dev += 1;
    }
}

}  // namespace adamw
}  // namespace fp8b200

using namespace fp8b200;

extern "C" {

static bool beta_ok(double b) { return b >= 0.0 && b < 1.0; }

fp8_status fp8_adamw_plan_size(const fp8_adamw_item* items, int64_t count, fp8_adamw_plan* plan) {
    using namespace fp8b200::adamw;
    if (!plan || (count > 0 && !items)) return FP8_ERR_NULL;
    if (count < 0) return FP8_ERR_SHAPE;
    if (count > 0x7FFFFFFF) return FP8_ERR_UNSUPPORTED;
    int64_t total = 0, amaxes = 0;
    for (int64_t i = 0; i < count; ++i) {
        const fp8_adamw_item& it = items[i];
        const bool codes = it.state == FP8_STATE_E4M3;
        if ((it.g_t != FP8_F32 && it.g_t != FP8_BF16) || (it.p_t != FP8_F32 && it.p_t != FP8_BF16) || (it.state != FP8_STATE_F32 && !codes) ||
            (it.copy && (it.copy_t < FP8_STORE_BF16 || it.copy_t > FP8_STORE_E5M2)))
            return FP8_ERR_ENUM;
        if (it.n < 0) return FP8_ERR_SHAPE;
        const bool coded = it.copy && it.copy_t >= FP8_STORE_E4M3;
        if (it.n > 0 && (!it.g || !it.p || !it.m || !it.v || (codes && (!it.m_scale || !it.v_scale)))) return FP8_ERR_NULL;
        if ((coded && !it.copy_scale_dev) || (it.copy_amax_dev && !coded)) return FP8_ERR_NULL;
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
    // Short lists are cut finer: about eight CTAs for each of 148 SMs.
    int64_t chunk = MOST_CHUNK;
    while (chunk > LEAST_CHUNK && total / chunk < 148 * 8) chunk /= 2;
    int64_t chunks = 0;
    for (int64_t i = 0; i < count; ++i) chunks += (items[i].n + chunk - 1) / chunk;
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
    if (plan->chunk < LEAST_CHUNK) return FP8_ERR_SHAPE;
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
    if (plan->count < 0 || plan->chunks < 0 || plan->chunks > 0x7FFFFFFF || plan->chunk < LEAST_CHUNK) return FP8_ERR_SHAPE;
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
