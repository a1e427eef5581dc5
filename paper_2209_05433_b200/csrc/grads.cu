// Gradient passes around the products (sm_100a): the backward pass of the fused epilogue (activation derivative,
// conversion, bias gradient in one pass over dy), and the global gradient norm with clipping over many tensors.
// All of it is bound by memory traffic.
#include <cuda_runtime.h>
#include <stdint.h>

#include <cmath>

#include "activation.cuh"
#include "codec.cuh"
#include "common.cuh"
#include "octet.cuh"

namespace fp8b200 {
namespace grads {

constexpr int THREADS = 256, WARPS = THREADS / 32;

// Not the read-only path: an output may be its own input.
__device__ __forceinline__ uint4 ld_stream_v4(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// Stores whose lines L2 may give up first: written once, read by no kernel here.
__device__ __forceinline__ uint64_t policy_once() {
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ void st_once_v4(void* p, const uint4& v, uint64_t policy) {
    asm volatile("st.global.L2::cache_hint.v4.b32 [%0], {%1,%2,%3,%4}, %5;" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w), "l"(policy) : "memory");
}

__device__ __forceinline__ void unpack_bf16(const uint4& w, float (&v)[8]) {
    v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xFFFF0000u);
    v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xFFFF0000u);
    v[4] = __uint_as_float(w.z << 16); v[5] = __uint_as_float(w.z & 0xFFFF0000u);
    v[6] = __uint_as_float(w.w << 16); v[7] = __uint_as_float(w.w & 0xFFFF0000u);
}

// Raw octet of a wide row: one 16-byte word of bf16, two of fp32.
template <bool BF16> struct Octet {
    uint4 w[BF16 ? 1 : 2];
    __device__ __forceinline__ void load(const uint8_t* p) {
        w[0] = ld_stream_v4(p);
        if (!BF16) w[BF16 ? 0 : 1] = ld_stream_v4(p + 16);
    }
    __device__ __forceinline__ void load_some(const uint8_t* p, int count) {
        uint32_t e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            e[i] = i >= count ? 0u : BF16 ? (uint32_t) reinterpret_cast<const uint16_t*>(p)[i] : reinterpret_cast<const uint32_t*>(p)[i];
        if (BF16) {
            w[0] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
        } else {
            w[0] = make_uint4(e[0], e[1], e[2], e[3]);
            w[BF16 ? 0 : 1] = make_uint4(e[4], e[5], e[6], e[7]);
        }
    }
    // Every value outside [-far, far] moved to the nearer end; NaN stays NaN.  `far` is a bf16 value.
    __device__ __forceinline__ void hold_within(float far) {
#pragma unroll
        for (int i = 0; i < (BF16 ? 1 : 2); ++i) {
            uint32_t e[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (BF16) {                                // both halves of the word at once
                    const uint32_t hi = (__float_as_uint(far) >> 16) * 0x10001u, lo = hi | 0x80008000u;
                    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(e[j]) : "r"(lo));
                    asm("min.NaN.bf16x2 %0, %0, %1;" : "+r"(e[j]) : "r"(hi));
                } else {
                    float f = __uint_as_float(e[j]);
                    asm("max.NaN.f32 %0, %0, %1;" : "+f"(f) : "f"(-far));
                    asm("min.NaN.f32 %0, %0, %1;" : "+f"(f) : "f"(far));
                    e[j] = __float_as_uint(f);
                }
            }
            w[i] = make_uint4(e[0], e[1], e[2], e[3]);
        }
    }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        if (BF16) {
            unpack_bf16(w[0], v);
        } else {
            const uint4 a = w[0], b = w[BF16 ? 0 : 1];
            v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
            v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
        }
    }
};

__device__ __forceinline__ uint4 pack8_bf16(const float (&v)[8]) {
    return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// ---- backward pass of the epilogue -------------------------------------------------------------------------------

constexpr int STRIP = 32 * 8;                              // columns of a block: one octet per lane
constexpr int UNROLL = 2;                                  // rows in flight per warp in the row loop

struct BackwardParams {
    int64_t M, N, ldy, ldp, ldo;
    const void* dy;
    const void* pre;
    void* out;
    const float* scale;
    float* dbias;
    uint32_t* amax_bits;
    unsigned int* counters;                                // one per strip, zero between calls
    unsigned int* amax_words;                              // two more, or null: *amax_bits is zero when the kernel starts
    float* partial;                                        // [row chunks][N]
    int64_t rows;                                          // of a chunk
    int store, nosat;
};

// A block takes a strip of 256 columns and a chunk of rows, a warp every eighth row.  Each thread keeps the sums of its
// eight columns; the block adds its warps' sums in order and the last block of a strip adds the chunks' in order.
// What bounds it: 5 bytes per bf16 element against some fourteen instructions, two of them exp2 and reciprocal: 8192 x 16384
// bf16 -> E5M2 with gelu_tanh and bias gradient 117 us (5.7 TB/s), without activation 82 us; the column sums are 9 of them.
// Wider strips (up to 2048 columns) or more rows in flight measured the same.  Addresses
// advance by pointers, bounds are settled outside the row loop and the stored type is fixed at compile time, because
// branches and address arithmetic were as many instructions as the mathematics (27 per element in all).
// STORE: FP8_STORE_E4M3, FP8_STORE_E5M2, or a wide type (which one is p.store).
template <int ACT, bool DY_BF16, bool PRE_BF16, int STORE>
__global__ void __launch_bounds__(THREADS, 4)
k_epilogue_backward(const BackwardParams p) {
    __shared__ float sums[WARPS][STRIP];
    __shared__ uint32_t red[32];
    __shared__ unsigned int last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t col = (int64_t)blockIdx.x * STRIP + lane * 8;
    const int64_t row_lo = (int64_t)blockIdx.y * p.rows, row_hi = min(p.M, row_lo + p.rows);
    const int count = (int)max((int64_t)0, min((int64_t)8, p.N - col));
    float acc[8], top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.0f;
    grid_dependency_wait();
    const float scale = STORE >= FP8_STORE_E4M3 ? __ldg(p.scale) : 1.0f;
    constexpr int YS = DY_BF16 ? 2 : 4, ZS = PRE_BF16 ? 2 : 4;
    const int os = STORE >= FP8_STORE_E4M3 ? 1 : p.store == FP8_STORE_BF16 ? 2 : 4;
    const int64_t first = row_lo + warp;
    const uint8_t* y = reinterpret_cast<const uint8_t*>(p.dy) + (first * p.ldy + col) * YS;
    const uint8_t* z = reinterpret_cast<const uint8_t*>(p.pre) + (first * p.ldp + col) * ZS;
    uint8_t* o = reinterpret_cast<uint8_t*>(p.out) + (first * p.ldo + col) * os;
    const int64_t y_step = WARPS * p.ldy * YS, z_step = WARPS * p.ldp * ZS, o_step = WARPS * p.ldo * os;
    int rows = count > 0 && first < row_hi ? (int)((row_hi - first + WARPS - 1) / WARPS) : 0;      // of this warp
    // dz of one octet: magnitudes, column sums, v
    auto derive = [&](Octet<DY_BF16>& dy, Octet<PRE_BF16>& pre, float (&v)[8]) {
        dy.values(v);
        if (ACT != FP8_ACT_NONE) {
            float x[8];
            if (ACT != FP8_ACT_RELU) pre.hold_within(Far<ACT>::value);
            pre.values(x);
#pragma unroll
            for (int i = 0; i < 8; i += 2) (Pair(v[i], v[i + 1]) * slope_within<ACT>(x[i], x[i + 1])).split(v[i], v[i + 1]);
        }
        const float most = most8(v);
        top = max_nan(top, most);
#pragma unroll
        for (int i = 0; i < 8; i += 2) (Pair(acc[i], acc[i + 1]) + Pair(v[i], v[i + 1])).split(acc[i], acc[i + 1]);
        return most;
    };
    if (count == 8) {
        auto work = [&](Octet<DY_BF16>& dy, Octet<PRE_BF16>& pre, uint8_t* to) {
            float v[8];
            const float most = derive(dy, pre, v);
            if (STORE >= FP8_STORE_E4M3) {
                *reinterpret_cast<uint2*>(to) = encode8_as<STORE == FP8_STORE_E5M2 ? kE5M2 : kE4M3>(v, most, scale, p.nosat != 0);
            } else if (os == 2) {
                *reinterpret_cast<uint4*>(to) = pack8_bf16(v);
            } else {
                reinterpret_cast<float4*>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
                reinterpret_cast<float4*>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
            }
        };
        Octet<DY_BF16> dy[2];
        Octet<PRE_BF16> pre[2];
#pragma unroll 1
        for (; rows >= 2; rows -= 2) {                     // two rows in flight
            dy[0].load(y);
            dy[1].load(y + y_step);
            if (ACT != FP8_ACT_NONE) { pre[0].load(z); pre[1].load(z + z_step); }
            work(dy[0], pre[0], o);
            work(dy[1], pre[1], o + o_step);
            y += 2 * y_step; z += 2 * z_step; o += 2 * o_step;
        }
        if (rows > 0) {
            dy[0].load(y);
            if (ACT != FP8_ACT_NONE) pre[0].load(z);
            work(dy[0], pre[0], o);
        }
    } else {                                               // the last columns of rows whose length is no multiple of 8
#pragma unroll 1
        for (; rows > 0; --rows) {
            Octet<DY_BF16> dy;
            Octet<PRE_BF16> pre;
            dy.load_some(y, count);
            if (ACT != FP8_ACT_NONE) pre.load_some(z, count);
            float v[8];
            const float most = derive(dy, pre, v);
            uint2 w = make_uint2(0u, 0u);
            if (STORE >= FP8_STORE_E4M3) w = encode8_as<STORE == FP8_STORE_E5M2 ? kE5M2 : kE4M3>(v, most, scale, p.nosat != 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i < count) {
                    if (STORE >= FP8_STORE_E4M3) o[i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
                    else if (os == 2) reinterpret_cast<uint16_t*>(o)[i] = (uint16_t)pack_bf16(v[i], 0.0f);
                    else reinterpret_cast<float*>(o)[i] = v[i];
                }
            }
            y += y_step; z += z_step; o += o_step;
        }
    }
    grid_launch_dependents();
    if (p.amax_bits) {
        if (STORE < FP8_STORE_E4M3 && os == 2) top = __uint_as_float(pack_bf16(top, 0.0f) << 16);
        block_fold_amax(canonical_nan_bits(__float_as_uint(top)), red, p.amax_words, p.amax_bits);
    }
    if (!p.dbias) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[warp][lane * 8 + i] = acc[i];
    __syncthreads();
    const int64_t c = (int64_t)blockIdx.x * STRIP + threadIdx.x;
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) s += sums[w][threadIdx.x];
    if (gridDim.y == 1) {
        if (c < p.N) p.dbias[c] = s;
        return;
    }
    if (c < p.N) p.partial[(int64_t)blockIdx.y * p.N + c] = s;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(&p.counters[blockIdx.x], 1u) == gridDim.y - 1 ? 1u : 0u;
    __syncthreads();
    if (!last) return;
    __threadfence();
    if (threadIdx.x == 0) p.counters[blockIdx.x] = 0u;
    if (c >= p.N) return;
    s = 0.0f;
#pragma unroll 8
    for (unsigned int y = 0; y < gridDim.y; ++y) s += __ldcg(p.partial + (int64_t)y * p.N + c);
    p.dbias[c] = s;
}

// The counters lie at the start of the workspace in a region of fixed size, so that the partial sums of one shape never
// lie where another shape's counters are.  Tensors of more strips fill the GPU without cutting rows.
constexpr int64_t MAX_COUNTERS = 4092;                     // and four words, two of them for the amax
constexpr size_t COUNTER_BYTES = (MAX_COUNTERS + 4) * 4;

// Rows of a chunk: about sixteen blocks per SM over all strips, at least 16 rows (two per warp).
static int64_t chunk_rows(int64_t M, int64_t N) {
    const int64_t strips = (N + STRIP - 1) / STRIP;
    int64_t chunks = strips > MAX_COUNTERS ? 1 : (int64_t)sm_count() * 16 / strips;
    if (chunks < 1) chunks = 1;
    if (chunks > 65535) chunks = 65535;
    const int64_t unit = WARPS * UNROLL;
    int64_t rows = (M + chunks - 1) / chunks;
    rows = (rows + unit - 1) / unit * unit;
    return rows < unit ? unit : rows;
}

template <int ACT, bool DY_BF16, bool PRE_BF16>
static cudaError_t launch_backward_as(dim3 grid, cudaStream_t st, const BackwardParams& p) {
    switch (p.store) {
        case FP8_STORE_E4M3: return launch_programmatic(k_epilogue_backward<ACT, DY_BF16, PRE_BF16, FP8_STORE_E4M3>, grid, dim3(THREADS), st, p);
        case FP8_STORE_E5M2: return launch_programmatic(k_epilogue_backward<ACT, DY_BF16, PRE_BF16, FP8_STORE_E5M2>, grid, dim3(THREADS), st, p);
        default: return launch_programmatic(k_epilogue_backward<ACT, DY_BF16, PRE_BF16, FP8_STORE_BF16>, grid, dim3(THREADS), st, p);
    }
}
template <int ACT>
static cudaError_t launch_backward(bool dy_bf16, bool pre_bf16, dim3 grid, cudaStream_t st, const BackwardParams& p) {
    if (ACT == FP8_ACT_NONE) pre_bf16 = true;              // not read
    if (dy_bf16) return pre_bf16 ? launch_backward_as<ACT, true, true>(grid, st, p) : launch_backward_as<ACT, true, ACT == FP8_ACT_NONE>(grid, st, p);
    return pre_bf16 ? launch_backward_as<ACT, false, true>(grid, st, p) : launch_backward_as<ACT, false, ACT == FP8_ACT_NONE>(grid, st, p);
}

// ---- global norm and clipping -------------------------------------------------------------------------------------
//
// Bound by HBM: two reads and one write, because the factor needs the whole norm first; 805M bf16 elements 712 us, 6.8 TB/s.
// What fits L2 is found there the second time (24M elements 26 us), the more since the outputs are written evict-first
// (30 us without).  Small lists are bound by two launches: 288 tensors, 3M elements, 7.3 us.

constexpr int64_t CHUNK = 32768;                           // elements of a tensor handled by one block

struct Entry {
    const void* x;
    void* out;
    int64_t n;
    int64_t first_chunk;
    int32_t x_bf16, out_bf16, aligned, reserved;           // aligned: x and out start on 16 bytes
};
static_assert(sizeof(Entry) == 48, "table layout");

struct ClipParams {
    const Entry* entries;
    const int32_t* chunk_entry;                            // the entry that a chunk belongs to
    int64_t chunks;
    unsigned int* counter;
    double* partial;                                       // one per chunk
    float* norm;
    float max_norm;
};

template <bool BF16>
__device__ __forceinline__ double chunk_squares(const void* x, int64_t n, bool aligned) {
    constexpr int EPI = BF16 ? 8 : 4, BATCH = 8;           // elements of a 16-byte item, items in flight
    double sum = 0.0;
    int64_t done = 0;
    if (aligned) {
        const int64_t items = n / EPI;
        const uint4* v = reinterpret_cast<const uint4*>(x);
        for (int64_t i0 = threadIdx.x; i0 < items; i0 += THREADS * BATCH) {
            uint4 w[BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int64_t i = i0 + b * THREADS;
                w[b] = i < items ? ld_stream_v4(v + i) : make_uint4(0u, 0u, 0u, 0u);
            }
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const uint32_t e[4] = {w[b].x, w[b].y, w[b].z, w[b].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (BF16) {
                        const float lo = __uint_as_float(e[j] << 16), hi = __uint_as_float(e[j] & 0xFFFF0000u);
                        s[0] = fmaf(lo, lo, s[0]);
                        s[1] = fmaf(hi, hi, s[1]);
                    } else {
                        const float f = __uint_as_float(e[j]);
                        s[j & 1] = fmaf(f, f, s[j & 1]);
                    }
                }
            }
            sum += (double)(s[0] + s[1]);
        }
        done = items * EPI;
    }
    for (int64_t i = done + threadIdx.x; i < n; i += THREADS) {
        const float f = BF16 ? __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(x)[i] << 16) : reinterpret_cast<const float*>(x)[i];
        sum += (double)(f * f);
    }
    return sum;
}

// Sum over the block, the same for every call: lanes by halving distance, then the warps in order.
__device__ __forceinline__ double block_sum(double v, double* smem) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) s += smem[w];
    return s;
}

// One block per chunk; the last block to finish adds the chunks' sums in a fixed order and takes the root.
__global__ void __launch_bounds__(THREADS) k_grad_norm(const ClipParams p) {
    __shared__ double red[WARPS];
    __shared__ unsigned int last;
    // The table is the plan's own: copied to the device before the first call, written by no kernel.
    const Entry e = p.entries[p.chunk_entry[blockIdx.x]];
    grid_dependency_wait();
    const int64_t lo = ((int64_t)blockIdx.x - e.first_chunk) * CHUNK, n = min(CHUNK, e.n - lo);
    const double mine = e.x_bf16 ? chunk_squares<true>(reinterpret_cast<const uint16_t*>(e.x) + lo, n, e.aligned != 0)
                                 : chunk_squares<false>(reinterpret_cast<const float*>(e.x) + lo, n, e.aligned != 0);
    const double s = block_sum(mine, red);
    grid_launch_dependents();
    if (threadIdx.x == 0) {
        p.partial[blockIdx.x] = s;
        __threadfence();
        last = atomicAdd(p.counter, 1u) == gridDim.x - 1 ? 1u : 0u;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double total = 0.0;
    for (int64_t i = threadIdx.x; i < p.chunks; i += THREADS) total += __ldcg(p.partial + i);
    total = block_sum(total, red);
    if (threadIdx.x == 0) {
        *p.norm = (float)sqrt(total);
        *p.counter = 0u;
    }
}

// out = x * coef over one chunk.  The first items are loaded before the norm is waited for: this kernel is scheduled when
// every block of the norm kernel is past its own wait, so whatever wrote x has finished, and the norm kernel itself writes
// nothing but the norm and its workspace.
template <bool X_BF16, bool OUT_BF16>
__device__ __forceinline__ void clip_chunk(const ClipParams& p, const Entry& e, int64_t lo, int64_t n) {
    constexpr int BATCH = 4;
    const uint8_t* x = reinterpret_cast<const uint8_t*>(e.x) + lo * (X_BF16 ? 2 : 4);
    uint8_t* out = reinterpret_cast<uint8_t*>(e.out) + lo * (OUT_BF16 ? 2 : 4);
    const int64_t octets = e.aligned ? n / 8 : 0;
    const uint64_t once = policy_once();
    Octet<X_BF16> w[BATCH];
    auto fetch = [&](int64_t i0) {
#pragma unroll
        for (int b = 0; b < BATCH; ++b)
            if (i0 + b * THREADS < octets) w[b].load(x + (i0 + b * THREADS) * (X_BF16 ? 16 : 32));
    };
    fetch(threadIdx.x);
    grid_dependency_wait();
    const float norm = __ldcg(p.norm);
    const float coef = norm <= p.max_norm ? 1.0f : p.max_norm / norm;
    if (coef == 1.0f && e.x == e.out) return;              // in place: nothing changes
    for (int64_t i0 = threadIdx.x; i0 < octets; i0 += THREADS * BATCH) {
        if (i0 != threadIdx.x) fetch(i0);
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int64_t i = i0 + b * THREADS;
            if (i >= octets) continue;
            float v[8];
            w[b].values(v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= coef;
            if (OUT_BF16) {
                st_once_v4(out + i * 16, pack8_bf16(v), once);
            } else {
                st_once_v4(out + i * 32, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])), once);
                st_once_v4(out + i * 32 + 16, make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])), once);
            }
        }
    }
    for (int64_t i = octets * 8 + threadIdx.x; i < n; i += THREADS) {
        const float f = (X_BF16 ? __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(x)[i] << 16) : reinterpret_cast<const float*>(x)[i]) * coef;
        if (OUT_BF16) reinterpret_cast<uint16_t*>(out)[i] = (uint16_t)pack_bf16(f, 0.0f);
        else reinterpret_cast<float*>(out)[i] = f;
    }
}

// One block per chunk, from the last to the first: the end of what the norm has just read is still in L2.
__global__ void __launch_bounds__(THREADS) k_grad_clip(const ClipParams p) {
    const int64_t chunk = p.chunks - 1 - blockIdx.x;
    const Entry e = p.entries[p.chunk_entry[chunk]];
    const int64_t lo = (chunk - e.first_chunk) * CHUNK, n = min(CHUNK, e.n - lo);
    if (!e.out) {                                          // counted in the norm only
        grid_dependency_wait();
        return;
    }
    if (e.x_bf16) e.out_bf16 ? clip_chunk<true, true>(p, e, lo, n) : clip_chunk<true, false>(p, e, lo, n);
    else          e.out_bf16 ? clip_chunk<false, true>(p, e, lo, n) : clip_chunk<false, false>(p, e, lo, n);
}

static bool wide_ok(int t) { return t == FP8_F32 || t == FP8_BF16; }

static fp8_status clip_params(const fp8_clip_plan* plan, const void* table, void* ws, float* norm, ClipParams& p) {
    if (!plan || !norm) return FP8_ERR_NULL;
    if (plan->count < 0 || plan->chunks < 0) return FP8_ERR_SHAPE;
    if (plan->chunks > 0 && (!table || !ws)) return FP8_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(table) & 15u) || (reinterpret_cast<uintptr_t>(ws) & 15u)) return FP8_ERR_ALIGN;
    p.entries = reinterpret_cast<const Entry*>(table);
    p.chunk_entry = reinterpret_cast<const int32_t*>(reinterpret_cast<const uint8_t*>(table) + plan->count * (int64_t)sizeof(Entry));
    p.chunks = plan->chunks;
    p.counter = reinterpret_cast<unsigned int*>(ws);
    p.partial = reinterpret_cast<double*>(reinterpret_cast<uint8_t*>(ws) + 16);
    p.norm = norm;
    p.max_norm = 0.0f;
    return FP8_OK;
}

static fp8_status enqueue_norm(const ClipParams& p, cudaStream_t st) {
    if (p.chunks == 0) {
        if (cudaMemsetAsync(p.norm, 0, 4, st) != cudaSuccess) return FP8_ERR_CUDA;
    } else if (launch_programmatic(k_grad_norm, dim3((unsigned)p.chunks), dim3(THREADS), st, p) != cudaSuccess) {
        (void)cudaGetLastError();
        return FP8_ERR_CUDA;
    }
    count_launches(1);
    return launch_status();
}

}  // namespace grads
}  // namespace fp8b200

using namespace fp8b200;

extern "C" {

size_t fp8_epilogue_backward_workspace_bytes(int64_t M, int64_t N) {
    using namespace fp8b200::grads;
    if (M <= 0 || N <= 0) return COUNTER_BYTES;
    const int64_t chunks = (M + chunk_rows(M, N) - 1) / chunk_rows(M, N);
    return COUNTER_BYTES + (chunks > 1 ? (size_t)chunks * (size_t)N * 4 : 0);
}

fp8_status fp8_epilogue_backward(int64_t M, int64_t N, fp8_activation act, const void* dy, fp8_wide dy_t, int64_t ldy,
                                 const void* pre, fp8_wide pre_t, int64_t ldp, fp8_store store, fp8_overflow overflow,
                                 const float* scale_dz_dev, void* out, int64_t ldo, float* dbias_dev, float* amax_dev,
                                 void* workspace_dev, size_t workspace_bytes, void* stream) {
    using namespace fp8b200::grads;
    if (act < FP8_ACT_NONE || act > FP8_ACT_SILU || !wide_ok(dy_t) || !wide_ok(pre_t) || store < FP8_STORE_F32 || store > FP8_STORE_E5M2 ||
        (overflow != FP8_SATURATE && overflow != FP8_NOSAT))
        return FP8_ERR_ENUM;
    if (M < 0 || N < 0) return FP8_ERR_SHAPE;
    const bool some = M > 0 && N > 0;
    if (store >= FP8_STORE_E4M3 && !scale_dz_dev) return FP8_ERR_NULL;
    if (some) {
        if (!dy || !out || (act != FP8_ACT_NONE && !pre)) return FP8_ERR_NULL;
        if (ldy < N || ldo < N || (pre && ldp < N)) return FP8_ERR_SHAPE;
        const int64_t ys = dy_t == FP8_BF16 ? 2 : 4, ps = pre_t == FP8_BF16 ? 2 : 4, os = store == FP8_STORE_F32 ? 4 : store == FP8_STORE_BF16 ? 2 : 1;
        if ((reinterpret_cast<uintptr_t>(dy) & 15u) || (reinterpret_cast<uintptr_t>(out) & 15u) || (reinterpret_cast<uintptr_t>(pre) & 15u) ||
            ((ldy * ys) & 15) || ((ldo * os) & 15) || (pre && ((ldp * ps) & 15)))
            return FP8_ERR_ALIGN;
        if (N > ((int64_t)1 << 31) - 512 || M > (int64_t)1 << 40) return FP8_ERR_UNSUPPORTED;
        if (dbias_dev && !workspace_dev) return FP8_ERR_NULL;
        if (workspace_dev) {
            if (workspace_bytes < fp8_epilogue_backward_workspace_bytes(M, N)) return FP8_ERR_SHAPE;
            if (reinterpret_cast<uintptr_t>(workspace_dev) & 15u) return FP8_ERR_ALIGN;
        }
    }
    cudaStream_t st = (cudaStream_t)stream;
    if (amax_dev && (!workspace_dev || !some)) {
        const fp8_status rc = launch_zero_word(reinterpret_cast<uint32_t*>(amax_dev), st);
        if (rc != FP8_OK) return rc;
    }
    if (!some) {
        if (dbias_dev && N > 0) {
            if (cudaMemsetAsync(dbias_dev, 0, (size_t)N * 4, st) != cudaSuccess) return FP8_ERR_CUDA;
            count_launches(1);
        }
        return FP8_OK;
    }
    BackwardParams p = {};
    p.M = M; p.N = N; p.ldy = ldy; p.ldp = ldp; p.ldo = ldo;
    p.dy = dy; p.pre = pre; p.out = out; p.scale = scale_dz_dev; p.dbias = dbias_dev;
    p.amax_bits = reinterpret_cast<uint32_t*>(amax_dev);
    p.counters = reinterpret_cast<unsigned int*>(workspace_dev);
    p.amax_words = workspace_dev && amax_dev ? p.counters + MAX_COUNTERS : nullptr;
    p.partial = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(workspace_dev) + COUNTER_BYTES);
    p.rows = chunk_rows(M, N);
    p.store = store; p.nosat = overflow == FP8_NOSAT ? 1 : 0;
    const dim3 grid((unsigned)((N + STRIP - 1) / STRIP), (unsigned)((M + p.rows - 1) / p.rows), 1);
    const bool yb = dy_t == FP8_BF16, pb = pre_t == FP8_BF16;
    cudaError_t e;
    switch (act) {
        case FP8_ACT_RELU: e = launch_backward<FP8_ACT_RELU>(yb, pb, grid, st, p); break;
        case FP8_ACT_GELU: e = launch_backward<FP8_ACT_GELU>(yb, pb, grid, st, p); break;
        case FP8_ACT_GELU_TANH: e = launch_backward<FP8_ACT_GELU_TANH>(yb, pb, grid, st, p); break;
        case FP8_ACT_SILU: e = launch_backward<FP8_ACT_SILU>(yb, pb, grid, st, p); break;
        default: e = launch_backward<FP8_ACT_NONE>(yb, pb, grid, st, p); break;
    }
    if (e != cudaSuccess) { (void)cudaGetLastError(); return FP8_ERR_CUDA; }
    count_launches(1);
    return launch_status();
}

fp8_status fp8_clip_plan_size(const fp8_clip_item* items, int64_t count, fp8_clip_plan* plan) {
    using namespace fp8b200::grads;
    if (!plan || (count > 0 && !items)) return FP8_ERR_NULL;
    if (count < 0) return FP8_ERR_SHAPE;
    int64_t chunks = 0;
    for (int64_t i = 0; i < count; ++i) {
        const fp8_clip_item& it = items[i];
        if (!wide_ok(it.x_t) || !wide_ok(it.out_t)) return FP8_ERR_ENUM;
        if (it.n < 0) return FP8_ERR_SHAPE;
        if (it.n > 0 && !it.x) return FP8_ERR_NULL;
        if ((reinterpret_cast<uintptr_t>(it.x) & (it.x_t == FP8_BF16 ? 1u : 3u)) || (reinterpret_cast<uintptr_t>(it.out) & (it.out_t == FP8_BF16 ? 1u : 3u)))
            return FP8_ERR_ALIGN;
        if (it.out == it.x && it.n > 0 && it.out_t != it.x_t) return FP8_ERR_ENUM;      // in place keeps its type
        if (it.n > CHUNK << 31) return FP8_ERR_UNSUPPORTED;
        chunks += (it.n + CHUNK - 1) / CHUNK;
        if (chunks > 0x7FFFFFFF) return FP8_ERR_UNSUPPORTED;
    }
    plan->count = count;
    plan->chunks = chunks;
    plan->table_bytes = (size_t)count * sizeof(Entry) + (size_t)(chunks + 3) / 4 * 16;
    plan->workspace_bytes = 16 + (size_t)chunks * sizeof(double);
    return FP8_OK;
}

fp8_status fp8_clip_plan_fill(const fp8_clip_item* items, const fp8_clip_plan* plan, void* table_host) {
    using namespace fp8b200::grads;
    if (!plan || (plan->table_bytes > 0 && !table_host) || (plan->count > 0 && !items)) return FP8_ERR_NULL;
    Entry* e = reinterpret_cast<Entry*>(table_host);
    int32_t* map = reinterpret_cast<int32_t*>(reinterpret_cast<uint8_t*>(table_host) + plan->count * (int64_t)sizeof(Entry));
    int64_t chunk = 0;
    for (int64_t i = 0; i < plan->count; ++i) {
        const fp8_clip_item& it = items[i];
        const int64_t n = (it.n + CHUNK - 1) / CHUNK;
        if (it.n < 0 || chunk + n > plan->chunks) return FP8_ERR_SHAPE;      // not the items the plan was sized for
        e[i].x = it.x; e[i].out = it.out; e[i].n = it.n; e[i].first_chunk = chunk;
        e[i].x_bf16 = it.x_t == FP8_BF16; e[i].out_bf16 = it.out_t == FP8_BF16;
        e[i].aligned = ((reinterpret_cast<uintptr_t>(it.x) | reinterpret_cast<uintptr_t>(it.out)) & 15u) == 0;
        e[i].reserved = 0;
        for (int64_t j = 0; j < n; ++j) map[chunk + j] = (int32_t)i;
        chunk += n;
    }
    return chunk == plan->chunks ? FP8_OK : FP8_ERR_SHAPE;
}

fp8_status fp8_grad_norm(const fp8_clip_plan* plan, const void* table_dev, void* workspace_dev, float* norm_dev, void* stream) {
    using namespace fp8b200::grads;
    ClipParams p;
    const fp8_status rc = clip_params(plan, table_dev, workspace_dev, norm_dev, p);
    return rc != FP8_OK ? rc : enqueue_norm(p, (cudaStream_t)stream);
}

fp8_status fp8_grad_clip(const fp8_clip_plan* plan, const void* table_dev, void* workspace_dev, float max_norm,
                         float* norm_dev, void* stream) {
    using namespace fp8b200::grads;
    ClipParams p;
    fp8_status rc = clip_params(plan, table_dev, workspace_dev, norm_dev, p);
    if (rc != FP8_OK) return rc;
    if (!(max_norm >= 0.0f)) return FP8_ERR_UNSUPPORTED;
    p.max_norm = max_norm;
    if ((rc = enqueue_norm(p, (cudaStream_t)stream)) != FP8_OK || p.chunks == 0) return rc;
    if (launch_programmatic(k_grad_clip, dim3((unsigned)p.chunks), dim3(THREADS), (cudaStream_t)stream, p) != cudaSuccess) {
        (void)cudaGetLastError();
        return FP8_ERR_CUDA;
    }
    count_launches(1);
    return launch_status();
}

}  // extern "C"
