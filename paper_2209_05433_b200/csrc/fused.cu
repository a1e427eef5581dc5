// FP8 products with fused epilogues (sm_100a): bias + activation + residual, the gated feed-forward block, and the
// data gradient of its down projection fused with the gate's derivative.
//
// k_fused_rows: products with few rows (tokens).  Computed transposed: 128 columns of D (rows of the weights) are the
// M side of the tensor core's tile and T tokens its N side, so that a tile wastes no tensor work on absent rows and one
// CTA owns 128 weight rows.  K is cut into slices, one CTA of a cluster each; their binary32 partial sums meet in
// distributed shared memory and are added in slice order, so the result does not depend on timing.
//
// k_fused_tiles: products with many rows, on persistent CTA pairs with 256 x 256 accumulator tiles as the plain product.
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <mutex>

#include "activation.cuh"
#include "codec.cuh"
#include "common.cuh"
#include "octet.cuh"
#include "umma.cuh"

namespace fp8b200 {
namespace fused {

using namespace gemm;

constexpr int MODE_EPILOGUE = 0;        // act(z + bias) + residual
constexpr int MODE_GATED = 1;           // act(g) * u
constexpr int MODE_GATED_BWD = 2;       // dh -> dG, dU

constexpr int BK = 128;                 // K-block in elements = bytes = one swizzle row
constexpr int UMMA_K = 32;

struct Params {
    int64_t M, N, K;                    // rows (tokens), columns, contraction
    const float* sa_inv;
    const float* sb_inv[2];             // [1]: the up projection of the gated block
    const float* sb_inv_vec;            // optional, N entries
    const float* scale_d;
    const void* bias;                   // optional, N entries
    const void* in[2];                  // residual | gate, up
    void* keep[2];                      // pre | gate, up
    void* D[2];                         // D | dG, dU
    int64_t ld_in, ld_keep, ldd;        // elements
    int bias_bf16, in_bf16, keep_bf16;
    int store, nosat, act;
    uint32_t* amax_bits;                // may be null
    unsigned int* amax_words;           // two zero words, or null: *amax_bits is zero when the kernel starts
    uint32_t idesc;
    int a_mn, w_mn;                     // rows stored with M contiguous; weights stored with N contiguous
};

// codes written to the error latch (those of the plain products end at 9, the grid barrier's is 16)
enum : uint32_t { F_WAIT_EMPTY = 33, F_WAIT_FULL = 34, F_WAIT_ACC_EMPTY = 35, F_WAIT_ACC_FULL = 36, F_WAIT_DRAIN = 37, F_WAIT_IN = 38 };

// ---- element access ----------------------------------------------------------

// Up to four consecutive elements of a wide row (missing ones read as 0).  Rows start on 16 bytes and the first index
// is a multiple of 4, so a full group is one 8- or 16-byte access.
__device__ __forceinline__ void load4(const void* base, bool bf16, int64_t at, int count, float (&v)[4]) {
    if (count == 4) {
        if (bf16) {
            const uint2 w = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint16_t*>(base) + at);
            v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xFFFF0000u);
            v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xFFFF0000u);
        } else {
            const float4 w = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + at);
            v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= count) v[i] = 0.0f;
        else if (bf16) v[i] = __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(base)[at + i] << 16);
        else v[i] = reinterpret_cast<const float*>(base)[at + i];
    }
}

// The same without alignment (bias vectors, scale vectors).
__device__ __forceinline__ void load4_any(const void* base, bool bf16, int64_t at, int count, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= count) v[i] = 0.0f;
        else if (bf16) v[i] = __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(base)[at + i] << 16);
        else v[i] = reinterpret_cast<const float*>(base)[at + i];
    }
}

__device__ __forceinline__ void store4_wide(void* base, bool bf16, int64_t at, int count, const float (&v)[4]) {
    if (bf16) {
        const uint2 w = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
        uint16_t* p = reinterpret_cast<uint16_t*>(base) + at;
        if (count == 4) { *reinterpret_cast<uint2*>(p) = w; return; }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < count) p[i] = (uint16_t)(((i & 2) ? w.y : w.x) >> (16 * (i & 1)));
    } else {
        float* p = reinterpret_cast<float*>(base) + at;
        if (count == 4) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); return; }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < count) p[i] = v[i];
    }
}

template <int FMT>
__device__ __forceinline__ uint32_t encode4(const float (&v)[4], float scale_d, bool nosat) {
    float y[4], top = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) { y[i] = v[i] * scale_d; top = fmax_nan(top, fabsf(y[i])); }
    const bool over = Fmt<FMT>::nosat_limit_inclusive ? top >= Fmt<FMT>::nosat_limit : top > Fmt<FMT>::nosat_limit;
    if (top <= 3.402823466e38f && !(nosat && over)) return cvt_quad<FMT>(y[0], y[1], y[2], y[3]);
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t code;
        if (y[i] != y[i]) code = ((__float_as_uint(v[i]) >> 24) & 0x80u) | 0x7Fu;
        else code = nosat ? encode_scalar<FMT, true>(y[i]) : encode_scalar<FMT, false>(y[i]);
        word |= code << (8 * i);
    }
    return word;
}

// Stores a group as p.store says and folds its magnitudes into `top` (NaN once any is NaN): of the stored values for
// the wide types, of v before scaling for FP8.
__device__ __forceinline__ void store4(const Params& p, void* base, int64_t at, int count, float (&v)[4], float scale_d, float& top) {
    if (p.store == FP8_STORE_BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(pack_bf16(v[i], 0.0f) << 16);
        store4_wide(base, true, at, count, v);
    } else if (p.store == FP8_STORE_F32) {
        store4_wide(base, false, at, count, v);
    } else {
        const uint32_t w = p.store == FP8_STORE_E4M3 ? encode4<kE4M3>(v, scale_d, p.nosat != 0) : encode4<kE5M2>(v, scale_d, p.nosat != 0);
        uint8_t* d = reinterpret_cast<uint8_t*>(base) + at;
        if (count == 4) *reinterpret_cast<uint32_t*>(d) = w;
        else
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < count) d[i] = (uint8_t)(w >> (8 * i));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < count) top = fmax_nan(top, fabsf(v[i]));
}

// ---- products with few rows ---------------------------------------------------
//
// Bound by the stream of weights.  Two CTAs of 112 KB share an SM, so that some 200 KB per SM are in flight (one CTA alone
// draws 45 GB/s however deep its ring: the issue of its matrix instructions is its limit).  Measured in a graph that goes round
// enough different weights (530 to 800 MB) that none is still in L2: one token 16384 -> 4096 (67 MB) 13.6 us (10.3 at the
// measured copy rate), gated 4096 -> 2 x 16384 (134 MB) 22.7 us (20.5), 37 tokens 4096 -> 16384 18.0 us (10.4).  With one weight
// again and again, partly found in L2: 11.5, 20.7 and 16.4 us.  Of the first, 1.1 us are the latency of the first loads, 2.3
// partial sums and epilogue; the rest is the stream and the hand-over between kernels.

constexpr int ROWS_THREADS = 192;                  // loader warp, MMA warp, four accumulator warps
constexpr int ROWS_BN = 128;                       // columns of D per tile = the tensor core's M
// The tensor core's accumulator, whose additions truncate, is drained every 512 of K into sums that round: it costs nothing
// beside the stream of weights (1 to 64 tokens, three shapes: within 0.1 us of draining every 1024; every 256 costs up to 1 %).
// With the sizes of a layer the error is the plain form's, 6e-8 of the result in the 2-norm at K = 16384 (1.1e-7 at 1024).
constexpr int ROWS_SPLIT_BLOCKS = 4;
constexpr uint32_t ROWS_TMEM_COLS = 256;           // half of an SM's TMEM: two CTAs share an SM
constexpr uint32_t ROWS_SMEM = 112 * 1024;         // dynamic shared memory of a CTA: two fit an SM
constexpr int ROWS_MAX_STAGES = 8;

template <int MODE, int T> struct RowsGeo {
    static constexpr int NB = MODE == MODE_GATED ? 2 : 1;                          // weight operands
    static constexpr uint32_t W_BYTES = ROWS_BN * BK;
    static constexpr uint32_t X_BYTES = T * BK;
    // K-blocks per stage: a stage costs the loader and the MMA warp a fixed number of barrier operations, so one holds
    // two weight tiles of either kind (two K-blocks of one operand, or one of both) where shared memory allows it
    static constexpr int KB = NB == 2 || T > 32 ? 1 : 2;
    static constexpr uint32_t STAGE_BYTES = KB * (NB * W_BYTES + X_BYTES);
    static constexpr int ACCS = ROWS_TMEM_COLS / (T * NB) < 16 ? ROWS_TMEM_COLS / (T * NB) : 16;
    // partial sums of `rows` tokens that a CTA receives from the slices, and what is left for the ring
    static constexpr uint32_t exchange_bytes(int rows) { return (uint32_t)(NB * rows * ROWS_BN * 4); }
    static constexpr int stages(int rows) {
        const int n = (int)((ROWS_SMEM - 1024 - exchange_bytes(rows)) / STAGE_BYTES);
        return n < ROWS_MAX_STAGES ? n : ROWS_MAX_STAGES;
    }
    static_assert(ACCS >= 2 && (ROWS_SMEM - 1024 - NB * T * ROWS_BN * 4) / STAGE_BYTES >= 2, "TMEM and shared memory budgets");
};

struct alignas(8) RowsBarriers {
    uint64_t full[ROWS_MAX_STAGES], empty[ROWS_MAX_STAGES], acc_full[16], acc_empty[16];
    uint32_t tmem_base, abort_flag;
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void tma_prefetch_3d(const CUtensorMap* map, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];" ::"l"(map), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ float4 ld_shared_f4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}

template <int MODE, int T>
__global__ void __launch_bounds__(ROWS_THREADS, 2)
k_fused_rows(const __grid_constant__ CUtensorMap map_w0, const __grid_constant__ CUtensorMap map_w1,
             const __grid_constant__ CUtensorMap map_x, const Params p, const int stages) {
    using G = RowsGeo<MODE, T>;
    constexpr int NB = G::NB, ACCS = G::ACCS;
    extern __shared__ uint8_t smem_raw[];
    __shared__ RowsBarriers bars;
    __shared__ uint32_t red[32];
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t exchange = ring + (uint32_t)stages * G::STAGE_BYTES;
    volatile uint32_t* abort_flag = &bars.abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n0 = blockIdx.x * ROWS_BN, t0 = blockIdx.y * T;
    const uint32_t slices = gridDim.z, slice = blockIdx.z;                     // the cluster spans z
    const int k_blocks = (int)((p.K + BK - 1) / BK);
    const int kb_lo = (int)((int64_t)k_blocks * slice / slices), kb_hi = (int)((int64_t)k_blocks * (slice + 1) / slices);
    const int kb_n = kb_hi - kb_lo;

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) { mbar_init(smem_u32(&bars.full[s]), 1); mbar_init(smem_u32(&bars.empty[s]), 1); }
        for (int a = 0; a < ACCS; ++a) { mbar_init(smem_u32(&bars.acc_full[a]), 1); mbar_init(smem_u32(&bars.acc_empty[a]), 4); }
        bars.abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_map(&map_w0);
        if (NB == 2) prefetch_map(&map_w1);
        prefetch_map(&map_x);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem_base)), "r"(ROWS_TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (slices > 1) cluster_arrive();                       // first phase: every CTA of the cluster runs
    const uint32_t tmem = bars.tmem_base;
    // The first ring's worth of weights is on its way to L2 while the stream's earlier kernels finish (L2 is where all of
    // this GPU's writes meet, so a weight that one of them still writes is read as written): 14.7 -> 13.0 us for one token,
    // 16384 -> 4096; prefetching twice as much or the whole slice gains less.
    if (threadIdx.x == 0) {
        const int ahead = min(stages * G::KB, kb_n);
        for (int i = 0; i < ahead; ++i) {
            const int k0 = (kb_lo + i) * BK, x = p.w_mn ? n0 : k0, y = p.w_mn ? k0 : n0;
            tma_prefetch_3d(&map_w0, x, y, 0);
            if (NB == 2) tma_prefetch_3d(&map_w1, x, y, 0);
        }
    }
    // The next kernel of the stream may be scheduled from here on (this CTA holds its TMEM already); nothing that an
    // earlier kernel may still be writing is touched above this line.
    grid_launch_dependents();
    grid_dependency_wait();

    // The epilogue's items are groups of four columns of a token; each slice of the cluster finishes a contiguous share of
    // the tile's items.  A thread's items lie THREADS apart, a multiple of 32, so its columns are always the same ones.
    const int rows = (int)min((int64_t)T, p.M - t0);
    const int share = rows * (ROWS_BN / 4) / (int)slices;   // 32 items per token, at most 8 slices: always whole
    const int lo = share * (int)slice;
    const int quad = (lo + (int)threadIdx.x) & 31;
    const int64_t n = n0 + quad * 4;
    const int count = (int)max((int64_t)0, min((int64_t)4, p.N - n));
    float factor[4], bias[4] = {0.0f, 0.0f, 0.0f, 0.0f}, alpha1 = 0.0f, scale_d = 1.0f;
    auto fetch_columns = [&] {
        const float sa = __ldg(p.sa_inv);
        if (MODE == MODE_EPILOGUE && p.sb_inv_vec) {
            load4_any(p.sb_inv_vec, false, n, count, factor);
#pragma unroll
            for (int i = 0; i < 4; ++i) factor[i] *= sa;
        } else {
            const float f = sa * __ldg(p.sb_inv[0]);
#pragma unroll
            for (int i = 0; i < 4; ++i) factor[i] = f;
        }
        if (MODE == MODE_EPILOGUE && p.bias) load4_any(p.bias, p.bias_bf16 != 0, n, count, bias);
        if (NB == 2) alpha1 = sa * __ldg(p.sb_inv[1]);
        if (p.store >= FP8_STORE_E4M3) scale_d = __ldg(p.scale_d);
    };

    constexpr int KB = G::KB;
    const int groups = (kb_n + KB - 1) / KB;                // stages' worth of K
    if (warp == 0) {
        // ------------------------------------------------------------ loader (one lane)
        if (lane == 0) {
            bool ok = true;
            int st = 0, issued = 0;
            uint32_t phase = 1;
            const uint64_t keep = policy_evict_last(), weights = gridDim.y == 1 ? policy_evict_first() : keep;
            // the weights are read once (by this tile alone when one tile holds all tokens); the tokens by every tile
            for (int g = 0; g < groups; ++g) {
                ok = mbar_wait(smem_u32(&bars.empty[st]), phase, abort_flag, F_WAIT_EMPTY);
                if (!ok) break;
                const uint32_t sw = ring + (uint32_t)st * G::STAGE_BYTES, sx = sw + KB * NB * G::W_BYTES, full = smem_u32(&bars.full[st]);
                const int blocks = min(KB, kb_n - g * KB);
                mbar_arrive_expect_tx(full, (uint32_t)blocks * (NB * G::W_BYTES + G::X_BYTES));
#pragma unroll
                for (int h = 0; h < KB; ++h) {
                    if (h < blocks) {
                        const int k0 = (kb_lo + g * KB + h) * BK, x = p.w_mn ? n0 : k0, y = p.w_mn ? k0 : n0;
                        tma_load_3d(sw + h * NB * G::W_BYTES, &map_w0, x, y, 0, full, weights);
                        if (NB == 2) tma_load_3d(sw + G::W_BYTES, &map_w1, x, y, 0, full, weights);
                        tma_load_3d(sx + h * G::X_BYTES, &map_x, k0, t0, 0, full, keep);
                    }
                }
                issued = g + 1;
                if (++st == stages) { st = 0; phase ^= 1u; }
            }
            if (!ok) {                                      // given up: no copy may be in flight when the CTA leaves
                for (int g = issued > stages ? issued - stages : 0; g < issued; ++g) {
                    const uint32_t bar = smem_u32(&bars.full[g % stages]);
                    for (int spin = 0; spin < (1 << 20) && !mbar_try_wait(bar, (uint32_t)(g / stages) & 1u); ++spin) {}
                }
            }
        }
        __syncwarp();
        fetch_columns();
        if (slices > 1) cluster_wait();
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer (one lane)
        if (lane == 0) {
            const uint32_t a_kstep = (p.w_mn ? UMMA_K * 128 : UMMA_K) >> 4;                  // in descriptor units of 16 bytes
            const uint64_t dw0 = smem_desc(ring, p.w_mn ? BK * 128 : 16, 1024), dx0 = smem_desc(ring + KB * NB * G::W_BYTES, 16, 1024);
            bool ok = true;
            int st = 0, acc = 0, in_chunk = 0;
            uint32_t phase = 0, acc_phase = 1;
            for (int g = 0; g < groups; ++g) {
                if (in_chunk == 0) {
                    ok = mbar_wait(smem_u32(&bars.acc_empty[acc]), acc_phase, abort_flag, F_WAIT_ACC_EMPTY);
                    if (!ok) break;
                }
                ok = mbar_wait(smem_u32(&bars.full[st]), phase, abort_flag, F_WAIT_FULL);
                if (!ok) break;
                tc_fence_after();
                const uint32_t at = (uint32_t)st * (G::STAGE_BYTES >> 4);
                const int blocks = min(KB, kb_n - g * KB);
#pragma unroll
                for (int h = 0; h < KB; ++h) {
                    if (h < blocks) {
#pragma unroll
                        for (int b = 0; b < NB; ++b)
#pragma unroll
                            for (int k = 0; k < BK / UMMA_K; ++k)
                                tc_mma_f8(tmem + (uint32_t)((acc * NB + b) * T), dw0 + (at + (h * NB + b) * (G::W_BYTES >> 4) + k * a_kstep),
                                          dx0 + (at + h * (G::X_BYTES >> 4) + k * (UMMA_K >> 4)), p.idesc, (in_chunk | h | k) != 0 ? 1u : 0u);
                    }
                }
                tc_commit(smem_u32(&bars.empty[st]));
                in_chunk += KB;
                if (in_chunk == ROWS_SPLIT_BLOCKS || g == groups - 1) {
                    tc_commit(smem_u32(&bars.acc_full[acc]));
                    in_chunk = 0;
                    if (++acc == ACCS) { acc = 0; acc_phase ^= 1u; }
                }
                if (++st == stages) { st = 0; phase ^= 1u; }
            }
        }
        __syncwarp();
        fetch_columns();
        if (slices > 1) cluster_wait();
    } else {
        // ------------------------------------------------------------ accumulators: lane = column of D, TMEM column = token
        const int q = warp & 3;
        fetch_columns();
        float part[NB * T];
#pragma unroll
        for (int i = 0; i < NB * T; ++i) part[i] = 0.0f;
        bool ok = true;
        const int chunks = (kb_n + ROWS_SPLIT_BLOCKS - 1) / ROWS_SPLIT_BLOCKS;
        for (int c = 0; c < chunks; ++c) {
            const int acc = c % ACCS;
            ok = mbar_wait(smem_u32(&bars.acc_full[acc]), (uint32_t)(c / ACCS) & 1u, abort_flag, F_WAIT_ACC_FULL);
            if (!ok) break;
            tc_fence_after();
            const uint32_t taddr = tmem + (uint32_t)(acc * NB * T) + ((uint32_t)(q * 32) << 16);
#pragma unroll
            for (int j = 0; j < NB * T / 16; ++j) {
                uint32_t r[16];
                tc_ld16(taddr + j * 16, r);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) part[j * 16 + i] += __uint_as_float(r[i]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars.acc_empty[acc]));
        }
        // every partial sum goes to the slice that finishes its item: [from slice][operand][item][4]
        if (slices > 1) cluster_wait();
        const float inv_share = 1.0f / (float)share;
        if (ok) {
#pragma unroll
            for (int t = 0; t < T; ++t) {
                if (t < rows) {
                    const int item = t * 32 + q * 8 + (lane >> 2);
                    const int owner = (int)(((float)item + 0.5f) * inv_share);      // item / share: both below 2^11
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        const uint32_t at = exchange + (uint32_t)((((int)slice * NB + b) * share + item - owner * share) * 16 + (lane & 3) * 4);
                        if (slices > 1)
                            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(map_to_cta(at, (uint32_t)owner)), "f"(part[b * T + t]) : "memory");
                        else
                            asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(part[b * T + t]) : "memory");
                    }
                }
            }
        } else if (lane == 0) {                             // given up: the other slices must not use this one's sums
            for (uint32_t s = 0; s < slices; ++s)
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to_cta(smem_u32(&bars.abort_flag), s)), "r"(1u) : "memory");
        }
    }
    // the first items' inputs, on their way while the slices meet
    const int first = (int)threadIdx.x;
    constexpr int NIN = MODE == MODE_GATED_BWD ? 2 : 1;
    float in[NIN][4];
    const bool has_in = MODE == MODE_GATED_BWD || (MODE == MODE_EPILOGUE && p.in[0]);
    if (has_in && first < share && count > 0) {
        const int64_t at = (t0 + ((lo + first) >> 5)) * p.ld_in + n;
#pragma unroll
        for (int i = 0; i < NIN; ++i) load4(p.in[i], p.in_bf16 != 0, at, count, in[i]);
    }
    tc_fence_before();
    if (slices > 1) { cluster_arrive(); cluster_wait(); }
    else __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(ROWS_TMEM_COLS) : "memory");

    // ---------------------------------------------------------------- epilogue: nothing below reaches into another CTA
    float top = 0.0f;
    if (bars.abort_flag == 0u && count > 0) {
        for (int j = first; j < share; j += ROWS_THREADS) {
            const int64_t t = t0 + ((lo + j) >> 5);
            float a[NB][4];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                a[b][0] = a[b][1] = a[b][2] = a[b][3] = 0.0f;
                for (uint32_t s = 0; s < slices; ++s) {
                    const float4 v = ld_shared_f4(exchange + (uint32_t)((((int)s * NB + b) * share + j) * 16));
                    a[b][0] += v.x; a[b][1] += v.y; a[b][2] += v.z; a[b][3] += v.w;
                }
            }
            if (has_in && j != first) {
#pragma unroll
                for (int i = 0; i < NIN; ++i) load4(p.in[i], p.in_bf16 != 0, t * p.ld_in + n, count, in[i]);
            }
            if (MODE == MODE_EPILOGUE) {
                float z[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) z[i] = fmaf(a[0][i], factor[i], bias[i]);
                if (p.keep[0]) store4_wide(p.keep[0], p.keep_bf16 != 0, t * p.ld_keep + n, count, z);
                with_activation(p.act, [&](auto tag) {
                    activate<decltype(tag)::value>(z[0], z[1]);
                    activate<decltype(tag)::value>(z[2], z[3]);
                });
                if (has_in) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[i] += in[0][i];
                }
                store4(p, p.D[0], t * p.ldd + n, count, z, scale_d, top);
            } else if (MODE == MODE_GATED) {
                float g[4], u[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) { g[i] = a[0][i] * factor[0]; u[i] = a[NB - 1][i] * alpha1; }
                if (p.keep[0]) {
                    store4_wide(p.keep[0], p.keep_bf16 != 0, t * p.ld_keep + n, count, g);
                    store4_wide(p.keep[1], p.keep_bf16 != 0, t * p.ld_keep + n, count, u);
                }
                with_activation(p.act, [&](auto tag) {
                    activate<decltype(tag)::value>(g[0], g[1]);
                    activate<decltype(tag)::value>(g[2], g[3]);
                });
#pragma unroll
                for (int i = 0; i < 4; ++i) g[i] *= u[i];
                store4(p, p.D[0], t * p.ldd + n, count, g, scale_d, top);
            } else {
                float dg[4], du[4];
                with_activation(p.act, [&](auto tag) {
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        Pair value, slope;
                        activate_with_slope<decltype(tag)::value>(in[0][i], in[0][i + 1], value, slope);
                        const Pair dh = Pair(a[0][i], a[0][i + 1]) * Pair(factor[0]);
                        (dh * Pair(in[NIN - 1][i], in[NIN - 1][i + 1]) * slope).split(dg[i], dg[i + 1]);
                        (dh * value).split(du[i], du[i + 1]);
                    }
                });
                store4(p, p.D[0], t * p.ldd + n, count, dg, scale_d, top);
                store4(p, p.D[1], t * p.ldd + n, count, du, scale_d, top);
            }
        }
    }
    if (p.amax_bits) block_fold_amax(canonical_nan_bits(__float_as_uint(top)), red, p.amax_words, p.amax_bits);
}

// ---- products with many rows --------------------------------------------------
//
// Persistent CTA pairs on 256 x 256 accumulator tiles (each CTA holds 128 rows), organised as the plain product kernel: a
// loader warp, an MMA warp in the leader, eight epilogue warps.  The accumulator is moved into the epilogue warps'
// registers chunk by chunk of K and handed back at once, so the epilogue of a tile runs beside the matrix instructions of
// the next one.  Matrices that the epilogue reads (residual; gate and up) and writes move as boxes of 32 rows x 32 columns
// between global and shared memory by TMA: every warp has its own staging slots, a tile's reads are issued while its
// products are still being accumulated, and the TMA unit clips rows and columns past the edges.
// The gated block puts 128 columns of the gate projection and the same 128 of the up projection into one accumulator
// tile (each CTA of the pair stages the weights of one of the two), so that both factors of h meet in one thread.
//
// Bound by the tensor core under the power limit where K is long: 8192 rows, 4096 -> 16384, back to back 454 us without
// activation (the plain product with codes out 453), 502 with gelu_tanh and the pre-activation kept, gated with both products
// kept 940, its backward 588.  At K = 1024 the epilogue bounds (269 us; the plain product 145): each step of 32 columns costs
// some 2000 clocks of waiting and staging beside its arithmetic.

constexpr int BM = 128;
constexpr int TILE_M = 2 * BM;
constexpr int ACC_COLS = 256;
constexpr int TILES_MAX_STAGES = 5, TILES_FG = 2;                      // ring depth; K-blocks per barrier wait
constexpr uint32_t TILES_A_BYTES = BM * BK, TILES_B_BYTES = 128 * BK;
constexpr uint32_t TILES_STAGE_BYTES = TILES_A_BYTES + TILES_B_BYTES;
constexpr int TILES_EPI_WARPS = 8, TILES_EPI_BASE = 4;
constexpr int TILES_THREADS = 32 * (TILES_EPI_BASE + TILES_EPI_WARPS);
constexpr int TILES_REGS_FRONT = 56, TILES_REGS_EPILOGUE = 224;        // 4 x 32 x 56 + 8 x 32 x 224 = 64512 <= 384 x 168
constexpr int TILES_SPLIT_BLOCKS = 16;                                 // split accumulation: a chunk is 2048 of K
constexpr int TILES_GROUP_M = 16;
constexpr int MAX_SLOTS = 4;
// Shared memory holds the ring and the epilogue warps' staging: 5 stages leave 8 KB per warp, 4 leave 12.
constexpr uint32_t TILES_POOL = 224 * 1024, TILES_SMEM = TILES_POOL + 1024;
constexpr uint32_t tiles_warp_bytes(int stages) { return (TILES_POOL - (uint32_t)stages * TILES_STAGE_BYTES) / TILES_EPI_WARPS; }
constexpr uint32_t TILES_TMEM_COLS = 512;

// tile index -> (row-tile, column-tile): GROUP_M row-tiles advance together over the columns, sharing panels in L2
__device__ __forceinline__ void fused_tile_coords(int t, int tiles_m, int tiles_n, int& tm, int& tn) {
    const int per_group = TILES_GROUP_M * tiles_n, g = t / per_group, first_m = g * TILES_GROUP_M;
    const int rows = min(TILES_GROUP_M, tiles_m - first_m), r = t - g * per_group;
    tm = first_m + r % rows;
    tn = r / rows;
}

struct alignas(8) TilesBarriers {
    uint64_t full[TILES_MAX_STAGES], empty[TILES_MAX_STAGES], acc_full[2], acc_empty[2];
    uint64_t in[TILES_EPI_WARPS][MAX_SLOTS];
    uint32_t tmem_base, abort_flag;
};

// Where the pieces of a staging slot lie: byte offsets of the boxes read and written.
struct Staging {
    uint32_t in[2], out[2], keep[2];
    uint32_t slot_bytes, warp_bytes;
    int slots, stages;
    uint32_t in_tx;                     // bytes that arrive per slot
};

struct TilesParams {
    Params p;
    Staging s;
    int tiles_m, tiles_n, chunk_blocks;
};

struct TilesMaps {
    CUtensorMap a, b[2], in[2], out[2], keep[2];
};

// byte offset of 16-byte unit `unit` of row `row` in a box whose rows are 32 << LOG2 bytes long, as the TMA unit swizzles it
__device__ __forceinline__ uint32_t box_offset(int row_bytes, int row, int unit) {
    const int mask = row_bytes >> 4;                                   // units per row: 2, 4, 8
    const int turn = row_bytes == 128 ? row : row_bytes == 64 ? row >> 1 : row >> 2;
    return (uint32_t)(row * row_bytes + ((unit ^ (turn & (mask - 1))) << 4));
}

__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

// Eight consecutive columns (octet `o` of four) of this thread's row in a staged box.
__device__ __forceinline__ void box_load8(uint32_t box, bool bf16, int row, int o, float (&v)[8]) {
    if (bf16) {
        const uint4 w = ld_shared_v4(box + box_offset(64, row, o));
        v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xFFFF0000u);
        v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xFFFF0000u);
        v[4] = __uint_as_float(w.z << 16); v[5] = __uint_as_float(w.z & 0xFFFF0000u);
        v[6] = __uint_as_float(w.w << 16); v[7] = __uint_as_float(w.w & 0xFFFF0000u);
    } else {
        const uint4 w = ld_shared_v4(box + box_offset(128, row, 2 * o)), x = ld_shared_v4(box + box_offset(128, row, 2 * o + 1));
        v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
        v[4] = __uint_as_float(x.x); v[5] = __uint_as_float(x.y); v[6] = __uint_as_float(x.z); v[7] = __uint_as_float(x.w);
    }
}

// All 32 columns of this thread's row written to a staged box.  `v` is a run of the thread's registers.
__device__ __forceinline__ void box_store32_wide(uint32_t box, bool bf16, int row, const float* v) {
    if (bf16) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            st_shared_v4(box + box_offset(64, row, u), pack_bf16(v[8 * u], v[8 * u + 1]), pack_bf16(v[8 * u + 2], v[8 * u + 3]),
                         pack_bf16(v[8 * u + 4], v[8 * u + 5]), pack_bf16(v[8 * u + 6], v[8 * u + 7]));
    } else {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            st_shared_v4(box + box_offset(128, row, u), __float_as_uint(v[4 * u]), __float_as_uint(v[4 * u + 1]), __float_as_uint(v[4 * u + 2]), __float_as_uint(v[4 * u + 3]));
    }
}

// 32 columns of an output: conversion and staging; `most` is their largest magnitude.  One decision for all of them, so
// that the common path is straight-line code.  STORE: FP8_STORE_E4M3, FP8_STORE_E5M2, or a wide type (which one is p.store).
template <int STORE>
__device__ __forceinline__ void emit32(const Params& p, uint32_t box, int row, const float* v, float most, float scale_d) {
    if (STORE <= FP8_STORE_BF16) {
        box_store32_wide(box, p.store == FP8_STORE_BF16, row, v);
        return;
    }
    constexpr int FMT = STORE == FP8_STORE_E5M2 ? kE5M2 : kE4M3;
    uint32_t w[8];
    if (__builtin_expect(converts_packed(most, scale_d, FMT == kE4M3, p.nosat != 0), 1)) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            float y[4];
            (Pair(v[4 * u], v[4 * u + 1]) * Pair(scale_d)).split(y[0], y[1]);
            (Pair(v[4 * u + 2], v[4 * u + 3]) * Pair(scale_d)).split(y[2], y[3]);
            w[u] = cvt_quad<FMT>(y[0], y[1], y[2], y[3]);
        }
    } else {
#pragma unroll
        for (int o = 0; o < 4; ++o) {
            const float x[8] = {v[8 * o], v[8 * o + 1], v[8 * o + 2], v[8 * o + 3], v[8 * o + 4], v[8 * o + 5], v[8 * o + 6], v[8 * o + 7]};
            const uint2 c = encode8_special(x, scale_d, FMT == kE4M3, p.nosat != 0);
            w[2 * o] = c.x;
            w[2 * o + 1] = c.y;
        }
    }
    st_shared_v4(box + box_offset(32, row, 0), w[0], w[1], w[2], w[3]);
    st_shared_v4(box + box_offset(32, row, 1), w[4], w[5], w[6], w[7]);
}

__device__ __forceinline__ float most32(const float* v) {
    float m[4];
#pragma unroll
    for (int o = 0; o < 4; ++o) {
        const float x[8] = {v[8 * o], v[8 * o + 1], v[8 * o + 2], v[8 * o + 3], v[8 * o + 4], v[8 * o + 5], v[8 * o + 6], v[8 * o + 7]};
        m[o] = most8(x);
    }
    return most3(most3(m[0], m[1], m[2]), m[3], 0.0f);
}

// TMEM columns straight into the partial sums (the first chunk of K)
__device__ __forceinline__ void tc_ld32_sums(uint32_t taddr, float* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]),
          "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]),
          "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]),
          "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
        : "r"(taddr) : "memory");
}

// A staged box written to global memory element by element: where it crosses the right edge of rows whose length is not a
// multiple of 16 bytes (the TMA unit clips in such units).  Lane = column.
__device__ __forceinline__ void copy_box_out(void* base, int size, uint32_t box, int64_t row0, int rows, int64_t col, int64_t ld, int lane, bool inside) {
    __syncwarp();
    const int byte = lane * size;
#pragma unroll 1
    for (int r = 0; r < rows && inside; ++r) {
        const uint32_t at = box + box_offset(32 * size, r, byte >> 4) + (uint32_t)(byte & 15);
        uint8_t* to = reinterpret_cast<uint8_t*>(base) + ((row0 + r) * ld + col + lane) * size;
        uint32_t w;
        if (size == 4) {
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
            *reinterpret_cast<uint32_t*>(to) = w;
        } else if (size == 2) {
            asm volatile("ld.shared.u16 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
            *reinterpret_cast<uint16_t*>(to) = (uint16_t)w;
        } else {
            asm volatile("ld.shared.u8 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
            *to = (uint8_t)w;
        }
    }
}

template <int MODE, int ACT, int STORE>
__global__ void __launch_bounds__(TILES_THREADS, 1)
k_fused_tiles(const __grid_constant__ TilesMaps maps, const __grid_constant__ TilesParams tp) {
    const Params& p = tp.p;
    constexpr int OUT_COLS = MODE == MODE_GATED ? 128 : 256;           // columns of D per tile
    constexpr int WARP_COLS = OUT_COLS / 2;                            // two warps share a lane quarter
    constexpr int STEPS = WARP_COLS / 32;
    constexpr int NIN = MODE == MODE_GATED_BWD ? 2 : 1, NOUT = MODE == MODE_GATED_BWD ? 2 : 1;
    extern __shared__ uint8_t smem_raw[];
    __shared__ TilesBarriers bars;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    volatile uint32_t* abort_flag = &bars.abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t cta_rank = cluster_ctarank();
    const int worker = blockIdx.x / 2, num_workers = gridDim.x / 2;
    const int num_tiles = tp.tiles_m * tp.tiles_n;
    const int k_blocks = (int)((p.K + BK - 1) / BK);
    const int k_pad = (k_blocks + TILES_FG - 1) / TILES_FG * TILES_FG;
    const int chunk = tp.chunk_blocks, stages = tp.s.stages;

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) { mbar_init(smem_u32(&bars.full[s]), TILES_FG * 2); mbar_init(smem_u32(&bars.empty[s]), 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(smem_u32(&bars.acc_full[a]), 1); mbar_init(smem_u32(&bars.acc_empty[a]), TILES_EPI_WARPS * 2); }
        for (int w = 0; w < TILES_EPI_WARPS; ++w)
            for (int s = 0; s < MAX_SLOTS; ++s) mbar_init(smem_u32(&bars.in[w][s]), 1);
        bars.abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem_base)), "r"(TILES_TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = bars.tmem_base;
    grid_launch_dependents();               // as in the kernel for few rows
    grid_dependency_wait();

    if (warp < TILES_EPI_BASE) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TILES_REGS_FRONT));
        if (warp == 0) {
            // -------------------------------------------------------- loader: each CTA its rows of A and its half of B.
            // K-blocks go through the ring of stages one by one; each pair of them completes on one barrier of the leader,
            // the pairs' barriers going round on their own.
            int stage = 0, pair = 0;
            uint32_t phase = 1;
            bool ok = true;
            const uint64_t keep = policy_evict_last();
            const CUtensorMap* map_b = &maps.b[MODE == MODE_GATED ? cta_rank : 0];
            const bool a_mn = p.a_mn != 0, b_mn = p.w_mn != 0;
            int tile_no = 0;
            for (int t = worker; t < num_tiles && ok; t += num_workers) {
                int tm, tn;
                fused_tile_coords(t, tp.tiles_m, tp.tiles_n, tm, tn);
                const int m0 = tm * TILE_M + (int)cta_rank * BM;
                const int n0 = MODE == MODE_GATED ? tn * OUT_COLS : tn * OUT_COLS + (int)cta_rank * 128;
                const bool backwards = (tile_no++ & 1) != 0;           // K from its end: the wave meets again in L2
                for (int kb = 0; kb < k_pad; ++kb) {
                    ok = mbar_wait(smem_u32(&bars.empty[stage]), phase, abort_flag, F_WAIT_EMPTY);
                    if (!ok) break;
                    if (lane == 0) {
                        const uint32_t sa = ring + (uint32_t)stage * TILES_STAGE_BYTES, sb = sa + TILES_A_BYTES;
                        const int k0 = (backwards && kb < k_blocks ? k_blocks - 1 - kb : kb) * BK;
                        const uint32_t full = map_to_cta(smem_u32(&bars.full[pair]), 0);
                        if (kb < k_blocks) {
                            mbar_arrive_expect_tx_cluster(full, TILES_STAGE_BYTES);
                            tma_load_3d_pair(sa, &maps.a, a_mn ? m0 : k0, a_mn ? k0 : m0, 0, full, keep);
                            tma_load_3d_pair(sb, map_b, b_mn ? n0 : k0, b_mn ? k0 : n0, 0, full, keep);
                        } else {
                            mbar_arrive_cluster(full);                 // padding block
                        }
                    }
                    __syncwarp();
                    if (++stage == stages) { stage = 0; phase ^= 1u; }
                    if ((kb & 1) != 0 && ++pair == stages) pair = 0;
                }
            }
            if (!ok)                                                   // given up: a millisecond for copies still in flight (their
                for (const long long t0 = clock64(); clock64() - t0 < 2000000ll;) {}     // barrier may be in the other CTA)
        } else if (warp == 1) {
            // -------------------------------------------------------- MMA issuer (leader only)
            int stage = 0, pair = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 1;
            bool ok = cta_rank == 0;
            const uint32_t a_kstep = p.a_mn ? UMMA_K * 128 : UMMA_K, a_lbo = p.a_mn ? BK * 128 : 16;
            const uint32_t b_kstep = p.w_mn ? UMMA_K * 128 : UMMA_K, b_lbo = p.w_mn ? BK * 128 : 16;
            for (int t = worker; t < num_tiles && ok; t += num_workers) {
                for (int kc = 0; kc < k_pad && ok; kc += chunk) {
                    ok = mbar_wait(smem_u32(&bars.acc_empty[acc]), acc_phase, abort_flag, F_WAIT_ACC_EMPTY);
                    if (!ok) break;
                    tc_fence_after();
                    const int kend = min(k_pad, kc + chunk), last_real = min(k_blocks, kend) - 1;
                    for (int kb = kc; kb < kend; kb += TILES_FG) {
                        // one wait per two K-blocks: a barrier query between MMA issues costs about one MMA's time
                        ok = mbar_wait(smem_u32(&bars.full[pair]), phase, abort_flag, F_WAIT_FULL);
                        if (!ok) break;
                        tc_fence_after();
                        const int stage1 = stage + 1 == stages ? 0 : stage + 1;
                        if (lane == 0) {
#pragma unroll
                            for (int h = 0; h < TILES_FG; ++h) {
                                const int st = h == 0 ? stage : stage1;
                                if (kb + h < k_blocks) {
                                    const uint32_t sa = ring + (uint32_t)st * TILES_STAGE_BYTES, sb = sa + TILES_A_BYTES;
#pragma unroll
                                    for (int k = 0; k < BK / UMMA_K; ++k)
                                        tc_mma_f8_pair(tmem + (uint32_t)acc * ACC_COLS, smem_desc(sa + k * a_kstep, a_lbo, 1024),
                                                       smem_desc(sb + k * b_kstep, b_lbo, 1024), p.idesc, ((kb - kc) | h | k) != 0 ? 1u : 0u);
                                }
                                tc_commit_pair(smem_u32(&bars.empty[st]));
                                if (kb + h == last_real) tc_commit_pair(smem_u32(&bars.acc_full[acc]));
                            }
                        }
                        __syncwarp();
                        stage = stage1 + 1 == stages ? 0 : stage1 + 1;
                        if (++pair == stages) { pair = 0; phase ^= 1u; }
                    }
                    if ((acc ^= 1) == 0) acc_phase ^= 1u;
                }
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue: each CTA its own 128 rows
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(TILES_REGS_EPILOGUE));
        const int ew = warp - TILES_EPI_BASE, q = warp & 3, part_no = ew >> 2;
        const float sa_inv = __ldg(p.sa_inv);
        const float alpha0 = p.sb_inv_vec ? 0.0f : sa_inv * __ldg(p.sb_inv[0]);
        const float alpha1 = MODE == MODE_GATED ? sa_inv * __ldg(p.sb_inv[1]) : 0.0f;
        const float scale_d = p.store >= FP8_STORE_E4M3 ? __ldg(p.scale_d) : 1.0f;
        const uint32_t staging = ring + (uint32_t)stages * TILES_STAGE_BYTES + (uint32_t)ew * tp.s.warp_bytes;
        const uint64_t stream = policy_evict_first();
        const bool has_in = tp.s.in_tx != 0u, has_columns = p.bias || p.sb_inv_vec;
        const int out_size = p.store == FP8_STORE_F32 ? 4 : p.store == FP8_STORE_BF16 ? 2 : 1;
        const int keep_size = p.keep_bf16 ? 2 : 4, in_size = p.in_bf16 ? 2 : 4;
        const bool clip_out = ((p.N * out_size) & 15) != 0, clip_keep = ((p.N * keep_size) & 15) != 0;
        const uint32_t columns = staging + tp.s.warp_bytes - 1024;     // 128 factors, 128 biases of this warp's columns
        uint32_t in_phase = 0;                                         // bit s: parity of slot s
        uint32_t issued = 0;                                           // bit s: a read into slot s has not been waited for
        const int M = (int)p.M, N = (int)p.N;                          // below 2^31
        float top = 0.0f;
        float part[128];
        bool ok = true;
        int it = 0;
        const int slots = tp.s.slots;
        int slot = 0;                                                  // of the current step; every step takes the next one
        // lane 0: issue the reads of step `st` of a tile into a slot
        auto issue = [&](int slot, int st, int row0, int col0) {
            if (lane == 0) {
                const uint32_t bar = smem_u32(&bars.in[ew][slot]), at = staging + (uint32_t)slot * tp.s.slot_bytes;
                const int x = (col0 + st * 32) * in_size;
                mbar_arrive_expect_tx(bar, tp.s.in_tx);
#pragma unroll
                for (int i = 0; i < NIN; ++i) tma_load_3d(at + tp.s.in[i], &maps.in[i], x, row0, 0, bar, stream);
            }
            issued |= 1u << slot;
        };
        // factors and biases of this warp's columns of a tile, four columns per lane
        float factor[4], bias[4];
        auto fetch_columns = [&](int tn) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = tn * OUT_COLS + part_no * WARP_COLS + i * 32 + lane;
                factor[i] = alpha0;
                bias[i] = 0.0f;
                if (c < N) {
                    if (p.sb_inv_vec) factor[i] = sa_inv * __ldg(p.sb_inv_vec + c);
                    if (p.bias) bias[i] = p.bias_bf16 ? __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(p.bias) + c) << 16)
                                                      : __ldg(reinterpret_cast<const float*>(p.bias) + c);
                }
            }
        };
        int tm = 0, tn = 0;
        fused_tile_coords(worker, tp.tiles_m, tp.tiles_n, tm, tn);     // (every worker has a tile)
        if (MODE == MODE_EPILOGUE && has_columns) fetch_columns(tn);
        for (int t = worker; t < num_tiles && ok; t += num_workers) {
            const int row0 = tm * TILE_M + (int)cta_rank * BM + q * 32;
            const int col0 = tn * OUT_COLS + part_no * WARP_COLS;
            const bool row_ok = row0 + lane < M;
            // steps with something inside D
            const int steps = row0 < M && col0 < N ? min(STEPS, (N - col0 + 31) / 32) : 0;
            if (MODE == MODE_EPILOGUE && has_columns) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(columns + (uint32_t)(i * 32 + lane) * 4), "f"(factor[i]) : "memory");
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(columns + 512 + (uint32_t)(i * 32 + lane) * 4), "f"(bias[i]) : "memory");
                }
                __syncwarp();
            }
            if (t + num_workers < num_tiles) {                         // the next tile's are on their way during this one
                fused_tile_coords(t + num_workers, tp.tiles_m, tp.tiles_n, tm, tn);
                if (MODE == MODE_EPILOGUE && has_columns) fetch_columns(tn);
            }
            if (has_in && steps > 0) {
                if (lane == 0) bulk_wait_read<0>();                    // the previous tile's boxes have left the slots
                __syncwarp();
                for (int st = 0; st < min(steps, slots); ++st) issue(slot + st < slots ? slot + st : slot + st - slots, st, row0, col0);
            }
            for (int kc = 0; kc < k_pad && ok; kc += chunk, ++it) {
                const uint32_t acc = (uint32_t)it & 1u;
                ok = mbar_wait(smem_u32(&bars.acc_full[acc]), ((uint32_t)it >> 1) & 1u, abort_flag, F_WAIT_ACC_FULL);
                if (!ok) break;
                tc_fence_after();
                const uint32_t taddr = tmem + acc * ACC_COLS + ((uint32_t)(q * 32) << 16);
                // gated: 64 columns of the gate half, then the same 64 of the up half
                auto column = [&](int j) { return (uint32_t)(MODE == MODE_GATED ? (j >> 1) * 128 + part_no * 64 + (j & 1) * 32 : part_no * 128 + j * 32); };
                if (kc == 0) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) tc_ld32_sums(taddr + column(j), part + j * 32);
                    tc_wait_ld();
                } else {
#pragma unroll
                    for (int s2 = 0; s2 < 2; ++s2) {
                        uint32_t r[2][32];
#pragma unroll
                        for (int h = 0; h < 2; ++h) tc_ld32(taddr + column(2 * s2 + h), r[h]);
                        tc_wait_ld();
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                float* s = part + (2 * s2 + h) * 32 + i;
                                (Pair(s[0], s[1]) + Pair(__uint_as_float(r[h][i]), __uint_as_float(r[h][i + 1]))).split(s[0], s[1]);
                            }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to_cta(smem_u32(&bars.acc_empty[acc]), 0));
            }
            if (!ok) break;
            // The loop takes two steps a round: its body is hundreds of instructions, and the warps come through it at different
            // times, so fully unrolled they wait for instruction fetches more than for anything else.  A round works on the
            // first 64 sums, then moves the others down.  What is rarely needed (special values, ragged edges) is kept out of
            // the straight line.  (One step a round: gated backward at K = 1024 346 us instead of 329.)
#pragma unroll 1
            for (int round = 0; round < steps; round += 2) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int st = round + half;
                    if (st >= steps || !ok) break;
                    const uint32_t at = staging + (uint32_t)slot * tp.s.slot_bytes;
                    const int col = col0 + st * 32;
                    const bool ragged = col + 32 > N;
                    if (has_in) {
                        ok = mbar_wait(smem_u32(&bars.in[ew][slot]), (in_phase >> slot) & 1u, abort_flag, F_WAIT_IN);
                        if (!ok) break;
                        in_phase ^= 1u << slot;
                        issued &= ~(1u << slot);
                    } else {
                        if (lane == 0) {                                   // the boxes last stored from this slot have left it
                            if (slots >= 4) bulk_wait_read<3>();
                            else if (slots == 3) bulk_wait_read<2>();
                            else if (slots == 2) bulk_wait_read<1>();
                            else bulk_wait_read<0>();
                        }
                        __syncwarp();
                    }
                    float* x = part + half * 32;                                       // this step's sums become its results in place
                    float y[32];
                    if (MODE == MODE_EPILOGUE) {
                        if (has_columns) {
#pragma unroll
                            for (int u = 0; u < 8; ++u) {
                                const float4 f = ld_shared_f4(columns + (uint32_t)(st * 32 + u * 4) * 4), b = ld_shared_f4(columns + 512 + (uint32_t)(st * 32 + u * 4) * 4);
                                x[u * 4 + 0] = fmaf(x[u * 4 + 0], f.x, b.x);
                                x[u * 4 + 1] = fmaf(x[u * 4 + 1], f.y, b.y);
                                x[u * 4 + 2] = fmaf(x[u * 4 + 2], f.z, b.z);
                                x[u * 4 + 3] = fmaf(x[u * 4 + 3], f.w, b.w);
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[i] *= alpha0;
                        }
                        if (p.keep[0]) box_store32_wide(at + tp.s.keep[0], p.keep_bf16 != 0, lane, x);
#pragma unroll
                        for (int i = 0; i < 32; i += 2) activate<ACT>(x[i], x[i + 1]);
                        if (has_in) {
#pragma unroll
                            for (int o = 0; o < 4; ++o) {
                                float r[8];
                                box_load8(at + tp.s.in[0], p.in_bf16 != 0, lane, o, r);
#pragma unroll
                                for (int i = 0; i < 8; ++i) x[o * 8 + i] += r[i];
                            }
                        }
                    } else if (MODE == MODE_GATED) {
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            (Pair(x[i], x[i + 1]) * Pair(alpha0)).split(x[i], x[i + 1]);
                            (Pair(part[(64 + half * 32 + i) & 127], part[(65 + half * 32 + i) & 127]) * Pair(alpha1)).split(y[i], y[i + 1]);
                        }
                        if (p.keep[0]) {
                            box_store32_wide(at + tp.s.keep[0], p.keep_bf16 != 0, lane, x);
                            box_store32_wide(at + tp.s.keep[1], p.keep_bf16 != 0, lane, y);
                        }
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            activate<ACT>(x[i], x[i + 1]);
                            (Pair(x[i], x[i + 1]) * Pair(y[i], y[i + 1])).split(x[i], x[i + 1]);
                        }
                    } else {
#pragma unroll
                        for (int o = 0; o < 4; ++o) {
                            float g[8], u[8];
                            box_load8(at + tp.s.in[0], p.in_bf16 != 0, lane, o, g);
                            box_load8(at + tp.s.in[NIN - 1], p.in_bf16 != 0, lane, o, u);
#pragma unroll
                            for (int i = 0; i < 8; i += 2) {
                                Pair value, slope;
                                activate_with_slope<ACT>(g[i], g[i + 1], value, slope);
                                const Pair dh = Pair(x[o * 8 + i], x[o * 8 + i + 1]) * Pair(alpha0);
                                (dh * Pair(u[i], u[i + 1]) * slope).split(x[o * 8 + i], x[o * 8 + i + 1]);
                                (dh * value).split(y[o * 8 + i], y[o * 8 + i + 1]);
                            }
                        }
                    }
                    if (__builtin_expect(ragged, 0)) {                     // columns past N count for nothing
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (col + i >= N) { x[i] = 0.0f; if (MODE == MODE_GATED_BWD) y[i] = 0.0f; }
                    }
                    float most = most32(x);
                    emit32<STORE>(p, at + tp.s.out[0], lane, x, most, scale_d);
                    if (MODE == MODE_GATED_BWD) {
                        const float most_y = most32(y);
                        emit32<STORE>(p, at + tp.s.out[NOUT - 1], lane, y, most_y, scale_d);
                        most = fmax_nan(most, most_y);
                    }
                    if (row_ok) top = fmax_nan(top, most);
                    const bool by_hand = ragged && clip_out, keep_by_hand = ragged && clip_keep;
                    if (__builtin_expect(ragged, 0)) {
                        const int rows = min(32, M - row0);
                        const bool inside = col + lane < N;
                        if (by_hand) {
                            copy_box_out(p.D[0], out_size, at + tp.s.out[0], row0, rows, col, p.ldd, lane, inside);
                            if (MODE == MODE_GATED_BWD) copy_box_out(p.D[1], out_size, at + tp.s.out[NOUT - 1], row0, rows, col, p.ldd, lane, inside);
                        }
                        if (MODE != MODE_GATED_BWD && keep_by_hand && p.keep[0]) {
                            copy_box_out(p.keep[0], keep_size, at + tp.s.keep[0], row0, rows, col, p.ld_keep, lane, inside);
                            if (MODE == MODE_GATED) copy_box_out(p.keep[1], keep_size, at + tp.s.keep[1], row0, rows, col, p.ld_keep, lane, inside);
                        }
                    }
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        if (!by_hand) {
#pragma unroll
                            for (int i = 0; i < NOUT; ++i) tma_store_3d(&maps.out[i], at + tp.s.out[i], col * out_size, row0, 0, stream);
                        }
                        if (MODE != MODE_GATED_BWD && p.keep[0] && !keep_by_hand) {
#pragma unroll
                            for (int i = 0; i < (MODE == MODE_GATED ? 2 : 1); ++i) tma_store_3d(&maps.keep[i], at + tp.s.keep[i], col * keep_size, row0, 0, stream);
                        }
                        bulk_commit();
                    }
                    if (has_in && st + slots < steps) {                    // the slot's next read, once these boxes have left it
                        if (lane == 0) bulk_wait_read<0>();
                        __syncwarp();
                        issue(slot, st + slots, row0, col0);
                    }
                    if (++slot == slots) slot = 0;
                }
                if (MODE != MODE_GATED) {
#pragma unroll
                    for (int i = 0; i < 64; ++i) part[i] = part[64 + i];
                }
            }
        }
        if (!ok) {                                                     // given up: wait (bounded) for reads still in flight
            for (int s = 0; s < MAX_SLOTS; ++s)
                if ((issued >> s) & 1u)
                    for (int spin = 0; spin < (1 << 20) && !mbar_try_wait(smem_u32(&bars.in[ew][s]), (in_phase >> s) & 1u); ++spin) {}
        }
        if (lane == 0) bulk_wait_all();                                // every store has reached global memory before exit
        if (p.amax_bits) {
            if (p.store == FP8_STORE_BF16) top = __uint_as_float(pack_bf16(top, 0.0f) << 16);      // of the values as stored
            const uint32_t bits = warp_max_u32(canonical_nan_bits(__float_as_uint(top)));
            if (lane == 0) {
                if (p.amax_words) fold_amax(bits, gridDim.x * TILES_EPI_WARPS, p.amax_words, p.amax_bits);
                else if (bits != 0u) atomicMax(p.amax_bits, bits);
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                     // neither CTA leaves while the other may still touch its smem, barriers or TMEM
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TILES_TMEM_COLS) : "memory");
    }
}

// ---- host ------------------------------------------------------------------

static bool wide_ok(int t) { return t == FP8_F32 || t == FP8_BF16; }
static int64_t store_bytes(int store) { return store == FP8_STORE_F32 ? 4 : store == FP8_STORE_BF16 ? 2 : 1; }
static bool misaligned(const void* p, int64_t pitch_bytes) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0 || (pitch_bytes & 15) != 0; }

static fp8_status launch_cluster(const void* kernel, dim3 grid, dim3 cluster, int threads, uint32_t smem, cudaStream_t st, void** args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster.x;
    attr[0].val.clusterDim.y = cluster.y;
    attr[0].val.clusterDim.z = cluster.z;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (cudaLaunchKernelExC(&cfg, kernel, args) != cudaSuccess) { (void)cudaGetLastError(); return FP8_ERR_CUDA; }
    count_launches(1);
    return launch_status();
}

// A kernel's dynamic shared memory limit is raised once per (kernel, device).
static bool allow_smem(const void* kernel, uint32_t bytes) {
    static std::mutex mu;
    static const void* done[64][64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
    std::lock_guard<std::mutex> lock(mu);
    int i = 0;
    while (i < 64 && done[dev][i] && done[dev][i] != kernel) ++i;
    if (i < 64 && done[dev][i] == kernel) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) { (void)cudaGetLastError(); return false; }
    if (i < 64) done[dev][i] = kernel;
    return true;
}

// CTA pairs of a tiles kernel that can be resident at once on the current device (looked up once per kernel and device).
static int pair_workers(const void* kernel) {
    static std::mutex mu;
    static struct { const void* k; int n; } known[64][48] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return sm_count() / 2;
    std::lock_guard<std::mutex> lock(mu);
    int i = 0;
    while (i < 48 && known[dev][i].k && known[dev][i].k != kernel) ++i;
    if (i < 48 && known[dev][i].k == kernel) return known[dev][i].n;
    int n = sm_count() / 2, clusters = 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * n), 1, 1);
    cfg.blockDim = dim3(TILES_THREADS, 1, 1);
    cfg.dynamicSmemBytes = TILES_SMEM;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) == cudaSuccess && clusters > 0 && clusters < n) n = clusters;
    if (i < 48) { known[dev][i].k = kernel; known[dev][i].n = n; }
    return n;
}

// The start value of the amax where no workspace takes its place: enqueued when nothing but the kernel itself is left to do,
// so that a refused call leaves nothing behind.
static fp8_status start_amax(const Params& p, cudaStream_t st) {
    return p.amax_bits && !p.amax_words ? launch_zero_word(p.amax_bits, st) : FP8_OK;
}

constexpr int64_t MAX_GRID_Y = 65535;

static void skip_rows(Params& p, int64_t rows) {
    p.M -= rows;
    for (int i = 0; i < 2; ++i) {
        if (p.in[i]) p.in[i] = reinterpret_cast<const uint8_t*>(p.in[i]) + rows * p.ld_in * (p.in_bf16 ? 2 : 4);
        if (p.keep[i]) p.keep[i] = reinterpret_cast<uint8_t*>(p.keep[i]) + rows * p.ld_keep * (p.keep_bf16 ? 2 : 4);
        if (p.D[i]) p.D[i] = reinterpret_cast<uint8_t*>(p.D[i]) + rows * p.ldd * store_bytes(p.store);
    }
}

template <int MODE, int T>
static fp8_status launch_rows(const fp8_gemm_desc* d, const uint8_t* A, const uint8_t* B0, const uint8_t* B1, Params& p, cudaStream_t st) {
    using G = RowsGeo<MODE, T>;
    const bool w_mn = d->mb == FP8_MAJOR_MN;
    CUtensorMap w0 = {}, w1 = {}, x = {};
    if (d->K > 0) {
        bool ok = make_map(&x, A, (uint64_t)d->K, (uint64_t)d->M, (uint64_t)d->lda, 1, 0, BK, T);
        const uint64_t inner = (uint64_t)(w_mn ? d->N : d->K), outer = (uint64_t)(w_mn ? d->K : d->N);
        ok = ok && make_map(&w0, B0, inner, outer, (uint64_t)d->ldb, 1, 0, 128, 128);
        ok = ok && (!B1 || make_map(&w1, B1, inner, outer, (uint64_t)d->ldb, 1, 0, 128, 128));
        if (!ok) return FP8_ERR_CUDA;
    }
    p.w_mn = w_mn ? 1 : 0;
    // instruction descriptor: fp32 accumulate; the weights are the tensor core's A operand (M = 128), the tokens its B (N = T)
    p.idesc = (1u << 4) | ((uint32_t)d->fb << 7) | ((uint32_t)d->fa << 10) | ((w_mn ? 1u : 0u) << 15) |
              ((uint32_t)(T >> 3) << 17) | ((uint32_t)(ROWS_BN >> 4) << 24);
    const int64_t tiles_n = (d->N + ROWS_BN - 1) / ROWS_BN, tiles_t = (d->M + T - 1) / T;
    const int64_t k_blocks = (d->K + BK - 1) / BK;
    unsigned slices = 1;
    while (slices < 8 && tiles_n * tiles_t * slices * 2 <= 2 * (int64_t)sm_count() && k_blocks >= 8 * (int64_t)slices) slices *= 2;
    const void* k = reinterpret_cast<const void*>(&k_fused_rows<MODE, T>);
    const int rows = d->M < T ? (int)d->M : T;
    int stages = G::stages(rows);
    const uint32_t smem = (uint32_t)stages * G::STAGE_BYTES + G::exchange_bytes(rows) + 1024;
    if (!allow_smem(k, ROWS_SMEM)) return FP8_ERR_CUDA;
    fp8_status rc = start_amax(p, st);
    void* args[] = {&w0, &w1, &x, &p, &stages};
    // The tiles of a launch lie on grid y, which ends at 65535.  Only an empty sum (K == 0) can have more: it takes several
    // launches, which fold into one amax (no workspace is used for it).
    for (int64_t done = 0; rc == FP8_OK && done < tiles_t; done += MAX_GRID_Y) {
        const int64_t here = tiles_t - done < MAX_GRID_Y ? tiles_t - done : MAX_GRID_Y;
        rc = launch_cluster(k, dim3((unsigned)tiles_n, (unsigned)here, slices), dim3(1, 1, slices), ROWS_THREADS, smem, st, args);
        skip_rows(p, here * T);
    }
    return rc;
}

// Tensor map of a wide or FP8 matrix in boxes of 32 rows x 32 columns (`size` bytes per element).
static bool make_box_map(CUtensorMap* map, const void* base, const Params& p, int64_t ld, int size) {
    const CUtensorMapSwizzle swizzle = size == 4 ? CU_TENSOR_MAP_SWIZZLE_128B : size == 2 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B;
    return make_map(map, base, (uint64_t)(p.N * size), (uint64_t)p.M, (uint64_t)(ld * size), 1, 0, (uint32_t)(32 * size), 32, swizzle);
}

template <int MODE, int ACT, int STORE>
static fp8_status launch_tiles(const fp8_gemm_desc* d, const uint8_t* A, const uint8_t* B0, const uint8_t* B1, Params& p, cudaStream_t st) {
    const bool a_mn = d->ma == FP8_MAJOR_MN, w_mn = d->mb == FP8_MAJOR_MN;
    TilesMaps m = {};
    TilesParams tp = {};
    bool ok = a_mn ? make_map(&m.a, A, (uint64_t)d->M, (uint64_t)d->K, (uint64_t)d->lda, 1, 0, 128, BK)
                   : make_map(&m.a, A, (uint64_t)d->K, (uint64_t)d->M, (uint64_t)d->lda, 1, 0, BK, BM);
    const uint64_t inner = (uint64_t)(w_mn ? d->N : d->K), outer = (uint64_t)(w_mn ? d->K : d->N);
    ok = ok && make_map(&m.b[0], B0, inner, outer, (uint64_t)d->ldb, 1, 0, 128, 128);
    ok = ok && (!B1 || make_map(&m.b[1], B1, inner, outer, (uint64_t)d->ldb, 1, 0, 128, 128));
    // boxes of the epilogue and their places in a staging slot; an output of the size of an input takes its place
    const int out_size = (int)store_bytes(p.store), in_size = p.in_bf16 ? 2 : 4, keep_size = p.keep_bf16 ? 2 : 4;
    uint32_t at = 0;
    for (int i = 0; i < 2; ++i) {
        if (p.in[i]) {
            ok = ok && make_box_map(&m.in[i], p.in[i], p, p.ld_in, in_size);
            tp.s.in[i] = at;
            at += 1024u * in_size;
            tp.s.in_tx += 1024u * in_size;
        }
    }
    for (int i = 0; i < 2; ++i) {
        if (p.D[i]) {
            ok = ok && make_box_map(&m.out[i], p.D[i], p, p.ldd, out_size);
            if (p.in[i] && in_size == out_size) tp.s.out[i] = tp.s.in[i];
            else { tp.s.out[i] = at; at += 1024u * out_size; }
        }
    }
    for (int i = 0; i < 2; ++i) {
        if (p.keep[i]) {
            ok = ok && make_box_map(&m.keep[i], p.keep[i], p, p.ld_keep, keep_size);
            tp.s.keep[i] = at;
            at += 1024u * keep_size;
        }
    }
    if (!ok) return FP8_ERR_CUDA;
    // Five stages, or four where a warp would then have no slot, or only one although it reads boxes and K is short enough
    // for the epilogue to matter.  Measured (8192 rows, back to back): gated block with both products kept 985 us at five
    // stages and one slot, 1013 at four and two; its backward pass at K = 4096 626 and 605; six stages gain nothing.
    const uint32_t columns = MODE == MODE_EPILOGUE && (p.bias || p.sb_inv_vec) ? 1024 : 0;
    auto slots_at = [&](int stages) { return (int)((tiles_warp_bytes(stages) - columns) / at); };
    const int wanted = tp.s.in_tx != 0 && d->K <= 8192 ? 2 : 1;
    const int stages = slots_at(5) >= wanted ? 5 : 4;
    tp.s.stages = stages;
    tp.s.slot_bytes = at;
    tp.s.warp_bytes = tiles_warp_bytes(stages);
    tp.s.slots = slots_at(stages) < MAX_SLOTS ? slots_at(stages) : MAX_SLOTS;
    p.a_mn = a_mn ? 1 : 0; p.w_mn = w_mn ? 1 : 0;
    p.idesc = (1u << 4) | ((uint32_t)d->fa << 7) | ((uint32_t)d->fb << 10) | ((a_mn ? 1u : 0u) << 15) | ((w_mn ? 1u : 0u) << 16) |
              ((uint32_t)(ACC_COLS >> 3) << 17) | ((uint32_t)(TILE_M >> 4) << 24);
    const int out_cols = MODE == MODE_GATED ? 128 : 256;
    const int64_t tiles_m = (d->M + TILE_M - 1) / TILE_M, tiles_n = (d->N + out_cols - 1) / out_cols;
    const int k_pad = (int)((d->K + BK - 1) / BK + TILES_FG - 1) / TILES_FG * TILES_FG;
    tp.p = p;
    tp.tiles_m = (int)tiles_m; tp.tiles_n = (int)tiles_n;
    tp.chunk_blocks = d->acc == FP8_ACC_SPLIT ? TILES_SPLIT_BLOCKS : k_pad;
    const void* k = reinterpret_cast<const void*>(&k_fused_tiles<MODE, ACT, STORE>);
    if (!allow_smem(k, TILES_SMEM)) return FP8_ERR_CUDA;
    const int workers = pair_workers(k);
    const int64_t use = tiles_m * tiles_n < workers ? tiles_m * tiles_n : workers;
    const fp8_status rc = start_amax(p, st);
    if (rc != FP8_OK) return rc;
    void* args[] = {&m, &tp};
    return launch_cluster(k, dim3((unsigned)(2 * use), 1, 1), dim3(2, 1, 1), TILES_THREADS, TILES_SMEM, st, args);
}

template <int MODE, int ACT>
static fp8_status dispatch_tiles(const fp8_gemm_desc* d, const uint8_t* A, const uint8_t* B0, const uint8_t* B1, Params& p, cudaStream_t st) {
    switch (p.store) {
        case FP8_STORE_E4M3: return launch_tiles<MODE, ACT, FP8_STORE_E4M3>(d, A, B0, B1, p, st);
        case FP8_STORE_E5M2: return launch_tiles<MODE, ACT, FP8_STORE_E5M2>(d, A, B0, B1, p, st);
        default: return launch_tiles<MODE, ACT, FP8_STORE_BF16>(d, A, B0, B1, p, st);
    }
}

template <int MODE>
static fp8_status dispatch(const fp8_gemm_desc* d, const uint8_t* A, const uint8_t* B0, const uint8_t* B1, Params& p, cudaStream_t st) {
    // The kernel for few rows takes up to 64 rows, and up to 256 where its tiles (128 columns x 64 rows) still fit the SMs in
    // one go.  Measured against the other, 4096 -> 4096: 100 rows 11.7 and 20.5 us, 256 rows 16.7 and 20.7, 333 rows 23.7 and
    // 21.0; 16384 -> 4096 at 200 rows 35.5 and 56.4; 4096 -> 16384 at 100 rows, two rounds of tiles, 26.9 and 25.3.
    const int64_t small_tiles = ((d->N + ROWS_BN - 1) / ROWS_BN) * ((d->M + 63) / 64);
    const bool few_rows = d->M <= 64 || (MODE != MODE_GATED && d->M <= 256 && small_tiles <= sm_count());
    if (d->K > 0 && (!few_rows || d->ma == FP8_MAJOR_MN)) {
        switch (p.act) {
            case FP8_ACT_RELU: return dispatch_tiles<MODE, FP8_ACT_RELU>(d, A, B0, B1, p, st);
            case FP8_ACT_GELU: return dispatch_tiles<MODE, FP8_ACT_GELU>(d, A, B0, B1, p, st);
            case FP8_ACT_GELU_TANH: return dispatch_tiles<MODE, FP8_ACT_GELU_TANH>(d, A, B0, B1, p, st);
            case FP8_ACT_SILU: return dispatch_tiles<MODE, FP8_ACT_SILU>(d, A, B0, B1, p, st);
            default: return dispatch_tiles<MODE, FP8_ACT_NONE>(d, A, B0, B1, p, st);
        }
    }
    if (d->M <= 16) return launch_rows<MODE, 16>(d, A, B0, B1, p, st);
    if (d->M <= 32) return launch_rows<MODE, 32>(d, A, B0, B1, p, st);
    if (MODE != MODE_GATED && d->M <= 48) return launch_rows<MODE, MODE == MODE_GATED ? 32 : 48>(d, A, B0, B1, p, st);
    // (the two operands of the gated block leave no room for the sums of 64 rows)
    return launch_rows<MODE, MODE == MODE_GATED ? 32 : 64>(d, A, B0, B1, p, st);
}

// ---- validation shared by the three entry points: nothing is enqueued before every check has passed ----------------

static bool enums_ok(const fp8_gemm_desc* d, int act, int store, int overflow) {
    return (d->fa == FP8_E4M3 || d->fa == FP8_E5M2) && (d->fb == FP8_E4M3 || d->fb == FP8_E5M2) &&
           (d->ma == FP8_MAJOR_K || d->ma == FP8_MAJOR_MN) && (d->mb == FP8_MAJOR_K || d->mb == FP8_MAJOR_MN) &&
           (d->acc == FP8_ACC_FAST || d->acc == FP8_ACC_SPLIT) && act >= FP8_ACT_NONE && act <= FP8_ACT_SILU &&
           store >= FP8_STORE_F32 && store <= FP8_STORE_E5M2 && (overflow == FP8_SATURATE || overflow == FP8_NOSAT);
}
// operands and D; `B1` only where the mode has it
static fp8_status check_product(const fp8_gemm_desc* d, const uint8_t* A, const uint8_t* B0, const uint8_t* B1, bool two,
                                const void* D0, const void* D1, bool two_out, int store) {
    if (d->M < 0 || d->N < 0 || d->K < 0) return FP8_ERR_SHAPE;
    if (d->M == 0 || d->N == 0) return FP8_OK;
    if (!D0 || (two_out && !D1)) return FP8_ERR_NULL;
    if (d->ldd < d->N) return FP8_ERR_SHAPE;
    if (d->K > 0) {
        if (!A || !B0 || (two && !B1)) return FP8_ERR_NULL;
        if (d->lda < (d->ma == FP8_MAJOR_MN ? d->M : d->K) || d->ldb < (d->mb == FP8_MAJOR_MN ? d->N : d->K)) return FP8_ERR_SHAPE;
        if (misaligned(A, d->lda) || misaligned(B0, d->ldb) || (two && misaligned(B1, d->ldb))) return FP8_ERR_ALIGN;
    }
    if (misaligned(D0, d->ldd * store_bytes(store)) || (two_out && misaligned(D1, d->ldd * store_bytes(store)))) return FP8_ERR_ALIGN;
    const int64_t most = ((int64_t)1 << 31) - 512;
    // (byte coordinates along a row of four-byte elements are 32-bit)
    if (d->M > most || d->N > most / 4 || d->K > most || ((d->M + 127) / 128) * ((d->N + 127) / 128) > (int64_t)1 << 30) return FP8_ERR_UNSUPPORTED;
    return FP8_OK;
}

// How the amax gets its start value.  With the workspace the call is one launch (2.0 us less host time: one token 4096 -> 128
// with codes out 12.6 us, then 10.6), but the kernel ends with three more round trips to L2; without it the launch of the
// one-thread kernel hides behind the kernel before it.  So the workspace serves the short kernels, bound by launches, and calls
// that move more than 32 MB (5 us of HBM time) leave it alone: gated block of one token, 134 MB, 22.1 us without and 23.1 us
// with it.  Nor is it used where several launches may share the rows (see launch_rows).
// `done`: there is nothing to compute, and the amax is 0; `words`: the workspace, where it is to be used.
static fp8_status prepare_amax(const fp8_gemm_desc* d, int operands, float* amax, void* workspace, bool& done, void*& words, cudaStream_t st) {
    done = d->M == 0 || d->N == 0;
    const double bytes = (double)d->K * ((double)d->N * operands + (double)d->M) + 4.0 * (double)d->M * (double)d->N;
    words = workspace && d->K > 0 && bytes <= 32.0 * (1 << 20) ? workspace : nullptr;
    return amax && done ? launch_zero_word(reinterpret_cast<uint32_t*>(amax), st) : FP8_OK;
}

static Params common_params(const fp8_gemm_desc* d, int act, int store, int overflow, const float* scale_d, float* amax, void* workspace) {
    Params p = {};
    p.M = d->M; p.N = d->N; p.K = d->K; p.ldd = d->ldd;
    p.act = act; p.store = store; p.nosat = overflow == FP8_NOSAT ? 1 : 0;
    p.scale_d = scale_d;
    p.amax_bits = reinterpret_cast<uint32_t*>(amax);
    p.amax_words = amax ? reinterpret_cast<unsigned int*>(workspace) : nullptr;
    return p;
}

}  // namespace fused

// Reads and clears this file's error latch.
void fused_read_clear_latch(unsigned int out2[2]) {
    out2[0] = out2[1] = 0u;
    if (cudaMemcpyFromSymbol(out2, g_async_latch, 2 * sizeof(unsigned int)) != cudaSuccess || out2[0] == 0u) return;
    const unsigned int zero[2] = {0u, 0u};
    (void)cudaMemcpyToSymbol(g_async_latch, zero, sizeof(zero));
}

}  // namespace fp8b200

using namespace fp8b200;

extern "C" {

fp8_status fp8_gemm_epilogue(const fp8_gemm_desc* d, const fp8_epilogue* e, const uint8_t* A, const uint8_t* B, void* D,
                             const float* scale_inv_a_dev, const float* scale_inv_b_dev, const float* scale_d_dev,
                             float* amax_d_dev, void* workspace_dev, void* stream) {
    using namespace fp8b200::fused;
    if (!d || !e || !scale_inv_a_dev || (!scale_inv_b_dev && !e->scale_inv_b_vec_dev)) return FP8_ERR_NULL;
    if (!enums_ok(d, e->act, e->store, e->overflow) || !wide_ok(e->bias_t) || !wide_ok(e->residual_t) || !wide_ok(e->pre_t)) return FP8_ERR_ENUM;
    if (e->store >= FP8_STORE_E4M3 && !scale_d_dev) return FP8_ERR_NULL;
    fp8_status rc = check_product(d, A, B, nullptr, false, D, nullptr, false, e->store);
    if (rc != FP8_OK) return rc;
    if (reinterpret_cast<uintptr_t>(workspace_dev) & 15u) return FP8_ERR_ALIGN;
    const int64_t r_size = e->residual_t == FP8_BF16 ? 2 : 4, p_size = e->pre_t == FP8_BF16 ? 2 : 4;
    if (d->M > 0 && d->N > 0) {
        if ((e->residual && e->ldr < d->N) || (e->pre && e->ldp < d->N)) return FP8_ERR_SHAPE;
        if ((e->residual && misaligned(e->residual, e->ldr * r_size)) || (e->pre && misaligned(e->pre, e->ldp * p_size))) return FP8_ERR_ALIGN;
        if (e->bias && (reinterpret_cast<uintptr_t>(e->bias) & (e->bias_t == FP8_BF16 ? 1u : 3u))) return FP8_ERR_ALIGN;
    }
    cudaStream_t st = (cudaStream_t)stream;
    bool done = false;
    void* words = nullptr;
    if ((rc = prepare_amax(d, 1, amax_d_dev, workspace_dev, done, words, st)) != FP8_OK || done) return rc;
    Params p = common_params(d, e->act, e->store, e->overflow, scale_d_dev, amax_d_dev, words);
    p.sa_inv = scale_inv_a_dev; p.sb_inv[0] = scale_inv_b_dev; p.sb_inv_vec = e->scale_inv_b_vec_dev;
    p.bias = e->bias; p.bias_bf16 = e->bias_t == FP8_BF16;
    p.in[0] = e->residual; p.in_bf16 = e->residual_t == FP8_BF16; p.ld_in = e->ldr;
    p.keep[0] = e->pre; p.keep_bf16 = e->pre_t == FP8_BF16; p.ld_keep = e->ldp;
    p.D[0] = D;
    return dispatch<MODE_EPILOGUE>(d, A, B, nullptr, p, st);
}

static fp8_status check_gate(const fp8_gemm_desc* d, const fp8_gated* w) {
    if (d->M == 0 || d->N == 0 || !w->gate) return FP8_OK;
    if (w->ldg < d->N) return FP8_ERR_SHAPE;
    const int64_t size = w->gate_t == FP8_BF16 ? 2 : 4;
    return fp8b200::fused::misaligned(w->gate, w->ldg * size) || fp8b200::fused::misaligned(w->up, w->ldg * size) ? FP8_ERR_ALIGN : FP8_OK;
}

fp8_status fp8_gemm_gated(const fp8_gemm_desc* d, const fp8_gated* w, const uint8_t* A, const uint8_t* Bg, const uint8_t* Bu, void* H,
                          const float* scale_inv_a_dev, const float* scale_inv_bg_dev, const float* scale_inv_bu_dev,
                          const float* scale_h_dev, float* amax_h_dev, void* workspace_dev, void* stream) {
    using namespace fp8b200::fused;
    if (!d || !w || !scale_inv_a_dev || !scale_inv_bg_dev || !scale_inv_bu_dev || !w->gate != !w->up) return FP8_ERR_NULL;
    if (!enums_ok(d, w->act, w->store, w->overflow) || !wide_ok(w->gate_t)) return FP8_ERR_ENUM;
    if (w->store >= FP8_STORE_E4M3 && !scale_h_dev) return FP8_ERR_NULL;
    fp8_status rc = check_product(d, A, Bg, Bu, true, H, nullptr, false, w->store);
    if (rc == FP8_OK && (reinterpret_cast<uintptr_t>(workspace_dev) & 15u)) rc = FP8_ERR_ALIGN;
    if (rc != FP8_OK || (rc = check_gate(d, w)) != FP8_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    bool done = false;
    void* words = nullptr;
    if ((rc = prepare_amax(d, 2, amax_h_dev, workspace_dev, done, words, st)) != FP8_OK || done) return rc;
    Params p = common_params(d, w->act, w->store, w->overflow, scale_h_dev, amax_h_dev, words);
    p.sa_inv = scale_inv_a_dev; p.sb_inv[0] = scale_inv_bg_dev; p.sb_inv[1] = scale_inv_bu_dev;
    p.keep[0] = w->gate; p.keep[1] = w->up; p.keep_bf16 = w->gate_t == FP8_BF16; p.ld_keep = w->ldg;
    p.D[0] = H;
    return dispatch<MODE_GATED>(d, A, Bg, Bu, p, st);
}

fp8_status fp8_gemm_gated_backward(const fp8_gemm_desc* d, const fp8_gated* w, const uint8_t* A, const uint8_t* B, void* dG, void* dU,
                                   const float* scale_inv_a_dev, const float* scale_inv_b_dev, const float* scale_d_dev,
                                   float* amax_dev, void* workspace_dev, void* stream) {
    using namespace fp8b200::fused;
    if (!d || !w || !scale_inv_a_dev || !scale_inv_b_dev) return FP8_ERR_NULL;
    if (!enums_ok(d, w->act, w->store, w->overflow) || !wide_ok(w->gate_t)) return FP8_ERR_ENUM;
    if (w->store >= FP8_STORE_E4M3 && !scale_d_dev) return FP8_ERR_NULL;
    if (d->M > 0 && d->N > 0 && (!w->gate || !w->up)) return FP8_ERR_NULL;
    fp8_status rc = check_product(d, A, B, nullptr, false, dG, dU, true, w->store);
    if (rc == FP8_OK && (reinterpret_cast<uintptr_t>(workspace_dev) & 15u)) rc = FP8_ERR_ALIGN;
    if (rc != FP8_OK || (rc = check_gate(d, w)) != FP8_OK) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    bool done = false;
    void* words = nullptr;
    if ((rc = prepare_amax(d, 1, amax_dev, workspace_dev, done, words, st)) != FP8_OK || done) return rc;
    Params p = common_params(d, w->act, w->store, w->overflow, scale_d_dev, amax_dev, words);
    p.sa_inv = scale_inv_a_dev; p.sb_inv[0] = scale_inv_b_dev;
    p.in[0] = w->gate; p.in[1] = w->up; p.in_bf16 = w->gate_t == FP8_BF16; p.ld_in = w->ldg;
    p.D[0] = dG; p.D[1] = dU;
    return dispatch<MODE_GATED_BWD>(d, A, B, nullptr, p, st);
}

}  // extern "C"
