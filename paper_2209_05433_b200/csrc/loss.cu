// Softmax cross entropy of a vocabulary projection, and its gradients (sm_100a): the logits never reach memory.
//
//   z = (x . w^T) * (sx * sw)          T x V, in tiles of 256 x 256 in tensor memory
//   lse_t = log sum_v exp z[t,v],      loss_t = lse_t - z[t, target_t]
//   dz[t,v] = (exp(z[t,v] - lse_t) - [v = target_t]) * dloss_t,     dx = dz . w,     dw = dz^T . x
//
// Forward: the epilogue of a tile reduces its columns to one (maximum, sum of exponentials) pair per row; a second kernel
// joins the pairs of a row, in a fixed order.  Backward: the vocabulary in pieces; for each the tile is multiplied again,
// its epilogue turns it into dz (E5M2 codes for FP8 operands, bf16 for bf16), and two products read dz.  dx is added up
// over the pieces in binary32.
//
// A logit is rounded to binary32 before anything is subtracted from it, and only the difference is scaled to base 2: where one
// logit stands alone, its lse is that number, and the gradient there softmax - 1 = 0, however large it is.  So the backward pass has
// to find the forward pass's bits: both add the products in the same order.
//
// All products here are one kernel on persistent CTAs or CTA pairs: TMA-fed ring, tcgen05 into two TMEM accumulators, and
// eight epilogue warps that take the accumulator into registers every 2048 of K (logits of bf16 operands: 512; partial sums
// are added there with round-to-nearest: the tensor core's own additions truncate) and hand it back before they work on it.
//
// What bounds it.  Many tokens: the tensor core, under the power limit (4096 tokens, width 4096, vocabulary 65536, FP8: forward
// 866 us = 2.5 PFLOP/s among other calls, 703 us = 3.1 with pauses; with the backward pass 3.64 ms = 2.4 PFLOP/s).  Few tokens: the stream of
// weights (one token against 131072 x 4096 codes: 95 us in a graph, 113 us as a call; the product's kernel alone 91 us with cold
// caches, 5.9 TB/s).  Width up to 512: the epilogue, 5000 clocks a
// tile.  256 x 256 tiles on pairs as in the plain product: half of B per SM.
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <mutex>
#include <type_traits>

#include "activation.cuh"
#include "codec.cuh"
#include "common.cuh"
#include "umma.cuh"

namespace fp8b200 {
namespace loss {

using namespace gemm;

constexpr int MODE_STATS = 0;           // (maximum, sum of exponentials) of a row's columns, and the target's logit
constexpr int MODE_DZ = 1;              // gradient of the logits
constexpr int MODE_OUT = 2;             // the scaled product itself, of one or two independent products:
enum : int { OUT_ROUNDED = 0, OUT_WIDE = 1, OUT_ADDED = 2 };     // as bf16, as binary32, or added to what is there

constexpr int ROWS = 128;               // rows of a CTA's tile (one TMEM lane each)
constexpr int K_BYTES = 128;            // K-block: one 128-byte swizzle row, 128 elements of 8 bits or 64 of 16
constexpr int K_STEP_BYTES = 32;        // K of one tcgen05.mma
// Of K, what one use of the accumulator covers.  The tensor core truncates what it adds, once per K_STEP_BYTES: a logit that
// grows steadily loses up to that many steps times 2^-24 of itself.  bf16 products have more bits to lose and half the steps
// per use: with 2048 their loss was off by 6e-6 in root mean square (sums in binary32: 4e-6), with 512 by 1.8e-6 (FP8 with 2048, many tokens
// of width 8808: 4e-7, sums in binary32 9e-7).  Up to 128 tokens, where the stream of weights nearly hides it, FP8 takes 1024 (75 tokens of
// width 2306: lse off by 8e-7 instead of 1.7e-6; with 512 5e-7, but one token against 131072 x 4096 takes 116 us, with 1024 112.6, with 2048
// 111.3).  The gradient of the logits takes what the logits take, so that they are the same bits; the products behind it are rounded coarsely.
template <int ESZ, int CG, int MODE> constexpr int split_of = MODE == MODE_OUT || (ESZ == 1 && CG == 2) ? 2048 : ESZ == 1 ? 1024 : 512;
constexpr int FG = 2;                   // K-blocks consumed per barrier wait
constexpr int MAX_STAGES = 12;
constexpr uint32_t A_BYTES = ROWS * K_BYTES;
constexpr uint32_t RING_BYTES = 196608;
constexpr uint32_t BOX_BYTES = 4096;    // 32 rows x 128 B: staging of an epilogue warp
constexpr int MOST_BOXES = 3;           // of a warp, two stages of the ring in exchange for two of them
constexpr int EPI_BASE = 4, EPI_WARPS = 8, THREADS = 32 * (EPI_BASE + EPI_WARPS);
constexpr int REGS_FRONT = 56, REGS_EPILOGUE = 224;      // 128 x 56 + 256 x 224 = 64512, the launch's 384 x 168
constexpr uint32_t SMEM_BARRIERS = 512;
constexpr uint32_t SMEM_BYTES = RING_BYTES + EPI_WARPS * BOX_BYTES + SMEM_BARRIERS + 1024;
constexpr uint32_t TMEM_COLS = 512;
constexpr int SHORT_K = 4;              // K-blocks of a product that is bound by its output
constexpr int EPILOGUE_K = 8;           // K-blocks in whose time a tile's epilogue is done
constexpr int GROUP_M = 16;             // row tiles that advance together over the columns
constexpr float LOG2E = 1.44269504088896341f;

// codes written to the error latch
enum : uint32_t { L_WAIT_EMPTY = 49, L_WAIT_FULL = 50, L_WAIT_ACC_EMPTY = 51, L_WAIT_ACC_FULL = 52 };

struct Product {
    int64_t M, N, K;
    const float* s[2];                  // factors of the product; null counts as 1
    void* D;
    int64_t ldd;                        // elements
    int out;                            // what is stored
    int64_t whole;                      // columns of D up to the last 16-byte boundary
    uint32_t idesc;
    int tiles_m, tiles_n, tiles;        // tiles: of all slices
    int k_blocks, slices, slice_blocks; // K in slices of slice_blocks K-blocks, each with an output plane of its own
    int a_mn, b_mn;                     // operand stored with its M (N) index contiguous
};
struct Params {
    Product q[2];
    int products;
    int full, rest, extra;              // how the tiles of two products are dealt out, see item_at
    int stages;                         // of the ring
    int boxes;                          // staging boxes of an epilogue warp
    uint32_t a_bytes;                   // A's part of a stage (one CTA per tile)
    const int64_t* target;
    int64_t first, vocab;               // vocabulary column of the first column here; all columns of the vocabulary
    float2* part;                       // [2 tiles_n][M]
    float* logit;                       // [M]: the target's
    const float* lse;
    const float* dloss;
    float* dz_scale;                    // written: scale of dz's codes and its inverse
};

struct alignas(8) Barriers {
    uint64_t full[MAX_STAGES], empty[MAX_STAGES], acc_full[2], acc_empty[2];
    uint32_t tmem_base, abort_flag;
    uint32_t most[EPI_WARPS];
};
static_assert(sizeof(Barriers) <= SMEM_BARRIERS, "barrier block too large");

__device__ __forceinline__ void mma_bf16(uint32_t tmem_d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(tmem_d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_bf16_pair(uint32_t tmem_d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(tmem_d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void call_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void tma_add_3d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2) {
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

// (a - c, b - c) log2(e).  The differences one by one: as an addition of pairs they could come out fused with the product that made
// a and b.
__device__ __forceinline__ Pair base2(float a, float b, float c) { return Pair(__fsub_rn(a, c), __fsub_rn(b, c)) * Pair(LOG2E); }

// tile index -> (row tile, column tile): GROUP_M row tiles share each sweep over the columns
__device__ __forceinline__ void tile_at(int t, int tiles_m, int tiles_n, int& tm, int& tn) {
    const int per_group = GROUP_M * tiles_n;
    const int g = t / per_group, first = g * GROUP_M;
    const int rows = min(GROUP_M, tiles_m - first);
    const int r = t - g * per_group;
    tm = first + r % rows;
    tn = r / rows;
}

// The j-th item of a worker: a tile of one of the products.  The first product, the one with the longer K, is dealt out in rounds
// of all workers; in its last round only `rest` of them get a tile.  The others take `extra` tiles of the second product
// meanwhile, and the remaining ones are dealt out in rounds again: all workers end at about the same time.
__device__ __forceinline__ bool item_at(const Params& p, int j, int worker, int workers, int& which, int& t) {
    which = 0;
    t = worker + j * workers;
    if (t < p.q[0].tiles) return true;
    if (p.products == 1) return false;
    which = 1;
    const bool late = worker >= p.rest;
    int i = j - p.full - (late ? 0 : 1);
    if (late) {
        if (i < p.extra) {
            t = i * (workers - p.rest) + worker - p.rest;
            return true;
        }
        i -= p.extra;
    }
    t = p.extra * (workers - p.rest) + i * workers + worker;
    return t < p.q[1].tiles;
}

// ESZ: bytes of an operand's element (1: FP8, 2: bf16).  CG: CTAs of a tile.  BN: its columns.  The logits' gradient in tiles of 128
// columns takes four epilogue warps, each with whole rows of them: a staged box has 128 bytes a row either way.
template <int ESZ, int CG, int BN, int MODE>
__global__ void __launch_bounds__(THREADS, 1)
k_vocabulary(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_d,
             const __grid_constant__ CUtensorMap map_a1, const __grid_constant__ CUtensorMap map_b1, const __grid_constant__ CUtensorMap map_d1,
             const __grid_constant__ Params p) {
    constexpr int KE = K_BYTES / ESZ;                             // elements of a K-block
    constexpr int MNE = 128 / ESZ;                                // M or N elements of a 128-byte row of an MN-major box
    constexpr uint32_t MN_BOX = (uint32_t)KE * 128;               // such a box: MNE elements x one K-block
    constexpr int B_ROWS = BN / CG;                               // columns of the tile that this CTA loads
    const uint32_t a_bytes = CG == 2 ? A_BYTES : p.a_bytes, stage_bytes = a_bytes + B_ROWS * K_BYTES;
    const uint32_t stages = CG == 2 && MODE != MODE_OUT ? RING_BYTES / (A_BYTES + B_ROWS * K_BYTES) : (uint32_t)p.stages;
    constexpr int SPLIT = split_of<ESZ, CG, MODE> / KE;                   // K-blocks per use of an accumulator
    constexpr int PARTS = MODE == MODE_DZ && BN == 128 ? 1 : 2;   // warps that share a row of a tile
    constexpr int ACTIVE = 4 * PARTS;                             // epilogue warps with something to do
    constexpr int NC = BN / PARTS;                                // columns of an epilogue thread
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t ring = (raw + 1023u) & ~1023u;
    Barriers* bars = reinterpret_cast<Barriers*>(smem_raw + (ring - raw) + RING_BYTES + EPI_WARPS * BOX_BYTES);
    volatile uint32_t* abort_flag = &bars->abort_flag;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_ctarank() : 0u;       // 0 = leader of the pair
    const int worker = blockIdx.x / CG, workers = gridDim.x / CG;

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < stages; ++s) { mbar_init(smem_u32(&bars->full[s]), FG * CG); mbar_init(smem_u32(&bars->empty[s]), 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(smem_u32(&bars->acc_full[a]), 1); mbar_init(smem_u32(&bars->acc_empty[a]), ACTIVE * CG); }
        bars->abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2 && lane == 0) {                                 // on their way while the barriers are made
        call_map(&map_a);
        call_map(&map_b);
        if (MODE != MODE_STATS) call_map(&map_d);
        if (MODE == MODE_OUT && p.products > 1) { call_map(&map_a1); call_map(&map_b1); call_map(&map_d1); }
    }
    if (warp == 1) {
        if (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)), "r"(TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)), "r"(TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = bars->tmem_base;
    // Nothing that an earlier kernel may still be writing is touched above this line.
    grid_launch_dependents();
    grid_dependency_wait();

    if (warp < EPI_BASE) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_FRONT));
    if (warp == 0) {
        // ---- loads: this CTA's rows of A and columns of B, one destination each
        uint32_t stage = 0, phase = 0;
        bool ok = true;
        const uint64_t keep = policy_evict_last();
        int which, t;
        for (int j = 0; ok && item_at(p, j, worker, workers, which, t); ++j) {
            const Product& q = p.q[which];
            const CUtensorMap* ma = which ? &map_a1 : &map_a;
            const CUtensorMap* mb = which ? &map_b1 : &map_b;
            int tm, tn;
            const int plane_tiles = q.tiles_m * q.tiles_n, slice = q.slices > 1 ? t / plane_tiles : 0;
            tile_at(t - slice * plane_tiles, q.tiles_m, q.tiles_n, tm, tn);
            const int m0 = (tm * CG + (int)rank) * ROWS, n0 = tn * BN + (int)rank * B_ROWS;
            const int kb0 = slice * q.slice_blocks, kn = min(q.slice_blocks, q.k_blocks - kb0);
            const int kn_pad = (kn + FG - 1) / FG * FG;
            // Every second round of dx or dw starts at the end of K where the last one ended: L2 still has it.  The round is the tile's own,
            // not the worker's count: a product's bits do not depend on what else is in the launch.  Logits are always added up from the start, as
            // their bits must not depend on the tiling either.
            const bool backwards = MODE == MODE_OUT && (t / workers & 1) != 0;
            for (int kb = 0; kb < kn_pad; ++kb) {
                ok = mbar_wait(smem_u32(&bars->empty[stage]), phase ^ 1u, abort_flag, L_WAIT_EMPTY);
                if (!ok) break;
                if (lane == 0) {
                    const uint32_t sa = ring + stage * stage_bytes, sb = sa + a_bytes;
                    const uint32_t bar = smem_u32(&bars->full[stage / FG]);
                    const uint32_t full = CG == 2 ? map_to_cta(bar, 0) : bar;          // the leader's
                    if (kb < kn) {
                        const int k = kb0 + (backwards ? kn - 1 - kb : kb);
                        auto load = [&](uint32_t dst, const CUtensorMap* map, int c0, int c1) {
                            if (CG == 2) tma_load_3d_pair(dst, map, c0, c1, 0, full, keep);
                            else         tma_load_3d(dst, map, c0, c1, 0, full, keep);
                        };
                        if (CG == 2) mbar_arrive_expect_tx_cluster(full, stage_bytes);
                        else         mbar_arrive_expect_tx(full, stage_bytes);
                        if (MODE == MODE_OUT && q.a_mn) {
#pragma unroll
                            for (int i = 0; i < ROWS / MNE; ++i) load(sa + i * MN_BOX, ma, m0 * ESZ + i * 128, k * KE);
                        } else {
                            load(sa, ma, k * K_BYTES, m0);
                        }
                        if (MODE == MODE_OUT && q.b_mn) {
#pragma unroll
                            for (int i = 0; i < B_ROWS / MNE; ++i) load(sb + i * MN_BOX, mb, n0 * ESZ + i * 128, k * KE);
                        } else {
                            load(sb, mb, k * K_BYTES, n0);
                        }
                    } else if (CG == 2) {
                        mbar_arrive_cluster(full);                // padding block: nothing to load
                    } else {
                        mbar_arrive(full);
                    }
                }
                __syncwarp();
                if (++stage == stages) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        // ---- tensor core (leader only)
        uint32_t stage = 0, phase = 0;
        bool ok = rank == 0;
        int it = 0, which, t;
        for (int j = 0; ok && item_at(p, j, worker, workers, which, t); ++j) {
            const Product& q = p.q[which];
            // K-major: groups of 8 rows 1024 B apart, 32 B per step.  MN-major: groups of 8 k 1024 B apart, boxes MN_BOX apart.
            const bool a_mn = MODE == MODE_OUT && q.a_mn, b_mn = MODE == MODE_OUT && q.b_mn;
            const uint32_t a_step = a_mn ? K_STEP_BYTES / ESZ * 128 : K_STEP_BYTES, a_lbo = a_mn ? MN_BOX : 16;
            const uint32_t b_step = b_mn ? K_STEP_BYTES / ESZ * 128 : K_STEP_BYTES, b_lbo = b_mn ? MN_BOX : 16;
            const uint32_t idesc = q.idesc;
            const int slice = q.slices > 1 ? t / (q.tiles_m * q.tiles_n) : 0;
            const int kn = min(q.slice_blocks, q.k_blocks - slice * q.slice_blocks);
            const int kn_pad = (kn + FG - 1) / FG * FG;
            for (int kc = 0; kc < kn_pad && ok; kc += SPLIT, ++it) {
                const uint32_t acc = (uint32_t)it & 1u;
                ok = mbar_wait(smem_u32(&bars->acc_empty[acc]), (((uint32_t)it >> 1) & 1u) ^ 1u, abort_flag, L_WAIT_ACC_EMPTY);
                if (!ok) break;
                tc_fence_after();
                const uint32_t tmem_d = tmem_base + acc * BN;
                const int kend = min(kn_pad, kc + SPLIT), last = min(kn, kend) - 1;
                for (int kb = kc; kb < kend; kb += FG) {
                    ok = mbar_wait(smem_u32(&bars->full[stage / FG]), phase, abort_flag, L_WAIT_FULL);
                    if (!ok) break;
                    tc_fence_after();
                    if (lane == 0) {
#pragma unroll
                        for (int h = 0; h < FG; ++h) {
                            const uint32_t st = stage + h;
                            if (kb + h < kn) {
                                // With few rows A's part of a stage holds those alone, and the rows behind them are whatever
                                // follows: every row of a product is its own, and theirs are not looked at.
                                const uint32_t sa = ring + st * stage_bytes, sb = sa + a_bytes;
#pragma unroll
                                for (int k = 0; k < K_BYTES / K_STEP_BYTES; ++k) {
                                    const uint64_t da = smem_desc(sa + k * a_step, a_lbo, 1024), db = smem_desc(sb + k * b_step, b_lbo, 1024);
                                    const uint32_t more = ((kb - kc) | h | k) != 0 ? 1u : 0u;
                                    if (ESZ == 1) {
                                        if (CG == 2) tc_mma_f8_pair(tmem_d, da, db, idesc, more);
                                        else         tc_mma_f8(tmem_d, da, db, idesc, more);
                                    } else {
                                        if (CG == 2) mma_bf16_pair(tmem_d, da, db, idesc, more);
                                        else         mma_bf16(tmem_d, da, db, idesc, more);
                                    }
                                }
                            }
                            if (CG == 2) {
                                tc_commit_pair(smem_u32(&bars->empty[st]));
                                if (kb + h == last) tc_commit_pair(smem_u32(&bars->acc_full[acc]));
                            } else {
                                tc_commit(smem_u32(&bars->empty[st]));
                                if (kb + h == last) tc_commit(smem_u32(&bars->acc_full[acc]));
                            }
                        }
                    }
                    __syncwarp();
                    stage += FG;
                    if (stage == stages) { stage = 0; phase ^= 1u; }
                }
            }
        }
    }
    } else {
        // ---- epilogue: a warp has 32 rows and half of the tile's columns, a thread one row of them
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_EPILOGUE));
        const int q4 = warp & 3, half = (warp - EPI_BASE) >> 2;
        float dz_scale = 1.0f;
        if (MODE == MODE_DZ && ESZ == 1) {
            // the scale of dz's codes: |dz| is at most the |dloss| of a token that counts
            uint32_t bits = 0u;
#pragma unroll 4
            for (int64_t i = threadIdx.x - 32 * EPI_BASE; i < p.q[0].M; i += 32 * EPI_WARPS) {
                const int64_t target = __ldg(p.target + i);
                const uint32_t b = __float_as_uint(__ldg(p.dloss + i)) & 0x7FFFFFFFu;
                if (target >= 0 && target < p.vocab) bits = max(bits, b);
            }
            bits = warp_max_u32(bits);
            if (lane == 0) bars->most[warp - EPI_BASE] = bits;
            asm volatile("bar.sync 1, %0;" ::"n"(32 * EPI_WARPS) : "memory");
#pragma unroll
            for (int i = 0; i < EPI_WARPS; ++i) bits = max(bits, bars->most[i]);
            const float a = __uint_as_float(bits);                // a NaN is above every number
            if (a > 0.0f && a <= 3.402823466e38f) dz_scale = fminf(57344.0f / a, 3.402823466e38f);
            if (blockIdx.x == 0 && threadIdx.x == 32 * EPI_BASE) {
                p.dz_scale[0] = dz_scale;
                p.dz_scale[1] = 1.0f / dz_scale;
            }
        }
        // one staging box after the ring, or three that start where it ends early
        const bool three = MODE == MODE_OUT && p.boxes == MOST_BOXES;
        const uint32_t boxes = three ? ring + RING_BYTES - 16u * BOX_BYTES + (uint32_t)(warp - EPI_BASE) * (MOST_BOXES * BOX_BYTES)
                                     : ring + RING_BYTES + (uint32_t)(warp - EPI_BASE) * BOX_BYTES;
        uint32_t box = boxes, box_row = box + lane * 128;
        const uint64_t out_policy = MODE == MODE_DZ ? policy_evict_last() : policy_evict_first();      // dz is read next
        auto factor = [](const Product& q) { return (q.s[0] ? __ldg(q.s[0]) : 1.0f) * (q.s[1] ? __ldg(q.s[1]) : 1.0f); };
        const float alpha0 = factor(p.q[0]), alpha1 = MODE == MODE_OUT ? factor(p.q[1]) : 1.0f;
        bool ok = true;
        int it = 0, which, t;
        float v[NC];
        for (int j = 0; ok && half < PARTS && item_at(p, j, worker, workers, which, t); ++j) {
            const Product& q = p.q[which];
            const CUtensorMap* md = which ? &map_d1 : &map_d;
            int tm, tn;
            const int plane_tiles = q.tiles_m * q.tiles_n, slice = q.slices > 1 ? t / plane_tiles : 0;
            tile_at(t - slice * plane_tiles, q.tiles_m, q.tiles_n, tm, tn);
            const int kb0 = slice * q.slice_blocks, kn = min(q.slice_blocks, q.k_blocks - kb0);
            const int kn_pad = (kn + FG - 1) / FG * FG;
            const int64_t row0 = ((int64_t)tm * CG + rank) * ROWS + q4 * 32, row = row0 + lane;
            const int64_t col0 = (int64_t)tn * BN + half * NC;                 // first column of this warp
            const bool row_ok = row < q.M;
            const int cols = (int)max((int64_t)0, min((int64_t)NC, q.N - col0));
            const float alpha = MODE == MODE_OUT && which ? alpha1 : alpha0;
            int rel = -1;                                         // the target's column among this thread's, if it is there
            bool counted = false;
            float g = 0.0f, lse = 0.0f;
            if (MODE != MODE_OUT && row_ok) {
                const int64_t target = __ldg(p.target + row), at = target - p.first - col0;
                counted = target >= 0 && target < p.vocab;
                if (at >= 0 && at < cols) rel = (int)at;
                if (MODE == MODE_DZ) {
                    g = __ldg(p.dloss + row) * dz_scale;
                    if (ESZ == 1 && !(fabsf(g) <= 3.402823466e38f)) g = NAN;      // codes saturate: an infinity would leave them finite
                    lse = __ldg(p.lse + row);
                }
            }
            for (int kc = 0; kc < kn_pad && ok; kc += SPLIT, ++it) {
                const uint32_t acc = (uint32_t)it & 1u;
                ok = mbar_wait(smem_u32(&bars->acc_full[acc]), ((uint32_t)it >> 1) & 1u, abort_flag, L_WAIT_ACC_FULL);
                if (!ok) break;
                tc_fence_after();
                const uint32_t taddr = tmem_base + acc * BN + ((uint32_t)(q4 * 32) << 16) + half * NC;
                constexpr int LOADS = NC >= 64 ? 2 : 1;           // in flight, one wait for all
#pragma unroll
                for (int c = 0; c < NC; c += 32 * LOADS) {
                    uint32_t r[LOADS][32];
#pragma unroll
                    for (int l = 0; l < LOADS; ++l) tc_ld32(taddr + c + 32 * l, r[l]);
                    tc_wait_ld();
                    if (kc == 0) {
#pragma unroll
                        for (int i = 0; i < 32 * LOADS; ++i) v[c + i] = __uint_as_float(r[i >> 5][i & 31]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32 * LOADS; ++i) v[c + i] += __uint_as_float(r[i >> 5][i & 31]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (CG == 2) mbar_arrive_cluster(map_to_cta(smem_u32(&bars->acc_empty[acc]), 0));
                    else         mbar_arrive(smem_u32(&bars->acc_empty[acc]));
                }
            }
            if (!ok) break;
            if (MODE == MODE_STATS) {
                if (row0 >= q.M) continue;                        // the whole warp
                float top = -INFINITY;
#pragma unroll
                for (int i = 0; i < NC; i += 2) (Pair(v[i], v[i + 1]) * Pair(alpha)).split(v[i], v[i + 1]);
                if (cols < NC) {                                  // the tile at the right edge
#pragma unroll
                    for (int i = 0; i < NC; ++i) v[i] = i < cols ? v[i] : -INFINITY;
                }
#pragma unroll
                for (int i = 0; i < NC; ++i) top = fmaxf(top, v[i]);
                if (__any_sync(0xFFFFFFFFu, rel >= 0)) {
                    float z = 0.0f;
#pragma unroll
                    for (int i = 0; i < NC; ++i) z = i == rel ? v[i] : z;
                    if (rel >= 0) p.logit[row] = z;
                }
                // a row of minus infinities keeps a sum of zero; a NaN or plus infinity makes the sum NaN
                const float shift = top == -INFINITY ? 0.0f : top;
                Pair s[2] = {Pair(0.0f), Pair(0.0f)};
#pragma unroll
                for (int i = 0; i < NC; i += 2) {
                    float a, b;
                    base2(v[i], v[i + 1], shift).split(a, b);
                    s[i >> 1 & 1] = s[i >> 1 & 1] + Pair(exp2_fast(a), exp2_fast(b));
                }
                float s0, s1;
                (s[0] + s[1]).split(s0, s1);
                if (row_ok) p.part[(int64_t)(2 * tn + half) * q.M + row] = make_float2(top, s0 + s1);
                continue;
            }
            bool tail = false;                                    // this row's last columns are here, in `rest`
            uint4 rest = make_uint4(0u, 0u, 0u, 0u);
            // OSZ bytes of an element in boxes of 128 bytes a row
            auto store = [&](auto size) {
                constexpr int OSZ = decltype(size)::value;
                constexpr int BOX_COLS = 128 / OSZ, SUBS = BOX_COLS / 32, WORDS = 8 * OSZ;
#pragma unroll
                for (int c = 0; c < NC; c += BOX_COLS) {
                    const int64_t col = col0 + c;
                    if (lane == 0) {                              // what was last stored from this box has left it
                        if (three) bulk_wait_read<MOST_BOXES - 1>();
                        else       bulk_wait_read<0>();
                    }
                    __syncwarp();
#pragma unroll
                    for (int sub = 0; sub < SUBS; ++sub) {
                        float y[32];
                        uint32_t w[WORDS];
                        const int base = c + sub * 32;
                        if (MODE == MODE_DZ) {
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                float a, b;
                                (Pair(v[base + i], v[base + i + 1]) * Pair(alpha)).split(a, b);
                                base2(a, b, lse).split(a, b);
                                y[i] = exp2_fast(a);
                                y[i + 1] = exp2_fast(b);
                            }
                            if (__any_sync(0xFFFFFFFFu, rel >= base && rel < base + 32)) {
#pragma unroll
                                for (int i = 0; i < 32; ++i) y[i] -= base + i == rel ? 1.0f : 0.0f;
                            }
#pragma unroll
                            for (int i = 0; i < 32; ++i) y[i] *= g;
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) y[i] = v[base + i] * alpha;
                        }
                        if (OSZ == 4) {
#pragma unroll
                            for (int i = 0; i < WORDS; ++i) w[i] = __float_as_uint(y[i % 32]);
                        } else if (OSZ == 2) {
#pragma unroll
                            for (int i = 0; i < WORDS; ++i) w[i] = pack_bf16(y[2 * i % 32], y[(2 * i + 1) % 32]);
                        } else {
#pragma unroll
                            for (int i = 0; i < WORDS; ++i) w[i] = cvt_quad<kE5M2>(y[4 * i % 32], y[(4 * i + 1) % 32], y[(4 * i + 2) % 32], y[(4 * i + 3) % 32]);
                        }
                        if (MODE == MODE_DZ && !counted) {        // whatever its logits are
#pragma unroll
                            for (int i = 0; i < WORDS; ++i) w[i] = 0u;
                        }
#pragma unroll
                        for (int i = 0; i < WORDS / 4; ++i) {
                            const int pos = sub * (WORDS / 4) + i;
                            st_shared_v4(box_row + ((pos ^ (lane & 7)) << 4), w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
                        }
                    }
                    if (MODE == MODE_OUT && q.whole < q.N && col <= q.whole && col + BOX_COLS > q.whole) {
                        rest = ld_shared_v4(box_row + ((((int)(q.whole - col) * OSZ / 16) ^ (lane & 7)) << 4));
                        tail = row_ok;
                    }
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        if (row0 < q.M && col < q.whole) {
                            if (OSZ == 4 && q.out == OUT_ADDED) tma_add_3d(md, box, (int)col, (int)row0, slice);
                            else                                tma_store_3d(md, box, (int)(col * OSZ), (int)row0, slice, out_policy);
                        }
                        bulk_commit();
                    }
                    if (three) {
                        box = box == boxes + (MOST_BOXES - 1) * BOX_BYTES ? boxes : box + BOX_BYTES;
                        box_row = box + lane * 128;
                    }
                }
            };
            if (MODE == MODE_DZ) store(std::integral_constant<int, ESZ>());
            else if (q.out == OUT_ROUNDED) store(std::integral_constant<int, 2>());
            else store(std::integral_constant<int, 4>());
            // The TMA unit clips in units of 16 bytes: the map ends with the last whole one of a row, and the few columns behind it,
            // where there are any, are written one by one.  Last of the tile: a box's fence would wait for them.
            if (tail) {
                const int count = (int)(q.N - q.whole);
                if (q.out == OUT_ROUNDED) {
                    uint16_t* to = reinterpret_cast<uint16_t*>(q.D) + row * q.ldd + q.whole;
#pragma unroll
                    for (int i = 0; i < 7; ++i)
                        if (i < count) to[i] = (uint16_t)((i < 2 ? rest.x : i < 4 ? rest.y : i < 6 ? rest.z : rest.w) >> (16 * (i & 1)));
                } else {
                    uint32_t* to = reinterpret_cast<uint32_t*>(q.D) + row * q.ldd + q.whole;
#pragma unroll
                    for (int i = 0; i < 3; ++i)
                        if (i < count) to[i] = i == 0 ? rest.x : i == 1 ? rest.y : rest.z;
                }
            }
        }
        if (MODE != MODE_STATS && lane == 0) bulk_wait_all();
    }

    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync_all();        // neither CTA leaves while the other may still touch its memory, barriers or TMEM
    if (warp == 1) {
        tc_fence_after();
        if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
        else         asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
}

// Joins the pairs of a row.  A block has `rows` rows, a power of two up to 32 and no more than there are: each has 1024 / rows threads,
// which take every so-many-th pair and join theirs in a tree.
// Bound by latency: 7 to 8 us with cold caches, for one token's 2048 pairs as for 2048 rows of 128.
__global__ void __launch_bounds__(1024) k_loss_join(const float2* part, const float* logit, int64_t parts, int64_t M, int rows,
                                                    const int64_t* target, int64_t vocab, float* loss, float* lse) {
    __shared__ float2 got[1024];
    const int row_in = threadIdx.x & (rows - 1), across = 1024 / rows, slot = threadIdx.x / rows;
    grid_launch_dependents();
    grid_dependency_wait();
    auto join = [](float2 a, float2 b) {
        const float top = fmaxf(a.x, b.x), shift = top == -INFINITY ? 0.0f : top;
        return make_float2(top, a.y * exp2_fast((a.x - shift) * LOG2E) + b.y * exp2_fast((b.x - shift) * LOG2E));
    };
    const int64_t row = (int64_t)blockIdx.x * rows + row_in;
    float2 sum = make_float2(-INFINITY, 0.0f);
    if (row < M) {
        for (int64_t i0 = slot; i0 < parts; i0 += across * 8) {
            float2 w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = i0 + across * j < parts ? part[(i0 + across * j) * M + row] : make_float2(-INFINITY, 0.0f);
            float top = sum.x;
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, w[j].x);
            const float shift = top == -INFINITY ? 0.0f : top;
            float s = sum.y * exp2_fast((sum.x - shift) * LOG2E);
#pragma unroll
            for (int j = 0; j < 8; ++j) s += w[j].y * exp2_fast((w[j].x - shift) * LOG2E);
            sum = make_float2(top, s);
        }
    }
    got[threadIdx.x] = sum;
    for (int d = 512; d >= rows; d >>= 1) {
        __syncthreads();
        if (threadIdx.x < d) got[threadIdx.x] = sum = join(sum, got[threadIdx.x + d]);
    }
    if (threadIdx.x < rows && row < M) {
        const float l = logf(sum.y);
        const int64_t t = target[row];
        lse[row] = sum.x + l;
        // the largest logit and the target's are near each other where the loss is small: their difference first
        loss[row] = t >= 0 && t < vocab ? (sum.x - logit[row]) + l : 0.0f;
    }
}

// dx from its binary32 planes, added in order.  Bound by memory: 4096 x 4096 to bf16 16 us (6.4 TB/s), a few rows 4 us of latency.
template <bool BF16>
__global__ void __launch_bounds__(256) k_sum_planes(const float* planes, int count, int64_t M, int64_t N, int64_t pitch, void* out, int64_t ldo) {
    grid_launch_dependents();
    grid_dependency_wait();
    const int64_t octets = (N + 7) / 8, total = M * octets;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / octets, col = (i - row * octets) * 8;
        const float* at = planes + row * pitch + col;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        for (int s = 0; s < count; ++s, at += M * pitch) {
            const float4 a = *reinterpret_cast<const float4*>(at), b = *reinterpret_cast<const float4*>(at + 4);
            v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
        }
        if (col + 8 <= N) {
            if (BF16) {
                *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(out) + row * ldo + col) =
                    make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
            } else {
                float* o = reinterpret_cast<float*>(out) + row * ldo + col;
                *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4*>(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (col + j >= N) continue;
                if (BF16) reinterpret_cast<uint16_t*>(out)[row * ldo + col + j] = (uint16_t)pack_bf16(v[j], 0.0f);
                else      reinterpret_cast<float*>(out)[row * ldo + col + j] = v[j];
            }
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

static int64_t round_up(int64_t n, int64_t unit) { return (n + unit - 1) / unit * unit; }

struct Operand {
    const void* p;
    int64_t ld;                         // elements
    bool mn;
};

struct Maps { CUtensorMap a, b, d; };

template <int ESZ, int CG, int BN, int MODE>
static fp8_status launch(const Maps* m, Params p, cudaStream_t st) {
    auto k = k_vocabulary<ESZ, CG, BN, MODE>;
    constexpr int MAX_DEVICES = 64;
    static std::mutex mu;
    static int cached_workers[MAX_DEVICES] = {0};                 // 0 = not looked up yet
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM_BYTES;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CG;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    int dev = 0, workers = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return FP8_ERR_CUDA;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (dev >= 0 && dev < MAX_DEVICES) workers = cached_workers[dev];
        if (workers == 0) {
            if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM_BYTES) != cudaSuccess) return FP8_ERR_CUDA;
            workers = sm_count() / CG;
            if (CG == 2) {
                cfg.gridDim = dim3(2 * workers);
                int clusters = 0;
                if (cudaOccupancyMaxActiveClusters(&clusters, k, &cfg) == cudaSuccess && clusters > 0 && clusters < workers) workers = clusters;
            }
            if (dev >= 0 && dev < MAX_DEVICES) cached_workers[dev] = workers;
        }
    }
    const int64_t tiles = (int64_t)p.q[0].tiles + (p.products > 1 ? p.q[1].tiles : 0);
    if ((int64_t)workers > tiles) workers = (int)tiles;
    p.full = p.q[0].tiles / workers;
    p.rest = p.q[0].tiles % workers;
    p.extra = 0;
    if (p.products > 1 && p.rest > 0) {                           // a last round of the first product lasts as long as so many tiles of the second
        const int k0 = p.q[0].slice_blocks > EPILOGUE_K ? p.q[0].slice_blocks : EPILOGUE_K;
        const int k1 = p.q[1].slice_blocks > EPILOGUE_K ? p.q[1].slice_blocks : EPILOGUE_K;
        const int others = workers - p.rest, lasts = (k0 + k1 / 2) / k1;
        p.extra = lasts < p.q[1].tiles / others ? lasts : p.q[1].tiles / others;
    }
    cfg.gridDim = dim3(workers * CG);
    const Maps& m1 = m[p.products - 1];
    if (cudaLaunchKernelEx(&cfg, k, m[0].a, m[0].b, m[0].d, m1.a, m1.b, m1.d, p) != cudaSuccess) { (void)cudaGetLastError(); return FP8_ERR_CUDA; }
    count_launches(1);
    return launch_status();
}

// Output planes of a product: bytes for stores, binary32 elements for additions (the unit adds what the map's type says).
static bool make_plane_map(CUtensorMap* map, void* base, int64_t cols, int64_t rows, int64_t ld, int planes, int osz, bool add) {
    if (!add) return make_map(map, base, (uint64_t)(cols * osz), (uint64_t)rows, (uint64_t)(ld * osz), (uint64_t)planes, (uint64_t)(ld * osz * rows), 128, 32);
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes}, strides[2] = {(cuuint64_t)ld * 4, (cuuint64_t)(ld * 4 * rows)};
    const cuuint32_t box[3] = {32, 32, 1}, step[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, base, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Columns of a tile for products with at most 128 rows (one CTA per tile).  A tile takes as long as its columns and rows are
// loaded, and a little more; the width with the shortest rounds of all SMs is taken.  (69 tokens x
// 11082, vocabulary 3055, FP8: backward pass 57 us, 74 with tiles of 256 columns alone.)
static int few_rows_width(int64_t M, int64_t N, int least) {
    const int64_t sms = sm_count();
    int best = 256;
    int64_t best_cost = 0;
    for (int bn = 256; bn >= least; bn /= 2) {
        const int64_t cost = ((N + bn - 1) / bn + sms - 1) / sms * (bn + round_up(M, 8) + 16);
        if (bn == 256 || cost < best_cost) { best = bn; best_cost = cost; }
    }
    return best;
}

// Fills in what follows from a product's sizes, layouts and formats, and its tensor maps.  q holds M, N, K, the factors, D, ldd,
// `out` and the wanted slices; a_rows: rows of A that a CTA loads.
static bool lay_out(Product& q, Maps& m, int esz, int fa, int fb, const Operand& A, const Operand& B, int cg, int bn, int a_rows, int64_t out_cols, int out_size) {
    const int ke = K_BYTES / esz;
    auto map = [&](CUtensorMap* t, const Operand& o, int64_t mn, int rows) {
        return o.mn ? make_map(t, o.p, (uint64_t)(mn * esz), (uint64_t)q.K, (uint64_t)(o.ld * esz), 1, 0, 128, (uint32_t)ke)
                    : make_map(t, o.p, (uint64_t)(q.K * esz), (uint64_t)mn, (uint64_t)(o.ld * esz), 1, 0, K_BYTES, (uint32_t)rows);
    };
    q.whole = out_cols * out_size / 16 * 16 / (out_size > 0 ? out_size : 1);
    if (!map(&m.a, A, q.M, a_rows) || !map(&m.b, B, q.N, bn / cg)) return false;
    if (!q.D) m.d = m.a;                                          // nothing is stored through it
    else if (q.whole == 0) m.d = m.a;                             // rows of less than 16 bytes
    else if (!make_plane_map(&m.d, q.D, q.whole, q.M, q.ldd, q.slices, out_size, q.out == OUT_ADDED)) return false;
    q.a_mn = A.mn ? 1 : 0;
    q.b_mn = B.mn ? 1 : 0;
    q.tiles_m = (int)((q.M + ROWS * cg - 1) / (ROWS * cg));
    q.tiles_n = (int)((q.N + bn - 1) / bn);
    q.k_blocks = (int)((q.K + ke - 1) / ke);
    q.slice_blocks = (q.k_blocks + q.slices - 1) / q.slices;
    q.slices = (q.k_blocks + q.slice_blocks - 1) / q.slice_blocks;
    q.tiles = q.tiles_m * q.tiles_n * q.slices;
    // binary32 accumulator; formats (bf16 is 1), layouts, N / 8, M / 16
    q.idesc = (1u << 4) | ((uint32_t)(esz == 2 ? 1 : fa) << 7) | ((uint32_t)(esz == 2 ? 1 : fb) << 10) | ((uint32_t)q.a_mn << 15) | ((uint32_t)q.b_mn << 16) |
              ((uint32_t)(bn >> 3) << 17) | ((uint32_t)(ROWS * cg >> 4) << 24);
    return true;
}

// The product x . w^T with the epilogue of MODE_STATS or MODE_DZ (D: dz, of pitch q.ldd = out_cols).
template <int MODE>
static fp8_status logits(const fp8_cross_entropy_desc* d, const void* x, const void* w, Params& p, cudaStream_t st) {
    Product& q = p.q[0];
    const int esz = d->x_t == FP8_OPERAND_BF16 ? 2 : 1;
    // (the part of a stage that the rows of A do not fill is read as rows that nobody looks at; behind the last stage that is the staging boxes)
    const int cg = q.M > ROWS ? 2 : 1, bn = cg == 1 ? few_rows_width(q.M, q.N, MODE == MODE_STATS ? 64 : 128) : 256;
    const int a_rows = cg == 2 ? ROWS : (int)round_up(q.M, 8);
    Maps m;
    q.slices = 1;
    if (!lay_out(q, m, esz, d->x_t, d->w_t, Operand{x, d->ldx, false}, Operand{w, d->ldw, false}, cg, bn, a_rows, q.ldd, esz)) return FP8_ERR_CUDA;
    p.products = 1;
    p.a_bytes = (uint32_t)a_rows * K_BYTES;
    p.stages = (int)(RING_BYTES / (p.a_bytes + (uint32_t)(bn / cg) * K_BYTES)) / FG * FG;
    if (p.stages > MAX_STAGES) p.stages = MAX_STAGES;
    if (cg == 2) return esz == 1 ? launch<1, 2, 256, MODE>(&m, p, st) : launch<2, 2, 256, MODE>(&m, p, st);
    if constexpr (MODE == MODE_STATS) {
        if (bn == 64) return esz == 1 ? launch<1, 1, 64, MODE>(&m, p, st) : launch<2, 1, 64, MODE>(&m, p, st);
    }
    if (bn == 128) return esz == 1 ? launch<1, 1, 128, MODE>(&m, p, st) : launch<2, 1, 128, MODE>(&m, p, st);
    return esz == 1 ? launch<1, 1, 256, MODE>(&m, p, st) : launch<2, 1, 256, MODE>(&m, p, st);
}

// One product, or two in one launch, on CTA pairs.  Short sums are bound by their output: where one of them has at most SHORT_K
// K-blocks, two stages of the ring become staging boxes, whose stores drain while the next boxes are filled (300 tokens, width
// 8192, vocabulary 32000, FP8: backward pass 411 -> 343 us; with 8 K-blocks the other product's shorter ring costs more: 1001 tokens 560 -> 589).
static fp8_status products(int esz, const Maps* m, Params& p, cudaStream_t st) {
    const bool is_short = p.q[0].slice_blocks <= SHORT_K || (p.products > 1 && p.q[1].slice_blocks <= SHORT_K);
    p.boxes = is_short ? MOST_BOXES : 1;
    p.stages = (int)(RING_BYTES / (2 * A_BYTES)) - (is_short ? 2 : 0);
    return esz == 1 ? launch<1, 2, 256, MODE_OUT>(m, p, st) : launch<2, 2, 256, MODE_OUT>(m, p, st);
}

template <typename... KArgs, typename... Args>
static fp8_status launch_small(void (*k)(KArgs...), unsigned grid, unsigned block, cudaStream_t st, Args... args) {
    if (launch_programmatic(k, dim3(grid), dim3(block), st, args...) != cudaSuccess) { (void)cudaGetLastError(); return FP8_ERR_CUDA; }
    count_launches(1);
    return launch_status();
}

// How the backward pass cuts its work.
struct Cut {
    int64_t cols;                       // vocabulary columns of a piece (the last may have fewer)
    int pieces;
    int slices;                         // K-slices of dx's product
    bool planes;                        // dx goes through binary32 planes
    int64_t pitch_z, pitch_x;           // of dz and of the planes, elements
    size_t z_bytes, x_bytes;
};

constexpr int64_t Z_BYTES = 64 << 20;   // dz of a piece: half of L2, so that the two products that read it find it there
constexpr int64_t LEAST_COLS = 8192;    // but no fewer columns: dx's planes are read and written once per piece

static Cut cut_of(int64_t T, int64_t K, int64_t V, int esz) {
    Cut c;
    int64_t most = Z_BYTES / (T * esz);
    if (most < LEAST_COLS) most = LEAST_COLS;
    c.pieces = (int)((V + most - 1) / most);
    c.cols = round_up((V + c.pieces - 1) / c.pieces, 256);
    c.pieces = (int)((V + c.cols - 1) / c.cols);
    // Few rows: dx has few tiles and a long contraction.  It is cut into slices while that pays: a pair needs about 0.25 us for a
    // K-block it waits for, the planes of several slices cost a launch and their traffic.
    const int64_t tiles = (T + 255) / 256 * ((K + 255) / 256), workers = sm_count() / 2;
    const int64_t ke = K_BYTES / esz, blocks = ((V < c.cols ? V : c.cols) + ke - 1) / ke;
    const double plane_us = (c.pieces > 1 ? 0.0 : 4.0), each_us = 8.0 * (double)T * (double)K / 4e6;
    double best = 0.0;
    c.slices = 1;
    for (int64_t s = 1; s <= 16 && s <= blocks && (s == 1 || tiles * s <= workers); ++s) {
        const int64_t each = (blocks + s - 1) / s;
        const double us = 0.25 * (double)each + (s > 1 ? plane_us + each_us * (double)s : 0.0);
        if (s == 1 || us < best) { best = us; c.slices = (int)((blocks + each - 1) / each); }      // as lay_out counts them for the first piece, which writes every plane
    }
    c.planes = c.slices > 1 || c.pieces > 1;
    c.pitch_z = c.cols;
    c.pitch_x = round_up(K, 32);
    c.z_bytes = (size_t)round_up(T * c.pitch_z * esz, 256);
    c.x_bytes = c.planes ? (size_t)c.slices * (size_t)T * (size_t)c.pitch_x * 4 : 0;
    return c;
}

static int64_t parts_of(int64_t T, int64_t V) {
    const int bn = T > ROWS ? 256 : few_rows_width(T, V, 64);
    return 2 * ((V + bn - 1) / bn);
}
static size_t forward_bytes(int64_t T, int64_t V) { return T > 0 ? (size_t)parts_of(T, V) * (size_t)T * 8 + (size_t)T * 4 : 0; }
static size_t backward_bytes(int64_t T, int64_t K, int64_t V, int esz) {
    if (T <= 0) return 0;
    const Cut c = cut_of(T, K, V, esz);
    return 256 + c.z_bytes + c.x_bytes;
}

static fp8_status check(const fp8_cross_entropy_desc* d) {
    if (!d) return FP8_ERR_NULL;
    if (d->x_t < FP8_OPERAND_E4M3 || d->x_t > FP8_OPERAND_BF16 || d->w_t < FP8_OPERAND_E4M3 || d->w_t > FP8_OPERAND_BF16 ||
        (d->x_t == FP8_OPERAND_BF16) != (d->w_t == FP8_OPERAND_BF16))
        return FP8_ERR_ENUM;
    if (d->tokens < 0 || d->width < 1 || d->vocab < 1) return FP8_ERR_SHAPE;
    const int64_t far = ((int64_t)1 << 30) - 512;                 // 32-bit coordinates in bytes
    if (d->tokens > far || d->width > far / 2 || d->vocab > far) return FP8_ERR_UNSUPPORTED;
    const int64_t tiles = ((d->tokens + 127) / 128) * ((d->vocab + 127) / 128), across = ((d->width + 255) / 256);
    if (tiles > (int64_t)1 << 29 || ((d->vocab + 127) / 128) * across > (int64_t)1 << 29 || ((d->tokens + 127) / 128) * across > (int64_t)1 << 25)
        return FP8_ERR_UNSUPPORTED;
    return FP8_OK;
}

static fp8_status check_operands(const fp8_cross_entropy_desc* d, const void* x, const void* w, const float* sx, const float* sw) {
    const int esz = d->x_t == FP8_OPERAND_BF16 ? 2 : 1;
    if (!x || !w || (esz == 1 && (!sx || !sw))) return FP8_ERR_NULL;
    if (d->ldx < d->width || d->ldw < d->width) return FP8_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(x) & 15u) || (reinterpret_cast<uintptr_t>(w) & 15u) || ((d->ldx * esz) & 15) || ((d->ldw * esz) & 15)) return FP8_ERR_ALIGN;
    return FP8_OK;
}

}  // namespace loss

void loss_read_clear_latch(unsigned int out2[2]) {
    out2[0] = out2[1] = 0u;
    if (cudaMemcpyFromSymbol(out2, g_async_latch, 2 * sizeof(unsigned int)) != cudaSuccess || out2[0] == 0u) return;
    const unsigned int zero[2] = {0u, 0u};
    (void)cudaMemcpyToSymbol(g_async_latch, zero, sizeof(zero));
}

}  // namespace fp8b200

using namespace fp8b200;

extern "C" {

fp8_status fp8_cross_entropy_workspace_bytes(const fp8_cross_entropy_desc* d, size_t* forward_bytes_out, size_t* backward_bytes_out) {
    using namespace fp8b200::loss;
    const fp8_status rc = check(d);
    if (rc != FP8_OK) return rc;
    if (forward_bytes_out) *forward_bytes_out = forward_bytes(d->tokens, d->vocab);
    if (backward_bytes_out) *backward_bytes_out = backward_bytes(d->tokens, d->width, d->vocab, d->x_t == FP8_OPERAND_BF16 ? 2 : 1);
    return FP8_OK;
}

fp8_status fp8_cross_entropy(const fp8_cross_entropy_desc* d, const void* x, const void* w, const float* scale_inv_x_dev, const float* scale_inv_w_dev,
                             const int64_t* target_dev, float* loss_dev, float* lse_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
    using namespace fp8b200::loss;
    fp8_status rc = check(d);
    if (rc != FP8_OK) return rc;
    const int64_t T = d->tokens, V = d->vocab;
    if (T == 0) return FP8_OK;
    if (!target_dev || !loss_dev || !lse_dev || !workspace_dev) return FP8_ERR_NULL;
    if ((rc = check_operands(d, x, w, scale_inv_x_dev, scale_inv_w_dev)) != FP8_OK) return rc;
    if (workspace_bytes < forward_bytes(T, V)) return FP8_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(workspace_dev) & 15u) || (reinterpret_cast<uintptr_t>(target_dev) & 7u) ||
        ((reinterpret_cast<uintptr_t>(loss_dev) | reinterpret_cast<uintptr_t>(lse_dev)) & 3u))
        return FP8_ERR_ALIGN;
    cudaStream_t st = (cudaStream_t)stream;
    Params p = {};
    Product& q = p.q[0];
    q.M = T; q.N = V; q.K = d->width;
    q.s[0] = scale_inv_x_dev; q.s[1] = scale_inv_w_dev;
    p.target = target_dev; p.vocab = V;
    p.part = reinterpret_cast<float2*>(workspace_dev);
    p.logit = reinterpret_cast<float*>(p.part + parts_of(T, V) * T);
    if ((rc = logits<MODE_STATS>(d, x, w, p, st)) != FP8_OK) return rc;
    int rows = 32;
    while (rows > T) rows /= 2;
    return launch_small(k_loss_join, (unsigned)((T + rows - 1) / rows), 1024u, st, (const float2*)p.part, (const float*)p.logit, (int64_t)q.tiles_n * 2, T, rows,
                        target_dev, V, loss_dev, lse_dev);
}

fp8_status fp8_cross_entropy_backward(const fp8_cross_entropy_desc* d, const void* x, const void* w, const float* scale_inv_x_dev, const float* scale_inv_w_dev,
                                      const int64_t* target_dev, const float* lse_dev, const float* dloss_dev, void* dx, fp8_wide dx_t, int64_t lddx,
                                      void* dw, fp8_wide dw_t, int64_t lddw, void* workspace_dev, size_t workspace_bytes, void* stream) {
    using namespace fp8b200::loss;
    fp8_status rc = check(d);
    if (rc != FP8_OK) return rc;
    if ((dx_t != FP8_F32 && dx_t != FP8_BF16) || (dw_t != FP8_F32 && dw_t != FP8_BF16)) return FP8_ERR_ENUM;
    const int64_t T = d->tokens, K = d->width, V = d->vocab;
    const int xo = dx_t == FP8_BF16 ? 2 : 4, wo = dw_t == FP8_BF16 ? 2 : 4;
    if (dw) {
        if (lddw < K) return FP8_ERR_SHAPE;
        if ((reinterpret_cast<uintptr_t>(dw) & 15u) || ((lddw * wo) & 15)) return FP8_ERR_ALIGN;
    }
    cudaStream_t st = (cudaStream_t)stream;
    if (T == 0) {                                                 // an empty sum
        if (!dw) return FP8_OK;
        if (cudaMemset2DAsync(dw, (size_t)(lddw * wo), 0, (size_t)(K * wo), (size_t)V, st) != cudaSuccess) { (void)cudaGetLastError(); return FP8_ERR_CUDA; }
        count_launches(1);
        return FP8_OK;
    }
    if (dx) {
        if (lddx < K) return FP8_ERR_SHAPE;
        if ((reinterpret_cast<uintptr_t>(dx) & 15u) || ((lddx * xo) & 15)) return FP8_ERR_ALIGN;
    }
    if (!target_dev || !lse_dev || !dloss_dev || !workspace_dev) return FP8_ERR_NULL;
    if ((rc = check_operands(d, x, w, scale_inv_x_dev, scale_inv_w_dev)) != FP8_OK) return rc;
    const int esz = d->x_t == FP8_OPERAND_BF16 ? 2 : 1;
    if (workspace_bytes < backward_bytes(T, K, V, esz)) return FP8_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(workspace_dev) & 15u) || (reinterpret_cast<uintptr_t>(target_dev) & 7u) ||
        ((reinterpret_cast<uintptr_t>(lse_dev) | reinterpret_cast<uintptr_t>(dloss_dev)) & 3u))
        return FP8_ERR_ALIGN;
    if (!dx && !dw) return FP8_OK;
    const Cut c = cut_of(T, K, V, esz);
    uint8_t* ws = reinterpret_cast<uint8_t*>(workspace_dev);
    float* scale = reinterpret_cast<float*>(ws);
    void* dz = ws + 256;
    float* planes = reinterpret_cast<float*>(ws + 256 + c.z_bytes);
    const float* back = esz == 1 ? scale + 1 : nullptr;
    const int fz = FP8_E5M2;
    for (int i = 0; i < c.pieces; ++i) {
        const int64_t v0 = i * c.cols, cols = V - v0 < c.cols ? V - v0 : c.cols;
        const uint8_t* wp = reinterpret_cast<const uint8_t*>(w) + v0 * d->ldw * esz;
        Params z = {};
        z.q[0].M = T; z.q[0].N = cols; z.q[0].K = K;
        z.q[0].s[0] = scale_inv_x_dev; z.q[0].s[1] = scale_inv_w_dev;
        z.q[0].D = dz; z.q[0].ldd = c.pitch_z;
        z.target = target_dev; z.first = v0; z.vocab = V;
        z.lse = lse_dev; z.dloss = dloss_dev; z.dz_scale = scale;
        if ((rc = logits<MODE_DZ>(d, x, wp, z, st)) != FP8_OK) return rc;
        // the two products that read dz: one launch
        Product of_x = {}, of_w = {};
        Maps mx, mw;
        if (dx) {
            of_x.M = T; of_x.N = K; of_x.K = cols;
            of_x.s[0] = back; of_x.s[1] = scale_inv_w_dev;
            of_x.slices = c.slices;
            const Operand A{dz, c.pitch_z, false}, B{wp, d->ldw, true};
            of_x.out = c.planes ? (i == 0 ? OUT_WIDE : OUT_ADDED) : dx_t == FP8_BF16 ? OUT_ROUNDED : OUT_WIDE;
            of_x.D = c.planes ? planes : dx;
            of_x.ldd = c.planes ? c.pitch_x : lddx;
            if (!lay_out(of_x, mx, esz, fz, d->w_t, A, B, 2, 256, ROWS, c.planes ? c.pitch_x : K, of_x.out == OUT_ROUNDED ? 2 : 4)) return FP8_ERR_CUDA;
        }
        if (dw) {
            of_w.M = cols; of_w.N = K; of_w.K = T;
            of_w.s[0] = back; of_w.s[1] = scale_inv_x_dev;
            of_w.slices = 1;
            of_w.D = reinterpret_cast<uint8_t*>(dw) + v0 * lddw * wo; of_w.ldd = lddw;
            of_w.out = dw_t == FP8_BF16 ? OUT_ROUNDED : OUT_WIDE;
            const Operand A{dz, c.pitch_z, true}, B{x, d->ldx, true};
            if (!lay_out(of_w, mw, esz, fz, d->x_t, A, B, 2, 256, ROWS, K, wo)) return FP8_ERR_CUDA;
        }
        Params p = {};
        Maps m[2];
        const bool x_first = dx && (!dw || of_x.slice_blocks >= of_w.slice_blocks);      // the longer K first
        p.products = dx && dw ? 2 : 1;
        p.q[0] = x_first ? of_x : of_w; m[0] = x_first ? mx : mw;
        p.q[1] = x_first ? of_w : of_x; m[1] = x_first ? mw : mx;
        if ((rc = products(esz, m, p, st)) != FP8_OK) return rc;
    }
    if (dx && c.planes) {
        const int64_t octets = T * ((K + 7) / 8);
        int64_t grid = (octets + 255) / 256;
        if (grid > (int64_t)sm_count() * 16) grid = (int64_t)sm_count() * 16;
        rc = dx_t == FP8_BF16 ? launch_small(k_sum_planes<true>, (unsigned)grid, 256u, st, (const float*)planes, c.slices, T, K, c.pitch_x, dx, lddx)
                              : launch_small(k_sum_planes<false>, (unsigned)grid, 256u, st, (const float*)planes, c.slices, T, K, c.pitch_x, dx, lddx);
    }
    return rc;
}

}  // extern "C"
