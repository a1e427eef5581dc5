/*
 * fp8_b200 — C ABI of the B200 (sm_100a) FP8 hot path of
 * "FP8 Formats for Deep Learning" (arXiv 2209.05433).
 *
 * Conventions shared by every call
 *   - Every pointer whose name ends in _dev, and every tensor pointer (x, c,
 *     out, A, B, D), is a DEVICE pointer owned by the caller.  The library
 *     never allocates or frees device memory and keeps no per-call state.
 *   - Scalars that flow between calls (amax, scale, scale_inv) live in device
 *     memory, so amax -> scale -> quantize -> gemm chain on one stream with no
 *     host synchronisation.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the default stream).
 *     Calls only enqueue work and return; argument errors are found on the
 *     host before anything is launched.
 *   - The return value is a status code; nothing aborts or throws.  A launch
 *     failure is reported as FP8_ERR_CUDA.  A device-side wait that ran out of
 *     patience (never expected) is latched and read by fp8_async_status().
 *   - bf16 tensors are arrays of 16-bit patterns (the upper half of binary32);
 *     FP8 tensors are arrays of 8-bit codes in the paper's S.E.M layout.
 */
#ifndef FP8_B200_H
#define FP8_B200_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    FP8_OK = 0,
    FP8_ERR_NULL = 1,        /* a required pointer is NULL */
    FP8_ERR_ENUM = 2,        /* an enum argument is out of range */
    FP8_ERR_SHAPE = 3,       /* negative size, or a leading dimension smaller than the row */
    FP8_ERR_ALIGN = 4,       /* GEMM operand base or leading dimension not 16-byte aligned */
    FP8_ERR_UNSUPPORTED = 5, /* a size beyond what the launch geometry can address */
    FP8_ERR_CUDA = 6,        /* the CUDA runtime / driver reported an error */
    FP8_ERR_TIMEOUT = 7      /* a bounded device-side wait expired (see fp8_async_status) */
} fp8_status;

/* The two encodings of Section 3 / Table 1. */
typedef enum { FP8_E4M3 = 0, FP8_E5M2 = 1 } fp8_format;
/* The wider type a tensor is converted from / to (Section 2). */
typedef enum { FP8_F32 = 0, FP8_BF16 = 1 } fp8_wide;
/* Section 2: overflow saturates to the maximum finite value (default), or, in the
 * non-saturating mode, becomes NaN (E4M3, which has no infinity) / Inf (E5M2). */
typedef enum { FP8_SATURATE = 0, FP8_NOSAT = 1 } fp8_overflow;
/* Which index of a GEMM operand is contiguous in memory. */
typedef enum { FP8_MAJOR_K = 0, FP8_MAJOR_MN = 1 } fp8_major;
/* how a GEMM accumulates over K (see fp8_gemm) */
typedef enum { FP8_ACC_SPLIT = 0, FP8_ACC_FAST = 1 } fp8_accumulate;

/*
 * fp8_amax — maximum magnitude of a tensor (Section 2: the quantity the scale
 * factor is chosen from).
 *   x         device, n elements of type t, any element-aligned address.
 *   amax_dev  device, one float, OVERWRITTEN with max_i |x_i| (+0 when n == 0).
 *             If any element is NaN the result is NaN (pattern 0x7FC00000);
 *             otherwise an infinity gives +Inf.  The result is exact and does
 *             not depend on reduction order.
 */
fp8_status fp8_amax(const void* x, fp8_wide t, size_t n, float* amax_dev, void* stream);

/*
 * fp8_scale_from_amax — Section 2: the scale factor that moves the tensor's
 * maximum magnitude onto the format's maximum (Table 1: 448 / 57344).
 *   scale = fmax / amax (binary32 division); amax of 0, NaN or Inf gives 1; a
 *   quotient that overflows is clamped to the largest finite binary32.
 *   scale_inv = 1 / scale.  All three pointers are device floats.
 */
fp8_status fp8_scale_from_amax(const float* amax_dev, fp8_format f,
                               float* scale_dev, float* scale_inv_dev, void* stream);

/*
 * fp8_quantize — Section 2: multiply by the per-tensor scale factor, convert to
 * FP8 (Table 1 encodings) with round-to-nearest-even.
 *   out_i = encode_f( binary32(x_i) * scale ), the product rounded to binary32
 *   first.  Special values convert to special values in both overflow modes:
 *   NaN -> sign|0x7F; +-Inf -> E4M3 sign|0x7F (NaN), E5M2 sign|0x7C (Inf); this
 *   rule is applied to the scaled value.  Finite overflow follows `o`.  The sign
 *   of zero and of values that round to zero is kept.
 *   x          device, n elements of type t.
 *   scale_dev  device float, read by the kernel.
 *   out        device, n bytes.
 *   amax_dev   NULL, or a device float OVERWRITTEN with amax(x) of the same pass
 *              (same definition as fp8_amax), for callers that scale with the
 *              previous step's amax.
 *   Fast path: x and out both 16-byte aligned; other alignments take a slower
 *   element-wise path with identical results.
 */
fp8_status fp8_quantize(const void* x, fp8_wide t, size_t n, fp8_format f, fp8_overflow o,
                        const float* scale_dev, uint8_t* out, float* amax_dev, void* stream);

/*
 * fp8_quantize_current — Section 2, the whole current-scaling conversion of one tensor in ONE call:
 * the scale is chosen from the tensor's own maximum magnitude, then the tensor is converted with it.
 * Results are identical, bit for bit, to fp8_amax + fp8_scale_from_amax + fp8_quantize:
 *   *amax_dev = amax(x); *scale_dev = fmax/amax (same guards); *scale_inv_dev = 1/scale;
 *   out_i = encode_f( binary32(x_i) * scale ).
 * Tensors below 256 MB take ONE kernel, launched cooperatively (all of its blocks resident at once), which
 * crosses one grid-wide barrier between the two passes; the second pass re-reads the tail of x from L2.  A tensor
 * small enough for the shared memory of the whole GPU (about 33 MB on a B200) is kept there between the passes and
 * read from global memory only once.
 * Larger tensors (and pointers without 16-byte alignment) take the three streaming kernels back to back on the
 * stream, the conversion walking the tensor from its end, where the amax pass has just been: on long streams
 * that is the faster form, and the workspace is then not touched.
 *   workspace  device, fp8_quantize_current_workspace_bytes() bytes, 16-byte aligned, owned by the
 *              caller.  It must hold zeros before the first call; every call leaves it zeroed again,
 *              so one buffer serves any number of calls on one stream.  Calls that may overlap on the
 *              GPU (different streams) need different workspaces.
 * The grid barrier is a bounded wait (about two seconds).  If it expires in any block, fp8_async_status
 * reports FP8_ERR_TIMEOUT and the contents of out, amax_dev, scale_dev and scale_inv_dev are undefined (blocks
 * that gave up write nothing, blocks that got through may have written their share).  The workspace is left
 * zeroed in that case too: the last block to leave clears it whether or not the barrier held.
 */
fp8_status fp8_quantize_current(const void* x, fp8_wide t, size_t n, fp8_format f, fp8_overflow o,
                                uint8_t* out, float* amax_dev, float* scale_dev, float* scale_inv_dev,
                                void* workspace, void* stream);

/* Size in bytes of the workspace fp8_quantize_current needs. */
size_t fp8_quantize_current_workspace_bytes(void);

/*
 * fp8_quantize_current_static — the paper has no counterpart; this entry point exists for callers
 * that cannot obtain device memory for a workspace.
 *
 * Who that is: code that runs where cudaMalloc is off limits or would fail — a plug-in called from
 * inside another framework's memory pool that already owns all of the GPU's memory, a latency-bound
 * serving loop in which an allocation (an implicit device synchronisation) is not acceptable, or a
 * component that is only ever handed its input and output buffers.  Such a caller still wants the
 * one-launch current-scaling conversion of fp8_quantize_current, but has no 16 spare bytes to pass.
 *
 * What it does: exactly fp8_quantize_current (same kernel, same results bit for bit), with the
 * kernel's three control words kept in a 256-byte array that is part of the library image.  Every GPU
 * that loads the library holds those 256 bytes until the process exits.  The call allocates nothing:
 * no cudaMalloc, no cudaFree, no allocating library routine.  The caller passes inputs and outputs only.
 *
 * Rules of use
 *   - The first call on a device looks up the array's device address (once per device, with that
 *     device current).  Make that first call outside any stream capture.
 *   - All calls on a device share the one array.  Each call clears the words it needs before its
 *     kernel runs, so a call never depends on what the previous one left behind; but two calls that
 *     overlap on the GPU (different streams, or different host threads on different streams) race on
 *     it and give undefined results.  Issue them on one stream, or serialise them yourself.
 *   - n may not exceed FP8_STATIC_MAX_ELEMENTS; larger tensors return FP8_ERR_UNSUPPORTED and nothing
 *     is enqueued.  (The scratch need of this kernel does not grow with n; the bound is simply the
 *     stated maximum of this entry point.)
 *   - Arguments, alignment rules and the bounded grid barrier are those of fp8_quantize_current.
 */
#define FP8_STATIC_MAX_ELEMENTS ((size_t)1 << 32)
fp8_status fp8_quantize_current_static(const void* x, fp8_wide t, size_t n, fp8_format f, fp8_overflow o,
                                       uint8_t* out, float* amax_dev, float* scale_dev, float* scale_inv_dev,
                                       void* stream);

/*
 * fp8_dequantize — Section 2: convert back and multiply by the inverse of the
 * scale factor.  out_i = round_t( decode_f(c_i) * scale_inv ), one binary32
 * multiply, then round-to-nearest-even to bf16 when t is FP8_BF16.  NaN codes
 * give NaN (payload unspecified), E5M2 infinities give infinities.
 */
fp8_status fp8_dequantize(const uint8_t* c, size_t n, fp8_format f,
                          const float* scale_inv_dev, void* out, fp8_wide t, void* stream);

/*
 * fp8_fake_quantize — Section 4: the paper's own experiments simulated FP8: tensors were converted
 * to FP8 (scale factor, rounding and saturation included) and straight back to the wider type, and the
 * arithmetic stayed in that wider type.  This is that round trip in one pass over the tensor:
 *   out_i = round_t( decode_f( encode_f( binary32(x_i) * scale ) ) * scale_inv ),  out has the type of x.
 * Bit for bit the composition of fp8_quantize and fp8_dequantize, without the intermediate code tensor
 * (4 B per bf16 element of traffic instead of 6).
 */
fp8_status fp8_fake_quantize(const void* x, fp8_wide t, size_t n, fp8_format f, fp8_overflow o,
                             const float* scale_dev, const float* scale_inv_dev, void* out, void* stream);

/*
 * fp8_scale_pow2_from_amax — Section 3.2: a programmable exponent bias amounts to restricting the scale
 * factors to powers of two.  scale = the largest power of two not above fmax/amax (same guards
 * as fp8_scale_from_amax), scale_inv = 1/scale (exact).  Converting with this scale is converting to an
 * E4M3/E5M2 variant whose exponent bias is shifted by log2(scale) (the bias sweep of Section 4.3).
 */
fp8_status fp8_scale_pow2_from_amax(const float* amax_dev, fp8_format f,
                                    float* scale_dev, float* scale_inv_dev, void* stream);

/*
 * fp8_gemm — Sections 2, 3 and 4.1: the matrix multiply on FP8 inputs with a
 * higher-precision result, unscaled once per dot product.
 *   D[i,j] = round_out( (sum_k decode_fa(A[i,k]) * decode_fb(B[k,j])) * (sa_inv * sb_inv) )
 * with binary32 accumulation on the tensor cores.
 * Operand roles (Section 3: E4M3 for weights and activations, E5M2 for
 * gradients): forward  fa=E4M3, fb=E4M3;  dgrad  fa=E5M2 (dY), fb=E4M3 (W);
 * wgrad  fa=E4M3 (X^T), fb=E5M2 (dY).  Any of the four pairs is accepted.
 *   A   M x K codes.  ma == FP8_MAJOR_K : A[i,k] at A[i*lda + k] (lda >= K);
 *                     ma == FP8_MAJOR_MN: A[i,k] at A[k*lda + i] (lda >= M).
 *   B   K x N codes.  mb == FP8_MAJOR_K : B[k,j] at B[j*ldb + k] (ldb >= K);
 *                     mb == FP8_MAJOR_MN: B[k,j] at B[k*ldb + j] (ldb >= N).
 *   D   M x N, row-major, D[i,j] at D[i*ldd + j], of type `out` (ldd in elements).
 *   scale_inv_a_dev / scale_inv_b_dev  device floats (the operands' inverse scales).
 *   amax_d_dev  NULL, or a device float OVERWRITTEN with amax of D as stored
 *               (after rounding), same definition as fp8_amax.
 * Alignment: A, B, D base addresses, lda, ldb (bytes) and ldd*sizeof(out) must
 * be multiples of 16, else FP8_ERR_ALIGN.  M, N, K are otherwise arbitrary
 * (edges are zero-filled on load and clipped on store).  M*N == 0 is a no-op
 * (amax = 0); K == 0 writes zeros.
 * Accumulation (`acc`): the products are exact and the tensor core adds them, 32 of K at a time, into a
 * binary32 accumulator whose additions round toward zero.
 *   FP8_ACC_SPLIT  (0, the default of a zero-initialised descriptor) the accumulator is drained every 2048 of K and the
 *                  partial sums are added in registers with round-to-nearest: below 1e-5 * sum_k|a.b| for ANY data and
 *                  any K.  For K <= 2048 it is the single accumulator.
 *   FP8_ACC_FAST   one accumulator over all of K, 2.5-4 % faster at K = 4096 .. 49152.  The error is below
 *                  1e-5 * sum_k|a.b| for K <= 2048 on any data; on products of mixed sign (training tensors: zero-mean
 *                  weights and gradients) it grows slowly with K (measured 1.4e-7 at K = 49152 on the workloads'
 *                  tensors, 1.2e-5 at K = 2^20 on heavy-tailed codes); products that all share one sign lose up to
 *                  (K/32) * 2^-23 of their sum (measured 3.7-5.3e-5 at K = 49152).  For callers who know their operands.
 * Every GEMM entry point that takes this descriptor honours `acc`; other values give FP8_ERR_ENUM.
 * Reproducibility: a call is bit-reproducible for a given problem (shapes, layouts, data) on a given device.  The
 * order in which the K-blocks of an output tile are accumulated (from the start or from the end of K) depends on
 * the tile's place in the kernel's schedule, so two equal dot products in different tiles may differ in the last
 * bits, within the stated tolerance.
 */
typedef struct {
    int64_t M, N, K;
    fp8_format fa, fb;
    fp8_major ma, mb;
    int64_t lda, ldb, ldd;
    fp8_wide out;
    fp8_accumulate acc;
} fp8_gemm_desc;

fp8_status fp8_gemm(const fp8_gemm_desc* d, const uint8_t* A, const uint8_t* B, void* D,
                    const float* scale_inv_a_dev, const float* scale_inv_b_dev,
                    float* amax_d_dev, void* stream);

/*
 * fp8_gemm_fp8out — Section 2: operations on FP8 inputs produce higher-precision results, which may
 * be converted to FP8 before they are written to memory.  Same contraction as fp8_gemm, but the
 * epilogue converts instead of storing a wide value:
 *   v[i,j] = (sum_k decode_fa(A[i,k]) * decode_fb(B[k,j])) * (sa_inv * sb_inv)      (binary32)
 *   D[i,j] = encode_fd( v[i,j] * scale_d )       conversion rules of fp8_quantize (RNE, specials, `od`)
 *   *amax_d_dev = amax over v, i.e. BEFORE the output scale and the conversion: it is the quantity the
 *                 next scale factor for this tensor is chosen from (scale_d itself comes from an earlier
 *                 step, as the scale-history recipes the paper leaves to software do).
 *   D            M x N codes, D[i,j] at D[i*ldd + j]; d->out is ignored; D and ldd 16-byte aligned.
 *   scale_d_dev  device float.
 * Everything else (operands, layouts, alignment, edge cases) as fp8_gemm.
 */
fp8_status fp8_gemm_fp8out(const fp8_gemm_desc* d, const uint8_t* A, const uint8_t* B, uint8_t* D,
                           fp8_format fd, fp8_overflow od,
                           const float* scale_inv_a_dev, const float* scale_inv_b_dev, const float* scale_d_dev,
                           float* amax_d_dev, void* stream);

/*
 * fp8_quantize_transpose — Sections 3 and 4.1: the same FP8 tensor is consumed by two matrix multiplies
 * that contract over different axes (an activation by the forward product and by the weight-gradient
 * product, an output gradient by both backward products), so its codes are produced once in both
 * orientations:
 *   code(r,c) = encode_f( binary32(x[r*ldx + c]) * scale )        conversion rules of fp8_quantize
 *   out  [r*ldo + c] = code(r,c)        (rows x cols; `out` may be NULL: transposed copy only)
 *   out_t[c*ldt + r] = code(r,c)        (cols x rows)
 *   *amax_dev (nullable) OVERWRITTEN with amax of x, same pass (definition of fp8_amax).
 * x is rows x cols, row-major, pitch ldx elements; ldo >= cols, ldt >= rows (bytes), else FP8_ERR_SHAPE.
 * One pass: 128 x 128 tiles, transposed through shared memory, every global access a full 128-byte line.
 * The tiled path needs rows and cols multiples of 4, x aligned to 4 elements with ldx a multiple of 4, and
 * out / out_t / ldo / ldt multiples of 4 bytes; anything else takes an element-wise kernel with identical
 * results.  rows*cols == 0 is a no-op (amax = 0).
 */
fp8_status fp8_quantize_transpose(const void* x, fp8_wide t, int64_t rows, int64_t cols, int64_t ldx,
                                  fp8_format f, fp8_overflow o, const float* scale_dev,
                                  uint8_t* out, int64_t ldo, uint8_t* out_t, int64_t ldt,
                                  float* amax_dev, void* stream);

/*
 * Per-channel scale factors — Section 4.2: post-training quantization scales weights channel by channel and
 * activations with one factor per tensor.  A channel is a row or a column of a 2-D tensor
 * x (rows x cols, row-major, pitch ld elements): axis 0 = one channel per column, axis 1 = one per row.
 *
 * fp8_amax_channels      amax_vec[c] = amax over channel c (definition of fp8_amax), OVERWRITTEN.
 * fp8_scales_from_amax   `count` scale factors at once, arithmetic of fp8_scale_from_amax; pow2 != 0 gives
 *                        the power-of-two scales of fp8_scale_pow2_from_amax.
 * fp8_quantize_channels  out[r*ld_out + c] = encode_f( binary32(x[r*ld + c]) * scale_vec[channel of (r,c)] ),
 *                        conversion rules of fp8_quantize.
 * Fast paths need 16-byte aligned rows (base and pitch); anything else takes element-wise kernels with
 * identical results.
 */
fp8_status fp8_amax_channels(const void* x, fp8_wide t, int64_t rows, int64_t cols, int64_t ld, int axis,
                             float* amax_vec_dev, void* stream);
fp8_status fp8_scales_from_amax(const float* amax_vec_dev, int64_t count, fp8_format f, int pow2,
                                float* scale_vec_dev, float* scale_inv_vec_dev, void* stream);
fp8_status fp8_quantize_channels(const void* x, fp8_wide t, int64_t rows, int64_t cols, int64_t ld, int axis,
                                 fp8_format f, fp8_overflow o, const float* scale_vec_dev,
                                 uint8_t* out, int64_t ld_out, void* stream);

/*
 * fp8_gemm_channel_scales — fp8_gemm for a B operand (the weights) quantized with per-channel scales:
 *   D[i,j] = round_out( (sum_k decode(A[i,k]) * decode(B[k,j])) * (sa_inv * sb_inv_vec[j]) )
 * scale_inv_b_vec_dev holds N device floats, one per column j of B (per output channel).  A keeps its
 * per-tensor inverse scale.  Everything else as fp8_gemm.
 */
fp8_status fp8_gemm_channel_scales(const fp8_gemm_desc* d, const uint8_t* A, const uint8_t* B, void* D,
                                   const float* scale_inv_a_dev, const float* scale_inv_b_vec_dev,
                                   float* amax_d_dev, void* stream);

/*
 * fp8_gemm_batched — Section 4.2 quantizes the inputs of every matrix multiply, the batched
 * products of attention among them.  `batch` independent products with the same shape, layouts,
 * formats and per-tensor scales (one scale for the whole batched tensor), in one launch:
 *   D_b = (A_b . B_b) * (sa_inv * sb_inv),   A_b = A + b*stride_a, B_b = B + b*stride_b, D_b = D + b*stride_d
 * Strides are in elements of the respective tensor and 16-byte aligned (in bytes).  The members of D lie at
 * least one whole matrix apart (they are written); the members of A and of B are only read, so any positive
 * stride is accepted: members may interleave (heads stored side by side inside a row, slices of K of one
 * matrix) or overlap.  amax_d_dev (optional) receives the amax over all batch members.  batch == 0 is a no-op
 * (amax = 0); batch <= 65535.  Everything else as fp8_gemm.
 */
fp8_status fp8_gemm_batched(const fp8_gemm_desc* d, int64_t batch,
                            const uint8_t* A, int64_t stride_a, const uint8_t* B, int64_t stride_b,
                            void* D, int64_t stride_d,
                            const float* scale_inv_a_dev, const float* scale_inv_b_dev,
                            float* amax_d_dev, void* stream);

/*
 * fp8_gemm_splitk — fp8_gemm for problems with few output tiles and a long contraction (a weight-bandwidth-
 * bound product of a few rows with a wide weight matrix): K is cut into `splits` slices that run as members of
 * one batched launch, each writing an fp32 partial product (already multiplied by sa_inv * sb_inv) into the
 * caller's workspace, and a second kernel adds the partials in slice order, rounds to `out` and records amax.
 *   D[i,j] = round_out( sum_s fl32( (sum_{k in slice s} a.b) * (sa_inv * sb_inv) ) )
 * Same tolerance as fp8_gemm (the extra binary32 roundings are ~1e-7 relative).  Deterministic.
 * fp8_gemm_splitk_workspace reports, for a descriptor, the number of slices the library will use on the
 * current device and the workspace it needs: splits = 1 (bytes = 0) whenever a cost model of the kernel (operand
 * bytes over min(tiles x 90 GB/s, HBM), plus the second launch and the partials) predicts less than 15 % gain,
 * K < 2048, N is not a multiple of 4, or K does not divide into slices that are multiples of 256; then
 * fp8_gemm_splitk is exactly fp8_gemm.  Otherwise splits is a power of two up to 16 and
 * bytes = splits * M * N * 4.  workspace_dev: 16-byte aligned device memory of at least that size (else
 * FP8_ERR_ALIGN / FP8_ERR_SHAPE), owned by the caller, contents undefined afterwards.  With splits > 1, D needs
 * only element alignment and ldd >= N.
 */
fp8_status fp8_gemm_splitk_workspace(const fp8_gemm_desc* d, int* splits_out, size_t* bytes_out);
fp8_status fp8_gemm_splitk(const fp8_gemm_desc* d, const uint8_t* A, const uint8_t* B, void* D,
                           const float* scale_inv_a_dev, const float* scale_inv_b_dev, float* amax_d_dev,
                           void* workspace_dev, size_t workspace_bytes, void* stream);

/*
 * Fused epilogues — Sections 2 and 4.1: what surrounds the matrix multiplies of a transformer layer (bias, activation,
 * residual addition, the gate of a gated feed-forward block) is applied to the binary32 dot products before they leave
 * the chip, and the result is stored in a wider type or converted to FP8 on the way out.
 *
 * What a result is stored as: a wide type, or FP8 codes  encode(v * scale_d)  by the rules of fp8_quantize.
 *
 * The three products below take an optional workspace (NULL, or 16 bytes of device memory on 16 bytes): with it the amax
 * needs no launch of its own for its start value.  It must hold zeros before its first use and is left zeroed by every
 * call, so one serves all calls of a stream; calls that may overlap on the GPU need different ones.
 */
typedef enum { FP8_STORE_F32 = 0, FP8_STORE_BF16 = 1, FP8_STORE_E4M3 = 2, FP8_STORE_E5M2 = 3 } fp8_store;
/*
 * Activations: relu max(z,0); gelu z*Phi(z) with the normal distribution function Phi; gelu_tanh
 * z*(1 + tanh(sqrt(2/pi)*(z + 0.044715 z^3)))/2; silu z/(1 + exp(-z)).  Computed in binary32 with the hardware's exponential
 * (2 ulp) and reciprocal (1 ulp), Phi by a fitted polynomial: values are within 3e-7 times max(1, |z|), slopes within 3e-7.
 * Relative to the value the error grows where the functions vanish (z = -6: gelu 6e-6, gelu_tanh 1e-5, silu 1e-6), and what is
 * below the normal range becomes 0.  At -inf they are 0 (their limit), NaN stays NaN.  The derivative of relu at 0 and at NaN is 0.
 */
typedef enum { FP8_ACT_NONE = 0, FP8_ACT_RELU = 1, FP8_ACT_GELU = 2, FP8_ACT_GELU_TANH = 3, FP8_ACT_SILU = 4 } fp8_activation;

/*
 * fp8_gemm_epilogue — the product of fp8_gemm with bias, activation and residual:
 *   z[i,j] = (sum_k decode_fa(A[i,k]) * decode_fb(B[k,j])) * (sa_inv * sb_inv) + bias[j]
 *   v[i,j] = act(z[i,j]) + residual[i,j]                       (all in binary32)
 *   D[i,j] = v rounded to the wide type, or encode(v * scale_d)
 *   pre[i,j] = z rounded to pre_t: what fp8_epilogue_backward reads
 *   *amax_d_dev = amax of D as stored (wide types), of v before scaling and conversion (FP8); as the other products.
 * d->out is ignored (e->store names the type).  In *e, NULL leaves a part out: bias (N elements), residual (M x N, pitch
 * ldr), pre (M x N, pitch ldp), scale_inv_b_vec_dev (N floats, one inverse scale per column of B, taken in place of
 * scale_inv_b_dev, which may then be NULL).  scale_d_dev is required for the FP8 stores.  residual may be D itself (same
 * address, pitch and type), otherwise the written matrices overlap nothing.
 * bias needs the alignment of its type; residual, pre and D are 16-byte aligned with pitches that are multiples of 16
 * bytes (FP8_ERR_ALIGN); pitches at least N (FP8_ERR_SHAPE).  K == 0 is an empty sum: z = bias.  M*N == 0 is a no-op
 * (amax = 0).  `acc` is accepted as by fp8_gemm; partial sums are added in registers in both of its values where the
 * kernel for few rows is taken.
 */
typedef struct {
    fp8_activation act;
    fp8_store store;
    fp8_overflow overflow;
    fp8_wide bias_t, residual_t, pre_t;
    const float* scale_inv_b_vec_dev;
    const void* bias;
    const void* residual;
    void* pre;
    int64_t ldr, ldp;
} fp8_epilogue;

fp8_status fp8_gemm_epilogue(const fp8_gemm_desc* d, const fp8_epilogue* e, const uint8_t* A, const uint8_t* B, void* D,
                             const float* scale_inv_a_dev, const float* scale_inv_b_dev, const float* scale_d_dev,
                             float* amax_d_dev, void* workspace_dev, void* stream);

/*
 * fp8_gemm_gated — the two up projections of a gated feed-forward block, the activation and the product, in one kernel:
 *   g = (A . Bg) * (sa_inv * sbg_inv),  u = (A . Bu) * (sa_inv * sbu_inv),  h = act(g) * u      (binary32)
 *   H = h rounded to the wide type, or encode(h * scale_h);  amax as fp8_gemm_epilogue.
 *   d         M, N, K of ONE projection (N = the block's inner width), formats, layouts, ldb of both B operands, ldd of H.
 *   w->gate, w->up   both or neither: M x N, pitch ldg, OVERWRITTEN with g and u rounded to gate_t, for the backward pass.
 * The two B operands may be halves of one matrix ([K, 2N] or [2N, K]): ldb is its pitch.
 * Alignment and special cases as fp8_gemm_epilogue (K == 0 gives g = u = 0).
 */
typedef struct {
    fp8_activation act;
    fp8_store store;
    fp8_overflow overflow;
    fp8_wide gate_t;
    void* gate;
    void* up;
    int64_t ldg;
} fp8_gated;

fp8_status fp8_gemm_gated(const fp8_gemm_desc* d, const fp8_gated* w, const uint8_t* A, const uint8_t* Bg, const uint8_t* Bu, void* H,
                          const float* scale_inv_a_dev, const float* scale_inv_bg_dev, const float* scale_inv_bu_dev,
                          const float* scale_h_dev, float* amax_h_dev, void* workspace_dev, void* stream);

/*
 * fp8_gemm_gated_backward — the data gradient of the down projection and the derivative of the gate in one kernel; the
 * gradient of h never reaches memory:
 *   dh = (A . B) * (sa_inv * sb_inv)           A = dY codes (M x K), B = the down weights as K x N, N = the inner width
 *   dG = dh * u * act'(g),  dU = dh * act(g)   g, u = w->gate, w->up as fp8_gemm_gated stored them (read)
 * stored as wide values or as encode(. * scale_d): ONE scale and one amax for both, so that [dG | dU] can be the two halves
 * of one M x 2N tensor of pitch ldd, the operand of the two remaining products (dX = [dG|dU] . [Bg|Bu]^T and
 * d[Bg|Bu] = X^T . [dG|dU], both fp8_gemm).  *amax_dev covers both.
 */
fp8_status fp8_gemm_gated_backward(const fp8_gemm_desc* d, const fp8_gated* w, const uint8_t* A, const uint8_t* B, void* dG, void* dU,
                                   const float* scale_inv_a_dev, const float* scale_inv_b_dev, const float* scale_d_dev,
                                   float* amax_dev, void* workspace_dev, void* stream);

/*
 * fp8_epilogue_backward — the backward pass of fp8_gemm_epilogue up to its product, in one pass over the output gradient:
 *   dz[i,j] = dy[i,j] * act'(pre[i,j])                          (binary32)
 *   out[i,j] = dz rounded to the wide type, or encode(dz * scale_dz): the E5M2 operand of the data and weight gradients
 *   dbias[j] = sum_i dz[i,j]                                    (binary32, from dz before its conversion; OVERWRITTEN)
 *   *amax_dev = amax of out as stored (wide types), of dz before scaling and conversion (FP8)
 * (the gradient of the residual is dy itself).  dy, pre: M x N wide, pitches ldy, ldp; pre may be NULL when act is
 * FP8_ACT_NONE.  dbias_dev (N floats) and amax_dev may be NULL.  M == 0 gives dbias = 0.  The sums are added in an order
 * that depends on the shape alone: repeated calls give the same bits.
 * Alignment: dy, pre and out 16-byte aligned with pitches that are multiples of 16 bytes (FP8_ERR_ALIGN).  out may be dy
 * itself (same address, pitch and type).
 *   workspace  fp8_epilogue_backward_workspace_bytes(M, N) bytes, 16-byte aligned; required when dbias_dev is given, else it
 *              may be NULL (then the amax takes a launch of its own for its start value).  It must hold zeros before its
 *              first use; every call leaves the part that matters zeroed again, so one buffer of the largest size serves any
 *              number of calls on one stream.  Calls that may overlap need different workspaces.
 */
size_t fp8_epilogue_backward_workspace_bytes(int64_t M, int64_t N);
fp8_status fp8_epilogue_backward(int64_t M, int64_t N, fp8_activation act, const void* dy, fp8_wide dy_t, int64_t ldy,
                                 const void* pre, fp8_wide pre_t, int64_t ldp, fp8_store store, fp8_overflow overflow,
                                 const float* scale_dz_dev, void* out, int64_t ldo, float* dbias_dev, float* amax_dev,
                                 void* workspace_dev, size_t workspace_bytes, void* stream);

/*
 * Global gradient norm and clipping over many tensors — Section 4.1 trains with the recipes of the higher-precision
 * baselines, of which norm clipping is a part; weight gradients are wide tensors.
 *   norm = sqrt(sum over all tensors of x^2);   coef = norm <= max_norm ? 1 : max_norm / norm;   out = round(x * coef)
 * The squares and the sums of up to 64 of them are binary32, the rest of the sum binary64.  So a magnitude above 1.8e19, or 64 of
 * more than 2.3e18 together, overflows to an infinite norm; below 1e-19 squares lose precision, below 2.6e-23 they count as 0.
 * The order of the additions depends on the plan alone.  The norm is that of the plan's tensors: where gradients are sharded
 * over ranks, their norms have to be combined by the caller, and the factor of fp8_grad_clip is each rank's own.  A NaN anywhere
 * gives a NaN norm and NaN everywhere in out; an infinite norm gives coef = 0 (0 for finite x, NaN for infinite x).
 *
 * A plan is made once for a list of tensors and holds their addresses, sizes and types: it is good as long as they stay where
 * they are, and a list whose tensors are freed or replaced (gradients dropped after a step) needs a new plan.
 *   fp8_clip_plan_size   fills *plan with the sizes of the table and of the workspace for these items.
 *   fp8_clip_plan_fill   writes the table (plan->table_bytes) to HOST memory; the caller copies it to the device.
 * fp8_grad_norm writes *norm_dev.  fp8_grad_clip writes *norm_dev and every out (out == x clips in place; then nothing is
 * written when coef is 1).  The workspace: device, plan->workspace_bytes, 16-byte aligned, zero before its first use; every
 * call leaves the part that matters zeroed.  Items need the alignment of their elements only (16 bytes are faster); x_t and
 * out_t may differ, and out may overlap nothing but its own x.  max_norm below 0 or NaN: FP8_ERR_UNSUPPORTED.
 */
typedef struct {
    const void* x;
    void* out;                  /* NULL: counted in the norm, not written */
    int64_t n;
    fp8_wide x_t, out_t;
} fp8_clip_item;
typedef struct {
    int64_t count, chunks;
    size_t table_bytes, workspace_bytes;
} fp8_clip_plan;

fp8_status fp8_clip_plan_size(const fp8_clip_item* items, int64_t count, fp8_clip_plan* plan);
fp8_status fp8_clip_plan_fill(const fp8_clip_item* items, const fp8_clip_plan* plan, void* table_host);
fp8_status fp8_grad_norm(const fp8_clip_plan* plan, const void* table_dev, void* workspace_dev, float* norm_dev, void* stream);
fp8_status fp8_grad_clip(const fp8_clip_plan* plan, const void* table_dev, void* workspace_dev, float max_norm,
                         float* norm_dev, void* stream);

/*
 * AdamW over many tensors — Section 4.1 trains with the optimisers of the higher-precision baselines; parameters, gradients and
 * the arithmetic stay wide, the copy that the next step's products read is FP8.  One launch over a plan, like fp8_grad_clip:
 *   coef = norm <= max_norm ? 1 : max_norm / norm      (norm_dev NULL: 1),   g' = g * coef
 *   m = beta1 m + (1 - beta1) g',   v = beta2 v + (1 - beta2) g'^2
 *   p = p (1 - lr weight_decay) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 * in binary32, each operation rounded to nearest, in the order written with the factors lr / (1 - beta1^t) and
 * 1 / sqrt(1 - beta2^t) rounded once; p is rounded to p_t.  (A quotient may, rarely, be off by its last bit, or by two where its
 * numerator is below 2^-100.)
 * A norm that is not finite skips the step: parameters, moments and the step counter stay as they are (the copies and their
 * amax are written from the parameters as they are).  Without norm_dev a gradient that is not finite makes its element NaN.
 *
 * States.  FP8_STATE_F32: m and v are n floats.  FP8_STATE_E4M3: n codes each, in blocks of 256 consecutive elements with a
 * scale each (m_scale, v_scale: ceil(n / 256) floats), value = code * scale.  With top = the block's largest magnitude,
 * scale = top * binary32(1 / 448), and what becomes a code is x * ((1 / top) * 448), each operation rounded (0 where top is 0):
 *   m holds the first moment, rounded to nearest;
 *   v holds the SQUARE ROOT of the second moment, rounded up or down with the probability of its distance (to nearest it would
 *     stand still: with beta2 near 1 it moves less than half a step at a time); one that is not zero keeps at least code 1.
 *   A first moment's scale below 2^-126 has few bits, and is 0 for a top of 3.1e-43 or less.  For a top below 2^-119 the codes are
 *     those of (m * 2^100) * (1 / (scale * 2^100)), so that code * scale is m as nearly as the scale allows, or 0 where the scale is.
 * With independent normal gradients v's root then scatters around its exact value by 9 % (beta2 = 0.9), 11 % (0.95), 15 % (0.99) or
 * 16 % (0.999) of it, its square is 1 to 5 % high in the mean, and the updates differ by 8 to 14 % of their mean from those
 * with binary32 moments.
 * The update of p uses the moments before they are rounded.  All zeros (codes and scales) is the state to start from.  A block
 * in which a moment is not finite holds nothing finite afterwards.  The random numbers are 16 bits per element, a function of
 * seed, t (both modulo 2^32 words of it) and the element's place in the plan: items are numbered one after the other, each from a
 * multiple of 256.  The same plan, seed and t give the same bits.
 *
 * Copy (NULL: none): the new parameters as stored, in bf16, or as codes encode(p * copy_scale) with saturation, rules of
 * fp8_quantize; copy_amax_dev (may be NULL; codes only) is OVERWRITTEN with amax of the new parameters, from which the next
 * step's copy_scale is chosen.
 *
 * lr_dev (binary32), step_dev take the place of lr, step where they are given, so that a captured call goes on from step to step: step_dev
 * counts the steps taken; the call uses t = *step_dev + 1 and adds one when it is done.
 * Plans as those of fp8_grad_clip: made on the host, addresses and sizes must stay.  The workspace must hold zeros before its
 * first use and is left zeroed; calls that may overlap need plans of their own.  Items need the alignment of their elements
 * only (32 bytes for binary32, 16 for bf16 and 8 for codes are faster); no two overlap.
 * beta1, beta2 in [0, 1), eps >= 0, step >= 1, max_norm >= 0 and weight_decay >= 0 finite, else FP8_ERR_UNSUPPORTED.
 */
typedef enum { FP8_STATE_F32 = 0, FP8_STATE_E4M3 = 1 } fp8_state;
typedef struct {
    const void* g;
    void* p;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    void* copy;
    const float* copy_scale_dev;
    float* copy_amax_dev;
    int64_t n;
    float weight_decay;
    fp8_wide g_t, p_t;
    fp8_state state;
    fp8_store copy_t;
} fp8_adamw_item;
typedef struct {
    int64_t count, chunks, chunk, amaxes;
    size_t table_bytes, workspace_bytes;
} fp8_adamw_plan;
typedef struct {
    double lr, beta1, beta2, eps;
    int64_t step;
    uint64_t seed;
    const float* norm_dev;
    const float* lr_dev;
    int64_t* step_dev;
    float max_norm;
} fp8_adamw_options;

fp8_status fp8_adamw_plan_size(const fp8_adamw_item* items, int64_t count, fp8_adamw_plan* plan);
fp8_status fp8_adamw_plan_fill(const fp8_adamw_item* items, const fp8_adamw_plan* plan, void* table_host);
fp8_status fp8_adamw_step(const fp8_adamw_plan* plan, const void* table_dev, void* workspace_dev, const fp8_adamw_options* o, void* stream);

/*
 * Softmax cross entropy of a vocabulary projection — Sections 3.1 and 4.1: the loss that the language models are trained and
 * evaluated with (perplexity is its exponential), and the first gradient of their backward pass.  The logits never reach
 * memory: the vocabulary is gone through in pieces, forward and backward.
 *   z[t,v] = (sum_k x[t,k] * w[v,k]) * (sx_inv * sw_inv)          binary32
 *   lse[t] = log sum_v exp(z[t,v]),   loss[t] = lse[t] - z[t, target[t]]
 *   dz[t,v] = (exp(z[t,v] - lse[t]) - [v == target[t]]) * dloss[t]
 *   dx = dz . w,   dw = dz^T . x       rounded to dx_t, dw_t
 * Operands: x (tokens x width, pitch ldx) and w (vocab x width, pitch ldw), rows contiguous, both FP8 codes (any pair of
 * formats, inverse scales required) or both bf16 (the inverse scales may be NULL, which counts as 1).
 * Targets: 64-bit indices.  A token whose target is not in 0 .. vocab-1 does not count: its loss is 0, its row of dz is 0 and
 * dloss is not looked at; its lse is written all the same.  (Its row of x still meets these zeros in dw: NaN or infinities
 * there give NaN.)
 * The gradient of the logits: FP8 operands take E5M2 codes encode(dz * s) with s = 57344 / max |dloss[t]| over the tokens that
 * count (1 where that is 0 or not finite): |dz| never exceeds it, so no amax of dz is needed, and what is below 1.2e-10 of it
 * becomes 0.  bf16 operands take bf16.  dz never leaves the workspace.  A dloss that is not finite, of a token that counts, makes
 * that token's row of dx and all of dw NaN or (bf16) infinite.
 * Precision: products are exact, their sums as FP8_ACC_SPLIT; exponentials by the hardware (2 ulp).  z and lse are binary32
 * numbers, so exp(z - lse) may be off by 2^-24 |lse| of itself; but where one logit of a row stands alone, lse is that number,
 * and dz is exactly dloss, -dloss or 0, as a backward pass of the same descriptor adds up the same z.  A row with a NaN or a
 * plus-infinite logit gives NaN; a row of minus infinities has lse = -inf.
 * fp8_cross_entropy_backward reads the lse that the forward pass wrote and the per-token factors dloss (1/tokens for a mean).
 * dx and dw are OVERWRITTEN; either may be NULL.  tokens == 0: dw = 0, nothing else is touched.  width and vocab are at least 1.
 * x, w, dx, dw are 16-byte aligned with pitches that are multiples of 16 bytes (FP8_ERR_ALIGN) and at least width
 * (FP8_ERR_SHAPE); the written matrices overlap nothing.
 * Workspace: device, 16-byte aligned, of the size that fp8_cross_entropy_workspace_bytes gives for the descriptor on the
 * current device; its contents before and after do not matter.  Calls that may overlap need different ones.
 * Results depend on the shape and the device alone, not on timing: repeated calls give the same bits.
 */
typedef enum { FP8_OPERAND_E4M3 = 0, FP8_OPERAND_E5M2 = 1, FP8_OPERAND_BF16 = 2 } fp8_operand;
typedef struct {
    int64_t tokens, width, vocab;
    fp8_operand x_t, w_t;
    int64_t ldx, ldw;                  /* elements */
} fp8_cross_entropy_desc;

fp8_status fp8_cross_entropy_workspace_bytes(const fp8_cross_entropy_desc* d, size_t* forward_bytes_out, size_t* backward_bytes_out);
fp8_status fp8_cross_entropy(const fp8_cross_entropy_desc* d, const void* x, const void* w, const float* scale_inv_x_dev,
                             const float* scale_inv_w_dev, const int64_t* target_dev, float* loss_dev, float* lse_dev,
                             void* workspace_dev, size_t workspace_bytes, void* stream);
fp8_status fp8_cross_entropy_backward(const fp8_cross_entropy_desc* d, const void* x, const void* w, const float* scale_inv_x_dev,
                                      const float* scale_inv_w_dev, const int64_t* target_dev, const float* lse_dev,
                                      const float* dloss_dev, void* dx, fp8_wide dx_t, int64_t lddx, void* dw, fp8_wide dw_t,
                                      int64_t lddw, void* workspace_dev, size_t workspace_bytes, void* stream);

/*
 * fp8_async_status — reads and clears the device-side error latch of the
 * current device (synchronises the device).  FP8_OK, or FP8_ERR_TIMEOUT if a
 * kernel gave up on a bounded wait since the last call; *detail (optional, host
 * pointer) receives a code naming the wait.  Not part of the paper: it exists
 * so that a pipeline fault ends in an error code instead of a hung GPU.
 */
fp8_status fp8_async_status(uint32_t* detail);

/*
 * fp8_self_test_expire_wait — the paper has no counterpart; a self-test of the library's safety net.  Every
 * device-side wait in the library (the mbarrier waits of the GEMM pipeline, the grid barrier of
 * fp8_quantize_current) counts SM clocks and gives up after a limit, so that a pipeline fault ends in
 * FP8_ERR_TIMEOUT instead of a hung GPU.  This call makes one such wait run out ON PURPOSE, in a way that
 * cannot hang or fault: it launches a small kernel whose wait can never be satisfied and whose limit is
 * `limit_cycles` SM clocks (1 .. 2e9, i.e. at most about a second; FP8_ERR_UNSUPPORTED otherwise).
 *   FP8_WAIT_MBARRIER      one block waits on an mbarrier nobody arrives on, through the same bounded-wait
 *                          routine the GEMM roles use; detail code 9.
 *   FP8_WAIT_GRID_BARRIER  the fp8_quantize_current kernel runs on an empty tensor with its grid barrier told to
 *                          expect one block more than the grid has: every block gives up, nothing is written, the
 *                          control words (those of fp8_quantize_current_static) are left zeroed; detail code 16.
 * Afterwards fp8_async_status returns FP8_ERR_TIMEOUT once, with the detail code above, then FP8_OK again;
 * the stream and the library remain fully usable.
 */
typedef enum { FP8_WAIT_MBARRIER = 0, FP8_WAIT_GRID_BARRIER = 1 } fp8_wait_kind;
fp8_status fp8_self_test_expire_wait(int which, uint64_t limit_cycles, void* stream);

/*
 * fp8_sm_clock_probe — the paper has no counterpart; a measurement aid.  Launches a one-warp kernel that reads the SM
 * cycle counter and the device's nanosecond timer, waits `duration_us` microseconds (1 .. 100000, else
 * FP8_ERR_UNSUPPORTED; the wait is bounded by an iteration count as well) and reads both again.
 *   out_dev  device, two 64-bit words, OVERWRITTEN: [0] = SM clocks elapsed, [1] = nanoseconds elapsed;
 *            clocks * 1000 / nanoseconds = SM clock in MHz during the window.
 * Enqueued on a second stream it runs beside other kernels (it needs one warp and no shared memory), which is how the
 * benchmark reads the clock the tensor cores actually ran at under the power cap: the management interface samples
 * too coarsely for that.
 */
fp8_status fp8_sm_clock_probe(uint64_t* out_dev, uint32_t duration_us, void* stream);

/* Human-readable name of a status code (static storage, never NULL). */
const char* fp8_status_string(fp8_status s);

/* Number of kernel launches (and memset nodes) the library has enqueued since
 * it was loaded; host-side counter used by benchmarks to report launch counts. */
uint64_t fp8_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* FP8_B200_H */
