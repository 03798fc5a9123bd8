/*
 * sqp.h -- C ABI of the SmoothQuant+ W4A16 linear-layer library for AMD MI355X (gfx950).
 *
 * The operations are those of arXiv 2312.03788: per-channel smoothing (Eq. 5, Eq. 6),
 * group-wise asymmetric 4-bit weight quantisation (Eq. 1, Sec 2.2) and the quantised
 * linear layer Y = X * W_hat with FP16 input/output and INT4 weights (Eq. 3, Fig. 7).
 *
 * Conventions for every entry point
 *   - Orientation follows Eq. 2: X is [M x K] (tokens x input channels), W is [K x N]
 *     (input channels x output channels), Y is [M x N]; all row-major, last index
 *     contiguous.
 *   - Every pointer is a DEVICE pointer owned by the caller and must be 16-byte aligned
 *     (the fp64 outputs of the loss calls: 8-byte).  fp16 data is IEEE binary16.  The
 *     library allocates no device memory, frees none, and keeps no caller memory except
 *     the workspace pointer handed to sqp_set_workspace.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Work is
 *     only enqueued; no call synchronises the device or allocates, so every call may be
 *     recorded into a HIP graph.
 *   - Return value: SQP_OK (0), or a negative error code, in which case nothing was
 *     enqueued.  sqp_status_string() names a code.
 *   - Shape rules: M, N, K > 0; N % 8 == 0; K % 8 == 0; group % 8 == 0, group >= 8,
 *     K % group == 0; every tensor has fewer than 2^31 elements.
 *
 * Storage format of a quantised weight (what sqp_quantize_pack writes and
 * sqp_dequantize / sqp_w4a16_gemm read):
 *   packed[K/8][N]      uint32; word (j, n) holds the 4-bit codes of input channels
 *                       k = 8j .. 8j+7 of output column n, the code of k = 8j+i in bits
 *                       [4i+3 : 4i] (lowest nibble = lowest k).
 *   scales[K/group][N]  fp16 step size Delta of group t = k / group, column n.
 *   zeros [K/group][N]  uint8 zero point Z in [0, 15] of the same group.
 */
#ifndef SQP_H
#define SQP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif
#pragma GCC visibility push(default) /* the library is built with hidden visibility: these are its exports */

#define SQP_OK 0
#define SQP_ERR_NULL (-1)    /* a required pointer is NULL */
#define SQP_ERR_SHAPE (-2)   /* a shape rule above is violated */
#define SQP_ERR_ALIGN (-3)   /* a pointer is not 16-byte aligned */
#define SQP_ERR_ARG (-4)     /* alpha outside [0, 1] or not finite; eps, scale or type out of range */
#define SQP_ERR_LAUNCH (-5)  /* the HIP runtime reported an error at launch */
#define SQP_ERR_WORKSPACE (-6) /* the workspace is too small for the launch plan of this shape */

const char *sqp_status_string(int status);

/* Smoothing factor of Eq. 6:  s[j] = max_t|x_cal[t][j]|^alpha / max_n|w[j][n]|^(1-alpha),
 * j = input channel.  Both maxima are floored at 1e-5 (Eq. 6 is 0 or infinite on a dead
 * channel); the quotient is evaluated in fp64 and rounded once to fp32.
 *   x_cal [T][K] fp16  calibration activations (Sec 2.2: per-channel maxima over the
 *                      calibration tokens)
 *   w     [K][N] fp16  the unsmoothed weight
 *   s     [K]    fp32  out; also used as scratch while the call runs
 * alpha in [0, 1]. */
int sqp_smooth_scales(int T, int K, int N, float alpha, const void *x_cal, const void *w,
                      float *s, void *stream);

/* Activation side of Eq. 5:  x_out[m][j] = fp16(x[m][j] / s[j]), fp32 divide, one rounding.
 * x, x_out [M][K] fp16 (may alias), s [K] fp32. */
int sqp_smooth_apply_x(int M, int K, const void *x, const float *s, void *x_out, void *stream);

/* Weight side of Eq. 5:  w_out[j][n] = fp16(s[j] * w[j][n]), fp32 multiply, one rounding.
 * w, w_out [K][N] fp16 (may alias), s [K] fp32. */
int sqp_smooth_apply_w(int K, int N, const void *w, const float *s, void *w_out, void *stream);

/* The merged gate/up projection of a LlamaMLP block with its activation fused (Fig. 5: the
 * block whose smoothing factors are folded into the preceding layers).  packed/scales/zeros
 * hold the quantised merged weight [K][N] whose columns alternate (gate j, up j)
 * (sqp_interleave_gate_up); the result is
 *   y[m][j] = fp16( SiLU(g) * u ),  g, u = the fp32 sums of Eq. 3 for columns 2j and 2j+1,
 * y [M][N/2] fp16.  N % 16 == 0; group 32, 64 or a multiple of 128.  Otherwise as sqp_w4a16_gemm. */
int sqp_w4a16_gemm_silu_mul(int M, int N, int K, int group, const void *x, const uint32_t *packed,
                            const void *scales, const uint8_t *zeros, void *y, void *stream);

/* LlamaRMSNorm: y[m][j] = fp16( x[m][j] / sqrt(mean_j x[m][j]^2 + eps) * gamma[j] ), fp32
 * arithmetic.  gamma [H] fp16 may already contain the division by the smoothing factor of the
 * layers it feeds (Sec 2.2: fused into post_attention_layernorm; fold it with
 * sqp_smooth_apply_x on the 1 x H weight).  x, y [M][H] fp16, H % 8 == 0, 0 <= eps < 1. */
int sqp_rmsnorm(int M, int H, const void *x, const void *gamma, float eps, void *y, void *stream);

/* w_out[k][n] = fp16(w[k][n] / s[n]): divides the OUTPUT columns of a layer by the smoothing
 * factor of the layer it feeds (Sec 2.2: down_proj's factor fused into up_proj's weights).
 * w, w_out [K][N] fp16 (may alias), s [N] fp32, N % 8 == 0. */
int sqp_scale_columns(int K, int N, const void *w, const float *s, void *w_out, void *stream);

/* w_out [K][2I] with column 2j = w_gate[.][j] and column 2j+1 = w_up[.][j] (exact copies), the
 * merged layout sqp_w4a16_gemm_silu_mul expects.  w_gate, w_up [K][I] fp16, I % 8 == 0. */
int sqp_interleave_gate_up(int K, int I, const void *w_gate, const void *w_up, void *w_out, void *stream);

/* Orientation helper: w_nk [N][K] fp16 (one row per output feature, as checkpoints store a
 * linear layer) -> w_kn [K][N] fp16, the orientation of Eq. 2 (X W with W of shape Ci x Co) that
 * every other entry point takes.  Exact copy of the values; the buffers must not overlap. */
int sqp_transpose_nk(int N, int K, const void *w_nk, void *w_kn, void *stream);

/* Group-wise asymmetric 4-bit quantisation of Eq. 1 along K (Sec 2.2) and packing.
 * For each column n and group t (rows t*group .. (t+1)*group-1):
 *   lo = min(min w, 0), hi = max(max w, 0)           (range widened to contain 0)
 *   Delta = fp16((hi - lo) / 15), replaced by 2^-24 if that is zero
 *   Z = clamp(round(-lo / Delta), 0, 15)
 *   code = clamp(round(w / Delta) + Z, 0, 15)        round = half-to-even, fp32 divide
 * w [K][N] fp16 (already smoothed); packed/scales/zeros as described above (out). */
int sqp_quantize_pack(int N, int K, int group, const void *w, uint32_t *packed, void *scales,
                      uint8_t *zeros, void *stream);

/* Second line of Eq. 1:  w_hat[k][n] = fp16((code - Z) * Delta).  w_hat [K][N] fp16 out. */
int sqp_dequantize(int N, int K, int group, const uint32_t *packed, const void *scales,
                   const uint8_t *zeros, void *w_hat, void *stream);

/* The quantised linear layer of Eq. 3 (Fig. 7: FP16 in, INT4 weights, FP16 out):
 *   y[m][n] = fp16( sum_k x[m][k] * (code[k][n] - Z[k/group][n]) * Delta[k/group][n] )
 * with fp32 accumulation and one rounding to fp16 at the end.  The result is
 * run-to-run deterministic.  x [M][K] fp16, y [M][N] fp16 out (must not alias x).
 * Rows M <= 64 take the weight-streaming (memory-bound) path, larger M the tiled
 * matrix-core path.  When the output has too few tiles to occupy the chip, the launch plan
 * splits the inner dimension across workgroups and passes fp32 partial sums through the
 * workspace set with sqp_set_workspace.  sqp_w4a16_gemm_workspace_bytes() is 0 for the shapes
 * that never touch it: with few rows, or few rows and a short K, groups of 128 (they split K
 * inside each workgroup); M <= 64 with a K of fewer than eight chunks of 128 (or of one group of 32 or
 * 64); larger M with more tiles of 128 x 512 than a quarter of the chip's compute units (those can
 * split too, but only in a scratch buffer of their own: sqp_w4a16_gemm_scratch).  For the others:
 *   - no workspace set: a plan without a split across workgroups runs (same result within the
 *     tolerance of Eq. 3's fp32 accumulation, slower on narrow layers with long K);
 *   - workspace smaller than sqp_w4a16_gemm_workspace_bytes() of the shape: a plan that fits
 *     it runs, down to sqp_w4a16_gemm_workspace_least_bytes(); below that SQP_ERR_WORKSPACE,
 *     nothing enqueued.
 * (Up to 32 rows some of these shapes run a plan that leaves the workspace untouched; sizes and
 * refusals are the same for them.)
 * Calls that use the workspace must not overlap on the device (order them on one stream, or
 * with events): they share its tickets and partial sums.  Calls of shapes whose
 * sqp_w4a16_gemm_workspace_bytes() is 0 may overlap with anything. */
int sqp_w4a16_gemm(int M, int N, int K, int group, const void *x, const uint32_t *packed,
                   const void *scales, const uint8_t *zeros, void *y, void *stream);

/* The same call (silu_mul != 0: sqp_w4a16_gemm_silu_mul) with a scratch buffer of its own, where a grid
 * that fills the chip leaves a last round of few tiles, or tiles of another height fit better with K
 * split: the partial sums of those K parts go there.  The buffer belongs to this call until the work
 * enqueued by it has run, needs no preparation and holds nothing afterwards; NULL or a smaller
 * one: a plan that fits runs (as sqp_w4a16_gemm without any).  Everything else, the workspace of
 * the shapes that use it included, is as for sqp_w4a16_gemm. */
int sqp_w4a16_gemm_scratch(int M, int N, int K, int group, int silu_mul, const void *x, const uint32_t *packed,
                           const void *scales, const uint8_t *zeros, void *y, void *scratch, size_t scratch_bytes,
                           void *stream);

/* Bytes of scratch the preferred plan of sqp_w4a16_gemm_scratch uses (0: none).  Host arithmetic only. */
size_t sqp_w4a16_gemm_scratch_bytes(int M, int N, int K, int group);

/* Bytes of workspace the launch plan of sqp_w4a16_gemm / sqp_w4a16_gemm_silu_mul uses for
 * this shape on the current device: 0 if the plan does not split the inner dimension,
 * otherwise 512 KB of tickets plus the fp32 partial sums.  Host arithmetic only. */
size_t sqp_w4a16_gemm_workspace_bytes(int M, int N, int K, int group);

/* The smallest workspace with which a call of this shape is not refused (at most the bytes above;
 * the two differ where the preferred plan splits more than it has to).  Host arithmetic only. */
size_t sqp_w4a16_gemm_workspace_least_bytes(int M, int N, int K, int group);

/* Hands the library a caller-owned device buffer for the partial sums of Eq. 3's split
 * launches on the CURRENT device (process-wide, one per device; the library keeps only the
 * pointer).  The call enqueues one kernel on `stream` that zeroes the ticket area (the first
 * 512 KB); GEMM calls must be ordered after it.  Every split launch leaves the tickets zero
 * again, so the buffer is set once; after an aborted launch set it again.  The caller keeps
 * the buffer alive until it sets another one or none: (NULL, 0) removes it.
 * Errors: SQP_ERR_ALIGN; SQP_ERR_WORKSPACE if bytes <= 512 KB.  Not to be called while
 * another thread is inside a GEMM call. */
int sqp_set_workspace(void *dev_ptr, size_t bytes, void *stream);

/* Quantisation loss of one layer, Eq. 4:  *loss = || x w - x_hat w_hat ||_F^2  with
 * w_hat the dequantised weights of (packed, scales, zeros) (Eq. 1) - the quantity the search
 * over the smoothing strength alpha minimises (Sec 2.2, Eq. 6), for one layer.  Both products
 * are accumulated together in fp32, 16 k of each in turn (the difference is formed before any
 * rounding to fp16, and rounding is relative to it and not to x w),
 * the squares are summed in fp64 in a fixed order (run-to-run deterministic).
 *   x     [M][K] fp16  calibration activations        w [K][N] fp16  the unsmoothed weight
 *   x_hat [M][K] fp16  smoothed activations (Eq. 5)   packed/scales/zeros: quantised smoothed weight
 *   scratch  device, at least sqp_quant_loss_scratch_doubles(M, N) doubles, overwritten
 *   loss     device, one double (out)
 * All device pointers (scratch and loss 8-byte aligned); nothing is allocated. */
long sqp_quant_loss_scratch_doubles(int M, int N);
int sqp_quant_loss(int M, int N, int K, int group, const void *x, const void *w, const void *x_hat,
                   const uint32_t *packed, const void *scales, const uint8_t *zeros, double *scratch,
                   double *loss, void *stream);

/* sqp_w4a16_gemm for callers that cannot allocate device memory and own no workspace: code
 * recorded under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same arguments, kernels, launch plans and results as sqp_w4a16_gemm with a sufficient
 * workspace set (bit-identical), but the tickets and partial sums of split launches live in a
 * static device array of the library: 512 KB + SQP_STATIC_PARTIAL_BYTES per device, held
 * until the process ends.  The call allocates nothing and ignores sqp_set_workspace.
 *   - A shape whose plan needs more partial sums than SQP_STATIC_PARTIAL_BYTES
 *     (sqp_w4a16_gemm_workspace_bytes(shape) - 512 KB) is refused with SQP_ERR_WORKSPACE,
 *     nothing enqueued.  The library's own plans stay below the limit for every shape.
 *   - The first call on a device looks the array up and enqueues one extra kernel that zeroes
 *     its tickets; make that call outside a graph capture.
 *   - All calls on one device share the array: calls that overlap on the device race (order
 *     them on one stream or with events), as do overlaps with nothing else in this library. */
#define SQP_STATIC_PARTIAL_BYTES ((size_t)48 << 20)
int sqp_w4a16_gemm_static(int M, int N, int K, int group, const void *x, const uint32_t *packed,
                          const void *scales, const uint8_t *zeros, void *y, void *stream);

/* Search of the smoothing strength for one layer (Sec 2.2: alpha is chosen on a grid to
 * minimise the quantisation loss of Eq. 4; the paper's grid is 0, 0.05, ..., 1).  The
 * per-channel maxima of Eq. 6 do not depend on alpha and are computed once; then for each
 * alphas[i], in order:  s = Eq. 6,  x_hat = x_cal / s and w_s = s * w (Eq. 5),  w_s quantised
 * (Eq. 1),  loss[i] = Eq. 4 on the calibration rows.  *best = index of the smallest loss (the
 * lowest index on ties).  loss[i] equals what the entry points above would give, bit for bit.
 *   alphas   HOST array of n_alpha values in [0, 1], 1 <= n_alpha <= 4096
 *   x_cal [T][K] fp16, w [K][N] fp16                                    (in)
 *   amax [2K] fp32, s [K] fp32, x_hat [T][K] fp16, w_s [K][N] fp16, packed / scales / zeros of
 *   the layer's shape, scratch (sqp_quant_loss_scratch_doubles(T, N) doubles): device work
 *   buffers, overwritten; on return they hold the last alpha's values
 *   loss [n_alpha] fp64 device (out), best: one int, device (out)
 * Nothing is allocated and nothing synchronises; errors as for the single calls. */
int sqp_alpha_search(int T, int N, int K, int group, int n_alpha, const float *alphas, const void *x_cal,
                     const void *w, float *amax, float *s, void *x_hat, void *w_s, uint32_t *packed,
                     void *scales, uint8_t *zeros, double *scratch, double *loss, int *best, void *stream);

/* The same search for callers that want the losses alone: all work buffers lie in one scratch buffer, which
 * may be larger, so that several alphas share a launch and the next ones are prepared beside them.
 * The losses are those of sqp_alpha_search, bit for bit.
 *   scratch  device, 16-byte aligned, overwritten; nothing in it is needed before or after the call
 *   scratch_bytes  sqp_alpha_search_scratch_bytes() for the preferred plan; with less a plan that fits
 *                  runs, and below sqp_alpha_search_scratch_least_bytes(), where not even one alpha's
 *                  operands fit, the call is refused with SQP_ERR_WORKSPACE, nothing enqueued
 * The two sizes: host arithmetic only, 0 for invalid arguments. */
size_t sqp_alpha_search_scratch_bytes(int T, int N, int K, int group, int n_alpha);
size_t sqp_alpha_search_scratch_least_bytes(int T, int N, int K, int group, int n_alpha);
int sqp_alpha_search_scratch(int T, int N, int K, int group, int n_alpha, const float *alphas, const void *x_cal,
                             const void *w, void *scratch, size_t scratch_bytes, double *loss, int *best, void *stream);

/* Element types of a key / value cache and of quantised activations.  SQP_E4M3: 8 bits, 4 of exponent and 3 of mantissa, no
 * infinities, largest value 448.  An 8-bit row has one fp32 scale: it stands for code * scale, with
 *   scale = max|row| / 127 (SQP_INT8) or / 448 (SQP_E4M3),  code = round-to-nearest-even(row * (127 or 448) / max|row|);
 * a row whose largest magnitude is below 2^-100 is stored as zeros with scale 0, one with an infinity or NaN with scale NaN. */
#define SQP_FP16 0
#define SQP_INT8 1
#define SQP_E4M3 2
/* Microscaled numbers: blocks of 32 values along a row.  SQP_E2M1: 4 bits, 2 of exponent and 1 of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and
 * their negatives, two to a byte, the first in the low half; or elements SQP_E4M3.  A block has one scale in a byte b: its values are
 * code * 2^(b - 127).  The scale of a block is the least power of two with which its largest magnitude rounds to a value of the type,
 * so that no value is cut off; code = round-to-nearest-even(value / scale).  A block whose largest magnitude is below 2^-100 is
 * stored as zeros with b = 0, one with an infinity or NaN as zeros with b = 255, which stands for NaN: all of it reads back as NaN.
 * Negative values that round to zero keep their sign. */
#define SQP_E2M1 4

/* Rows into blocks of `type` (SQP_E2M1 or SQP_E4M3) and back.  x [R][K] fp16, K % 32 == 0; codes [R][K/2] bytes (e2m1) or [R][K];
 * scales [R][K/32] bytes.  Back: x = fp16(code * scale), one rounding (values beyond fp16's largest become infinite). */
int sqp_mx_quantize(int R, int K, int type, const void *x, void *codes, uint8_t *scales, void *stream);
int sqp_mx_dequantize(int R, int K, int type, const void *codes, const uint8_t *scales, void *x, void *stream);

/* A weight w [K][N] fp16 (the orientation of Eq. 2, already smoothed) into e2m1 blocks along K: one row per output column, codes
 * [N][K/2], scales [N][K/32], which is what sqp_mx_quantize gives for w transposed.  K % 32 == 0, K <= 16776960, N % 8 == 0. */
int sqp_mx_quantize_weight(int N, int K, const void *w, void *codes, uint8_t *scales, void *stream);

/* The linear layer on blocks: y[m][n] = fp16( sum_k x[m][k] w[n][k] ), the products of the codes multiplied by both blocks' scales on
 * the matrix cores and summed in fp32, one rounding at the end.  Products of e2m1 by e2m1 are exact.  Of e4m3 by e2m1 the matrix cores take
 * eight neighbouring k (k / 8) together and cut, towards zero, what lies below 2^-13 of the largest power of two among them: a product
 * smaller than 2^-7 of the largest of its eight is off by up to 2^-12 of that largest, the others by nothing.  So the sum is off by up to
 * 7 * 2^-12 of the sum of the eights' largest products, besides fp32's own additions; beside a channel of outliers, or where large products cancel, that is
 * what is left of its seven neighbours.  (Uniformly random codes lose up to 2e-4 of sum |x w|, a sum's outputs 2.1e-4 rms with their rounding.)
 * x: M rows of x_type (SQP_E2M1 or SQP_E4M3) with their scales, w: N rows of e2m1 with theirs.  M, N, K > 0, N % 8 == 0, K % 32 == 0.
 * silu_mul != 0: the columns alternate (gate j, up j) (sqp_interleave_gate_up), N % 16 == 0, and y [M][N/2] = fp16(SiLU(g) u) of the fp32 sums.  A block that is NaN makes NaN of its row (x) or column (w).  Deterministic.
 * scratch: of this call alone until its work has run, sqp_mx_gemm_scratch_bytes() for the preferred plan (at most 96 MiB); smaller or NULL:
 * a plan that fits.  No other workspace: calls may overlap with anything. */
size_t sqp_mx_gemm_scratch_bytes(int M, int N, int K, int x_type);
int sqp_mx_gemm(int M, int N, int K, int x_type, int silu_mul, const void *x, const uint8_t *x_scales, const void *w, const uint8_t *w_scales,
                void *y, void *scratch, size_t scratch_bytes, void *stream);

/* The residual's addition and the RMS norm behind it: sum = fp16(x + residual), y = sqp_rmsnorm(sum) (fp32 arithmetic, one
 * rounding at the end).  x, residual, sum, y [M][H] fp16, gamma [H] fp16, H % 8 == 0, 0 <= eps < 1.  sum may be x or residual
 * itself; y may be none of the others. */
int sqp_add_rmsnorm(int M, int H, const void *x, const void *residual, const void *gamma, float eps, void *y, void *sum, void *stream);

/* The same with y quantised per row (type SQP_INT8 or SQP_E4M3) before any rounding to fp16: codes [M][H], scales [M] fp32. */
int sqp_add_rmsnorm_quant(int M, int H, int type, const void *x, const void *residual, const void *gamma, float eps, void *codes,
                          float *scales, void *sum, void *stream);

/* The same with y in blocks of `type` (SQP_E2M1 or SQP_E4M3), H % 32 == 0: codes [M][H/2] or [M][H], scales [M][H/32] bytes.  The codes are
 * those of y in 64-bit arithmetic, rounded once. */
int sqp_add_rmsnorm_mx(int M, int H, int type, const void *x, const void *residual, const void *gamma, float eps, void *codes,
                       uint8_t *scales, void *sum, void *stream);

/* Paged cache of keys and values, D = 64 or 128 values per token and head, `page` tokens per page (a power of two from 16 to 65536):
 *   k_cache, v_cache    [pages][kv_heads][page][D] of `type`; pages * page < 2^31, the tensors may have more elements than that
 *   k_scales, v_scales  [pages][kv_heads][page] fp32 (8-bit types; NULL for SQP_FP16)
 * or blocks of SQP_E2M1: k_cache, v_cache [pages][kv_heads][page][D/2] bytes, k_scales, v_scales [pages][kv_heads][page][D/32] bytes.
 * A slot is a token's place: page number * page + place in the page.  Index arrays (slots, positions, page tables, lengths,
 * starts) are int32 and need 4-byte alignment only.
 *
 * Writes the keys and values of T tokens into their slots; on the way keys, and queries if there are any, are rotated:
 *   y[j] = x[j] c[j] - x[D/2 + j] s[j],  y[D/2 + j] = x[D/2 + j] c[j] + x[j] s[j],  c | s = cos_sin[position], fp32
 * (cos_sin [n_positions][D] fp32: D/2 cosines, D/2 sines; NULL: no rotation; every product and sum rounded for itself), and keys and
 * values are quantised from these fp32 values.  q [T][heads][D], k, v [T][kv_heads][D] fp16 with the given distances between tokens (elements, multiples of 8),
 * q_out [T][heads][D] fp16 (heads == 0: no queries, q and q_out unused).  A token whose slot lies outside the cache (-1, say)
 * is not written; one whose position lies outside the table becomes NaN.  Two tokens in one slot: a mixture of both may end there.
 * T == 0 enqueues nothing. */
int sqp_kv_cache_write(int T, int heads, int kv_heads, int D, int type, int page, int pages, const void *q, long q_stride, const void *k,
                       long k_stride, const void *v, long v_stride, const int *slots, const float *cos_sin, const int *positions,
                       int n_positions, void *k_cache, void *v_cache, void *k_scales, void *v_scales, void *q_out, void *stream);

/* Reads T slots back: k, v [T][kv_heads][D] fp16 = fp16(code * scale); zeros for a slot outside the cache. */
int sqp_kv_cache_read(int T, int kv_heads, int D, int type, int page, int pages, const int *slots, const void *k_cache, const void *v_cache,
                      const void *k_scales, const void *v_scales, void *k, void *v, void *stream);

/* Attention of the newest tokens of B sequences over the paged cache, which holds these tokens' keys and values already:
 *   out[t][h] = sum_j p_j v_j,  p = softmax_j (scale q[t][h] . k_j),  h reading the cached head h / (heads / kv_heads)
 * Sequence b has seq_lens[b] cached tokens, token j in page page_table[b][j / page]; its new tokens are the rows
 * q_starts[b] .. q_starts[b + 1] - 1 of q (q_starts [B + 1], not decreasing; NULL: T == B, one token each).  The i-th of its n
 * new tokens sees the tokens j <= seq_lens[b] - n + i.  A token that sees nothing, all of whose scores are minus infinity, or that
 * belongs to no sequence, gets zeros.
 *   q [T][heads][D] fp16, q_stride elements between tokens; out [T][heads][D] fp16
 *   page_table [B][table_width] int32, table_width * page <= 2^30, table_stride entries between rows; entries past a
 *                   sequence's length may be anything
 *   max_q, max_len  the most new tokens and the greatest length of a sequence, as far as the caller knows: the work is laid
 *                   out by them.  Larger ones in the arrays are computed as well, only slower.  0: not known
 *                   (scratch_bytes: max_len = table_width * page then; max_q = 1 without q_starts).
 *   scratch         of this call alone until its work has run, sqp_paged_attention_scratch_bytes() for the preferred plan;
 *                   smaller or NULL: a plan that fits
 * Scores, softmax and sums are fp32; for the matrix cores a token's weight (p, for 8-bit caches times its value's scale) is rounded to
 * fp16, which is off by up to 2^-11 of it or 2^-35 of the row's largest weight, whichever is more; sequences of at most 16 rows per cached
 * head (new tokens * heads / kv_heads) take it as a sum of two fp16 numbers (2^-22 of it, or 2^-35 of the largest) where max_q makes no
 * more; beside longer ones they are rounded in one way or the other (e2m1 blocks: what a block stands for is rounded to
 * multiples of 2^-24, keys 2^-23, as in an fp16 cache).  What lies past a sequence's length is not used, whatever it holds; nor does a
 * token that sees less depend on the later ones, be they infinite or NaN.  Page numbers outside the cache, lengths past the table and
 * starts past T are taken as the nearest that is inside.  Deterministic.  B <= 65535. */
size_t sqp_paged_attention_scratch_bytes(int T, int B, int heads, int kv_heads, int D, int max_q, int max_len);
int sqp_paged_attention(int T, int B, int heads, int kv_heads, int D, int type, int page, int pages, int table_width, int max_q, int max_len,
                        float scale, const void *q, long q_stride, const void *k_cache, const void *v_cache, const void *k_scales,
                        const void *v_scales, const int *page_table, long table_stride, const int *seq_lens, const int *q_starts, void *out,
                        void *scratch, size_t scratch_bytes, void *stream);

#pragma GCC visibility pop
#ifdef __cplusplus
}
#endif
#endif /* SQP_H */
