/*
 * dhq_groups.h - operators on linear layers that are stored by groups of consecutive inputs: products with 4-bit
 * weights, and activations kept in 8 bits for the backward pass.
 *
 * A row of K values is cut into groups of G = 32, 64 or 128 consecutive ones; the last group is padded with zeros to
 * Kp = ceil(K / G) G.  With rotation = DHQ_ROT_INPUT every group is transformed on its own by the Walsh-Hadamard
 * matrix H_G (Eq. 3 of the paper, block by block: a distribution with a few outliers becomes close to normal before it
 * meets the quantizer); DHQ_ROT_NONE leaves it out; DHQ_ROT_BOTH is UNSUPPORTED here.  The fp32 rotation adds in the
 * order of dhq.h: in-place butterfly, strides 1, 2, 4, ..., G/2, (i, i+h) -> (a+b, a-b).
 *
 * Conventions are those of dhq.h: device pointers, `stream` a cudaStream_t, argument errors by return value with nothing
 * enqueued.  The calls have no handle.  They enqueue kernels only - no allocation, no synchronisation, no state kept
 * between calls - so they may be recorded into a CUDA graph, and calls on different streams or devices do not meet.
 * Every pointer belongs to the device that is current in the call.  Matrices are row-major with a leading dimension in
 * elements (ld >= columns) and need the alignment of their element type; `codes` needs 16 bytes, 4-bit scales need 2.
 * Inputs and outputs do not overlap except where a call says so.  Rows and columns of an output behind the stated sizes are not
 * touched.  Sizes: columns (N, K) 1 .. 2^24, rows (T) 0 .. 2^31 - 1; offsets are 64 bits wide.
 * Errors of every call: INVALID_ARG (NULL or misaligned pointer, size or leading dimension out of range, unknown type),
 * UNSUPPORTED (group, rotation or activation not named here), CUDA.
 */
#ifndef DHQ_GROUPS_H_
#define DHQ_GROUPS_H_

#include "dhq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of inputs and results.  Sums are held in fp32 whatever the type. */
typedef enum { DHQ_F32 = 0, DHQ_BF16 = 1, DHQ_F16 = 2 } dhq_dtype_t;

/*
 * Weight side, once per matrix (Eq. 4 by groups, and the quantizer of Section III-B with a scale per group):
 *     v = W, or W H_G / G group by group (fp32 butterfly, exact power of two)
 *     s = bf16(max |v| / 7), q = clamp(round_half_even(fl32(v * fl32(1 / s))), +-7);  s = 0 or 1 / s infinite: s = q = 0
 * A group with a value that is not finite gets the scale NaN: every product of that row is NaN.
 *   W       [N][K] of `dtype`, leading dimension ldw.
 *   codes   [N][Kp / 2] bytes.  Eight consecutive codes k0..k7 make a 32-bit little-endian word whose nibbles, from the lowest,
 *           hold k0, k2, k4, k6, k1, k3, k5, k7, each as q + 8: a word shifted by 4 i and masked with 0x000f000f is
 *           the pair (k_2i, k_2i+1), as 16-bit arithmetic on pairs wants it.
 *   scales  [N][Kp / G] bf16.
 */
DHQ_API dhq_status_t dhq_w4_pack(const void *W, dhq_dtype_t dtype, int64_t N, int64_t K, int64_t ldw, int group,
                                 dhq_rot_t rotation, uint8_t *codes, uint16_t *scales, void *stream);

/*
 * Products of few rows with 4-bit weights: out[t][n] = sum_g s[n][g] sum_{k in g} q[n][k] x~[t][k] + bias[n], with x~ = x
 * or, for weights that were packed with DHQ_ROT_INPUT, x~ = H_G x by groups.  Any T is taken;
 * the codes are read once for every 64 columns (rows times terms, see below).
 * Accuracy: products are summed in fp32 on the tensor cores, with one multiply by the scale per group and one rounding to the type
 * of `out`.  x~ goes there as fp16 numbers times a power of two per row and group: 16-bit x as one, exactly (below 2^-28 of its
 * group's largest value it may lose bits), rotated bf16 x as one (off by 2^-11 of a value at most; the result is rounded by up to 2^-8), fp32 and
 * rotated fp16 x as two terms (2^-23).  With 16-bit x a group's sum is formed as sum (q + 8) x~ - 8 sum x~: what fp32 rounds is relative
 * to the larger one of these, which costs up to 5 of its 24 bits where x~ has one sign.  A row of x with values that are not finite has no finite results
 * (with 16-bit x they may all be NaN); other rows are not touched by it.  Range: 16-bit x wants scales below 2^103 and magnitudes of x~ from 2^-126 on,
 * fp32 x 7 G max |x~| below 2^128 (sums of codes times values are taken before the scale).
 *   x     [T][K] of `dtype`, leading dimension ldx.     bias  [N] of `dtype`, or NULL.
 *   out   [T][N] of `dtype`, leading dimension ldout.
 *   workspace  device, `workspace_bytes` of at least what dhq_w4_linear_workspace says, 16-byte aligned; NULL where that is 0
 *              (few rows that are not very long).  Used until the call's work on `stream` is done: calls that may run at the same time need one each.
 * Errors: also ALLOC if the workspace is too small.
 */
DHQ_API dhq_status_t dhq_w4_linear_workspace(int64_t T, int64_t N, int64_t K, int group, dhq_rot_t rotation, dhq_dtype_t dtype, int64_t *bytes);
DHQ_API dhq_status_t dhq_w4_linear(const uint8_t *codes, const uint16_t *scales, int64_t N, int64_t K, int group,
                                   dhq_rot_t rotation, const void *x, dhq_dtype_t dtype, int64_t T, int64_t ldx,
                                   const void *bias, void *out, int64_t ldout, void *workspace, int64_t workspace_bytes,
                                   void *stream);

/*
 * What the backward pass keeps of x in place of x: 8-bit codes and a power of two per group, and beside it the layer's
 * activation, in one pass over x.
 *     v = x, or H_G x by groups;   e = the least integer with max |v| <= 127 2^e, at least -126
 *     q = round_half_even(v 2^-e);   x^ = q 2^e, or H_G (q 2^e) / G
 * Powers of two cost up to one of the 8 bits against max |v| / 127; in return q 2^e is exact in 16-bit types, so that the
 * products of dhq_checkpoint_weight_grad round nothing of it.  1 + 1/G bytes per value.
 *   x           [T][K] of `dtype`, leading dimension ldx.
 *   activation  DHQ_ACT_NONE (x is the input of a linear layer: no y), DHQ_ACT_SINE sin(omega0 x), DHQ_ACT_GABOR
 *               sin(omega0 x) exp(-(act_s0 x)^2), DHQ_ACT_SILU x / (1 + exp(-x)), DHQ_ACT_GELU x Phi(x) (Phi the normal
 *               distribution's, not the approximation with tanh).
 *               omega0 and act_s0 (finite; act_s0 > 0 for the wavelet) are ignored by the others.
 *               Accuracy of fp32 results, before the rounding to `dtype`: 2^-19 for the sine and the wavelet, with phases below 2^22 turns (beyond, sines
 *               of some phase; NaN where |omega0 x| / 2 pi is more than fp32 holds), 2^-19 |x| for the others.  These are bounds; root mean squares are 1.1e-7,
 *               and 6e-8 for silu and 1e-7 for gelu of x with a standard deviation of 2.
 *   codes       [T][Kp] int8.    exponents  [T][Kp / G] bytes: e + 127; 0 a group of zeros; 255, over codes of 0, a
 *               group with a value that is not finite (or whose rotation is not), which comes back as NaN.
 *               Both NULL: nothing is kept, as where no backward pass follows (not for DHQ_ACT_NONE); y has the same bits.
 *   y           [T][K] of `dtype`, leading dimension ldy; NULL for DHQ_ACT_NONE.  y may be x itself (same ldy).
 */
DHQ_API dhq_status_t dhq_checkpoint_save(const void *x, dhq_dtype_t dtype, int64_t T, int64_t K, int64_t ldx, int group,
                                         dhq_rot_t rotation, dhq_act_t activation, float omega0, float act_s0,
                                         int8_t *codes, uint8_t *exponents, void *y, int64_t ldy, void *stream);

/*
 * Backward pass of that activation from the checkpoint: dx = dy act'(x^).  DHQ_ACT_NONE is UNSUPPORTED (dx = dy).
 * Accuracy of act'(x^): 2^-19 of omega0 for the sine (phases as above), of omega0 + 2 act_s0 for the wavelet (NaN where 2 act_s0^2 x^ is more than fp32 holds), of 2 for
 * the others.
 *   dy, dx  [T][K] of `dtype`, leading dimensions lddy, lddx.  dx may be dy itself (same leading dimension).
 */
DHQ_API dhq_status_t dhq_checkpoint_act_grad(const int8_t *codes, const uint8_t *exponents, int64_t T, int64_t K, int group,
                                             dhq_rot_t rotation, dhq_act_t activation, float omega0, float act_s0,
                                             const void *dy, dhq_dtype_t dtype, int64_t lddy, void *dx, int64_t lddx, void *stream);

/*
 * Weight gradient of a linear layer y = x W^T (+ b) whose input x was kept as a checkpoint: dW = dy^T x^, the sum over the
 * T rows.  T = 0 writes zeros.  (A wait inside the kernel for copies or products of its own that lasts two seconds, which no sound GPU has, ends that block with NaN
 * in its part of dW; the call has returned OK by then.)  Every sum is taken in the same order in every call with the same sizes and types.
 *   dy         [T][N] of `dtype`, leading dimension lddy.
 *   dW         [N][K] of `dw_dtype` (DHQ_F32, or the type of dy), leading dimension lddw; overwritten.
 *   workspace  device, `workspace_bytes` of at least what dhq_checkpoint_weight_grad_workspace says for the same
 *              arguments, 16-byte aligned; NULL if that is 0.  (It holds parts of the sums, and a copy of 16-bit dy whose rows are not
 *              aligned to 16 bytes.)  Used until the call's work on `stream` is done: calls that may
 *              run at the same time need one each.
 * fp16 dy: the q 2^e of a group are fp16 numbers times a power of two, which is one for the rows that a block sums and such that the largest is
 * finite (1 while magnitudes before the quantizer stay within 65,024, and then nothing of q 2^e is rounded; else what lies 2^39 below the largest is, and the block takes twice the time).
 * Accuracy: products are exact and summed on the tensor cores, which cut off what does not fit an fp32 sum.  fp32 results take the sums of at most
 * 1,024 rows (512 of fp16 dy) from there and add these in fp32; for 16-bit results up to 65,536 rows of bf16 or 16,384 of fp16 stay there, by which a
 * sum of one sign is too small by some 5e-5 of itself (measured).  Range: |q 2^e| below 2^127; sums of dy times rotated values are taken before H_G / G.
 * Errors: also ALLOC if the workspace is too small, UNSUPPORTED for sizes that make more blocks than a launch has (far beyond any memory).
 */
DHQ_API dhq_status_t dhq_checkpoint_weight_grad_workspace(int64_t T, int64_t N, int64_t K, int group, dhq_rot_t rotation,
                                                          dhq_dtype_t dtype, const void *dy, int64_t lddy,
                                                          dhq_dtype_t dw_dtype, int64_t *bytes);
DHQ_API dhq_status_t dhq_checkpoint_weight_grad(const int8_t *codes, const uint8_t *exponents, int64_t T, int64_t K, int group,
                                                dhq_rot_t rotation, const void *dy, dhq_dtype_t dtype, int64_t N, int64_t lddy,
                                                void *dW, dhq_dtype_t dw_dtype, int64_t lddw, void *workspace,
                                                int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DHQ_GROUPS_H_ */
