/*
 * qc_w4.h - C ABI of the operators on 4-bit weights with a scale per group, for
 * MI355X (gfx950): their quantiser, linear layers from one row to many, the
 * gated half of a feed-forward block, and the gradients of both with respect to
 * their inputs.  The weights of qc_w8a8_linear have one scale per output row;
 * at 4 bits a scale (and a zero point) for every 32, 64 or 128 inputs keeps
 * more of the matrix, and the activations may stay in floating point.
 *
 * A weight matrix W [N, K] stands for
 *   w[n, k] = scale[n, g] (u[n, k] - zero[n, g]),  g = k / group,  u in 0..15
 * zero in 0..15 (unsigned convention, as for activations); zero 8 everywhere is
 * the symmetric case, for which the pointer may be NULL.  The codes are stored
 * as the two's complement nibbles u - 8, packed as in qc.h: element 2j of a row
 * in bits 0-3 of byte j, element 2j+1 in bits 4-7.  The last group of a row may
 * be shorter than the others (K is a multiple of 16, not of the group).
 *
 * Conventions are those of qc.h: QC_OK or a negative qc_status with a text in
 * qc_last_error(); "dev" pointers are device memory owned by the caller;
 * `stream` is a hipStream_t as void*; a call only enqueues work on that stream;
 * argument checks run before any device call.  The calls need no workspace,
 * allocate nothing and keep nothing, so that they may overlap freely and be
 * captured into graphs; the tensors have to lie on the current device.  Results
 * do not depend on anything but the arguments (sums run in a fixed order).
 * Outputs must not overlap inputs.
 *
 * Types of activations and gradients: float32, float16, bfloat16 (QC_TYPE_*);
 * products are summed in float32 and rounded once, to nearest even, at the end.
 * Where a call also takes 8-bit activation codes (QC_TYPE_I8: the paper's
 * unsigned code minus 128, as qc_quantize_act writes them), their real values
 * are x_scale (code + 128 - x_zp), the result is float32, and the products of a
 * group are summed exactly; for the other types x_scale and x_zp are ignored.
 *
 * Rows: a tensor argument has a leading dimension ld in elements, at least its
 * number of columns.  x rows, packed codes and the matrices given to
 * qc_w4_quantize start at multiples of 16 bytes (QC_ERR_ALIGN); results,
 * gradients of results and vectors need only the alignment of their elements.
 * Limits: M below 2^24, N, K and leading dimensions below 2^22, M times a
 * result's columns and N * ceil(K / 32) below 2^31; M = 0 and N = 0 are valid
 * and do nothing (the gradients of N = 0 outputs are zero).
 * Range: products are scaled after a group's are summed, or gradients before
 * they are multiplied.  Inputs of magnitude below 2^120 (the products of a group,
 * 128 of 15/16 of that, then stay in float32), scales below 2^124 and gradients
 * times scales below 2^124 give what the definition gives; beyond, a result may
 * be infinite or NaN where the definition's is not.  Float32 inputs, and in
 * gradients scales and their products, below 2^-110 may lose their last bits.
 * Infinite and NaN inputs reach the results of their row, and no others.
 */
#ifndef QC_W4_H_
#define QC_W4_H_

#include <stddef.h>
#include <stdint.h>
#include "qc.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { QC_TYPE_F32 = 0, QC_TYPE_F16 = 1, QC_TYPE_BF16 = 2, QC_TYPE_I8 = 3 };
enum { QC_ACT_SILU = 0, QC_ACT_GELU = 1 };   /* v / (1 + exp(-v)); the tanh form of GELU, as in the DiT block */

typedef struct qc_w4_weight {
  void *q;          /* dev [N, K/2] packed codes, 16-byte aligned                                   */
  float *scale;     /* dev [N, G], G = ceil(K / group); of magnitude below 2^124                     */
  uint8_t *zero;    /* dev [N, G] zero points 0..15, or NULL: 8 everywhere (symmetric)              */
  float *sum;       /* dev [N] sum over k of w[n, k]; read for QC_TYPE_I8 inputs only, else may be NULL */
  int32_t N, K;     /* K % 16 == 0                                                                  */
  int32_t group;    /* 32, 64 or 128                                                                */
} qc_w4_weight;

/* Quantises a matrix w: dev [N, K] of `type` (float32, float16 or bfloat16; finite, the range h - l too), rows ld apart, into out->q,
 * out->scale, out->zero (unless it is NULL) and out->sum (unless it is NULL).  Per group of a row, in float32:
 *   symmetric (out->zero NULL):  s = max|w| / 7,  u = clip(round(w / s), -7, 7) + 8
 *   with zero points:  l = min(min w, 0), h = max(max w, 0), s = (h - l) / 15, z = clip(round(-l / s), 0, 15),
 *                      u = clip(round(w / s) + z, 0, 15)
 * with IEEE divisions and rounding half to even; a group whose s is 0 gets s = 1.  sum is the float32 rounding of the
 * exact sum of the values the codes stand for (summed in float64). */
int qc_w4_quantize(const void *w, int type, int64_t ld, const qc_w4_weight *out, void *stream);

/* The matrix that a quantised weight stands for: out: dev [N, K] of `type` (float32, float16, bfloat16), rows ld apart. */
int qc_w4_expand(const qc_w4_weight *w, void *out, int type, int64_t ld, void *stream);

/* y[m, n] = sum_k x[m, k] w[n, k] + bias[n].  x: dev [M, K] of `type`, rows ldx apart; bias: dev fp32 [N] or NULL;
 * y: dev [M, N] of the same type (float32 for codes), rows ldy apart. */
int qc_w4_linear(const void *x, int type, int64_t ldx, float x_scale, int x_zp, const qc_w4_weight *w, const float *bias,
                 int M, void *y, int64_t ldy, void *stream);

/* The gated half of a feed-forward block in one kernel:
 *   h[m, n] = act(v[m, n]) u[m, n],  v = x Wgate^T + gate_bias,  u = x Wup^T + up_bias
 * Both weights have the same N, K and group, and both or neither have zero points.  v and u are not rounded in between.
 * The other half is qc_w4_linear on h. */
int qc_w4_gated(const void *x, int type, int64_t ldx, float x_scale, int x_zp, const qc_w4_weight *gate,
                const qc_w4_weight *up, const float *gate_bias, const float *up_bias, int act, int M, void *h,
                int64_t ldh, void *stream);

/* Gradient of a linear layer's input, and of the common input of two layers:
 *   dx[m, k] = sum_n dy[m, n] w[n, k]  (+ sum_n dy2[m, n] w2[n, k], if w2 is not NULL)
 * dy, dy2: dev [M, N] (each of its weight's N) of `type` (float32, float16, bfloat16); dx: dev [M, K] of that type.
 * w and w2 have the same K and group, and both or neither have zero points.  The weights are fixed: no gradient of
 * theirs is formed.  The scales vary along the summed axis and enter the matrix product: for float16 and bfloat16
 * either dy * scale, or scale * (u - zero) (and of float16 dy), is taken to 15 bits or more, whatever the type, for
 * float32 to 24.  For float32 a row of dy that is not finite gives results that are not, infinities or NaN. */
int qc_w4_linear_grad(const void *dy, int type, int64_t lddy, const qc_w4_weight *w, const void *dy2, int64_t lddy2,
                      const qc_w4_weight *w2, int M, void *dx, int64_t lddx, void *stream);

/* Gradients inside the gated block, from the gradient of h (v and u are computed again, nothing else is kept):
 *   dgate[m, n] = dh[m, n] u[m, n] act'(v[m, n]),  dup[m, n] = dh[m, n] act(v[m, n])
 * dh, dgate, dup: dev [M, N] of `type` (float32, float16, bfloat16); dgate and dup have rows ldd apart.  Their column
 * sums are the gradients of the biases; qc_w4_linear_grad(dgate, gate, dup, up) is the gradient of x. */
int qc_w4_gated_grad(const void *x, int type, int64_t ldx, const qc_w4_weight *gate, const qc_w4_weight *up,
                     const float *gate_bias, const float *up_bias, int act, const void *dh, int64_t lddh, int M,
                     void *dgate, void *dup, int64_t ldd, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* QC_W4_H_ */
