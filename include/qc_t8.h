/*
 * qc_t8.h - C ABI of the 8-bit layers with a scale for each token, for MI355X
 * (gfx950): root-mean-square norm and row quantiser that make the codes, the
 * linear layer that reads them, and the gradients of all three.  The
 * activations of qc_w8a8_linear have one scale and zero point that calibration
 * fixes beforehand; here every row (token) brings its own, found from the row
 * itself, and codes are symmetric, so that there is no zero point.
 *
 * Rows of codes: v[m, k] is stood for by scale[m] q[m, k], q in -127..127,
 *   scale = max_k |v| / 127        (an IEEE float32 division; 1 where it is 0)
 *   q     = clip(round(v / scale), -127, 127)   (float32 division, half to even)
 * v being float32.  A row that holds an infinity or a NaN gets the scale NaN
 * and codes 0, so that everything made from it is NaN, and no other row is.
 * Weights [N, K] are rows of codes too (one scale per output channel): the same
 * call quantises them, and qc_quantize_weight gives the same codes and scales.
 *
 * Conventions are those of qc.h: QC_OK or a negative qc_status with a text in
 * qc_last_error(); "dev" pointers are device memory owned by the caller;
 * `stream` is a hipStream_t as void*; a call only enqueues work on that stream;
 * argument checks run before any device call.  The calls allocate nothing and
 * keep nothing, so that they may overlap freely and be captured into graphs;
 * calls that take a workspace use it until their work has ended, and two that
 * may run at the same time need one each.  The tensors have to lie on the
 * current device.  Results do not depend on anything but the arguments (sums
 * run in a fixed order).  Outputs must not overlap inputs or each other, but
 * where a call says that one may be the other.
 *
 * Types of activations and gradients: float32, float16, bfloat16 (QC_TYPE_* of
 * qc_w4.h), one type for all of a call's.  Results are computed in float32 or
 * more and rounded once, to nearest even.
 *
 * Rows: a tensor argument has a leading dimension ld in elements, at least its
 * number of columns (any value where there is at most one row).  Rows need only
 * the alignment of their elements, but for the codes that the products read:
 * those start at multiples of 16 bytes (QC_ERR_ALIGN), and K % 16 == 0 there.
 * Vectors (scales, weights of norms, biases) are float32.
 * Limits: M below 2^24, N and K from 1 (N from 0) and below 2^17, leading
 * dimensions below 2^22.
 * M = 0 and N = 0 are valid: nothing is written but the gradients of a sum
 * without terms, which are zero.
 */
#ifndef QC_T8_H_
#define QC_T8_H_

#include <stddef.h>
#include <stdint.h>
#include "qc.h"
#include "qc_w4.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Root-mean-square norm of rows, with the addition of a residual stream in front and the row quantiser behind it:
 *   h = x + residual                                   (rounded to the type; h = x if residual is NULL)
 *   y = (h rho) weight,  rho = 1 / sqrt(sum_k h^2 / K + eps)
 * rho is the float32 rounding of the float64 expression; h rho and y are float32 products.  h is normalised as it is
 * stored: what the next layer adds to and what qc_t8_norm_grad reads.
 * x, residual, h, y: dev [M, K] of `type`; weight: dev [K] or NULL (ones); eps > 0.  residual and h belong together (both or
 * neither); h may be x or residual itself (the same pointer and leading dimension).  q, scale: the codes of y, dev int8
 * [M, K] and dev [M], both or neither; y: y in the type, or NULL; q or y has to be there. */
int qc_t8_norm(const void *x, int64_t ldx, const void *residual, int64_t ldr, const float *weight, float eps, int type, int M,
               int K, void *h, int64_t ldh, void *y, int64_t ldy, int8_t *q, int64_t ldq, float *scale, void *stream);

/* Gradient of qc_t8_norm, from dy, the gradient of y (rounding to codes is passed through: its gradient is taken to be 1),
 * and dh, the gradient that reaches h by other ways (the residual stream), or NULL:
 *   dx[m, k] = rho (g - h rho^2 sum_j g h / K) + dh,  g = dy weight          (the gradient of x and of the residual)
 *   dweight[k] = sum_m dy h rho                                              (NULL: not wanted)
 * h: dev [M, K], the input of the norm (h of the forward call, or x); dy, dh, dx: dev [M, K] of the same type; dx may be
 * dy or dh itself.  dweight: dev [K], written.  work: dev, at least qc_t8_norm_grad_bytes, 16-byte aligned; read only if
 * dweight is not NULL. */
int qc_t8_norm_grad_bytes(int M, int K, size_t *bytes_out);
int qc_t8_norm_grad(const void *h, int64_t ldh, const float *weight, float eps, const void *dy, int64_t lddy, const void *dh,
                    int64_t lddh, int type, int M, int K, void *dx, int64_t lddx, float *dweight, void *work,
                    size_t work_bytes, void *stream);

/* Rows to codes: v = x, or v = act(gate) x where gate is not NULL (the gated half of a feed-forward block, whose product is
 * never stored): the float32 rounding of the exact value (of magnitude below 2^127, or an infinity).
 * x, gate: dev [M, K] of `type`; act: QC_ACT_SILU or QC_ACT_GELU; q: dev int8 [M, K]; scale: dev [M]. */
int qc_t8_quantize(const void *x, int64_t ldx, const void *gate, int64_t ldg, int act, int type, int M, int K, int8_t *q,
                   int64_t ldq, float *scale, void *stream);

/* What rows of codes stand for: out = scale q.  out: dev [M, K] of `type`. */
int qc_t8_expand(const int8_t *q, int64_t ldq, const float *scale, int M, int K, void *out, int type, int64_t ldo,
                 void *stream);

/* Gradient of v = act(gate) x, from dv (rounding to codes passed through):
 *   dx = dv act(gate),  dgate = (dv x) act'(gate)
 * (dv x is a float32 product; where it is beyond float32 so is dgate, or NaN.)
 * All dev [M, K] of `type`; dx and dgate may each be x, gate or dv itself, but not each other. */
int qc_t8_gated_grad(const void *x, int64_t ldx, const void *gate, int64_t ldg, int act, const void *dv, int64_t lddv, int type,
                     int M, int K, void *dx, int64_t lddx, void *dgate, int64_t lddg, void *stream);

/* y[m, n] = x_scale[m] w_scale[n] sum_k qx[m, k] qw[n, k] + bias[n]
 * The sum is exact (32-bit integers; any bytes, -128 among them); the rest is float32: (float(sum) w_scale) x_scale + bias.
 * qx: dev int8 [M, K], rows ldx apart; qw: dev int8 [N, K], rows ldw apart; both start at multiples of 16 bytes, K % 16 == 0.
 * bias: dev [N] or NULL; y: dev [M, N] of `type`. */
int qc_t8_linear(const int8_t *qx, int64_t ldx, const float *x_scale, const int8_t *qw, int64_t ldw, const float *w_scale,
                 const float *bias, int M, int N, int K, void *y, int type, int64_t ldy, void *stream);

/* Gradient of its input (of v, the row that the codes stand for); the weights are fixed:
 *   dx[m, k] = sum_n dy[m, n] w_scale[n] qw[n, k]
 * The scales vary along the summed axis, so that dy w_scale enters the product: the float32 product, as a fixed-point number of
 * 24 bits (float16, bfloat16) or 32 bits (float32) of the row's largest |dy w_scale|, whose bytes meet the weights' in exact
 * integer sums.  The rounding of one term is thus at most 2^-23.9 (2^-31.9) of the largest in its row, whatever its own size:
 * beside an outlier a thousand times its size a term keeps 14 (22) bits.  A row of dy w_scale that is not finite gives NaN; one
 * with nothing of 2^-100 or above may be taken for zeros.
 * dy: dev [M, N] of `type`; qw: as above; dx: dev [M, K] of `type`.  work: dev, at least qc_t8_linear_grad_bytes, 256-byte
 * aligned. */
int qc_t8_linear_grad_bytes(int M, int N, int K, int type, size_t *bytes_out);
int qc_t8_linear_grad(const void *dy, int64_t lddy, int type, const int8_t *qw, int64_t ldw, const float *w_scale, int M, int N,
                      int K, void *dx, int64_t lddx, void *work, size_t work_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* QC_T8_H_ */
