// Host layer of include/qc_t8.h: argument checks, then the launches.  Every check runs before the first device call.
#include <cmath>

#include "t8_common.h"

using namespace qc;

#define QC_FAIL(code, ...)      \
  do {                          \
    qc::set_error(__VA_ARGS__); \
    return (code);              \
  } while (0)

#define QC_HIP(expr)                                                                          \
  do {                                                                                        \
    hipError_t e_ = (expr);                                                                   \
    if (e_ != hipSuccess) QC_FAIL(QC_ERR_HIP, "%s: %s", #expr, hipGetErrorString(e_));        \
  } while (0)

#define QC_TRY(expr)      \
  do {                    \
    const int rc_ = (expr); \
    if (rc_) return rc_;  \
  } while (0)

namespace {

constexpr int LIMIT_M = 1 << 24, LIMIT_N = 1 << 17, LIMIT_LD = 1 << 22;

int bytes_of(int type) { return type == QC_TYPE_F32 ? 4 : type == QC_TYPE_I8 ? 1 : 2; }
bool off_by(const void *p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes != 0; }

int check_type(int type) {
  if (type == QC_TYPE_F32 || type == QC_TYPE_F16 || type == QC_TYPE_BF16) return QC_OK;
  QC_FAIL(QC_ERR_UNSUPPORTED, "type %d is not one of this call's", type);
}

int check_shape(int M, int K) {
  if (M < 0 || M >= LIMIT_M) QC_FAIL(QC_ERR_SHAPE, "M (%d) out of range", M);
  if (K < 1 || K >= LIMIT_N) QC_FAIL(QC_ERR_SHAPE, "K (%d) out of range", K);
  return QC_OK;
}

int check_product(int M, int N, int K) {
  QC_TRY(check_shape(M, K));
  if (N < 0 || N >= LIMIT_N) QC_FAIL(QC_ERR_SHAPE, "N (%d) out of range", N);
  if (K % 16) QC_FAIL(QC_ERR_SHAPE, "K (%d) must be a multiple of 16", K);
  return QC_OK;
}

// a matrix of `cols` columns whose rows start at multiples of `align` bytes; one without elements may lie nowhere
int check_rows(const void *p, const char *name, int64_t ld, int64_t rows, int64_t cols, int type, int align) {
  if (rows == 0 || cols == 0) return QC_OK;
  if (!p) QC_FAIL(QC_ERR_NULL, "%s is NULL", name);
  if (rows > 1 && (ld < cols || ld >= LIMIT_LD)) QC_FAIL(QC_ERR_SHAPE, "%s: leading dimension %lld of %lld columns", name, (long long)ld, (long long)cols);
  if (off_by(p, align) || (rows > 1 && ld * bytes_of(type) % align)) QC_FAIL(QC_ERR_ALIGN, "%s: rows must start at multiples of %d bytes", name, align);
  return QC_OK;
}
int check_rows(const void *p, const char *name, int64_t ld, int64_t rows, int64_t cols, int type) {
  return check_rows(p, name, ld, rows, cols, type, bytes_of(type));
}

int check_vector(const void *p, const char *name, bool needed) {
  if (needed && !p) QC_FAIL(QC_ERR_NULL, "%s is NULL", name);
  if (off_by(p, 4)) QC_FAIL(QC_ERR_ALIGN, "%s must be aligned to its elements", name);
  return QC_OK;
}

int check_eps(float eps) {
  if (!(eps > 0.0f) || !std::isfinite(eps)) QC_FAIL(QC_ERR_RANGE, "eps must be positive and finite");
  return QC_OK;
}

int check_act(int act) {
  if (act != QC_ACT_SILU && act != QC_ACT_GELU) QC_FAIL(QC_ERR_UNSUPPORTED, "unknown activation %d", act);
  return QC_OK;
}

int check_work(const void *work, size_t bytes, size_t needed, int align) {
  if (needed && !work) QC_FAIL(QC_ERR_NULL, "work is NULL");
  if (off_by(work, align)) QC_FAIL(QC_ERR_ALIGN, "work must be %d-byte aligned", align);
  if (bytes < needed) QC_FAIL(QC_ERR_WORKSPACE, "workspace too small: %zu bytes given, %zu needed", bytes, needed);
  return QC_OK;
}

// the one row of a matrix has no leading dimension to speak of
int64_t row_step(int64_t ld, int M, int64_t cols) { return M > 1 ? ld : cols; }

// workspace of qc_t8_linear_grad: planes, row scales, partial sums, each from a multiple of 256 bytes on
struct GradWork {
  int64_t pitch, scale, part, total;
};
int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }
GradWork grad_work(int M, int N, int K, int type) {
  GradWork w{};
  const int P = t8_planes(type);
  w.pitch = ((int64_t)N + T8_SLAB - 1) / T8_SLAB * T8_SLAB;
  w.scale = up256(((int64_t)M + 15) / 16 * 16 * P * w.pitch);
  w.part = up256(w.scale + (int64_t)M * 4);
  w.total = w.part + (M && N ? t8_grad_part_bytes(M, N, K, type) : 0);
  return w;
}
int check_grad(int M, int N, int K, int type) {
  QC_TRY(check_product(M, N, K));
  QC_TRY(check_type(type));
  return QC_OK;
}
size_t norm_grad_work(int M, int K) { return (size_t)t8_norm_grad_groups(M, K) * (size_t)K * 4; }

}  // namespace

extern "C" {

int qc_t8_norm(const void *x, int64_t ldx, const void *residual, int64_t ldr, const float *weight, float eps, int type, int M, int K, void *h, int64_t ldh,
               void *y, int64_t ldy, int8_t *q, int64_t ldq, float *scale, void *stream) {
  QC_TRY(check_shape(M, K));
  QC_TRY(check_type(type));
  QC_TRY(check_eps(eps));
  if (!residual != !h) QC_FAIL(QC_ERR_NULL, "residual and h belong together");
  if (!q != !scale) QC_FAIL(QC_ERR_NULL, "q and scale belong together");
  if (M && !q && !y) QC_FAIL(QC_ERR_NULL, "q and y are both NULL");
  QC_TRY(check_rows(x, "x", ldx, M, K, type));
  if (residual) {
    QC_TRY(check_rows(residual, "residual", ldr, M, K, type));
    QC_TRY(check_rows(h, "h", ldh, M, K, type));
  }
  if (y) QC_TRY(check_rows(y, "y", ldy, M, K, type));
  if (q) QC_TRY(check_rows(q, "q", ldq, M, K, QC_TYPE_I8));
  QC_TRY(check_vector(weight, "weight", false));
  QC_TRY(check_vector(scale, "scale", false));
  if (M == 0) return QC_OK;
  T8RowArgs a{};
  a.x = x; a.ldx = row_step(ldx, M, K);
  a.add = residual; a.lda = row_step(ldr, M, K);
  a.w = weight; a.eps = eps; a.share = 1.0 / K;
  a.h = h; a.ldh = row_step(ldh, M, K);
  a.y = y; a.ldy = row_step(ldy, M, K);
  a.q = q; a.ldq = row_step(ldq, M, K);
  a.scale = scale;
  a.M = M; a.K = K;
  QC_HIP(launch_t8_rows(a, type, T8_NORM, static_cast<hipStream_t>(stream)));
  return QC_OK;
}

int qc_t8_norm_grad_bytes(int M, int K, size_t *bytes_out) {
  if (!bytes_out) QC_FAIL(QC_ERR_NULL, "bytes_out is NULL");
  QC_TRY(check_shape(M, K));
  *bytes_out = norm_grad_work(M, K);
  return QC_OK;
}

int qc_t8_norm_grad(const void *h, int64_t ldh, const float *weight, float eps, const void *dy, int64_t lddy, const void *dh, int64_t lddh, int type, int M,
                    int K, void *dx, int64_t lddx, float *dweight, void *work, size_t work_bytes, void *stream) {
  QC_TRY(check_shape(M, K));
  QC_TRY(check_type(type));
  QC_TRY(check_eps(eps));
  QC_TRY(check_rows(h, "h", ldh, M, K, type));
  QC_TRY(check_rows(dy, "dy", lddy, M, K, type));
  if (dh) QC_TRY(check_rows(dh, "dh", lddh, M, K, type));
  QC_TRY(check_rows(dx, "dx", lddx, M, K, type));
  QC_TRY(check_vector(weight, "weight", false));
  QC_TRY(check_vector(dweight, "dweight", false));
  if (dweight) QC_TRY(check_work(work, work_bytes, norm_grad_work(M, K), 16));
  if (M == 0 && !dweight) return QC_OK;
  T8NormGradArgs a{};
  a.h = h; a.ldh = row_step(ldh, M, K);
  a.dy = dy; a.lddy = row_step(lddy, M, K);
  a.dh = dh; a.lddh = row_step(lddh, M, K);
  a.dx = dx; a.lddx = row_step(lddx, M, K);
  a.w = weight; a.eps = eps; a.share = 1.0 / K;
  a.dw = dweight; a.part = static_cast<float *>(work);
  a.M = M; a.K = K;
  QC_HIP(launch_t8_norm_grad(a, type, static_cast<hipStream_t>(stream)));
  return QC_OK;
}

int qc_t8_quantize(const void *x, int64_t ldx, const void *gate, int64_t ldg, int act, int type, int M, int K, int8_t *q, int64_t ldq, float *scale,
                   void *stream) {
  QC_TRY(check_shape(M, K));
  QC_TRY(check_type(type));
  if (gate) QC_TRY(check_act(act));
  QC_TRY(check_rows(x, "x", ldx, M, K, type));
  if (gate) QC_TRY(check_rows(gate, "gate", ldg, M, K, type));
  QC_TRY(check_rows(q, "q", ldq, M, K, QC_TYPE_I8));
  QC_TRY(check_vector(scale, "scale", M > 0));
  if (M == 0) return QC_OK;
  T8RowArgs a{};
  a.x = x; a.ldx = row_step(ldx, M, K);
  a.add = gate; a.lda = row_step(ldg, M, K);
  a.q = q; a.ldq = row_step(ldq, M, K);
  a.scale = scale;
  a.M = M; a.K = K;
  QC_HIP(launch_t8_rows(a, type, gate ? (act == QC_ACT_SILU ? T8_SILU : T8_GELU) : T8_PLAIN, static_cast<hipStream_t>(stream)));
  return QC_OK;
}

int qc_t8_expand(const int8_t *q, int64_t ldq, const float *scale, int M, int K, void *out, int type, int64_t ldo, void *stream) {
  QC_TRY(check_shape(M, K));
  QC_TRY(check_type(type));
  QC_TRY(check_rows(q, "q", ldq, M, K, QC_TYPE_I8));
  QC_TRY(check_rows(out, "out", ldo, M, K, type));
  QC_TRY(check_vector(scale, "scale", M > 0));
  if (M == 0) return QC_OK;
  QC_HIP(launch_t8_expand(q, row_step(ldq, M, K), scale, M, K, out, type, row_step(ldo, M, K), static_cast<hipStream_t>(stream)));
  return QC_OK;
}

int qc_t8_gated_grad(const void *x, int64_t ldx, const void *gate, int64_t ldg, int act, const void *dv, int64_t lddv, int type, int M, int K, void *dx,
                     int64_t lddx, void *dgate, int64_t lddg, void *stream) {
  QC_TRY(check_shape(M, K));
  QC_TRY(check_type(type));
  QC_TRY(check_act(act));
  QC_TRY(check_rows(x, "x", ldx, M, K, type));
  QC_TRY(check_rows(gate, "gate", ldg, M, K, type));
  QC_TRY(check_rows(dv, "dv", lddv, M, K, type));
  QC_TRY(check_rows(dx, "dx", lddx, M, K, type));
  QC_TRY(check_rows(dgate, "dgate", lddg, M, K, type));
  if (M == 0) return QC_OK;
  QC_HIP(launch_t8_gated_grad(x, row_step(ldx, M, K), gate, row_step(ldg, M, K), act, dv, row_step(lddv, M, K), type, M, K, dx, row_step(lddx, M, K), dgate,
                              row_step(lddg, M, K), static_cast<hipStream_t>(stream)));
  return QC_OK;
}

int qc_t8_linear(const int8_t *qx, int64_t ldx, const float *x_scale, const int8_t *qw, int64_t ldw, const float *w_scale, const float *bias, int M, int N,
                 int K, void *y, int type, int64_t ldy, void *stream) {
  QC_TRY(check_product(M, N, K));
  QC_TRY(check_type(type));
  QC_TRY(check_rows(qx, "qx", ldx, M, K, QC_TYPE_I8, 16));
  QC_TRY(check_rows(qw, "qw", ldw, N, K, QC_TYPE_I8, 16));
  QC_TRY(check_rows(y, "y", ldy, M, N, type));
  QC_TRY(check_vector(x_scale, "x_scale", M > 0));
  QC_TRY(check_vector(w_scale, "w_scale", N > 0));
  QC_TRY(check_vector(bias, "bias", false));
  if (M == 0 || N == 0) return QC_OK;
  T8Product a{};
  a.a = qx; a.lda = row_step(ldx, M, K); a.xs = x_scale;
  a.w = qw; a.ldw = row_step(ldw, N, K); a.ws = w_scale; a.bias = bias;
  a.M = M; a.N = N; a.K = K;
  a.y = y; a.ldy = row_step(ldy, M, N);
  QC_HIP(launch_t8_linear(a, type, static_cast<hipStream_t>(stream)));
  return QC_OK;
}

int qc_t8_linear_grad_bytes(int M, int N, int K, int type, size_t *bytes_out) {
  if (!bytes_out) QC_FAIL(QC_ERR_NULL, "bytes_out is NULL");
  QC_TRY(check_grad(M, N, K, type));
  *bytes_out = (size_t)grad_work(M, N, K, type).total;
  return QC_OK;
}

int qc_t8_linear_grad(const void *dy, int64_t lddy, int type, const int8_t *qw, int64_t ldw, const float *w_scale, int M, int N, int K, void *dx, int64_t lddx,
                      void *work, size_t work_bytes, void *stream) {
  QC_TRY(check_grad(M, N, K, type));
  QC_TRY(check_rows(dy, "dy", lddy, M, N, type));
  QC_TRY(check_rows(qw, "qw", ldw, N, K, QC_TYPE_I8, 16));
  QC_TRY(check_rows(dx, "dx", lddx, M, K, type));
  QC_TRY(check_vector(w_scale, "w_scale", N > 0));
  const GradWork w = grad_work(M, N, K, type);
  QC_TRY(check_work(work, work_bytes, (size_t)w.total, 256));
  if (M == 0) return QC_OK;
  char *base = static_cast<char *>(work);
  hipStream_t st = static_cast<hipStream_t>(stream);
  T8RowArgs r{};
  r.x = dy; r.ldx = row_step(lddy, M, N);
  r.w = w_scale;
  r.q = (int8_t *)base; r.scale = (float *)(base + w.scale);
  r.M = M; r.K = N; r.pitch = (int)w.pitch;
  T8Product a{};
  a.a = r.q; a.lda = w.pitch; a.xs = r.scale;
  a.w = qw; a.ldw = row_step(ldw, N, K);
  a.M = M; a.N = N; a.K = K;
  a.y = dx; a.ldy = row_step(lddx, M, K);
  a.part = (int32_t *)(base + w.part);
  if (N == 0) {
    QC_HIP(launch_t8_zero(dx, type, M, K, a.ldy, st));
    return QC_OK;
  }
  QC_HIP(launch_t8_rows(r, type, T8_PLANES, st));
  QC_HIP(launch_t8_grad(a, type, st));
  return QC_OK;
}

}  // extern "C"
