// Host layer of include/qc_w4.h: argument checks, then one launch.  Every check runs before the first device call.
#include <cmath>

#include "w4_common.h"

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

constexpr int LIMIT_M = 1 << 24, LIMIT = 1 << 22;     // rows; features and leading dimensions (32-bit offsets inside 128 rows)

int bytes_of(int type) { return type == QC_TYPE_F32 ? 4 : type == QC_TYPE_I8 ? 1 : 2; }
bool off_by(const void *p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes != 0; }

int check_type(int type, bool codes) {
  if (type == QC_TYPE_F32 || type == QC_TYPE_F16 || type == QC_TYPE_BF16 || (codes && type == QC_TYPE_I8)) return QC_OK;
  QC_FAIL(QC_ERR_UNSUPPORTED, "type %d is not one of this call's", type);
}

int check_weight(const qc_w4_weight *w, const char *name) {
  if (!w || (w->N > 0 && (!w->q || !w->scale))) QC_FAIL(QC_ERR_NULL, "%s, its codes or its scales are NULL", name);
  if (w->N < 0 || w->K < 1 || w->N >= LIMIT || w->K >= LIMIT) QC_FAIL(QC_ERR_SHAPE, "%s: N (%d) or K (%d) out of range", name, w->N, w->K);
  if (w->K % 16) QC_FAIL(QC_ERR_SHAPE, "%s: K (%d) must be a multiple of 16", name, w->K);
  if (w->group != 32 && w->group != 64 && w->group != 128) QC_FAIL(QC_ERR_UNSUPPORTED, "%s: group (%d) must be 32, 64 or 128", name, w->group);
  if ((int64_t)w->N * ((w->K + 31) / 32) >= (1ll << 31)) QC_FAIL(QC_ERR_UNSUPPORTED, "%s: %d x %d is too large", name, w->N, w->K);
  if (off_by(w->q, 16)) QC_FAIL(QC_ERR_ALIGN, "%s: the codes must be 16-byte aligned", name);
  if (off_by(w->scale, 4) || off_by(w->sum, 4)) QC_FAIL(QC_ERR_ALIGN, "%s: scales and sums must be aligned to their elements", name);
  return QC_OK;
}

// two weights of one call; one without rows has no zero points to have or not (its pointers may be NULL)
int check_pair(const qc_w4_weight *a, const qc_w4_weight *b, bool rows) {
  if (a->K != b->K || a->group != b->group || (rows && a->N != b->N))
    QC_FAIL(QC_ERR_SHAPE, "the weights differ: %d x %d in groups of %d, %d x %d in groups of %d", a->N, a->K, a->group, b->N, b->K, b->group);
  if (a->N && b->N && !a->zero != !b->zero) QC_FAIL(QC_ERR_UNSUPPORTED, "one of the weights has zero points, the other has none");
  return QC_OK;
}

// a matrix of `cols` columns whose rows start at multiples of `align` bytes; one without elements may lie nowhere
int check_rows(const void *p, const char *name, int64_t ld, int64_t rows, int64_t cols, int type, int align) {
  if (rows == 0 || cols == 0) return QC_OK;
  if (!p) QC_FAIL(QC_ERR_NULL, "%s is NULL", name);
  if (ld < cols || ld >= LIMIT) QC_FAIL(QC_ERR_SHAPE, "%s: leading dimension %lld of %lld columns", name, (long long)ld, (long long)cols);
  if (off_by(p, align) || ld * bytes_of(type) % align) QC_FAIL(QC_ERR_ALIGN, "%s: rows must start at multiples of %d bytes", name, align);
  return QC_OK;
}

int check_rows_of_call(int M, int64_t cols) {
  if (M < 0 || M >= LIMIT_M) QC_FAIL(QC_ERR_SHAPE, "M (%d) out of range", M);
  if (M * cols >= (1ll << 31)) QC_FAIL(QC_ERR_UNSUPPORTED, "a result of %d x %lld is too large", M, (long long)cols);
  return QC_OK;
}

int check_codes(int type, float x_scale, int x_zp, const qc_w4_weight *w) {
  if (type != QC_TYPE_I8) return QC_OK;
  if (!(x_scale > 0.0f) || !std::isfinite(x_scale)) QC_FAIL(QC_ERR_RANGE, "scale must be positive and finite");
  if (x_zp < 0 || x_zp > 255) QC_FAIL(QC_ERR_RANGE, "zero point %d outside 0..255", x_zp);
  if (w->N && !w->sum) QC_FAIL(QC_ERR_NULL, "8-bit inputs need the weight's row sums");
  return QC_OK;
}

int check_bias(const float *b) {
  if (off_by(b, 4)) QC_FAIL(QC_ERR_ALIGN, "a bias must be aligned to its elements");
  return QC_OK;
}

W4Mat mat(const qc_w4_weight *w, const float *bias) { return W4Mat{(const uint8_t *)w->q, w->scale, w->zero, w->sum, bias}; }

W4Args args(const void *x, int type, int64_t ldx, float x_scale, int x_zp, const qc_w4_weight *w, const float *bias, int M, void *y, int64_t ldy) {
  W4Args a{};
  a.x = x; a.ldx = ldx;
  a.w[0] = a.w[1] = mat(w, bias);
  a.M = M; a.N = w->N; a.K = w->K; a.group = w->group; a.G = (w->K + w->group - 1) / w->group;
  a.xs = x_scale; a.zp = x_zp - 128;
  a.y = y; a.ldy = ldy;
  return a;
}

hipError_t launch(const W4Args &a, int type, int op, void *stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  return w4_tile_pays(a, type, op) ? launch_w4_tile(a, type, op, st) : launch_w4_rows(a, type, op, st);
}

int result_type(int type) { return type == QC_TYPE_I8 ? QC_TYPE_F32 : type; }

}  // namespace

extern "C" {

int qc_w4_quantize(const void *w, int type, int64_t ld, const qc_w4_weight *out, void *stream) {
  QC_TRY(check_weight(out, "out"));
  QC_TRY(check_type(type, false));
  QC_TRY(check_rows(w, "w", ld, out->N, out->K, type, 16));
  if (out->N == 0) return QC_OK;
  QC_HIP(launch_w4_quantize(w, type, ld, *out, static_cast<hipStream_t>(stream)));
  return QC_OK;
}

int qc_w4_expand(const qc_w4_weight *w, void *out, int type, int64_t ld, void *stream) {
  QC_TRY(check_weight(w, "w"));
  QC_TRY(check_type(type, false));
  QC_TRY(check_rows(out, "out", ld, w->N, w->K, type, bytes_of(type)));
  if (w->N == 0) return QC_OK;
  QC_HIP(launch_w4_expand(*w, out, type, ld, static_cast<hipStream_t>(stream)));
  return QC_OK;
}

int qc_w4_linear(const void *x, int type, int64_t ldx, float x_scale, int x_zp, const qc_w4_weight *w, const float *bias, int M, void *y,
                 int64_t ldy, void *stream) {
  QC_TRY(check_weight(w, "w"));
  QC_TRY(check_type(type, true));
  QC_TRY(check_rows_of_call(M, w->N));
  QC_TRY(check_codes(type, x_scale, x_zp, w));
  QC_TRY(check_rows(x, "x", ldx, M, w->K, type, 16));
  QC_TRY(check_rows(y, "y", ldy, M, w->N, result_type(type), bytes_of(result_type(type))));
  QC_TRY(check_bias(bias));
  if (M == 0 || w->N == 0) return QC_OK;
  QC_HIP(launch(args(x, type, ldx, x_scale, x_zp, w, bias, M, y, ldy), type, W4_LINEAR, stream));
  return QC_OK;
}

int qc_w4_gated(const void *x, int type, int64_t ldx, float x_scale, int x_zp, const qc_w4_weight *gate, const qc_w4_weight *up,
                const float *gate_bias, const float *up_bias, int act, int M, void *h, int64_t ldh, void *stream) {
  QC_TRY(check_weight(gate, "gate"));
  QC_TRY(check_weight(up, "up"));
  QC_TRY(check_pair(gate, up, true));
  QC_TRY(check_type(type, true));
  if (act != QC_ACT_SILU && act != QC_ACT_GELU) QC_FAIL(QC_ERR_UNSUPPORTED, "unknown activation %d", act);
  QC_TRY(check_rows_of_call(M, gate->N));
  QC_TRY(check_codes(type, x_scale, x_zp, gate));
  QC_TRY(check_codes(type, x_scale, x_zp, up));
  QC_TRY(check_rows(x, "x", ldx, M, gate->K, type, 16));
  QC_TRY(check_rows(h, "h", ldh, M, gate->N, result_type(type), bytes_of(result_type(type))));
  QC_TRY(check_bias(gate_bias));
  QC_TRY(check_bias(up_bias));
  if (M == 0 || gate->N == 0) return QC_OK;
  W4Args a = args(x, type, ldx, x_scale, x_zp, gate, gate_bias, M, h, ldh);
  a.w[1] = mat(up, up_bias);
  a.act = act;
  QC_HIP(launch(a, type, W4_GATED, stream));
  return QC_OK;
}

int qc_w4_linear_grad(const void *dy, int type, int64_t lddy, const qc_w4_weight *w, const void *dy2, int64_t lddy2, const qc_w4_weight *w2, int M,
                      void *dx, int64_t lddx, void *stream) {
  QC_TRY(check_weight(w, "w"));
  QC_TRY(check_type(type, false));
  QC_TRY(check_rows_of_call(M, w->K));
  QC_TRY(check_rows(dy, "dy", lddy, M, w->N, type, bytes_of(type)));
  if (w2) {
    QC_TRY(check_weight(w2, "w2"));
    QC_TRY(check_pair(w, w2, false));
    QC_TRY(check_rows(dy2, "dy2", lddy2, M, w2->N, type, bytes_of(type)));
  }
  QC_TRY(check_rows(dx, "dx", lddx, M, w->K, type, bytes_of(type)));
  if (M == 0) return QC_OK;
  W4GradArgs a{};
  a.dy[0] = dy; a.lddy[0] = lddy; a.w[0] = mat(w, nullptr); a.N[0] = w->N; a.nw = 1;
  if (w2) {
    a.dy[1] = dy2; a.lddy[1] = lddy2; a.w[1] = mat(w2, nullptr); a.N[1] = w2->N; a.nw = 2;
  }
  a.M = M; a.K = w->K; a.group = w->group; a.G = (w->K + w->group - 1) / w->group;
  a.dx = dx; a.lddx = lddx;
  QC_HIP(launch_w4_grad(a, type, static_cast<hipStream_t>(stream)));
  return QC_OK;
}

int qc_w4_gated_grad(const void *x, int type, int64_t ldx, const qc_w4_weight *gate, const qc_w4_weight *up, const float *gate_bias,
                     const float *up_bias, int act, const void *dh, int64_t lddh, int M, void *dgate, void *dup, int64_t ldd, void *stream) {
  QC_TRY(check_weight(gate, "gate"));
  QC_TRY(check_weight(up, "up"));
  QC_TRY(check_pair(gate, up, true));
  QC_TRY(check_type(type, false));
  if (act != QC_ACT_SILU && act != QC_ACT_GELU) QC_FAIL(QC_ERR_UNSUPPORTED, "unknown activation %d", act);
  QC_TRY(check_rows_of_call(M, gate->N));
  QC_TRY(check_rows(x, "x", ldx, M, gate->K, type, 16));
  QC_TRY(check_rows(dh, "dh", lddh, M, gate->N, type, bytes_of(type)));
  QC_TRY(check_rows(dgate, "dgate", ldd, M, gate->N, type, bytes_of(type)));
  QC_TRY(check_rows(dup, "dup", ldd, M, gate->N, type, bytes_of(type)));
  QC_TRY(check_bias(gate_bias));
  QC_TRY(check_bias(up_bias));
  if (M == 0 || gate->N == 0) return QC_OK;
  W4Args a = args(x, type, ldx, 1.0f, 128, gate, gate_bias, M, dgate, ldd);
  a.w[1] = mat(up, up_bias);
  a.act = act;
  a.dh = dh; a.lddh = lddh; a.y2 = dup;
  QC_HIP(launch(a, type, W4_GATED_GRAD, stream));
  return QC_OK;
}

}  // extern "C"
