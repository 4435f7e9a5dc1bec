// Shared by the kernels of the 8-bit layers with a scale for each token (include/qc_t8.h).
#pragma once
#include "qc_t8.h"
#include "w4_common.h"

namespace qc {

// rows to codes, by what is quantised (t8_rows.hip)
enum T8Source { T8_PLAIN = 0, T8_SILU = 1, T8_GELU = 2, T8_NORM = 3, T8_PLANES = 4 };

struct T8RowArgs {
  const void *x;            // [M, K]; T8_PLANES: the gradients
  int64_t ldx;
  const void *add;          // T8_SILU, T8_GELU: gates; T8_NORM: residual, or null
  int64_t lda;
  const float *w;           // [K]: the norm's weight, or null; T8_PLANES: the scales of the weights' rows
  void *h, *y;              // T8_NORM: the sum with the residual, the normalised rows, or null
  int64_t ldh, ldy;
  int8_t *q;                // T8_PLANES: the planes, rows of `pitch` bytes, and behind `scale` the rows' scales
  int64_t ldq;
  float *scale;
  int M, K;
  float eps;
  double share;             // 1 / K
  int pitch;                // T8_PLANES
};

struct T8NormGradArgs {
  const void *h, *dy, *dh;
  int64_t ldh, lddy, lddh;
  const float *w;
  void *dx;
  int64_t lddx;
  float *dw, *part;         // part: [groups, K]
  int M, K, groups;
  float eps;
  double share;             // 1 / K
  int waves;                // of a row
};

// T8_PLANES: bytes that stand for a gradient, and the rows of the matrix of planes.  Three hold as much of the row's largest number as a float32 product
// does (two left the others of a row with an outlier fewer bits than float16 has: 1 % off beside one of a thousand times their size).
// Row m's plane p (the lowest byte is 0) is row (m / 16 P + p) 16 + m % 16: the 16-row operands of a matrix instruction, a row block's planes one
// behind the other.
constexpr int t8_planes(int type) { return type == QC_TYPE_F32 ? 4 : 3; }
// A row's scale counts its number's high bytes from the third on, so that it is a normal float32 for all rows that are kept (most / 127 2^24 would not be)
constexpr double T8_PLANE_TOP = 127.0 * 65536.0;
__host__ __device__ inline int64_t t8_plane_row(int m, int p, int planes) { return ((int64_t)(m >> 4) * planes + p) * 16 + (m & 15); }

struct T8Product {
  const int8_t *a;          // [rows, lda]: codes, or the planes of gradients
  int64_t lda;
  const int8_t *w;          // [N, K], rows ldw apart
  int64_t ldw;
  const float *xs, *ws, *bias;   // scales of the rows and of the columns (the gradient has none: null)
  int M, N, K;              // rows and columns of the result, length of the summed axis
  int arows;                // rows of `a` (M, or M's blocks of planes)
  void *y;
  int64_t ldy;
  int tm, tn;               // grid of tiles
  int stream;               // whether the result's stores pass the caches
  int split, per;           // parts of the summed axis, slabs of each; their sums
  int32_t *part;
};

constexpr int T8_SLAB = 128;     // the summed axis of the planes is padded to it

hipError_t launch_t8_rows(const T8RowArgs &a, int type, int source, hipStream_t st);
hipError_t launch_t8_expand(const int8_t *q, int64_t ldq, const float *scale, int M, int K, void *out, int type, int64_t ldo, hipStream_t st);
hipError_t launch_t8_gated_grad(const void *x, int64_t ldx, const void *g, int64_t ldg, int act, const void *dv, int64_t lddv, int type, int M, int K,
                                void *dx, int64_t lddx, void *dg, int64_t lddg, hipStream_t st);
int t8_norm_grad_groups(int M, int K);
hipError_t launch_t8_norm_grad(const T8NormGradArgs &a, int type, hipStream_t st);
hipError_t launch_t8_linear(T8Product a, int type, hipStream_t st);
// the forward product by large tiles, and what it takes in us
hipError_t launch_t8_tile(const T8Product &a, int type, hipStream_t st);
float t8_tile_time(int M, int N, int K);
// bytes of the partial sums of a gradient (0: the summed axis is not split)
int64_t t8_grad_part_bytes(int M, int N, int K, int type);
hipError_t launch_t8_grad(T8Product a, int type, hipStream_t st);
// rows of zeros: the gradient of a sum without terms
hipError_t launch_t8_zero(void *x, int type, int M, int K, int64_t ld, hipStream_t st);

// ---- vectors of 16 bytes at any alignment of their elements
typedef w4_u4 t8_u4 __attribute__((aligned(1)));
typedef w4_u2 t8_u2 __attribute__((aligned(1)));
typedef unsigned t8_u1 __attribute__((aligned(1)));

template <int TYPE>
constexpr int t8_vl = TYPE == QC_TYPE_F32 ? 4 : 8;        // elements of such a vector

// Elements e .. of a row of K >= VL, zeros beyond it: the row's last vector is loaded in their place and shifted (a branch that whole vectors do not
// take; element by element it would be many, whose masks fill the scalar registers).
template <int TYPE>
__device__ __forceinline__ w4_u4 t8_raw(const typename W4Mem<TYPE>::T *row, int e, int K) {
  constexpr int VL = t8_vl<TYPE>, BITS = 128 / VL;
  w4_u4 r = {0, 0, 0, 0};
  if (e < K) {
    const int from = min(e, K - VL), by = (e - from) * BITS;
    r = *(const t8_u4 *)((const char *)row + (unsigned)from * (unsigned)sizeof(*row));
    if (by > 0) {
      unsigned long long lo = (unsigned long long)r[1] << 32 | r[0], hi = (unsigned long long)r[3] << 32 | r[2];
      lo = by >= 64 ? hi >> (by - 64) : lo >> by | hi << (64 - by);
      hi = by >= 64 ? 0 : hi >> by;
      r = w4_u4{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
    }
  }
  return r;
}
template <int TYPE>
__device__ __forceinline__ void t8_values(w4_u4 raw, float v[t8_vl<TYPE>]) {
  constexpr int VL = t8_vl<TYPE>;
  typedef typename W4Mem<TYPE>::T vec __attribute__((ext_vector_type(VL)));
  const vec r = __builtin_bit_cast(vec, raw);
#pragma unroll
  for (int i = 0; i < VL; ++i) v[i] = W4Mem<TYPE>::get(r[i]);
}
template <int TYPE>
__device__ __forceinline__ void t8_load(const typename W4Mem<TYPE>::T *row, int e, int K, float v[t8_vl<TYPE>]) {
  t8_values<TYPE>(t8_raw<TYPE>(row, e, K), v);
}
// (Rows stream past the L2 caches: the norm of 16384 x 1152 bfloat16 and the reading of its codes 42.3 -> 36.8 us, gated rows of 16384 x 4608 125 -> 110;
// with the next kernel reading them, 1 - 400 MB in all, from the same time to 9 % less.)
template <int TYPE>
__device__ __forceinline__ void t8_store(typename W4Mem<TYPE>::T *row, int e, int K, const float v[t8_vl<TYPE>]) {
  constexpr int VL = t8_vl<TYPE>;
  using T = typename W4Mem<TYPE>::T;
  typedef T vec __attribute__((ext_vector_type(VL)));
  if (e + VL <= K) {
    vec r;
#pragma unroll
    for (int i = 0; i < VL; ++i) r[i] = W4Mem<TYPE>::put(v[i]);
    __builtin_nontemporal_store(__builtin_bit_cast(w4_u4, r), (t8_u4 *)((char *)row + (unsigned)e * (unsigned)sizeof(T)));
  } else {
#pragma unroll
    for (int i = 0; i < VL; ++i)
      if (e + i < K) row[e + i] = W4Mem<TYPE>::put(v[i]);
  }
}
// the same of a float32 vector, VL elements
template <int VL>
__device__ __forceinline__ void t8_load_f32(const float *w, int e, int K, float v[VL]) {
#pragma unroll
  for (int i = 0; i < VL; ++i) v[i] = 0.0f;
  if (e < K) {
    const int from = min(e, K - VL), over = e - from;
#pragma unroll
    for (int i = 0; i < VL; i += 4) {
      const w4_f4 r = __builtin_bit_cast(w4_f4, (w4_u4) * (const t8_u4 *)((const char *)w + (unsigned)(from + i) * 4u));
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i + j] = r[j];
    }
    if (over > 0) {
#pragma unroll
      for (int by = VL / 2; by; by /= 2)
        if (over & by) {
#pragma unroll
          for (int i = 0; i < VL; ++i) v[i] = i + by < VL ? v[i + by] : 0.0f;
        }
    }
  }
}
// the low bytes of VL words, as bytes e .. of a row
template <int VL>
__device__ __forceinline__ void t8_store_bytes(int8_t *row, int e, int K, const unsigned b[VL]) {
  if (e + VL <= K) {
    unsigned w[VL / 4];
#pragma unroll
    for (int i = 0; i < VL / 4; ++i)
      w[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x0c0c0400u), __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u),
                                   0x05040100u);
    if constexpr (VL == 8) *(t8_u2 *)(row + (unsigned)e) = w4_u2{w[0], w[1]};
    else *(t8_u1 *)(row + (unsigned)e) = w[0];
  } else {
#pragma unroll
    for (int i = 0; i < VL; ++i)
      if (e + i < K) row[e + i] = (int8_t)b[i];
  }
}

// ---- reductions over a wavefront, the same value in every lane
template <int CTRL>
__device__ __forceinline__ unsigned t8_dpp(unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false); }
__device__ __forceinline__ unsigned t8_wave_max(unsigned v) {
  v = max(v, t8_dpp<0xB1>(v));
  v = max(v, t8_dpp<0x4E>(v));
  v = max(v, t8_dpp<0x141>(v));
  v = max(v, t8_dpp<0x140>(v));
  const unsigned a = max((unsigned)__builtin_amdgcn_readlane((int)v, 0), (unsigned)__builtin_amdgcn_readlane((int)v, 16));
  return max(a, max((unsigned)__builtin_amdgcn_readlane((int)v, 32), (unsigned)__builtin_amdgcn_readlane((int)v, 48)));
}
// for what lies in LDS (not __syncthreads(), which would wait for loads that are on their way too)
__device__ __forceinline__ void t8_lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
// the same over the entries of up to 16 wavefronts, in LDS
__device__ __forceinline__ unsigned t8_across_max(const unsigned *u, int waves, int lane) {
  unsigned v = (lane & 15) < waves ? u[lane & 15] : 0u;
  v = max(v, t8_dpp<0xB1>(v));
  v = max(v, t8_dpp<0x4E>(v));
  v = max(v, t8_dpp<0x141>(v));
  v = max(v, t8_dpp<0x140>(v));
  return (unsigned)__builtin_amdgcn_readfirstlane((int)v);
}
__device__ __forceinline__ double t8_across_sum(const double *d, int waves, int lane) {
  double v = (lane & 15) < waves ? d[lane & 15] : 0.0;
  v += dpp_move_d<0xB1>(v);
  v += dpp_move_d<0x4E>(v);
  v += dpp_move_d<0x141>(v);
  v += dpp_move_d<0x140>(v);
  return readlane_d(v, 0);
}
// the larger of two magnitudes, a NaN if either is one
__device__ __forceinline__ float t8_larger(float a, float b) { return __builtin_elementwise_maximum(fabsf(a), fabsf(b)); }
// |v| as a word: ordered as the magnitudes are, infinities above them and NaN above those
__device__ __forceinline__ unsigned t8_mag(float v) { return __builtin_bit_cast(unsigned, v) & 0x7FFFFFFFu; }

// 1 / sqrt(v) in float64 and its float32 rounding: the hardware's estimate and two Newton steps (v is normal and positive;
// infinite and NaN sums give 0 or NaN, whose rows are NaN either way)
__device__ __forceinline__ double t8_rsqrt(double v) {
  double y = __builtin_amdgcn_rsq(v);
#pragma unroll
  for (int i = 0; i < 2; ++i) y = __builtin_fma(y * 0.5, __builtin_fma(-v * y, y, 1.0), y);
  return y;
}

// ---- the gated block's activations
// exact to float64: v times a logistic function, v / (1 + exp(-t)); (1 + tanh(y)) / 2 is the logistic function of 2 y
__device__ __forceinline__ double t8_gate_exact(int act, float gate, float x) {
  const double g = gate, t = act == QC_ACT_SILU ? g : g * (1.5957691216057307117 + 1.5957691216057307117 * 0.044715 * g * g);
  return g / (1.0 + exp(-t)) * (double)x;
}
// float32: `s` the logistic function, `o` one minus it.  The exponent's argument is taken in float64 and handed on as two float32
// numbers, so that the error does not grow with it: off by at most 9 e (e = 2^-24) of the value while that is above 2^-100; below,
// s 2^100 (o 2^100) is returned in its place and `deep` is set.
__device__ __forceinline__ void t8_logistic(int act, float gate, float &s, float &o, bool &deep) {
  const double g = gate;
  double u = act == QC_ACT_SILU ? g * 1.4426950408889634 : g * (2.302208198144325 + 0.1029432395800235 * (g * g));
  u = fmin(fmax(u, -400.0), 400.0);                       // 2^-400 is 0 to any product below; a NaN comes back through `gate`
  const double a = fabs(u);
  const float hi = (float)a, lo = (float)(a - (double)hi);
  deep = hi > 100.0f;
  const float e = __builtin_amdgcn_exp2f(deep ? 100.0f - hi : -hi);
  const float z = __builtin_fmaf(e, lo * -0.6931471805599453f, e);
  const float r = deep ? 1.0f : __builtin_amdgcn_rcpf(1.0f + z);
  s = u < 0.0 ? z * r : r;
  o = u < 0.0 ? r : z * r;
}
// act(gate) x by the same formula without the cases, for gates above T8_DEEP: to 1.8e-6 of its value.  The logistic function is
// 1 / (1 + exp(-t)), which keeps the digits of small values; above LIMIT it is 1, below -LIMIT it is what it is there: too large, so that products of gates
// below T8_DEEP are not to be used.  An infinite or NaN gate gives an infinite or NaN product.
template <int ACT>
__device__ __forceinline__ float t8_gate(float gate, float x) {
  constexpr float LIMIT = ACT == QC_ACT_SILU ? 85.0f : 9.9f;             // exp(-t) up to 2^123
  const float b = __builtin_amdgcn_fmed3f(gate, -LIMIT, LIMIT);
  float hi, lo;                                          // -t = hi log(2) + lo
  if constexpr (ACT == QC_ACT_SILU) {
    hi = b * -1.4426950408889634f;
    lo = -__builtin_fmaf(hi, 0.6931471805599453f, b);
  } else {
    const double g = b, u = g * (-2.302208198144325 - 0.1029432395800235 * (g * g));
    hi = (float)u;
    lo = (float)(u - (double)hi) * 0.6931471805599453f;
  }
  const float e = __builtin_amdgcn_exp2f(hi);
  // (the gate last: a subnormal one times the logistic function would have lost its digits when a large x brings it back.  A subnormal x meets a
  // logistic function below 1 only where the gate, and with it the product, is small.)
  return __builtin_amdgcn_rcpf(1.0f + __builtin_fmaf(e, lo, e)) * x * gate;
}
template <int ACT>
constexpr float T8_DEEP = ACT == QC_ACT_SILU ? -69.0f : -9.0f;       // exp(-t) = 2^100, about
template <int ACT>
constexpr float T8_GONE = ACT == QC_ACT_SILU ? -400.0f : -20.0f;     // the product is below any float32, for finite x

// Value and derivative of the activation, for gates of a magnitude below T8_FAR (2^-100, about): t8_logistic without what lies beyond.  The products with
// log2(e) are float32 with what they lose (SiLU; of GELU's third power float64 is as short).
template <int ACT>
constexpr float T8_FAR = ACT == QC_ACT_SILU ? 69.0f : 9.0f;
template <int ACT>
__device__ __forceinline__ float t8_act_near(float gate, float &d) {
  float hi, lo;
  if constexpr (ACT == QC_ACT_SILU) {
    const float a = fabsf(gate);
    hi = a * -0x1.715476p+0f;
    lo = __builtin_fmaf(a, 0x1.4ae0cp-26f, __builtin_fmaf(a, 0x1.715476p+0f, hi));
  } else {
    const double g = fabsf(gate), u = g * (2.302208198144325 + 0.1029432395800235 * (g * g));
    hi = -(float)u;
    lo = (float)(u + (double)hi);
  }
  const float e = __builtin_amdgcn_exp2f(hi), z = __builtin_fmaf(e, lo * -0.6931471805599453f, e), r = __builtin_amdgcn_rcpf(1.0f + z);
  const float s = gate < 0.0f ? z * r : r, o = gate < 0.0f ? r : z * r;
  if constexpr (ACT == QC_ACT_SILU) d = __builtin_fmaf(gate * o, s, s);
  else d = __builtin_fmaf(gate * (1.5957691216057308f * (1.0f + 0.134145f * (gate * gate))) * o, s, s);
  return gate * s;
}

// of any gate
__device__ __forceinline__ float t8_act(int act, float gate, float &d) {
  float s, o;
  bool deep;
  t8_logistic(act, gate, s, o, deep);
  const bool low = deep && gate < 0.0f;                   // s is 2^100 times what it stands for; else o, which is nothing beside 1
  if (deep && !low) o *= 0x1p-100f;
  if (act == QC_ACT_SILU) {
    d = __builtin_fmaf(gate * o, s, s);
  } else {
    const float b = fabsf(gate) > 30.0f ? copysignf(30.0f, gate) : gate;      // beyond, s o is 0 (the comparison leaves NaN as it is)
    d = __builtin_fmaf(b * (1.5957691216057308f * (1.0f + 0.134145f * (b * b))) * o, s, s);
  }
  const float v = gate * s;
  d = low ? d * 0x1p-100f : d;
  return low ? v * 0x1p-100f : v;
}

}  // namespace qc
