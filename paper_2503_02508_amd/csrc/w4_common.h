// Shared by the kernels on 4-bit weights with a scale per group (include/qc_w4.h).
#pragma once
#include <algorithm>

#include "qc_internal.h"
#include "qc_w4.h"

namespace qc {

typedef __bf16 w4_bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 w4_h8 __attribute__((ext_vector_type(8)));
typedef float w4_f8 __attribute__((ext_vector_type(8)));
typedef float w4_f4 __attribute__((ext_vector_type(4)));
typedef int w4_i4 __attribute__((ext_vector_type(4)));
typedef unsigned w4_u4 __attribute__((ext_vector_type(4)));
typedef unsigned w4_u2 __attribute__((ext_vector_type(2)));
// rows of packed codes start at multiples of 8 bytes (K % 16 == 0)
typedef w4_u4 w4_u4_a8 __attribute__((aligned(8)));

struct W4Mat {
  const uint8_t *q;
  const float *scale;
  const uint8_t *zero;   // null: 8 everywhere
  const float *sum;
  const float *bias;     // null: none
};

enum W4Op { W4_LINEAR = 0, W4_GATED = 1, W4_GATED_GRAD = 2 };

struct W4Args {
  const void *x;         // [M, K], rows ldx apart
  int64_t ldx;
  W4Mat w[2];
  int M, N, K, group, G;
  float xs;              // codes: scale and zero point (unsigned minus 128)
  int zp;
  int act;
  void *y, *y2;          // [M, N], rows ldy apart; y2: the second gradient
  int64_t ldy;
  const void *dh;        // gradient of h
  int64_t lddh;
};

struct W4GradArgs {
  const void *dy[2];     // [M, N_i], rows lddy_i apart
  int64_t lddy[2];
  W4Mat w[2];
  int N[2], nw;
  int M, K, group, G;
  void *dx;
  int64_t lddx;
};

// launchers (every argument checked by the host layer)
hipError_t launch_w4_quantize(const void *w, int type, int64_t ld, const qc_w4_weight &out, hipStream_t st);
hipError_t launch_w4_expand(const qc_w4_weight &w, void *out, int type, int64_t ld, hipStream_t st);
hipError_t launch_w4_rows(const W4Args &a, int type, int op, hipStream_t st);
hipError_t launch_w4_grad(const W4GradArgs &a, int type, hipStream_t st);

// ---- element types in memory
template <int TYPE>
struct W4Mem;
template <>
struct W4Mem<QC_TYPE_F32> {
  using T = float;
  static __device__ __forceinline__ float get(T v) { return v; }
  static __device__ __forceinline__ T put(float v) { return v; }
};
template <>
struct W4Mem<QC_TYPE_F16> {
  using T = _Float16;
  static __device__ __forceinline__ float get(T v) { return (float)v; }
  static __device__ __forceinline__ T put(float v) { return (_Float16)v; }
};
template <>
struct W4Mem<QC_TYPE_BF16> {
  using T = __bf16;
  static __device__ __forceinline__ float get(T v) { return (float)v; }
  static __device__ __forceinline__ T put(float v) { return (__bf16)v; }
};
template <>
struct W4Mem<QC_TYPE_I8> : W4Mem<QC_TYPE_F32> {};

// ---- codes.  The nibble at bits 0-3 as a signed number over 16; one instruction (v_cvt_off_f32_i4), exact.  The scales are
// multiplied by 16 to match.
__device__ __forceinline__ float w4_nibble(unsigned w) { return __builtin_amdgcn_cvt_off_f32_i4((int)w); }

// the upper halves of two float32 words: exact for numbers of at most 8 significant bits
__device__ __forceinline__ unsigned w4_pack_bf16(float lo, float hi) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, hi), __builtin_bit_cast(unsigned, lo), 0x07060302u);
}

// ---- activation and derivative of the gated block, in float32
__device__ __forceinline__ float w4_act(int act, float v, float &d) {
  if (act == QC_ACT_SILU) {
    const float e = 1.0f / (1.0f + expf(-v));
    d = e * (1.0f + v * (1.0f - e));
    return v * e;
  }
  // (1 + tanh(y)) / 2 as 1 / (1 + exp(-2 y)), which keeps its digits where it is small; |v| > 30 is 0 or 1 already
  const float c0 = 0.7978845608028654f, c1 = 0.044715f;
  const float b = fminf(fmaxf(v, -30.0f), 30.0f), b2 = b * b;
  const float e = 1.0f / (1.0f + expf(-2.0f * c0 * (b + c1 * b * b2)));
  d = e + 2.0f * c0 * b * (1.0f + 3.0f * c1 * b2) * (e * (1.0f - e));
  return v * e;
}

}  // namespace qc
