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
// rows of gradients start at any element
typedef w4_u4 w4_u4_a4 __attribute__((aligned(4)));
typedef w4_u4 w4_u4_a2 __attribute__((aligned(2)));

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
// many rows: whether it pays, and the launch
bool w4_tile_pays(const W4Args &a, int type, int op);
int w4_tile_rows(const W4Args &a, int type);
hipError_t launch_w4_tile(const W4Args &a, int type, int op, hipStream_t st);
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
// all 8 of a word: the instruction reads any byte of a register, so that the odd ones cost one shift for all four
__device__ __forceinline__ void w4_nibbles(unsigned w, float v[8]) {
  unsigned odd = w >> 4;
  asm("" : "+v"(odd));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = w4_nibble((w >> (8 * i)) & 0xFF);
    v[2 * i + 1] = w4_nibble((odd >> (8 * i)) & 0xFF);
  }
}

// the upper halves of two float32 words: exact for numbers of at most 8 significant bits
__device__ __forceinline__ unsigned w4_pack_bf16(float lo, float hi) {
  return __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, hi), __builtin_bit_cast(unsigned, lo), 0x07060302u);
}

// One type's operands of a product of 16 x 32 by 32 x 16: lane l holds 8 inputs 8 (l / 16) .. of row (column) l % 16, the result's
// column l % 16 and rows 4 (l / 16) ..
template <int TYPE>
struct Frag;

template <>
struct Frag<QC_TYPE_BF16> {
  using X = w4_bf8;
  using W = w4_bf8;
  using Acc = w4_f4;
  template <bool ASYM>
  static __device__ __forceinline__ W weights(unsigned w, float z16, unsigned) {
    float v[8];
    w4_nibbles(w, v);
    w4_u4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = ASYM ? w4_pack_bf16(v[2 * i] - z16, v[2 * i + 1] - z16) : w4_pack_bf16(v[2 * i], v[2 * i + 1]);
    return __builtin_bit_cast(W, r);
  }
  static __device__ __forceinline__ Acc mma(X x, W w, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, w, c, 0, 0, 0); }
};

template <>
struct Frag<QC_TYPE_F16> {
  using X = w4_h8;
  using W = w4_h8;
  using Acc = w4_f4;
  template <bool ASYM>
  static __device__ __forceinline__ W weights(unsigned w, float z16, unsigned) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const _Float16 z = (_Float16)z16;
    float v[8];
    w4_nibbles(w, v);
    w4_u4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h2 p = __builtin_bit_cast(h2, __builtin_amdgcn_cvt_pkrtz(v[2 * i], v[2 * i + 1]));
      if (ASYM) p -= h2{z, z};
      r[i] = __builtin_bit_cast(unsigned, p);
    }
    return __builtin_bit_cast(W, r);
  }
  static __device__ __forceinline__ Acc mma(X x, W w, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w, c, 0, 0, 0); }
};

template <>
struct Frag<QC_TYPE_I8> {
  using X = w4_u2;
  using W = w4_u2;
  using Acc = w4_i4;
  // u - z in bytes: (u + 128) - z never borrows from its neighbour
  template <bool ASYM>
  static __device__ __forceinline__ W weights(unsigned w, float, unsigned zb) {
    if (!ASYM) zb = 0x08080808u;
    const unsigned even = (((w & 0x0F0F0F0Fu) ^ 0x88888888u) - zb) ^ 0x80808080u;
    const unsigned odd = ((((w >> 4) & 0x0F0F0F0Fu) ^ 0x88888888u) - zb) ^ 0x80808080u;
    W r;
    r[0] = __builtin_amdgcn_perm(odd, even, 0x05010400u);
    r[1] = __builtin_amdgcn_perm(odd, even, 0x07030602u);
    return r;
  }
  static __device__ __forceinline__ Acc mma(X x, W w, Acc c) {
    return __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, x), __builtin_bit_cast(long, w), c, 0, 0, 0);
  }
};

// words of four lanes 16 apart: word j of row i of the wavefront (16 lanes) changes places with word i of row j
__device__ __forceinline__ void w4_transpose(w4_u4 &v) {
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  u2 a = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
  u2 b = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
  u2 c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
  u2 d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  v[0] = c[0];
  v[1] = c[1];
  v[2] = d[0];
  v[3] = d[1];
}

// the first half of it: words 0 and 1 of the upper 32 lanes change places with words 2 and 3 of the lower
__device__ __forceinline__ void w4_swap32(w4_u4 &v) {
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  const u2 a = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false);
  const u2 b = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
  v = w4_u4{a[0], b[0], a[1], b[1]};
}

// float32 as three bfloat16 numbers whose sum it is exactly: truncation leaves 8 bits of the 24 each time.  What does not
// change when its upper half is taken away (infinities) leaves nothing.
template <bool FINITE = false>
__device__ __forceinline__ void w4_split(float v, float p[3]) {
  const float h = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, v) & 0xFFFF0000u);
  const float r = !FINITE && h == v ? 0.0f : v - h;
  const float m = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, r) & 0xFFFF0000u);
  p[0] = h;
  p[1] = m;
  p[2] = r - m;
}

// The matrix products' operands of float32 activations: bfloat16, three products for one
template <int TYPE>
using FragOf = Frag<TYPE == QC_TYPE_F32 ? QC_TYPE_BF16 : TYPE>;

// position of a launch's workgroup: the workgroups of one XCD (every eighth) take neighbouring tiles, groups of GM tile rows column by column
__device__ __forceinline__ void tile_at(int id, int total, int tm, int tn, int GM, int &mi, int &ni) {
  const int x = id & 7, q = total >> 3, r = total & 7;
  int t = x * q + min(x, r) + (id >> 3);
  const int per = GM * tn, g = t / per, rows = min(GM, tm - g * GM);
  t -= g * per;
  mi = g * GM + t % rows;
  ni = t / rows;
}

// ---- Loads through a buffer descriptor: `bytes` from p on; what lies beyond reads as zero, without a branch.  Offsets are 32 bits, so p is
// the first byte of a workgroup's own rows.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t w4_buffer(const void *p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)min(max(bytes, (int64_t)0), (int64_t)0x7FFFFFFF), 0x00027000);
}
constexpr unsigned W4_NOWHERE = 0x80000000u;      // an offset beyond every buffer

// ---- A wavefront's 16 weight rows, 64 bytes of each.  Sixteen neighbouring lanes are looked up together, a cache line a clock: loads
// therefore give 4 neighbouring lanes one row's 64 bytes (4 lines for 16 lanes, not 16), and lanes then fetch what is theirs
// from each other: lane l holds piece l / 16 of row l % 16 afterwards.
__device__ __forceinline__ unsigned w4_pull(unsigned v, int from4) { return (unsigned)__builtin_amdgcn_ds_bpermute(from4, (int)v); }
__device__ __forceinline__ int w4_from(int lane) { return ((lane & 15) * 4 + (lane >> 4)) * 4; }

// ---- activation and derivative of the gated block, in float32.  Both are v times a logistic function, 1 / (1 + exp(-t)), from the
// hardware's exponential and reciprocal: off by a few units in the last place, and exp2's argument by |t| of them.
__device__ __forceinline__ float w4_logistic(float t) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t * -1.4426950408889634f)); }
__device__ __forceinline__ float w4_act(int act, float v, float &d) {
  if (act == QC_ACT_SILU) {
    const float e = w4_logistic(v);
    d = e * (1.0f + v * (1.0f - e));
    return v * e;
  }
  // (1 + tanh(y)) / 2 = logistic(2 y), which keeps its digits where it is small; |v| > 30 is 0 or 1 already.  The
  // comparison leaves NaN as it is (minimum and maximum would not).
  const float c0 = 1.5957691216057308f, c1 = 0.044715f;
  const float b = fabsf(v) > 30.0f ? copysignf(30.0f, v) : v, b2 = b * b;
  const float e = w4_logistic(c0 * b * (1.0f + c1 * b2));
  d = e + c0 * b * (1.0f + 3.0f * c1 * b2) * (e * (1.0f - e));
  return v * e;
}

}  // namespace qc
