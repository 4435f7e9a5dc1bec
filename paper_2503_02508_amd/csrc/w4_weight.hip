// 4-bit weights with a scale per group: the quantiser, and the matrix that its codes stand for.
//
// Both move memory only: the quantiser reads a matrix once and writes an eighth (float32) or a quarter of its bytes, the
// expansion does the reverse.  A workgroup takes a row, a lane 8 neighbouring values (a group of 32, 64 or 128 lies in 4, 8 or
// 16 neighbouring lanes and is reduced without LDS).  16-bit matrices leave the quantiser between its bytes and its arithmetic: 8192 x 8192
// bfloat16 take 52 us (3.3 TB/s), of which 22 vector instructions a value need 37 to issue and the bytes 33; float32 59 us (5.2 TB/s, what a large copy reaches); with eight IEEE divisions a lane and reductions
// through LDS they took 65 and 70.  The expansion: 35 us (4.9 TB/s) and 67 us (4.5 TB/s).
#include "w4_common.h"

namespace qc {

template <int TYPE>
using W4Eight = typename W4Mem<TYPE>::T __attribute__((ext_vector_type(8)));

// a value of the other lanes of a group, by data-parallel primitives: the neighbour, the pair beside, the quad beside, the eight beside
template <int CTRL>
__device__ __forceinline__ float w4_beside(float v) {
  const int b = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, CTRL, 0xF, 0xF, false));
}
// minimum / maximum over 4, 8 or 16 neighbouring lanes, in each of them
template <bool MAX>
__device__ __forceinline__ float w4_group_reduce(float v, int lanes) {
  const auto with = [&](float o) { v = MAX ? fmaxf(v, o) : fminf(v, o); };
  with(w4_beside<0xB1>(v));      // quad_perm [1, 0, 3, 2]
  with(w4_beside<0x4E>(v));      // quad_perm [2, 3, 0, 1]
  if (lanes > 4) with(w4_beside<0x141>(v));      // row_half_mirror
  if (lanes > 8) with(w4_beside<0x140>(v));      // row_mirror
  return v;
}

template <int TYPE>
__global__ __launch_bounds__(256) void w4_quantize_kernel(const typename W4Mem<TYPE>::T *w, int64_t ld, int K, int group, int shift, int G, uint8_t *q,
                                                          float *scale, uint8_t *zero, float *sum) {
  __shared__ double part[4];
  const size_t n = blockIdx.x;
  const int lanes = group / 8, KR = (K + 127) / 128 * 128;       // whole groups, so that all lanes of one take part
  double total = 0.0;
  W4Eight<TYPE> next = {};
  if ((int)threadIdx.x * 8 < K) next = *(const W4Eight<TYPE> *)(w + n * ld + threadIdx.x * 8);
  for (int k = threadIdx.x * 8; k < KR; k += blockDim.x * 8) {
    const bool in = k < K;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = in ? W4Mem<TYPE>::get(next[i]) : 0.0f;
    const int kn = k + blockDim.x * 8;
    if (kn < K) next = *(const W4Eight<TYPE> *)(w + n * ld + kn);
    float lo = fminf(v[0], 0.0f), hi = fmaxf(v[0], 0.0f);
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      lo = fminf(lo, v[i]);
      hi = fmaxf(hi, v[i]);
    }
    lo = w4_group_reduce<false>(lo, lanes);
    hi = w4_group_reduce<true>(hi, lanes);
    // w / s by way of 1 / s, off by less than 4e-6 for |w / s| <= 15.5: only next to a half (or where 1 / s is infinite) does it take
    // the division to decide
    float s = zero ? (hi - lo) / 15.0f : fmaxf(hi, -lo) / 7.0f;
    if (s == 0.0f) s = 1.0f;
    const float inv = __builtin_amdgcn_rcpf(s);
    float r[8], z = 8.0f, off = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = v[i] * inv;
      r[i] = rintf(t);
      off = fmaxf(off, fabsf(t - r[i]));
    }
    if (zero) {
      const float t = -lo * inv;
      z = rintf(t);
      off = fmaxf(off, fabsf(t - z));
    }
    if (off > 0.49999f || !(inv < 3.0e38f)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = rintf(v[i] / s);
      if (zero) z = rintf(-lo / s);
    }
    z = fminf(fmaxf(z, 0.0f), 15.0f);
    const float low = (zero ? 0.0f : 1.0f) - z, high = 15.0f - z;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = __builtin_amdgcn_fmed3f(r[i], low, high);
    // four codes as one number below 65536, exact in float32; their sum is at most 60
    const auto four = [&](const float *c) { return (unsigned)fmaf(fmaf(fmaf(c[3], 16.0f, c[2]), 16.0f, c[1]), 16.0f, fmaf(z, 4369.0f, c[0])); };
    const unsigned code = (four(r) | four(r + 4) << 16) ^ 0x88888888u;   // u - 8 in two's complement
    if (in) {
      *(unsigned *)(q + n * (K / 2) + k / 2) = code;
      if ((k & (group - 1)) == 0) {
        const size_t at = n * G + (k >> shift);
        scale[at] = s;
        if (zero) zero[at] = (uint8_t)z;
      }
      const float isum = ((r[0] + r[1]) + (r[2] + r[3])) + ((r[4] + r[5]) + (r[6] + r[7]));
      total += (double)s * (double)isum;
    }
  }
  if (!sum) return;
  total = wave_sum_dpp(total);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = total;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (unsigned i = 1; i < blockDim.x / 64; ++i) total += part[i];
    sum[n] = (float)total;
  }
}

// VEC: rows of the result start at multiples of 16 bytes, which is what a lane stores
template <int TYPE, bool VEC>
__global__ __launch_bounds__(256) void w4_expand_kernel(const uint8_t *q, const float *scale, const uint8_t *zero, int K, int shift, int G,
                                                        typename W4Mem<TYPE>::T *out, int64_t ld) {
  using T = typename W4Mem<TYPE>::T;
  constexpr int E = 16 / sizeof(T);
  typedef T TE __attribute__((ext_vector_type(E)));
  typedef typename std::conditional<E == 8, unsigned, unsigned short>::type Code;
  const size_t n = blockIdx.x;
  for (int k = threadIdx.x * E; k < K; k += blockDim.x * E) {
    const unsigned code = *(const Code *)(q + n * (K / 2) + k / 2);
    const size_t g = n * G + (k >> shift);
    const float s = scale[g];
    const int z = zero ? (int)zero[g] - 8 : 0;
    TE t;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      float v = s * (float)(((int)(code << (28 - 4 * i)) >> 28) - z);
      asm("" : "+v"(v));          // rounded to float32, then to the type: not a product that is rounded to float16 directly
      t[i] = W4Mem<TYPE>::put(v);
    }
    T *o = out + n * ld + k;
    if (VEC) {
      *(TE *)o = t;
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) o[i] = t[i];
    }
  }
}

static int row_threads(int K) { return std::min(256, ((K + 127) / 128 * 16 + 63) / 64 * 64); }

template <int TYPE>
static void quantize(const void *w, int64_t ld, const qc_w4_weight &o, hipStream_t st) {
  const int G = (o.K + o.group - 1) / o.group;
  w4_quantize_kernel<TYPE><<<o.N, row_threads(o.K), 0, st>>>((const typename W4Mem<TYPE>::T *)w, ld, o.K, o.group, __builtin_ctz(o.group), G, (uint8_t *)o.q, o.scale,
                                                            o.zero, o.sum);
}

hipError_t launch_w4_quantize(const void *w, int type, int64_t ld, const qc_w4_weight &o, hipStream_t st) {
  if (type == QC_TYPE_F32) quantize<QC_TYPE_F32>(w, ld, o, st);
  else if (type == QC_TYPE_F16) quantize<QC_TYPE_F16>(w, ld, o, st);
  else quantize<QC_TYPE_BF16>(w, ld, o, st);
  return hipGetLastError();
}

template <int TYPE>
static void expand(const qc_w4_weight &w, void *out, int64_t ld, hipStream_t st) {
  using T = typename W4Mem<TYPE>::T;
  const int G = (w.K + w.group - 1) / w.group;
  const bool vec = (uintptr_t)out % 16 == 0 && ld * sizeof(T) % 16 == 0;
  auto kern = vec ? w4_expand_kernel<TYPE, true> : w4_expand_kernel<TYPE, false>;
  kern<<<w.N, row_threads(w.K), 0, st>>>((const uint8_t *)w.q, w.scale, w.zero, w.K, __builtin_ctz(w.group), G, (T *)out, ld);
}

hipError_t launch_w4_expand(const qc_w4_weight &w, void *out, int type, int64_t ld, hipStream_t st) {
  if (type == QC_TYPE_F32) expand<QC_TYPE_F32>(w, out, ld, st);
  else if (type == QC_TYPE_F16) expand<QC_TYPE_F16>(w, out, ld, st);
  else expand<QC_TYPE_BF16>(w, out, ld, st);
  return hipGetLastError();
}

}  // namespace qc
