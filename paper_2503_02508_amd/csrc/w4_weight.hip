// 4-bit weights with a scale per group: the quantiser, and the matrix that its codes stand for.
//
// Both move memory only: the quantiser reads a matrix once and writes an eighth (float32) or a quarter of its bytes, the
// expansion does the reverse.  A workgroup takes a row, a lane 8 neighbouring values (a group of 32, 64 or 128 lies in 4, 8 or
// 16 neighbouring lanes and is reduced without LDS).
#include "w4_common.h"

namespace qc {

template <int TYPE>
__device__ __forceinline__ void w4_load8(const typename W4Mem<TYPE>::T *p, float v[8]) {
  using T = typename W4Mem<TYPE>::T;
  typedef T T8 __attribute__((ext_vector_type(8)));
  const T8 t = *(const T8 *)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = W4Mem<TYPE>::get(t[i]);
}

// minimum / maximum over 4, 8 or 16 neighbouring lanes, in each of them
template <bool MAX>
__device__ __forceinline__ float w4_group_reduce(float v, int lanes) {
  for (int m = 1; m < lanes; m <<= 1) {
    const float o = __shfl_xor(v, m);
    v = MAX ? fmaxf(v, o) : fminf(v, o);
  }
  return v;
}

template <int TYPE>
__global__ __launch_bounds__(256) void w4_quantize_kernel(const typename W4Mem<TYPE>::T *w, int64_t ld, int K, int group, int G, uint8_t *q,
                                                          float *scale, uint8_t *zero, float *sum) {
  __shared__ double part[4];
  const size_t n = blockIdx.x;
  const int lanes = group / 8, KR = (K + 127) / 128 * 128;       // whole groups, so that all lanes of one take part
  double total = 0.0;
  for (int k = threadIdx.x * 8; k < KR; k += blockDim.x * 8) {
    float v[8] = {};
    const bool in = k < K;
    if (in) w4_load8<TYPE>(w + n * ld + k, v);
    float lo = fminf(v[0], 0.0f), hi = fmaxf(v[0], 0.0f);
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      lo = fminf(lo, v[i]);
      hi = fmaxf(hi, v[i]);
    }
    lo = w4_group_reduce<false>(lo, lanes);
    hi = w4_group_reduce<true>(hi, lanes);
    float s, z = 8.0f, low = 1.0f;
    if (zero) {
      s = (hi - lo) / 15.0f;
      if (s == 0.0f) s = 1.0f;
      z = fminf(fmaxf(rintf(-lo / s), 0.0f), 15.0f);
      low = 0.0f;
    } else {
      s = fmaxf(hi, -lo) / 7.0f;
      if (s == 0.0f) s = 1.0f;
    }
    // w / s by way of 1 / s, off by less than 3e-6 for |w / s| <= 15.5: only next to a half does it take the division to decide
    const float inv = 1.0f / s;
    float r[8];
    bool near = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = v[i] * inv;
      r[i] = rintf(t);
      near |= !(fabsf(t - r[i]) <= 0.49999f);                            // or 1 / s is infinite
    }
    if (near) {
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = rintf(v[i] / s);
    }
    unsigned code = 0;
    int isum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = (int)__builtin_amdgcn_fmed3f(r[i] + z, low, 15.0f);
      isum += c;
      code |= (unsigned)c << (4 * i);
    }
    code ^= 0x88888888u;                                                 // u - 8 in two's complement
    isum -= 8 * (int)z;
    if (in) {
      *(unsigned *)(q + n * (K / 2) + k / 2) = code;
      if (k % group == 0) {
        scale[n * G + k / group] = s;
        if (zero) zero[n * G + k / group] = (uint8_t)z;
      }
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
__global__ __launch_bounds__(256) void w4_expand_kernel(const uint8_t *q, const float *scale, const uint8_t *zero, int K, int group, int G,
                                                        typename W4Mem<TYPE>::T *out, int64_t ld) {
  using T = typename W4Mem<TYPE>::T;
  constexpr int E = 16 / sizeof(T);
  typedef T TE __attribute__((ext_vector_type(E)));
  typedef typename std::conditional<E == 8, unsigned, unsigned short>::type Code;
  const size_t n = blockIdx.x;
  for (int k = threadIdx.x * E; k < K; k += blockDim.x * E) {
    const unsigned code = *(const Code *)(q + n * (K / 2) + k / 2);
    const size_t g = n * G + k / group;
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
  w4_quantize_kernel<TYPE><<<o.N, row_threads(o.K), 0, st>>>((const typename W4Mem<TYPE>::T *)w, ld, o.K, o.group, G, (uint8_t *)o.q, o.scale,
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
  kern<<<w.N, row_threads(w.K), 0, st>>>((const uint8_t *)w.q, w.scale, w.zero, w.K, w.group, G, (T *)out, ld);
}

hipError_t launch_w4_expand(const qc_w4_weight &w, void *out, int type, int64_t ld, hipStream_t st) {
  if (type == QC_TYPE_F32) expand<QC_TYPE_F32>(w, out, ld, st);
  else if (type == QC_TYPE_F16) expand<QC_TYPE_F16>(w, out, ld, st);
  else expand<QC_TYPE_BF16>(w, out, ld, st);
  return hipGetLastError();
}

}  // namespace qc
