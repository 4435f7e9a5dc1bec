// Gradient of a linear layer's input through fixed 4-bit weights of groups: dx = dy W (+ dy2 W2).
//
// The summed axis is the rows of W, and the scales vary along it, so every weight is scaled before it enters a product.  A lane reads
// 4 bytes of a weight row, 8 neighbouring inputs, and nibble t is its operand of product t: after the sum over all rows it
// holds 8 neighbouring results of each of its rows of dx.
#include "w4_common.h"

namespace qc {

// 16 rows of dx by 128 columns; the workgroup's four wavefronts take the weight rows in turn, four at a time
template <int TYPE>
__global__ __launch_bounds__(256) void w4_grad_kernel(W4GradArgs a) {
  using T = typename W4Mem<TYPE>::T;
  __shared__ float red[3][16 * 128];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, kb = lane >> 4;
  const int ntk = (a.K + 127) / 128, k0 = (int)(blockIdx.x % ntk) * 128, m0 = (int)(blockIdx.x / ntk) * 16;
  const int k = min(k0 + r16 * 8, a.K - 8), g = k / a.group, KB = a.K / 2;
  const int64_t m = min(m0 + r16, a.M - 1);
  w4_f4 acc[8] = {};
  for (int i = 0; i < a.nw; ++i) {
    const T *dy = (const T *)a.dy[i] + m * a.lddy[i];
    const W4Mat &w = a.w[i];
    const int N = a.N[i];
    for (int n = wave * 4; n < N; n += 16) {
      const size_t row = min(n + kb, N - 1);
      const float x = n + kb < N ? W4Mem<TYPE>::get(dy[n + kb]) : 0.0f;
      const unsigned q = *(const unsigned *)(w.q + row * KB + k / 2);
      const float s = w.scale[row * a.G + g] * 16.0f;
      const float z16 = w.zero ? (float)((int)w.zero[row * a.G + g] - 8) * 0.0625f : 0.0f;
#pragma unroll
      for (int t = 0; t < 8; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, s * (w4_nibble(q >> (4 * t)) - z16), acc[t], 0, 0, 0);
    }
  }
  if (wave) {
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) red[wave - 1][(kb * 4 + e) * 128 + r16 * 8 + t] = acc[t][e];
  }
  __syncthreads();
  if (wave || k0 + r16 * 8 >= a.K) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int row = m0 + kb * 4 + e;
    if (row >= a.M) break;
    T *o = (T *)a.dx + (int64_t)row * a.lddx + k;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const int at = (kb * 4 + e) * 128 + r16 * 8 + t;
      o[t] = W4Mem<TYPE>::put(((acc[t][e] + red[0][at]) + red[1][at]) + red[2][at]);
    }
  }
}

template <int TYPE>
static void grad(const W4GradArgs &a, hipStream_t st) {
  w4_grad_kernel<TYPE><<<(unsigned)((a.K + 127) / 128) * (unsigned)((a.M + 15) / 16), 256, 0, st>>>(a);
}

hipError_t launch_w4_grad(const W4GradArgs &a, int type, hipStream_t st) {
  if (type == QC_TYPE_F32) grad<QC_TYPE_F32>(a, st);
  else if (type == QC_TYPE_F16) grad<QC_TYPE_F16>(a, st);
  else grad<QC_TYPE_BF16>(a, st);
  return hipGetLastError();
}

}  // namespace qc
