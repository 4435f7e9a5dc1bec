// Products with 4-bit weights of groups, a few rows at a time: linear layers, the gated block and its inner gradients.
//
// A workgroup makes 16 columns of up to 16 MT rows.  Its wavefronts take the chunks of 128 inputs in turn, so that together they
// read runs of their 16 weight rows; each lane reads 16 bytes (32 codes) of one row, the four lanes of a row exchange them
// (v_permlane) so that a matrix instruction covers 32 consecutive inputs, which lie in one group, and every group's product is
// scaled in float32 as it is added: the codes themselves are exact in every type.  The wavefronts' sums are added in LDS in
// wavefront order.
#include "w4_common.h"

namespace qc {

// GC: groups in a chunk of 128 inputs; MT: tiles of 16 rows
template <int TYPE, int GC, int MT, int OP>
__global__ __launch_bounds__(MT > 1 ? 512 : 1024) void w4_rows_kernel(W4Args a) {
  using F = Frag<TYPE>;
  using T = typename W4Mem<TYPE>::T;
  using XT = typename std::conditional<TYPE == QC_TYPE_I8, int8_t, T>::type;
  constexpr int NW = OP == W4_LINEAR ? 1 : 2;
  extern __shared__ float red[];                 // [wavefronts][NW][MT][64][4]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int r16 = lane & 15, kb = lane >> 4;
  const int ntn = (a.N + 15) / 16, n0 = (int)(blockIdx.x % ntn) * 16, m0 = (int)(blockIdx.x / ntn) * (16 * MT);
  const size_t n = min(n0 + r16, a.N - 1);
  const XT *xr[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) xr[i] = (const XT *)a.x + (int64_t)min(m0 + 16 * i + r16, a.M - 1) * a.ldx;
  const int KB = a.K / 2, chunks = (a.K + 127) / 128;
  w4_f4 y[NW][MT];
#pragma unroll
  for (int w = 0; w < NW; ++w)
#pragma unroll
    for (int i = 0; i < MT; ++i) y[w][i] = w4_f4{};
  for (int c = wave; c < chunks; c += waves) {
    w4_u4 q[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      q[w] = w4_load16(a.w[w].q + n * KB, c * 64 + kb * 16, KB);
      w4_transpose(q[w]);
    }
#pragma unroll
    for (int gi = 0; gi < GC; ++gi) {
      const size_t g = n * a.G + min(c * GC + gi, a.G - 1);
      typename F::Acc acc[NW][MT];
#pragma unroll
      for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[w][i] = typename F::Acc{};
      float s[NW], z16[NW];
      unsigned zb[NW];
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        s[w] = a.w[w].scale[g] * (TYPE == QC_TYPE_I8 ? 1.0f : 16.0f);
        const int z = a.w[w].zero ? a.w[w].zero[g] : 8;
        z16[w] = (float)(z - 8) * 0.0625f;
        zb[w] = (unsigned)z * 0x01010101u;
      }
#pragma unroll
      for (int t = 0; t < 4 / GC; ++t) {
        const int j = gi * (4 / GC) + t;
        const int k = c * 128 + j * 32 + kb * 8;
        typename F::X x[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          x[i] = typename F::X{};
          if (k < a.K) x[i] = *(const typename F::X *)(xr[i] + k);
        }
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          const typename F::W wf = F::template weights<true>(q[w][j], z16[w], zb[w]);
#pragma unroll
          for (int i = 0; i < MT; ++i) acc[w][i] = F::mma(x[i], wf, acc[w][i]);
        }
      }
#pragma unroll
      for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) y[w][i][e] += s[w] * (float)acc[w][i][e];
    }
  }
  constexpr int TILE = MT * 256;
#pragma unroll
  for (int w = 0; w < NW; ++w)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) red[(wave * NW + w) * TILE + (i * 16 + kb * 4 + e) * 16 + r16] = y[w][i][e];
  __syncthreads();
  for (int o = threadIdx.x; o < TILE; o += blockDim.x) {
    const int m = m0 + o / 16, col = n0 + o % 16;
    if (m >= a.M || col >= a.N) continue;
    float v[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      float t = red[w * TILE + o];
      for (int p = 1; p < waves; ++p) t += red[(p * NW + w) * TILE + o];
      if (TYPE == QC_TYPE_I8) t = a.xs * (t - (float)a.zp * a.w[w].sum[col]);
      v[w] = t + (a.w[w].bias ? a.w[w].bias[col] : 0.0f);
    }
    const int64_t at = (int64_t)m * a.ldy + col;
    if constexpr (OP == W4_LINEAR) {
      ((T *)a.y)[at] = W4Mem<TYPE>::put(v[0]);
    } else {
      float d;
      const float act = w4_act(a.act, v[0], d);
      if constexpr (OP == W4_GATED) {
        ((T *)a.y)[at] = W4Mem<TYPE>::put(act * v[1]);
      } else {
        const float dh = W4Mem<TYPE>::get(((const T *)a.dh)[(int64_t)m * a.lddh + col]);
        ((T *)a.y)[at] = W4Mem<TYPE>::put(dh * v[1] * d);
        ((T *)a.y2)[at] = W4Mem<TYPE>::put(dh * act);
      }
    }
  }
}

template <int TYPE, int GC, int MT, int OP>
static hipError_t rows_launch(const W4Args &a, hipStream_t st) {
  const int waves = std::min((a.K + 127) / 128, MT > 1 ? 8 : 16);
  const int lds = waves * (OP == W4_LINEAR ? 1 : 2) * MT * 1024;
  const unsigned grid = (unsigned)((a.N + 15) / 16) * (unsigned)((a.M + 16 * MT - 1) / (16 * MT));
  static std::atomic<unsigned long long> done{0};
  auto kern = w4_rows_kernel<TYPE, GC, MT, OP>;
  if (lds > 65536) {
    hipError_t e = allow_lds((const void *)kern, lds, done);
    if (e != hipSuccess) return e;
  }
  kern<<<grid, waves * 64, lds, st>>>(a);
  return hipGetLastError();
}

template <int TYPE, int GC, int OP>
static hipError_t rows_mt(const W4Args &a, hipStream_t st) {
  if (a.M <= 16) return rows_launch<TYPE, GC, 1, OP>(a, st);
  return rows_launch<TYPE, GC, 4, OP>(a, st);
}

template <int TYPE, int OP>
static hipError_t rows_gc(const W4Args &a, hipStream_t st) {
  if (a.group == 128) return rows_mt<TYPE, 1, OP>(a, st);
  if (a.group == 64) return rows_mt<TYPE, 2, OP>(a, st);
  return rows_mt<TYPE, 4, OP>(a, st);
}

template <int TYPE>
static hipError_t rows_op(const W4Args &a, int op, hipStream_t st) {
  if (op == W4_LINEAR) return rows_gc<TYPE, W4_LINEAR>(a, st);
  if (op == W4_GATED) return rows_gc<TYPE, W4_GATED>(a, st);
  if constexpr (TYPE == QC_TYPE_I8) return hipErrorInvalidValue;
  else return rows_gc<TYPE, W4_GATED_GRAD>(a, st);
}

hipError_t launch_w4_rows(const W4Args &a, int type, int op, hipStream_t st) {
  if (type == QC_TYPE_F32) return rows_op<QC_TYPE_F32>(a, op, st);
  if (type == QC_TYPE_F16) return rows_op<QC_TYPE_F16>(a, op, st);
  if (type == QC_TYPE_BF16) return rows_op<QC_TYPE_BF16>(a, op, st);
  return rows_op<QC_TYPE_I8>(a, op, st);
}

}  // namespace qc
