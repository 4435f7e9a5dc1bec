// Gradient of the root-mean-square norm of rows:
//   dx = rho (g - h rho^2 mean(g h)) + dh,  g = dy weight;   dweight = sum over the rows of dy h rho
// A row's h and dy are read once and stay in registers while its two sums are formed, so that the kernel moves what it has to: h, dy, dh in,
// dx out.  A workgroup walks rows M / groups apart and keeps its columns' part of dweight in registers from row to row; the groups' parts
// go to the workspace, and a second kernel adds them in their order.
#include "t8_common.h"

namespace qc {

// FULL: a workgroup a row (else a wavefront); C: vectors a lane
template <int TYPE, bool FULL, int C>
__global__ __launch_bounds__(FULL ? 1024 : 256) void t8_norm_grad_kernel(T8NormGradArgs a) {
  using T = typename W4Mem<TYPE>::T;
  constexpr int VL = t8_vl<TYPE>;
  __shared__ double red[2][2][16];                          // alternating, as in t8_rows.hip
  __shared__ float join[FULL ? 1 : 4 * 64 * C * VL];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = FULL ? (int)blockDim.x >> 6 : 1, step = 64 * waves * VL, e0 = (FULL ? (int)threadIdx.x : lane) * VL;
  float dw[C][VL] = {};
  int turn = 0;
  for (int64_t row = FULL ? blockIdx.x : blockIdx.x * 4 + wave; row < a.M; row += FULL ? gridDim.x : gridDim.x * 4, turn ^= 1) {
    float h[C][VL], g[C][VL];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      t8_load<TYPE>((const T *)a.h + row * a.ldh, e0 + c * step, a.K, h[c]);
      t8_load<TYPE>((const T *)a.dy + row * a.lddy, e0 + c * step, a.K, g[c]);
    }
    double ss = 0.0;
    float gh = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float w[VL];
      if (a.w) t8_load_f32<VL>(a.w, e0 + c * step, a.K, w);
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        ss = __builtin_fma((double)h[c][i], (double)h[c][i], ss);
        gh = __builtin_fmaf(a.w ? g[c][i] * w[i] : g[c][i], h[c][i], gh);
      }
    }
    ss = wave_sum_dpp(ss);
    double dot = wave_sum_dpp((double)gh);
    if constexpr (FULL) {
      if (lane == 0) {
        red[turn][0][wave] = ss;
        red[turn][1][wave] = dot;
      }
      __syncthreads();
      ss = red[turn][0][0];
      dot = red[turn][1][0];
      for (int i = 1; i < waves; ++i) {
        ss += red[turn][0][i];
        dot += red[turn][1][i];
      }
    }
    const double r = t8_rsqrt(ss / (double)a.K + (double)a.eps);
    const float rho = (float)r, along = (float)(r * r * r * (dot / (double)a.K));
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float w[VL], add[VL], d[VL];
      if (a.w) t8_load_f32<VL>(a.w, e0 + c * step, a.K, w);
      if (a.dh) t8_load<TYPE>((const T *)a.dh + row * a.lddh, e0 + c * step, a.K, add);
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        d[i] = __builtin_fmaf(-h[c][i], along, rho * (a.w ? g[c][i] * w[i] : g[c][i]));
        if (a.dh) d[i] += add[i];
        dw[c][i] = __builtin_fmaf(g[c][i], h[c][i] * rho, dw[c][i]);
      }
      t8_store<TYPE>((T *)a.dx + row * a.lddx, e0 + c * step, a.K, d);
    }
  }
  if (!a.dw) return;
  float *part = a.part + (size_t)blockIdx.x * a.K;
  if constexpr (FULL) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int i = 0; i < VL; ++i)
        if (e0 + c * step + i < a.K) part[e0 + c * step + i] = dw[c][i];
    }
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < VL; ++i) join[wave * 64 * C * VL + e0 + c * step + i] = dw[c][i];
    __syncthreads();
    for (int e = threadIdx.x; e < a.K; e += 256) {
      float t = join[e];
#pragma unroll
      for (int i = 1; i < 4; ++i) t += join[i * 64 * C * VL + e];
      part[e] = t;
    }
  }
}

// Rows of any length, read twice, element after element; a group's part of dweight lives in the workspace, each element with the thread
// that owns its column
template <int TYPE>
__global__ __launch_bounds__(1024) void t8_norm_grad_long_kernel(T8NormGradArgs a) {
  using T = typename W4Mem<TYPE>::T;
  using Mem = W4Mem<TYPE>;
  __shared__ double red[2][2][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float *part = a.dw ? a.part + (size_t)blockIdx.x * a.K : nullptr;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x, turn ^= 1) {
    const T *h = (const T *)a.h + row * a.ldh, *dy = (const T *)a.dy + row * a.lddy, *dh = (const T *)a.dh + row * a.lddh;
    T *dx = (T *)a.dx + row * a.lddx;
    double ss = 0.0, dot = 0.0;
    for (int e = threadIdx.x; e < a.K; e += 1024) {
      const float v = Mem::get(h[e]), g = Mem::get(dy[e]);
      ss = __builtin_fma((double)v, (double)v, ss);
      dot = __builtin_fma((double)(a.w ? g * a.w[e] : g), (double)v, dot);
    }
    ss = wave_sum_dpp(ss);
    dot = wave_sum_dpp(dot);
    if (lane == 0) {
      red[turn][0][wave] = ss;
      red[turn][1][wave] = dot;
    }
    __syncthreads();
    ss = red[turn][0][0];
    dot = red[turn][1][0];
    for (int i = 1; i < 16; ++i) {
      ss += red[turn][0][i];
      dot += red[turn][1][i];
    }
    const double r = t8_rsqrt(ss / (double)a.K + (double)a.eps);
    const float rho = (float)r, along = (float)(r * r * r * (dot / (double)a.K));
    for (int e = threadIdx.x; e < a.K; e += 1024) {
      const float v = Mem::get(h[e]), g = Mem::get(dy[e]);
      float d = __builtin_fmaf(-v, along, rho * (a.w ? g * a.w[e] : g));
      if (a.dh) d += Mem::get(dh[e]);
      if (part) part[e] = __builtin_fmaf(g, v * rho, row == blockIdx.x ? 0.0f : part[e]);
      dx[e] = Mem::put(d);
    }
  }
}

// dweight: 64 columns a workgroup, its 16 wavefronts every sixteenth group, float64 sums in the groups' order
__global__ __launch_bounds__(1024) void t8_weight_grad_kernel(const float *part, int groups, int K, float *dw) {
  __shared__ double red[16][64];
  const int col = blockIdx.x * 64 + (threadIdx.x & 63), wave = threadIdx.x >> 6;
  double t = 0.0;
  if (col < K)
    for (int g = wave; g < groups; g += 16) t += (double)part[(size_t)g * K + col];
  red[wave][threadIdx.x & 63] = t;
  __syncthreads();
  if (wave == 0 && col < K) {
    for (int i = 1; i < 16; ++i) t += red[i][threadIdx.x];
    dw[col] = (float)t;
  }
}

struct NormGradShape {
  int waves, c, groups;      // waves 0: the kernel of long rows
};
// One rule for every type, so that the workspace does not depend on it: vectors of 4 elements would be 8 of the 16-bit types'.
static NormGradShape norm_grad_shape(int M, int K, int vl) {
  const int vectors = (K + vl - 1) / vl;
  NormGradShape s{};
  s.groups = std::min(M, 512);
  if (vectors > 64 * 16 * 2) return s;
  s.waves = 1;
  while (vectors > 64 * 2 * s.waves || (s.waves < 16 && vectors > 64 * s.waves && (int64_t)M * s.waves < 1024)) s.waves *= 2;
  s.c = (vectors + 64 * s.waves - 1) / (64 * s.waves);
  if (s.waves == 1) s.groups = std::min((M + 3) / 4, 512);
  return s;
}

int t8_norm_grad_groups(int M, int K) { return std::max(norm_grad_shape(M, K, 4).groups, norm_grad_shape(M, K, 8).groups); }

template <int TYPE>
static hipError_t norm_grad_launch(T8NormGradArgs a, hipStream_t st) {
  const NormGradShape s = norm_grad_shape(a.M, a.K, t8_vl<TYPE>);
  a.groups = s.groups;
  if (a.M > 0) {
    if (s.waves == 0) t8_norm_grad_long_kernel<TYPE><<<s.groups, 1024, 0, st>>>(a);
    else if (s.waves == 1 && s.c == 1) t8_norm_grad_kernel<TYPE, false, 1><<<s.groups, 256, 0, st>>>(a);
    else if (s.waves == 1) t8_norm_grad_kernel<TYPE, false, 2><<<s.groups, 256, 0, st>>>(a);
    else if (s.c == 1) t8_norm_grad_kernel<TYPE, true, 1><<<s.groups, 64 * s.waves, 0, st>>>(a);
    else t8_norm_grad_kernel<TYPE, true, 2><<<s.groups, 64 * s.waves, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dw) t8_weight_grad_kernel<<<(a.K + 63) / 64, 1024, 0, st>>>(a.part, s.groups, a.K, a.dw);
  return hipGetLastError();
}

hipError_t launch_t8_norm_grad(const T8NormGradArgs &a, int type, hipStream_t st) {
  if (type == QC_TYPE_F32) return norm_grad_launch<QC_TYPE_F32>(a, st);
  if (type == QC_TYPE_F16) return norm_grad_launch<QC_TYPE_F16>(a, st);
  return norm_grad_launch<QC_TYPE_BF16>(a, st);
}

}  // namespace qc
