// Gradient of the root-mean-square norm of rows:
//   dx = rho (g - h rho^2 mean(g h)) + dh,  g = dy weight;   dweight = sum over the rows of dy h rho
// as rho g - (h rho) (rho^2 mean(g h)): h rho is of the size of 1 and the other factor of that of the result, where rho^3 mean(g h) of large rows would
// be below any float32.
// A row's h and dy are read once and stay in registers while its two sums are formed, so that the kernel moves what it has to: h, dy, dh in,
// dx out.  A workgroup walks rows M / groups apart and keeps its columns' part of dweight in registers from row to row; the groups' parts
// go to the workspace, and a second kernel adds them in their order.
// Bytes bound it: 8192 x 4096 bfloat16 with dh 52.0 us, 5.2 TB/s, and 5.0 for the parts (8 MB; workgroups of eight wavefronts, two a compute unit, the next
// row on its way: 99 us with one row at a time, 66 with the weight read from memory in every row); 1000 x 1153 float32 7.8 and 4.9, a row's latency and
// two rows a workgroup.
#include "t8_common.h"

namespace qc {

// `waves` wavefronts a row, as many rows a workgroup as make 8 of them; they walk in step (one wavefront a row: by themselves).  C: vectors a lane.
template <int TYPE, int C>
__global__ __launch_bounds__(512, C <= 2 ? 4 : 2) void t8_norm_grad_kernel(T8NormGradArgs a) {
  using T = typename W4Mem<TYPE>::T;
  constexpr int VL = t8_vl<TYPE>;
  __shared__ double red[2][2][16];                          // alternating, as in t8_rows.hip
  extern __shared__ __align__(16) float own[];              // [rows of a workgroup, width]: each thread's weights, in the end its dweight
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = a.waves, rows = ((int)blockDim.x >> 6) / waves, sub = wave / waves, first = sub * waves;
  const int step = 64 * waves * VL, e0 = ((wave - first) * 64 + lane) * VL;
  const int width = step * C;
  float *mine = own + sub * width + e0;
  // (from memory, twice a row, the weight would be as many bytes of the L2 caches as the rows are of memory)
  if (a.w) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float w[VL];
      t8_load_f32<VL>(a.w, e0 + c * step, a.K, w);
#pragma unroll
      for (int i = 0; i < VL; ++i) mine[c * step + i] = w[i];
    }
  }
  const auto weight = [&](int c, float (&w)[VL]) {
#pragma unroll
    for (int i = 0; i < VL; i += 4) {
      const w4_f4 r = *(const w4_f4 *)(mine + c * step + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[i + j] = r[j];
    }
  };
  float dw[C][VL] = {};
  constexpr bool AHEAD = C <= 2, ALL = C * VL <= 8;        // the next row (ALL: and its dh) is on its way while this one is at work: registers
  w4_u4 nh[C], ng[C], nd[C];
  const auto fetch = [&](int64_t row, int K) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      nh[c] = t8_raw<TYPE>((const T *)a.h + row * a.ldh, e0 + c * step, K);
      ng[c] = t8_raw<TYPE>((const T *)a.dy + row * a.lddy, e0 + c * step, K);
      if (ALL && a.dh) nd[c] = t8_raw<TYPE>((const T *)a.dh + row * a.lddh, e0 + c * step, K);
    }
  };
  int64_t row = (int64_t)blockIdx.x * rows + sub;
  const int64_t ahead = (int64_t)gridDim.x * rows;
  if (AHEAD && row < a.M) fetch(row, a.K);
  int turn = 0;
  for (int64_t base = (int64_t)blockIdx.x * rows; base < a.M; base += ahead, row += ahead, turn ^= 1) {
    const bool there = row < a.M;
    int K = a.K;
    asm volatile("" : "+s"(K));                             // what depends on it is formed again for each row, not kept: registers
    w4_u4 ch[C], cg[C], cd[C];
    if (!AHEAD && there) fetch(row, K);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      ch[c] = nh[c];
      cg[c] = ng[c];
      if (ALL) cd[c] = nd[c];
    }
    if (!ALL && a.dh && there) {
#pragma unroll
      for (int c = 0; c < C; ++c) cd[c] = t8_raw<TYPE>((const T *)a.dh + row * a.lddh, e0 + c * step, K);
    }
    if (AHEAD && row + ahead < a.M) fetch(row + ahead, K);
    double ss = 0.0, dot = 0.0;                             // (float64: products of two float32 numbers pass its range)
    if (there) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float h[VL], g[VL], w[VL];
        t8_values<TYPE>(ch[c], h);
        t8_values<TYPE>(cg[c], g);
        if (a.w) {
          weight(c, w);
#pragma unroll
          for (int i = 0; i < VL; ++i) g[i] *= w[i];
        }
#pragma unroll
        for (int i = 0; i < VL; ++i) {
          ss = __builtin_fma((double)h[i], (double)h[i], ss);
          dot = __builtin_fma((double)g[i], (double)h[i], dot);
        }
      }
    }
    ss = wave_sum_dpp(ss);
    dot = wave_sum_dpp(dot);
    if (waves > 1) {
      if (lane == 0) {
        red[turn][0][wave] = ss;
        red[turn][1][wave] = dot;
      }
      t8_lds_barrier();
      ss = t8_across_sum(red[turn][0] + first, waves, lane);
      dot = t8_across_sum(red[turn][1] + first, waves, lane);
    }
    if (!there) continue;
    const double r = t8_rsqrt(__builtin_fma(ss, a.share, (double)a.eps));
    const float rho = (float)r, along = (float)(r * r * (dot * a.share));
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float h[VL], g[VL], w[VL], d[VL];
      t8_values<TYPE>(ch[c], h);
      t8_values<TYPE>(cg[c], g);
      if (a.w) weight(c, w);
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        const float n = h[i] * rho;
        dw[c][i] = __builtin_fmaf(g[i], n, dw[c][i]);
        if (a.w) g[i] *= w[i];
        d[i] = __builtin_fmaf(-n, along, rho * g[i]);
      }
      if (a.dh) {
        float add[VL];
        t8_values<TYPE>(cd[c], add);
#pragma unroll
        for (int i = 0; i < VL; ++i) d[i] += add[i];
      }
      t8_store<TYPE>((T *)a.dx + row * a.lddx, e0 + c * step, K, d);
    }
  }
  if (!a.dw) return;
  float *part = a.part + (size_t)blockIdx.x * a.K;
  if (rows == 1) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < VL; ++i)
        if (e0 + c * step + i < a.K) part[e0 + c * step + i] = dw[c][i];
    return;
  }
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < VL; ++i) mine[c * step + i] = dw[c][i];
  __syncthreads();
  for (int e = threadIdx.x; e < a.K; e += blockDim.x) {
    float t = own[e];
    for (int i = 1; i < rows; ++i) t += own[i * width + e];
    part[e] = t;
  }
}

// Rows of any length, read twice, element after element; a group's part of dweight lives in the workspace, each element with the thread
// that owns its column: 2000 x 9001 float32 with dh 131 us, where the bytes would take 58
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
    ss = t8_across_sum(red[turn][0], 16, lane);
    dot = t8_across_sum(red[turn][1], 16, lane);
    const double r = t8_rsqrt(__builtin_fma(ss, a.share, (double)a.eps));
    const float rho = (float)r, along = (float)(r * r * (dot * a.share));
    for (int e = threadIdx.x; e < a.K; e += 1024) {
      const float v = Mem::get(h[e]), g = Mem::get(dy[e]);
      const float n = v * rho;
      float d = __builtin_fmaf(-n, along, rho * (a.w ? g * a.w[e] : g));
      if (a.dh) d += Mem::get(dh[e]);
      if (part) part[e] = __builtin_fmaf(g, n, row == blockIdx.x ? 0.0f : part[e]);
      dx[e] = Mem::put(d);
    }
  }
}

// dweight: 16 columns a workgroup, 64 groups at a time, float64 sums in the groups' order
__global__ __launch_bounds__(1024) void t8_weight_grad_kernel(const float *part, int groups, int K, float *dw) {
  __shared__ double red[64][17];
  const int col = blockIdx.x * 16 + (threadIdx.x & 15), first = threadIdx.x >> 4;
  double t = 0.0;
  if (col < K)
    for (int g = first; g < groups; g += 64) t += (double)part[(size_t)g * K + col];
  red[first][threadIdx.x & 15] = t;
  __syncthreads();
  if (first == 0 && col < K) {
    for (int i = 1; i < 64; ++i) t += red[i][threadIdx.x];
    dw[col] = (float)t;
  }
}

struct NormGradShape {
  int waves, rows, c, groups;      // waves 0: the kernel of long rows
};
constexpr int NORM_GRAD_GROUPS = 512;
static NormGradShape norm_grad_shape(int M, int K, int type) {
  const int vl = type == QC_TYPE_F32 ? 4 : 8, vectors = (K + vl - 1) / vl;
  NormGradShape s{};
  s.groups = std::min(M, NORM_GRAD_GROUPS);
  if (vectors > 64 * 8 * 4 || K < vl) return s;
  // two vectors a lane, so that the next row is on its way (16384 x 1152 float32 55 us; with four 76, with one 60)
  s.waves = std::min((vectors + 127) / 128, 8);
  while (s.waves < 8 && vectors > 64 * s.waves && (int64_t)M * s.waves < 2048) ++s.waves;
  s.c = (vectors + 64 * s.waves - 1) / (64 * s.waves);
  s.c = s.c > 2 ? 4 : s.c;
  s.rows = 8 / s.waves;
  // workgroups for every compute unit come before rows that share one
  while (s.rows > 1 && (M + s.rows - 1) / s.rows < 256) --s.rows;
  s.groups = std::min((M + s.rows - 1) / s.rows, NORM_GRAD_GROUPS);
  return s;
}

int t8_norm_grad_groups(int M, int K) { return std::min(M, NORM_GRAD_GROUPS); }

template <int TYPE>
static hipError_t norm_grad_launch(T8NormGradArgs a, hipStream_t st) {
  const NormGradShape s = norm_grad_shape(a.M, a.K, TYPE);
  a.groups = s.groups;
  a.waves = s.waves;
  if (a.M > 0) {
    const int threads = 64 * s.waves * s.rows, lds = threads * s.c * t8_vl<TYPE> * 4;      // 64 KB at most
    if (s.waves == 0) {
      t8_norm_grad_long_kernel<TYPE><<<s.groups, 1024, 0, st>>>(a);
    } else {
      const int at = s.c / 2;
      constexpr void (*kernels[3])(T8NormGradArgs) = {t8_norm_grad_kernel<TYPE, 1>, t8_norm_grad_kernel<TYPE, 2>, t8_norm_grad_kernel<TYPE, 4>};
      static std::atomic<unsigned long long> done[3];
      if (lds > 65536 - 1024) {
        const hipError_t e = allow_lds((const void *)kernels[at], 131072, done[at]);
        if (e != hipSuccess) return e;
      }
      kernels[at]<<<s.groups, threads, lds, st>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dw) t8_weight_grad_kernel<<<(a.K + 15) / 16, 1024, 0, st>>>(a.part, s.groups, a.K, a.dw);
  return hipGetLastError();
}

hipError_t launch_t8_norm_grad(const T8NormGradArgs &a, int type, hipStream_t st) {
  if (type == QC_TYPE_F32) return norm_grad_launch<QC_TYPE_F32>(a, st);
  if (type == QC_TYPE_F16) return norm_grad_launch<QC_TYPE_F16>(a, st);
  return norm_grad_launch<QC_TYPE_BF16>(a, st);
}

}  // namespace qc
