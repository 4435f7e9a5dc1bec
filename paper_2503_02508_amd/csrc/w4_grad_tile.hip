// Gradient of a linear layer's input through fixed 4-bit weights of groups, many rows: dx = dy W (+ dy2 W2).
//
// A workgroup makes 16 MI rows by 256 columns of dx.  Its two halves take every second step, 64 rows of W, and add their sums at the end; a
// half's four wavefronts stand side by side along the columns.  A step's gradients, packed codes and scales go through LDS.  A lane expands, of 8 neighbouring rows of W, the 4 neighbouring columns it will hold
// results of (nibble t of its two bytes belongs to product t); the scales vary along the summed axis, so a weight is scaled before it
// enters a product.  float16 and bfloat16: it is rounded to the type.  float32: gradients and scaled weights are each the sum of
// three bfloat16 numbers, and six of the nine products are formed (the others are below 2^-22 of the largest).
#include "w4_common.h"

namespace qc {

constexpr int GT_N = 64, GT_WROW = 136;        // rows of W a step; bytes between rows of packed codes in LDS (four rows 8 apart share no bank)

template <int TYPE, int MI>
struct GradTile {
  static constexpr int P = TYPE == QC_TYPE_F32 ? 3 : 1;
  static constexpr int ES = TYPE == QC_TYPE_F32 ? 4 : 2;
  static constexpr int DY = 16 * MI * 128 * P;                           // bytes: planes of 16 MI rows of 64 gradients
  static constexpr int W = GT_N * GT_WROW;
  static constexpr int S = 8 * GT_N * 8;                                 // (scale, offset) of up to 8 groups of columns
  static constexpr int BUF = DY + W + S;
  // two halves with two buffers each; afterwards half of the sums of each half, on their way to the other
  static constexpr int LDS = 4 * BUF > MI / 2 * 4 * 512 * 16 ? 4 * BUF : MI / 2 * 4 * 512 * 16;
  static constexpr int UR = GT_N * ES / 16, NU = 16 * MI * UR / 256;
};

// 16-byte unit u of row r of a plane: 16 rows of one unit lie in 16 different slots of 256 bytes
__device__ __forceinline__ int gt_slot(int r, int u) { return r * 128 + ((u ^ ((r >> 1) & 7)) << 4); }

template <int TYPE, int MI, bool ASYM>
__global__ __launch_bounds__(512, 2) void w4_grad_tile_kernel(W4GradArgs a, int tm, int tk) {
  using T = typename W4Mem<TYPE>::T;
  using F = Frag<TYPE == QC_TYPE_F32 ? QC_TYPE_BF16 : TYPE>;
  using G = GradTile<TYPE, MI>;
  constexpr int P = G::P;
  extern __shared__ __align__(16) char lds[];
  const int half = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), tid = threadIdx.x & 255;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, kb = lane >> 4;
  int mi, ki;
  tile_at(blockIdx.x, gridDim.x, tm, tk, 8, mi, ki);
  const int m0 = mi * 16 * MI, k0 = ki * 256, KB = a.K / 2;
  const int last = a.M - 1 - m0, ncol = (256 + a.group - 1) / a.group;   // groups of the tile's columns
  const int g0 = k0 / a.group, mine = (wave * 64 + r16 * 4) / a.group;   // the lane's own
  const int steps0 = (a.N[0] + GT_N - 1) / GT_N, steps = steps0 + (a.nw > 1 ? (a.N[1] + GT_N - 1) / GT_N : 0);

  w4_u4 dyv[G::NU], wv[2];
  float sv[2];
  int zv[2];
  const auto fetch = [&](int step) {
    const int i = step >= steps0 && a.nw > 1, n0 = (step - (i ? steps0 : 0)) * GT_N, N = a.N[i];
    const T *dy = (const T *)a.dy[i] + (int64_t)m0 * a.lddy[i];
    const W4Mat &w = a.w[i];
    const int ld = (int)a.lddy[i];
#pragma unroll
    for (int v = 0; v < G::NU; ++v) {
      const int t = tid + 256 * v, r = t / G::UR, n = n0 + t % G::UR * (16 / G::ES);
      const T *p = dy + (size_t)min(r, last) * ld + n;
      dyv[v] = w4_u4{};
      if (n + 16 / G::ES <= N) {
        dyv[v] = *(const typename std::conditional<G::ES == 4, w4_u4_a4, w4_u4_a2>::type *)p;
      } else if (n < N) {
        T e[16 / G::ES];
#pragma unroll
        for (int x = 0; x < 16 / G::ES; ++x) {
          e[x] = (T)0.0f;
          if (n + x < N) e[x] = p[x];
        }
        dyv[v] = __builtin_bit_cast(w4_u4, e);
      }
    }
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int t = tid + 256 * v;
      wv[v] = w4_load16(w.q + (size_t)min(n0 + t / 8, N - 1) * KB, k0 / 2 + t % 8 * 16, KB);
      const int g = g0 + t / GT_N;                                       // entries [group][row], up to 512
      if (t < ncol * GT_N) {
        const size_t at = (size_t)min(n0 + t % GT_N, N - 1) * a.G + min(g, a.G - 1);
        sv[v] = w.scale[at];
        if (ASYM) zv[v] = w.zero[at];
      }
    }
  };
  const auto put = [&](char *buf) {
#pragma unroll
    for (int v = 0; v < G::NU; ++v) {
      const int t = tid + 256 * v, r = t / G::UR, u = t % G::UR;
      if constexpr (TYPE == QC_TYPE_F32) {
        float p[4][3];
#pragma unroll
        for (int e = 0; e < 4; ++e) w4_split(__builtin_bit_cast(w4_f4, dyv[v])[e], p[e]);
#pragma unroll
        for (int s = 0; s < 3; ++s)
          *(w4_u2 *)(buf + s * 16 * MI * 128 + gt_slot(r, u >> 1) + (u & 1) * 8) = w4_u2{w4_pack_bf16(p[0][s], p[1][s]), w4_pack_bf16(p[2][s], p[3][s])};
      } else {
        *(w4_u4 *)(buf + gt_slot(r, u)) = dyv[v];
      }
    }
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int t = tid + 256 * v;
      char *at = buf + G::DY + t / 8 * GT_WROW + t % 8 * 16;
      *(w4_u2 *)at = w4_u2{wv[v][0], wv[v][1]};
      *(w4_u2 *)(at + 8) = w4_u2{wv[v][2], wv[v][3]};
      if (t < ncol * GT_N) {
        float *s = (float *)(buf + G::DY + G::W);
        if (ASYM) {
          s[2 * t] = sv[v] * 16.0f;
          s[2 * t + 1] = -(float)(zv[v] - 8) * sv[v];
        } else {
          s[t] = sv[v] * 16.0f;
        }
      }
    }
  };

  w4_f4 acc[MI][4] = {};
  char *mybuf = lds + half * (2 * G::BUF);
  const int turns = (steps + 1) / 2;                                     // of both halves: the last step of one may lie beyond the rows
  if (turns) {
    fetch(half);
    put(mybuf);
  }
  __syncthreads();
  for (int turn = 0; turn < turns; ++turn) {
    const char *cur = mybuf + (turn & 1) * G::BUF;
    if (turn + 1 < turns) fetch(2 * (turn + 1) + half);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      unsigned short q[8];
      float s[8], o[8];
      const char *wq = cur + G::DY + (h * 32 + kb * 8) * GT_WROW + wave * 32 + r16 * 2;
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = *(const unsigned short *)(wq + i * GT_WROW);
      const float *sp = (const float *)(cur + G::DY + G::W) + (mine * GT_N + h * 32 + kb * 8) * (ASYM ? 2 : 1);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[i] = sp[ASYM ? 2 * i : i];
        o[i] = ASYM ? sp[2 * i + 1] : 0.0f;
      }
      w4_u4 wf[P][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {                                      // rows 2 i and 2 i + 1
        float v[2][4];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          unsigned even = q[2 * i + b], odd = even >> 4;
          asm("" : "+v"(odd));
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const float c = w4_nibble(((t & 1 ? odd : even) >> (t & 2 ? 8 : 0)) & 0xFF);
            v[b][t] = ASYM ? fmaf(c, s[2 * i + b], o[2 * i + b]) : c * s[2 * i + b];
          }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if constexpr (TYPE == QC_TYPE_F32) {
            float p0[3], p1[3];
            w4_split(v[0][t], p0);
            w4_split(v[1][t], p1);
#pragma unroll
            for (int p = 0; p < 3; ++p) wf[p][t][i] = w4_pack_bf16(p0[p], p1[p]);
          } else {
            typedef T T2 __attribute__((ext_vector_type(2)));
            typedef float f2 __attribute__((ext_vector_type(2)));
            asm("" : "+v"(v[0][t]), "+v"(v[1][t]));                      // rounded to float32 before it is rounded to the type
            wf[0][t][i] = __builtin_bit_cast(unsigned, __builtin_convertvector((f2{v[0][t], v[1][t]}), T2));
          }
        }
      }
#pragma unroll
      for (int i = 0; i < MI; ++i) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const typename F::X x = *(const typename F::X *)(cur + p * 16 * MI * 128 + gt_slot(16 * i + r16, h * 4 + kb));
#pragma unroll
          for (int pw = 0; pw < P - p; ++pw)
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[i][t] = F::mma(x, __builtin_bit_cast(typename F::W, wf[pw][t]), acc[i][t]);
        }
      }
    }
    if (turn + 1 < turns) put(mybuf + ((turn + 1) & 1) * G::BUF);
    __syncthreads();
  }

  // the first half of the workgroup finishes the tile's upper rows, the second the lower ones
  w4_f4 *there = (w4_f4 *)lds;
#pragma unroll
  for (int i = 0; i < MI / 2; ++i)
#pragma unroll
    for (int t = 0; t < 4; ++t) there[(i * 4 + t) * 512 + threadIdx.x] = half ? acc[i][t] : acc[i + MI / 2][t];
  __syncthreads();
  const int k = k0 + wave * 64 + r16 * 4;
  if (k >= a.K) return;
#pragma unroll
  for (int i = 0; i < MI / 2; ++i) {
    w4_f4 sum[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const w4_f4 o = there[(i * 4 + t) * 512 + (threadIdx.x ^ 256)];
      sum[t] = half ? o + acc[i + MI / 2][t] : acc[i][t] + o;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 16 * (i + half * (MI / 2)) + kb * 4 + e;
      if (r > last) continue;
      T *o = (T *)a.dx + (int64_t)(m0 + r) * a.lddx + k;
      typedef T T4 __attribute__((ext_vector_type(4)));
      T4 v;
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = W4Mem<TYPE>::put(sum[t][e]);
      if ((uintptr_t)o % sizeof(T4) == 0) {
        *(T4 *)o = v;
      } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) o[t] = v[t];
      }
    }
  }
}

template <int TYPE, int MI, bool ASYM>
static hipError_t launch(const W4GradArgs &a, hipStream_t st) {
  constexpr int lds = GradTile<TYPE, MI>::LDS;
  const int tm = (a.M + 16 * MI - 1) / (16 * MI), tk = (a.K + 255) / 256;
  static std::atomic<unsigned long long> done{0};
  auto kern = w4_grad_tile_kernel<TYPE, MI, ASYM>;
  if (lds > 65536) {
    hipError_t e = allow_lds((const void *)kern, lds, done);
    if (e != hipSuccess) return e;
  }
  kern<<<tm * tk, 512, lds, st>>>(a, tm, tk);
  return hipGetLastError();
}

// us of a step of both halves of a workgroup (128 rows of W), by row blocks of a tile: measured with bfloat16 at 4608 x 1152, 9216 x 1152
// and 4608 x 4608, 64 - 4096 rows.  A compute unit runs one workgroup at a time, two of the smallest.
static float step_time(int MI) { return MI == 8 ? 2.9f : MI == 6 ? 2.75f : MI == 4 ? 2.3f : 2.1f; }

template <int TYPE, bool ASYM>
static hipError_t rows(const W4GradArgs &a, hipStream_t st) {
  const int64_t tk = (a.K + 255) / 256;
  int best = 2;
  float time = 0.0f;
  for (int MI = 2; MI <= (TYPE == QC_TYPE_F32 ? 4 : 8); MI += 2) {       // float32: three planes of 64 rows fill LDS
    const int64_t groups = (a.M + 16 * MI - 1) / (16 * MI) * tk, slots = MI == 2 ? 512 : 256;
    const float t = step_time(MI) * (float)((groups + slots - 1) / slots);
    if (MI == 2 || t < time) {
      best = MI;
      time = t;
    }
  }
  if constexpr (TYPE != QC_TYPE_F32) {
    if (best == 8) return launch<TYPE, 8, ASYM>(a, st);
    if (best == 6) return launch<TYPE, 6, ASYM>(a, st);
  }
  return best == 4 ? launch<TYPE, 4, ASYM>(a, st) : launch<TYPE, 2, ASYM>(a, st);
}

bool w4_grad_tile_pays(const W4GradArgs &a, int) { return a.M > 16; }

hipError_t launch_w4_grad_tile(const W4GradArgs &a, int type, hipStream_t st) {
  const bool z = a.w[0].zero != nullptr;
  if (type == QC_TYPE_F32) return z ? rows<QC_TYPE_F32, true>(a, st) : rows<QC_TYPE_F32, false>(a, st);
  if (type == QC_TYPE_F16) return z ? rows<QC_TYPE_F16, true>(a, st) : rows<QC_TYPE_F16, false>(a, st);
  return z ? rows<QC_TYPE_BF16, true>(a, st) : rows<QC_TYPE_BF16, false>(a, st);
}

}  // namespace qc
