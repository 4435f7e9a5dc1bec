// Gradient of a linear layer's input through fixed 4-bit weights of groups: dx = dy W (+ dy2 W2).
//
// The summed axis is the rows of W.  A workgroup makes 16 MI rows by 64 CW columns of dx; its WV wavefronts are WV / CW parties that take
// the steps, 64 rows of W, in turn and add their sums at the end, so that a narrow dx still has every wavefront at work.  A step's
// gradients, packed codes and scales go through LDS.  A lane expands, of 8 neighbouring rows of W, the 4 neighbouring columns it will hold
// results of (nibble t of its two bytes belongs to product t).  The scales vary along the summed axis, so a weight is scaled before it
// enters a product, and is not a number of few bits any more.  All products are of bfloat16 parts, whose exponents are float32's:
//   bfloat16   gradients as they are; weights of two parts, the second rounded, off by 2^-15 of themselves at most: two products
//   float16    gradients of two parts, exactly; weights of two; the product of the two second parts, below 2^-15, is left out: three
//   float32    both of three parts, exactly; six of the nine products are formed (the others are below 2^-22 of the largest)
// Where a tile's columns lie in one group the scale can multiply the gradients instead (PRE below), and the codes stay exact.
#include "w4_common.h"

namespace qc {

constexpr int GT_N = 64;                       // rows of W a step

// MI: blocks of 16 rows; CW: wavefronts side by side, 64 columns each; the workgroup's WV wavefronts are WV / CW such parties.  A party of
// one wavefront (SOLO) has its part of LDS to itself: it needs no barrier and no second buffer, and the smallest tile has registers
// left to ask for its steps two ahead.
template <int TYPE, int MI, int CW, bool PRE>
struct GradTile {
  static constexpr int P = TYPE == QC_TYPE_F32 ? 3 : PRE || TYPE == QC_TYPE_F16 ? 2 : 1;   // parts of a gradient
  static constexpr int PW = PRE ? 1 : TYPE == QC_TYPE_F32 ? 3 : 2;       // of a weight
  static constexpr int TERMS = TYPE == QC_TYPE_F32 ? 3 : 2;              // parts p and q are multiplied where p + q is less
  static constexpr int ES = TYPE == QC_TYPE_F32 ? 4 : 2;
  static constexpr bool SOLO = CW == 1;
  static constexpr int AHEAD = SOLO && MI == 1 && TYPE != QC_TYPE_F32 ? 2 : 1;
  static constexpr int WV = AHEAD == 2 ? 16 : 8, BUFS = SOLO ? 1 : 2;
  static constexpr int S = WV / CW, TH = 64 * CW;                        // parties, threads of one
  static constexpr int WROW = 32 * CW + 8;                               // bytes between rows of packed codes in LDS: four rows 8 apart share no bank
  static constexpr int GR = CW < 2 ? 2 : 2 * CW;                         // groups of up to 64 CW columns
  static constexpr int DY = 16 * MI * 128 * P;                           // bytes: planes of 16 MI rows of 64 gradients
  static constexpr int W = GT_N * WROW;
  static constexpr int BUF = DY + W + (PRE ? 0 : GR * GT_N * 8);         // and (scale, zero point) of every row and group
  // buffers of all parties; afterwards the sums, of two parties only the half that the other finishes
  static constexpr int SUMS = (S == 2 ? MI / 2 : MI) * 4 * 64 * WV * 16;
  static constexpr int TABLES = PRE ? S * 3 * 2 * GT_N * 4 : 0;
  static constexpr int LDS = BUFS * S * BUF + TABLES > SUMS ? BUFS * S * BUF + TABLES : SUMS;
  static constexpr int UR = GT_N * ES / 16, NU = 16 * MI * UR / TH;
  static constexpr int WU = 2 * CW, NW = GT_N * WU / TH;                 // units of a row of codes, a thread's
  static constexpr int NS = GR * GT_N / TH;
  static_assert(16 * MI * UR % TH == 0 && (S > 2 || MI % 2 == 0), "whole loads");
};

// 16-byte unit u of row r of a plane: 16 rows of one unit lie in 16 different slots of 256 bytes
__device__ __forceinline__ int gt_slot(int r, int u) { return r * 128 + ((u ^ ((r >> 1) & 7)) << 4); }

// a weight in two parts.  The first is cut off below the weight itself, so that the second has its sign and is not zero either: what an
// infinite gradient gives is the weight's infinity, and NaN only where the weight is zero.
__device__ __forceinline__ void gt_weight(float v, float p[2]) {
  p[0] = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, v * (1.0f - 0x1p-22f)) & 0xFFFF0000u);
  p[1] = v - p[0];
}
__device__ __forceinline__ unsigned gt_round_bf16(float lo, float hi) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  typedef float f2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_convertvector((f2{lo, hi}), b2));
}

// PRE: the tile's columns lie in one group, so that the scale of a weight row multiplies the gradients as they go to LDS, and the
// weights are exact codes, of which nothing has to be split: three products for six (float32), two for three (float16), and few
// instructions a weight where there are few rows to pay for it
template <int TYPE, int MI, int CW, bool ASYM, bool PRE>
__global__ __launch_bounds__((64 * GradTile<TYPE, MI, CW, PRE>::WV), 2) void w4_grad_kernel(W4GradArgs a, int tm, int tk) {
  using T = typename W4Mem<TYPE>::T;
  using F = Frag<QC_TYPE_BF16>;
  using G = GradTile<TYPE, MI, CW, PRE>;
  constexpr int P = G::P, PW = G::PW;
  extern __shared__ __align__(16) char lds[];
  const int party = __builtin_amdgcn_readfirstlane(threadIdx.x / G::TH), tid = threadIdx.x % G::TH;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, kb = lane >> 4;
  int mi, ki;
  tile_at(blockIdx.x, gridDim.x, tm, tk, 8, mi, ki);
  const int m0 = mi * 16 * MI, k0 = ki * (64 * CW), KB = a.K / 2;
  const int last = a.M - 1 - m0, ncol = (64 * CW + a.group - 1) / a.group;  // groups of the tile's columns
  const int g0 = k0 / a.group, mine = (k0 + wave * 64 + r16 * 4) / a.group - g0;   // the lane's own
  const int steps0 = (a.N[0] + GT_N - 1) / GT_N, steps = steps0 + (a.nw > 1 ? (a.N[1] + GT_N - 1) / GT_N : 0);

  struct Stage {                                 // a step on its way to LDS
    w4_u4 dy[G::NU], w[G::NW];
    float s[G::NS];
    int z[G::NS];
  } stage[G::AHEAD];
  // Where a step lies: its weight, first row of W and how many are left.  Codes, scales and zero points beyond the last row read as
  // zero; what is read beyond a row's end belongs to columns that are not stored.
  const auto where = [&](int step, bool &second, int &n0) {
    second = step >= steps0 && a.nw > 1;
    n0 = (step - (second ? steps0 : 0)) * GT_N;
    return (second ? a.N[1] : a.N[0]) - n0;
  };
  const auto fetch_scales = [&](Stage &f, int step) {
    bool second;
    int n0;
    const int left = where(step, second, n0);
    const __amdgpu_buffer_rsrc_t sb = w4_buffer((second ? a.w[1].scale : a.w[0].scale) + ((size_t)n0 * a.G + g0), ((int64_t)left * a.G - g0) * 4);
    const __amdgpu_buffer_rsrc_t zb = w4_buffer((second ? a.w[1].zero : a.w[0].zero) + ((size_t)n0 * a.G + g0), (int64_t)left * a.G - g0);
#pragma unroll
    for (int v = 0; v < G::NS; ++v) {
      const int t = tid + G::TH * v, at = t % GT_N * a.G + t / GT_N;     // entries [group][row]
      if (t < ncol * GT_N) {
        f.s[v] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(sb, at * 4, 0, 0));
        if (ASYM) f.z[v] = __builtin_amdgcn_raw_buffer_load_b8(zb, at, 0, 0);
      }
    }
  };
  const auto put_scales = [&](const Stage &f, float *s) {
#pragma unroll
    for (int v = 0; v < G::NS; ++v) {
      const int t = tid + G::TH * v;
      if (t < ncol * GT_N) {
        if (PRE) {                                                       // [row] scales, then [row] zero points
          s[t] = f.s[v] * 16.0f;
          if (ASYM) s[GT_N + t] = (float)(f.z[v] - 8) * 0.0625f;
        } else if (ASYM) {
          s[2 * t] = f.s[v] * 16.0f;
          s[2 * t + 1] = (float)(f.z[v] - 8) * 0.0625f;
        } else {
          s[t] = f.s[v] * 16.0f;
        }
      }
    }
  };
  const auto fetch = [&](Stage &f, int step) {
    bool second;
    int n0;
    const int left = where(step, second, n0);
    const int64_t ld = second ? a.lddy[1] : a.lddy[0];
    const int row_bytes = (int)ld * G::ES;
    const char *dy = (const char *)(second ? a.dy[1] : a.dy[0]) + ((int64_t)m0 * ld + n0) * G::ES;
    if (left >= GT_N) {
#pragma unroll
      for (int v = 0; v < G::NU; ++v) {
        const int t = tid + G::TH * v, r = t / G::UR, u = t % G::UR;
        f.dy[v] = *(const typename std::conditional<G::ES == 4, w4_u4_a4, w4_u4_a2>::type *)(dy + (unsigned)(min(r, last) * row_bytes + u * 16));
      }
    } else {                                     // the last rows of W: zero beyond them
#pragma unroll
      for (int v = 0; v < G::NU; ++v) {
        const int t = tid + G::TH * v, r = t / G::UR, n = t % G::UR * (16 / G::ES);
        const T *p = (const T *)(dy + (unsigned)(min(r, last) * row_bytes)) + n;
        T e[16 / G::ES];
#pragma unroll
        for (int x = 0; x < 16 / G::ES; ++x) {
          e[x] = (T)0.0f;
          if (n + x < left) e[x] = p[x];
        }
        f.dy[v] = __builtin_bit_cast(w4_u4, e);
      }
    }
    const __amdgpu_buffer_rsrc_t qb = w4_buffer((second ? a.w[1].q : a.w[0].q) + ((size_t)n0 * KB + k0 / 2), (int64_t)left * KB - k0 / 2);
#pragma unroll
    for (int v = 0; v < G::NW; ++v) {
      const int t = tid + G::TH * v;
      f.w[v] = __builtin_bit_cast(w4_u4, __builtin_amdgcn_raw_buffer_load_b128(qb, t / G::WU * KB + t % G::WU * 16, 0, 0));
    }
    if (!PRE) fetch_scales(f, step);
  };
  const auto put = [&](const Stage &f, char *buf, const float *scales) {
#pragma unroll
    for (int v = 0; v < G::NU; ++v) {
      const int t = tid + G::TH * v, r = t / G::UR, u = t % G::UR;
      if constexpr (TYPE == QC_TYPE_F32) {
        float p[4][3];
#pragma unroll
        for (int e = 0; e < 4; ++e) w4_split(__builtin_bit_cast(w4_f4, f.dy[v])[e] * (PRE ? scales[u * 4 + e] : 1.0f), p[e]);
#pragma unroll
        for (int s = 0; s < 3; ++s)
          *(w4_u2 *)(buf + s * 16 * MI * 128 + gt_slot(r, u >> 1) + (u & 1) * 8) = w4_u2{w4_pack_bf16(p[0][s], p[1][s]), w4_pack_bf16(p[2][s], p[3][s])};
      } else if constexpr (PRE) {
        typedef T T8 __attribute__((ext_vector_type(8)));
        const T8 e = __builtin_bit_cast(T8, f.dy[v]);
        float p[8][2];                                                   // a part cut off, the rest rounded; of infinities nothing is left
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float t = (float)e[i] * scales[u * 8 + i];
          p[i][0] = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, t) & 0xFFFF0000u);
          p[i][1] = p[i][0] == t ? 0.0f : t - p[i][0];
        }
        w4_u4 h, rest;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          h[i] = w4_pack_bf16(p[2 * i][0], p[2 * i + 1][0]);
          rest[i] = gt_round_bf16(p[2 * i][1], p[2 * i + 1][1]);
        }
        *(w4_u4 *)(buf + gt_slot(r, u)) = h;
        *(w4_u4 *)(buf + 16 * MI * 128 + gt_slot(r, u)) = rest;
      } else if constexpr (TYPE == QC_TYPE_F16) {
        const w4_h8 e = __builtin_bit_cast(w4_h8, f.dy[v]);
        w4_u4 h, rest;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = (float)e[2 * i], b = (float)e[2 * i + 1];
          h[i] = gt_round_bf16(a, b);
          const float ah = __builtin_bit_cast(float, h[i] << 16), bh = __builtin_bit_cast(float, h[i] & 0xFFFF0000u);
          rest[i] = w4_pack_bf16(ah == a ? 0.0f : a - ah, bh == b ? 0.0f : b - bh);      // three bits of it are left, of infinities none
        }
        *(w4_u4 *)(buf + gt_slot(r, u)) = h;
        *(w4_u4 *)(buf + 16 * MI * 128 + gt_slot(r, u)) = rest;
      } else {
        *(w4_u4 *)(buf + gt_slot(r, u)) = f.dy[v];
      }
    }
#pragma unroll
    for (int v = 0; v < G::NW; ++v) {
      const int t = tid + G::TH * v;
      char *at = buf + G::DY + t / G::WU * G::WROW + t % G::WU * 16;
      *(w4_u2 *)at = w4_u2{f.w[v][0], f.w[v][1]};
      *(w4_u2 *)(at + 8) = w4_u2{f.w[v][2], f.w[v][3]};
    }
    if (!PRE) put_scales(f, (float *)(buf + G::DY + G::W));
  };

  w4_f4 acc[MI][4] = {};
  char *mybuf = lds + party * (G::BUFS * G::BUF);
  const int turns = (steps + G::S - 1) / G::S;                           // of every party: the last step of one may lie beyond the rows
  const auto turned = [&]() {
    if constexpr (G::SOLO) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    } else {
      __syncthreads();
    }
  };
  // PRE: three tables of scales, since a step's are needed when its gradients are stored, a step before its weights are used
  float *tables = (float *)(lds + G::BUFS * G::S * G::BUF) + party * (3 * 2 * GT_N);
  if (turns) {
    if (PRE) {
      fetch_scales(stage[0], party);
      put_scales(stage[0], tables);
      fetch_scales(stage[0], G::S + party);
      put_scales(stage[0], tables + 2 * GT_N);
      turned();
    }
#pragma unroll
    for (int d = 0; d < G::AHEAD; ++d) fetch(stage[d], G::S * d + party);
    put(stage[0], mybuf, tables);
  }
  turned();
  int table = 0;                                                         // of the present step
  const auto work = [&](int turn, Stage &later, Stage &next) {
    const char *cur = mybuf + (turn % G::BUFS) * G::BUF;
    const float *now = tables + table * (2 * GT_N);
    if (PRE && turn + 2 < turns) fetch_scales(later, G::S * (turn + 2) + party);
    if (turn + G::AHEAD < turns) fetch(later, G::S * (turn + G::AHEAD) + party);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      unsigned short q[8];
      float s[8], o[8];
      const char *wq = cur + G::DY + (h * 32 + kb * 8) * G::WROW + wave * 32 + r16 * 2;
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = *(const unsigned short *)(wq + i * G::WROW);
      const float *sp = PRE ? now + GT_N + h * 32 + kb * 8 : (const float *)(cur + G::DY + G::W) + (mine * GT_N + h * 32 + kb * 8) * (ASYM ? 2 : 1);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s[i] = PRE ? 1.0f : sp[ASYM ? 2 * i : i];
        o[i] = !ASYM ? 0.0f : sp[PRE ? i : 2 * i + 1];
      }
      w4_u4 wf[PW][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {                                      // rows 2 i and 2 i + 1
        float v[2][4];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          unsigned even = q[2 * i + b], odd = even >> 4;
          asm("" : "+v"(odd));
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            float c = w4_nibble(((t & 1 ? odd : even) >> (t & 2 ? 8 : 0)) & 0xFF);
            if (ASYM) c -= o[2 * i + b];                                 // among the codes, where it is exact: u = z is a weight of zero
            v[b][t] = PRE ? c : c * s[2 * i + b];
          }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if constexpr (PRE) {
            wf[0][t][i] = w4_pack_bf16(v[0][t], v[1][t]);
          } else if constexpr (TYPE == QC_TYPE_F32) {
            float p0[3], p1[3];
            w4_split<true>(v[0][t], p0);
            w4_split<true>(v[1][t], p1);
#pragma unroll
            for (int p = 0; p < 3; ++p) wf[p][t][i] = w4_pack_bf16(p0[p], p1[p]);
          } else {
            float p0[2], p1[2];
            gt_weight(v[0][t], p0);
            gt_weight(v[1][t], p1);
            wf[0][t][i] = w4_pack_bf16(p0[0], p1[0]);
            wf[1][t][i] = gt_round_bf16(p0[1], p1[1]);
          }
        }
      }
      // the operands of a row block are read while the products of the one before run
      typename F::X x[2][P];
      const auto read = [&](int i) {
#pragma unroll
        for (int p = 0; p < P; ++p) x[i & 1][p] = *(const typename F::X *)(cur + p * 16 * MI * 128 + gt_slot(16 * i + r16, h * 4 + kb));
      };
      read(0);
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        if (i + 1 < MI) read(i + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
          for (int pw = 0; pw < (PW < G::TERMS - p ? PW : G::TERMS - p); ++pw)
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[i][t] = F::mma(x[i & 1][p], __builtin_bit_cast(typename F::W, wf[pw][t]), acc[i][t]);
      }
    }
    const int after = table == 2 ? 0 : table + 1;
    if (G::SOLO) turned();                                               // its one buffer is read
    if (turn + 1 < turns) put(next, mybuf + ((turn + 1) % G::BUFS) * G::BUF, tables + after * (2 * GT_N));
    if (PRE && turn + 2 < turns) put_scales(later, tables + (after == 2 ? 0 : after + 1) * (2 * GT_N));
    table = after;
    turned();
  };
  for (int turn = 0; turn < turns; turn += G::AHEAD) {
    work(turn, stage[0], stage[G::AHEAD - 1]);
    if (G::AHEAD == 2 && turn + 1 < turns) work(turn + 1, stage[G::AHEAD - 1], stage[0]);
  }
  if (G::SOLO) __syncthreads();

  w4_f4 *there = (w4_f4 *)lds;
  const auto store = [&](int row0, int k, const w4_f4 sum[4]) {
    if (k >= a.K) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = row0 + e;
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
  };
  if constexpr (G::S == 2) {                     // the first party finishes the tile's upper rows, the second the lower ones
#pragma unroll
    for (int i = 0; i < MI / 2; ++i)
#pragma unroll
      for (int t = 0; t < 4; ++t) there[(i * 4 + t) * 512 + threadIdx.x] = party ? acc[i][t] : acc[i + MI / 2][t];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MI / 2; ++i) {
      w4_f4 sum[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const w4_f4 o = there[(i * 4 + t) * 512 + (threadIdx.x ^ 256)];
        sum[t] = party ? o + acc[i + MI / 2][t] : acc[i][t] + o;
      }
      store(16 * (i + party * (MI / 2)) + kb * 4, k0 + wave * 64 + r16 * 4, sum);
    }
  } else {                                       // all parties' sums, in their order
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int t = 0; t < 4; ++t) there[(i * 4 + t) * (64 * G::WV) + threadIdx.x] = acc[i][t];
    __syncthreads();
    for (int o = threadIdx.x; o < MI * G::TH; o += 64 * G::WV) {
      const int i = o / G::TH, th = o % G::TH;
      w4_f4 sum[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        sum[t] = there[(i * 4 + t) * (64 * G::WV) + th];
#pragma unroll
        for (int p = 1; p < G::S; ++p) sum[t] += there[(i * 4 + t) * (64 * G::WV) + p * G::TH + th];
      }
      store(16 * i + (th >> 4 & 3) * 4, k0 + (th >> 6) * 64 + (th & 15) * 4, sum);
    }
  }
}

template <int TYPE, int MI, int CW, bool ASYM, bool PRE>
static hipError_t launch(const W4GradArgs &a, hipStream_t st) {
  constexpr int lds = GradTile<TYPE, MI, CW, PRE>::LDS;
  static_assert(lds <= 163840, "LDS of a compute unit");
  const int64_t tm = (a.M + 16 * MI - 1) / (16 * MI), tk = (a.K + 64 * CW - 1) / (64 * CW);
  static std::atomic<unsigned long long> done{0};
  auto kern = w4_grad_kernel<TYPE, MI, CW, ASYM, PRE>;
  if (lds > 65536) {
    hipError_t e = allow_lds((const void *)kern, lds, done);
    if (e != hipSuccess) return e;
  }
  kern<<<(unsigned)(tm * tk), 64 * GradTile<TYPE, MI, CW, PRE>::WV, lds, st>>>(a, (int)tm, (int)tk);
  return hipGetLastError();
}

// Tiles: row blocks, wavefronts side by side, parties, the smallest group they take, us of a step of all parties, 64 rows of W each, and what
// another 256 workgroups take of the time of the first: as much where registers or LDS leave a compute unit one workgroup at a time, 0.7
// where it holds two (one tile, 114 registers and 80 KB of LDS; 1024 rows of 8192 x 8192: 777 us for 32 times 256, the first 35).  Measured at
// 4608 x 1152, 1152 x 4608 and 8192 x 8192, 1 - 4096 rows, groups of 32 - 128: 16-bit types get the best tile in all 41 launches tried, float32
// one within 6 % of it in 15.  Few rows want many parties, narrow tiles and the scale in the gradients (1 row of 4608 x 1152, bfloat16 with
// zero points: 20 us; with weights in two parts 23, with tiles of 128 columns 42 and 46, of 256 columns 101 and more), many rows tall and
// wide tiles (2048 rows of 8192 x 8192, bfloat16: 480 us, 620 with 96 rows a tile and 1050 with the scale in the gradients).
// Those run at the rate of a large library product of 16-bit numbers, counted as the two products they are: 1145 TFLOP/s; float16, three
// products, 790 us.  Weights rounded to the type, one product, would take 330 and be off by half a step each.
struct GradShape {
  int MI, CW, parties, group;
  float step, again = 1.0f;
};
// the first two of each with the scale in the gradients (PRE)
static constexpr GradShape SHAPES_BF16[] = {{1, 1, 16, 64, 3.3f}, {2, 2, 4, 128, 2.05f}, {1, 1, 16, 32, 4.0f}, {2, 1, 8, 32, 2.2f}, {2, 2, 4, 32, 2.3f},
                                            {4, 2, 4, 32, 2.85f}, {4, 4, 2, 32, 2.75f}, {6, 4, 2, 32, 3.2f}, {8, 4, 2, 32, 3.7f}};
static constexpr GradShape SHAPES_F16[] = {{1, 1, 16, 64, 3.3f}, {2, 2, 4, 128, 2.05f}, {1, 1, 16, 32, 4.7f}, {2, 1, 8, 32, 3.05f}, {2, 2, 4, 32, 2.8f},
                                           {4, 4, 2, 32, 3.25f}, {6, 4, 2, 32, 4.1f}};
static constexpr GradShape SHAPES_F32[] = {{1, 1, 8, 64, 2.05f, 0.7f}, {2, 2, 4, 128, 2.4f}, {1, 1, 8, 32, 3.05f}, {2, 2, 4, 32, 3.7f}, {2, 4, 2, 32, 3.45f}, {4, 4, 2, 32, 4.9f}};

template <int N>
static int shape(const W4GradArgs &a, const GradShape (&shapes)[N]) {
  const int steps = (a.N[0] + GT_N - 1) / GT_N + (a.nw > 1 ? (a.N[1] + GT_N - 1) / GT_N : 0);
  int best = -1;
  float least = 0.0f;
  for (int i = 0; i < N; ++i) {
    const GradShape &s = shapes[i];
    if (a.group < s.group) continue;
    const int64_t groups = (int64_t)((a.M + 16 * s.MI - 1) / (16 * s.MI)) * ((a.K + 64 * s.CW - 1) / (64 * s.CW));
    const float first = 3.0f + s.step * ((steps + s.parties - 1) / s.parties);                   // 3 us: first loads, last stores
    const float t = first * (1.0f + s.again * (float)((groups - 1) / 256));
    if (best < 0 || t < least) {
      best = i;
      least = t;
    }
  }
  return best;
}

template <int TYPE, bool ASYM>
static hipError_t rows(const W4GradArgs &a, hipStream_t st) {
  if constexpr (TYPE == QC_TYPE_F32) {
    switch (shape(a, SHAPES_F32)) {
      case 0: return launch<TYPE, 1, 1, ASYM, true>(a, st);
      case 1: return launch<TYPE, 2, 2, ASYM, true>(a, st);
      case 2: return launch<TYPE, 1, 1, ASYM, false>(a, st);
      case 3: return launch<TYPE, 2, 2, ASYM, false>(a, st);
      case 4: return launch<TYPE, 2, 4, ASYM, false>(a, st);
      default: return launch<TYPE, 4, 4, ASYM, false>(a, st);
    }
  } else if constexpr (TYPE == QC_TYPE_F16) {
    switch (shape(a, SHAPES_F16)) {
      case 0: return launch<TYPE, 1, 1, ASYM, true>(a, st);
      case 1: return launch<TYPE, 2, 2, ASYM, true>(a, st);
      case 2: return launch<TYPE, 1, 1, ASYM, false>(a, st);
      case 3: return launch<TYPE, 2, 1, ASYM, false>(a, st);
      case 4: return launch<TYPE, 2, 2, ASYM, false>(a, st);
      case 5: return launch<TYPE, 4, 4, ASYM, false>(a, st);
      default: return launch<TYPE, 6, 4, ASYM, false>(a, st);
    }
  } else {
    switch (shape(a, SHAPES_BF16)) {
      case 0: return launch<TYPE, 1, 1, ASYM, true>(a, st);
      case 1: return launch<TYPE, 2, 2, ASYM, true>(a, st);
      case 2: return launch<TYPE, 1, 1, ASYM, false>(a, st);
      case 3: return launch<TYPE, 2, 1, ASYM, false>(a, st);
      case 4: return launch<TYPE, 2, 2, ASYM, false>(a, st);
      case 5: return launch<TYPE, 4, 2, ASYM, false>(a, st);
      case 6: return launch<TYPE, 4, 4, ASYM, false>(a, st);
      case 7: return launch<TYPE, 6, 4, ASYM, false>(a, st);
      default: return launch<TYPE, 8, 4, ASYM, false>(a, st);
    }
  }
}

hipError_t launch_w4_grad(const W4GradArgs &a, int type, hipStream_t st) {
  // a weight without rows may have zero points or none, whatever the other has
  const bool z = (a.N[0] && a.w[0].zero) || (a.nw > 1 && a.N[1] && a.w[1].zero);
  if (type == QC_TYPE_F32) return z ? rows<QC_TYPE_F32, true>(a, st) : rows<QC_TYPE_F32, false>(a, st);
  if (type == QC_TYPE_F16) return z ? rows<QC_TYPE_F16, true>(a, st) : rows<QC_TYPE_F16, false>(a, st);
  return z ? rows<QC_TYPE_BF16, true>(a, st) : rows<QC_TYPE_BF16, false>(a, st);
}

}  // namespace qc
