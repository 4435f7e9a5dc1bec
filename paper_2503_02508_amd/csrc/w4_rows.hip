// Products with 4-bit weights of groups, a few rows at a time: linear layers, the gated block and its inner gradients.
//
// A workgroup makes 16 NT columns (of each of its matrices) of up to 16 MT rows.  Its wavefronts take the chunks of 128 inputs in turn,
// so that together they read runs of their weight rows; each lane reads 16 bytes (32 codes) of one row, the four lanes of a row
// exchange them (v_permlane) so that a matrix instruction covers 32 consecutive inputs, which lie in one group, and every group's
// product is scaled in float32 as it is added: the codes themselves are exact in every type, and float32 inputs are three bfloat16
// numbers each.  The wavefronts' sums are added in LDS in wavefront order.
//
// One row takes the weights' bytes and the instructions that expand them, and fills neither limit: 28672 x 8192 float16 in groups of 64
// with zero points takes 42 us, 3.2 TB/s of codes and scales, its SIMDs issuing vector instructions 64 % of the time (8-bit inputs, which
// need fewest, 4.4 TB/s without zero points; a large copy reads and writes 5.2).  Sixteen neighbouring lanes are looked up in the cache together, a
// line a clock: with lanes in the products' order, 16 rows in each look-up, the same took 80 us, and 16 rows of 8192 x 8192
// bfloat16 29 us instead of 16.  Loads that ran further ahead, whole cache lines a row and scales asked for a pair of chunks earlier
// changed nothing or cost registers.
#include "w4_common.h"

namespace qc {

template <int TYPE>
struct RowsX {                                                           // a lane's 8 inputs of a product
  using X = typename std::conditional<TYPE == QC_TYPE_F32, w4_f8, typename FragOf<TYPE>::X>::type;
  static constexpr int ES = TYPE == QC_TYPE_F32 ? 4 : TYPE == QC_TYPE_I8 ? 1 : 2;
  static __device__ __forceinline__ X load(__amdgpu_buffer_rsrc_t buf, unsigned at, int chunk) {
    if constexpr (TYPE == QC_TYPE_I8) {
      return __builtin_bit_cast(w4_u2, __builtin_amdgcn_raw_buffer_load_b64(buf, at, chunk, 0));
    } else if constexpr (TYPE == QC_TYPE_F32) {
      const w4_f4 a = __builtin_bit_cast(w4_f4, __builtin_amdgcn_raw_buffer_load_b128(buf, at, chunk, 0));
      const w4_f4 b = __builtin_bit_cast(w4_f4, __builtin_amdgcn_raw_buffer_load_b128(buf, at + 16, chunk, 0));
      return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      return __builtin_bit_cast(X, __builtin_amdgcn_raw_buffer_load_b128(buf, at, chunk, 0));
    }
  }
};

// wavefronts of a workgroup at most: 16 where 128 registers hold a wavefront's tile
constexpr int rows_most(int type, int MT, int NW) { return type == QC_TYPE_F32 || MT * NW > 2 ? 8 : 16; }

// GC: groups in a chunk of 128 inputs; MT: tiles of 16 rows; NT: of 16 columns (of each matrix)
// PULL: inputs are loaded like weight rows, four lanes a row, and pulled into place (a few rows cost less as they are)
template <int TYPE, int GC, int MT, int NT, int OP, bool ASYM, bool PULL>
__global__ __launch_bounds__(64 * rows_most(TYPE, MT, NT * (OP == W4_LINEAR ? 1 : 2))) void w4_rows_kernel(W4Args a) {
  using F = FragOf<TYPE>;
  using T = typename W4Mem<TYPE>::T;
  constexpr int P = TYPE == QC_TYPE_F32 ? 3 : 1, ES = RowsX<TYPE>::ES, MATS = OP == W4_LINEAR ? 1 : 2, NW = MATS * NT;
  constexpr int AHEAD = MT == 1 ? 2 : 1;         // chunks that registers hold: with two the next one is asked for before this one is used
  constexpr bool LATE = TYPE == QC_TYPE_F32 && MT > 1;                  // inputs a product ahead only: a chunk's are 32 MT registers
  constexpr int XJ = LATE ? 2 : 4;
  extern __shared__ float red[];                 // [wavefronts][NW][MT][64][4]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int r16 = lane & 15, kb = lane >> 4;
  const int ntn = (a.N + 16 * NT - 1) / (16 * NT), n0 = (int)(blockIdx.x % ntn) * (16 * NT), m0 = (int)(blockIdx.x / ntn) * (16 * MT);
  const int KB = a.K / 2, chunks = (a.K + 127) / 128, rest = a.N - n0;
  const __amdgpu_buffer_rsrc_t xb = w4_buffer((const char *)a.x + (int64_t)m0 * a.ldx * ES, ((int64_t)(a.M - 1 - m0) * a.ldx + a.K) * ES);
  __amdgpu_buffer_rsrc_t qb[MATS], sb[MATS], zb[MATS];
#pragma unroll
  for (int w = 0; w < MATS; ++w) {
    qb[w] = w4_buffer(a.w[w].q + (size_t)n0 * KB, (int64_t)rest * KB);
    sb[w] = w4_buffer(a.w[w].scale + (size_t)n0 * a.G, (int64_t)rest * a.G * 4);
    if (ASYM) zb[w] = w4_buffer(a.w[w].zero + (size_t)n0 * a.G, (int64_t)rest * a.G);
  }
  // offsets of the lane; a chunk's own offset is uniform
  unsigned xat[MT], qat[NT], gat[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) xat[i] = (unsigned)(16 * i + (PULL ? lane >> 2 : r16)) * (unsigned)a.ldx * ES + (PULL ? lane & 3 : kb) * 8 * ES;
#pragma unroll
  for (int w = 0; w < NT; ++w) {
    qat[w] = (unsigned)((16 * w + (lane >> 2)) * KB + (lane & 3) * 16);
    gat[w] = (unsigned)((16 * w + (lane >> 2)) * a.G + (lane & 3));
  }
  const int from = w4_from(lane), fromg = r16 * 16;                     // four groups of a row lie in four neighbouring lanes

  struct Slot {
    w4_u4 q[NW];
    typename RowsX<TYPE>::X x[MT][XJ];
  } slot[AHEAD];
  constexpr int PER = 4 / GC;                    // chunks to four groups
  unsigned s4[NW], z4[NW];
  w4_f4 y[NW][MT] = {};
  const auto fetch_x = [&](Slot &f, int c, int j) {
    const bool in = c * 128 + j * 32 + (PULL ? lane & 3 : kb) * 8 < a.K;
#pragma unroll
    for (int i = 0; i < MT; ++i) f.x[i][j % XJ] = RowsX<TYPE>::load(xb, in ? xat[i] + j * 32 * ES : W4_NOWHERE, c * 128 * ES);
  };
  const auto fetch = [&](Slot &f, int c) {
#pragma unroll
    for (int w = 0; w < NW; ++w) f.q[w] = __builtin_bit_cast(w4_u4, __builtin_amdgcn_raw_buffer_load_b128(qb[w / NT], qat[w % NT], c * 64, 0));
    if ((c + 1) * 128 <= a.K) {
#pragma unroll
      for (int j = 0; j < (LATE ? 1 : 4); ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) f.x[i][j] = RowsX<TYPE>::load(xb, xat[i] + j * 32 * ES, c * 128 * ES);
    } else {                                     // a row's end is not the buffer's
#pragma unroll
      for (int j = 0; j < (LATE ? 1 : 4); ++j) fetch_x(f, c, j);
    }
  };
  const auto fetch4 = [&](int c) {               // scales and zero points of the four groups that chunk c's are among
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      s4[w] = __builtin_amdgcn_raw_buffer_load_b32(sb[w / NT], gat[w % NT] * 4, (c & -PER) * GC * 4, 0);
      if (ASYM) z4[w] = __builtin_amdgcn_raw_buffer_load_b8(zb[w / NT], gat[w % NT], (c & -PER) * GC, 0);
    }
  };
  const auto use = [&](Slot &f, int c) {
    float sc[NW][GC];
    int z[NW][GC];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
#pragma unroll
      for (int e = 0; e < 4; ++e) f.q[w][e] = w4_pull(f.q[w][e], from);
#pragma unroll
      for (int g = 0; g < GC; ++g) {
        const int at = fromg + ((c & (PER - 1)) * GC + g) * 4;
        const float s = __builtin_bit_cast(float, w4_pull(s4[w], at));
        // beyond the last group nothing is added, whatever was read there
        sc[w][g] = c * GC + g < a.G ? s * (TYPE == QC_TYPE_I8 ? 1.0f : 16.0f) : 0.0f;
        z[w][g] = ASYM ? (int)w4_pull(z4[w], at) : 8;
      }
      w4_transpose(f.q[w]);
    }
#pragma unroll
    for (int g = 0; g < GC; ++g) {
      typename F::Acc acc[NW][MT] = {};
#pragma unroll
      for (int t = 0; t < 4 / GC; ++t) {
        const int j = g * (4 / GC) + t;
        if (LATE && j < 3) fetch_x(f, c, j + 1);
        typename F::W wf[NW];
#pragma unroll
        for (int w = 0; w < NW; ++w)
          wf[w] = F::template weights<ASYM>(f.q[w][j], ASYM ? (float)(z[w][g] - 8) * 0.0625f : 0.0f, ASYM ? (unsigned)z[w][g] * 0x01010101u : 0u);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          typename RowsX<TYPE>::X x = f.x[i][j % XJ];
          if (PULL) {
            typedef unsigned XU __attribute__((ext_vector_type(2 * ES)));
            XU v = __builtin_bit_cast(XU, x);
#pragma unroll
            for (int e = 0; e < 2 * ES; ++e) v[e] = w4_pull(v[e], from);
            x = __builtin_bit_cast(typename RowsX<TYPE>::X, v);
          }
          typename F::X xf[P];
          if constexpr (TYPE == QC_TYPE_F32) {
            float p[8][3];
#pragma unroll
            for (int e = 0; e < 8; ++e) w4_split(x[e], p[e]);
#pragma unroll
            for (int s = 0; s < 3; ++s)
              xf[s] = __builtin_bit_cast(w4_bf8, w4_u4{w4_pack_bf16(p[0][s], p[1][s]), w4_pack_bf16(p[2][s], p[3][s]),
                                                       w4_pack_bf16(p[4][s], p[5][s]), w4_pack_bf16(p[6][s], p[7][s])});
          } else {
            xf[0] = x;
          }
#pragma unroll
          for (int p = 0; p < P; ++p)
#pragma unroll
            for (int w = 0; w < NW; ++w) acc[w][i] = F::mma(xf[p], wf[w], acc[w][i]);
        }
      }
#pragma unroll
      for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) y[w][i][e] += sc[w][g] * (float)acc[w][i][e];
    }
  };
  // Wavefronts take pairs of chunks, 128 bytes of every weight row: whole cache lines
  if constexpr (AHEAD == 2) {
    // four groups serve the pair, or (groups of 32) each chunk its own four
    const int step = 2 * waves;
    int c = 2 * wave;
    if (c < chunks) {
      fetch4(c);
      fetch(slot[0], c);
    }
    if (c + 1 < chunks) fetch(slot[1], c + 1);
    for (; c < chunks; c += step) {
      use(slot[0], c);
      if (GC == 4 && c + 1 < chunks) fetch4(c + 1);
      if (c + step < chunks) fetch(slot[0], c + step);
      if (c + 1 < chunks) use(slot[1], c + 1);
      if (c + step < chunks) fetch4(c + step);
      if (c + 1 + step < chunks) fetch(slot[1], c + 1 + step);
    }
  } else {
    for (int c = wave; c < chunks; c += waves) {
      fetch4(c);
      fetch(slot[0], c);
      use(slot[0], c);
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
  for (int o = threadIdx.x; o < TILE * NT; o += blockDim.x) {
    const int nt = o / TILE, in = o % TILE, m = m0 + in / 16, col = n0 + nt * 16 + in % 16;
    if (m >= a.M || col >= a.N) continue;
    float v[MATS];
#pragma unroll
    for (int w = 0; w < MATS; ++w) {
      const float *r = red + (w * NT + nt) * TILE + in;
      float t = r[0];
      for (int p = 1; p < waves; ++p) t += r[p * NW * TILE];
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

// wavefronts of a workgroup: up to 16 (8 of the larger tiles), no more than chunks (pairs of chunks) and than fill the chip
static int rows_waves(const W4Args &a, int type, int MT, int NW, int groups) {
  const int chunks = (a.K + 127) / 128, turns = MT == 1 ? (chunks + 1) / 2 : chunks, most = rows_most(type, MT, NW);
  int waves = 1;
  while (waves < most && waves < turns && groups * waves < 4096) waves *= 2;
  return waves;
}

template <int TYPE, int GC, int MT, int NW, int OP, bool PULL>
static hipError_t rows_launch(const W4Args &a, hipStream_t st) {
  constexpr int NT = NW / (OP == W4_LINEAR ? 1 : 2);
  const int ntn = (a.N + 16 * NT - 1) / (16 * NT), ntm = (a.M + 16 * MT - 1) / (16 * MT), waves = rows_waves(a, TYPE, MT, NW, ntn * ntm);
  const int lds = waves * NW * MT * 1024;
  static std::atomic<unsigned long long> done[2];
  auto kern = a.w[0].zero ? w4_rows_kernel<TYPE, GC, MT, NT, OP, true, PULL> : w4_rows_kernel<TYPE, GC, MT, NT, OP, false, PULL>;
  if (lds > 65536) {
    hipError_t e = allow_lds((const void *)kern, lds, done[a.w[0].zero != nullptr]);
    if (e != hipSuccess) return e;
  }
  kern<<<(unsigned)ntn * (unsigned)ntm, waves * 64, lds, st>>>(a);
  return hipGetLastError();
}

// Tiles of this kernel, MT row blocks by NW column blocks of both matrices, and what a step (a chunk of every wavefront of a workgroup)
// of theirs takes in us: alone, and for each 8 or 16 wavefronts (rows_most) that a compute unit has to run.  And what a chunk takes the
// kernel of large tiles (w4_tile.hip), alone and with every compute unit holding as many of its workgroups as fit, `full_at` in all.
// Measured with groups of 128 at 4608 x 1152, 1152 x 4608 and 8192 x 8192, 1 - 512 rows and, the large tiles, 4096 and 8192; smaller groups
// are taken to cost their kernels alike.  A launch takes what comes to least; against the best there that loses up to a fifth, and mostly
// nothing.
struct RowsTile {
  int MT, NW;
  float alone, full;
};
struct RowsCosts {
  int tiles;
  RowsTile tile[5];
  float alone, full;
  int full_at;
};
static constexpr RowsCosts COSTS_16 = {5, {{1, 1, 0.7f, 1.2f}, {1, 2, 0.9f, 2.0f}, {2, 2, 1.9f, 1.4f}, {4, 2, 2.3f, 2.6f}, {4, 4, 3.7f, 4.0f}}, 2.0f, 2.8f, 512};
static constexpr RowsCosts COSTS_F32 = {4, {{1, 1, 1.5f, 1.75f}, {1, 2, 1.8f, 2.1f}, {2, 2, 3.8f, 3.4f}, {4, 2, 6.2f, 6.6f}}, 3.4f, 3.9f, 256};
static constexpr RowsCosts COSTS_I8 = {5, {{1, 1, 0.7f, 0.95f}, {1, 2, 0.9f, 1.6f}, {2, 2, 1.3f, 1.15f}, {4, 2, 1.9f, 2.0f}, {4, 4, 3.2f, 3.3f}}, 1.8f, 2.9f, 512};
static const RowsCosts &rows_costs(int type) { return type == QC_TYPE_F32 ? COSTS_F32 : type == QC_TYPE_I8 ? COSTS_I8 : COSTS_16; }

static float rows_time(const W4Args &a, int type, int op, const RowsTile &t) {
  const int cols = 16 * t.NW / (op == W4_LINEAR ? 1 : 2), groups = ((a.N + cols - 1) / cols) * ((a.M + 16 * t.MT - 1) / (16 * t.MT));
  const int waves = rows_waves(a, type, t.MT, t.NW, groups), chunks = (a.K + 127) / 128, steps = (chunks + waves - 1) / waves;
  return steps * std::max(t.alone, t.full * groups * waves / (256.0f * rows_most(type, t.MT, t.NW)));
}

static int rows_tile(const W4Args &a, int type, int op, float &time) {
  const RowsCosts &c = rows_costs(type);
  int best = -1;
  for (int i = op == W4_LINEAR ? 0 : 1; i < c.tiles; ++i) {              // the gated block has two column blocks at least
    const float t = rows_time(a, type, op, c.tile[i]);
    if (best < 0 || t < time) {
      best = i;
      time = t;
    }
  }
  return best;
}

bool w4_tile_pays(const W4Args &a, int type, int op) {
  float rows;
  rows_tile(a, type, op, rows);
  const RowsCosts &c = rows_costs(type);
  const int tr = w4_tile_rows(a, type), tc = op == W4_LINEAR ? 256 : 128;
  const float tiles = (float)((a.M + tr - 1) / tr) * (float)((a.N + tc - 1) / tc);
  return (a.K + 127) / 128 * std::max(c.alone, c.full * tiles / c.full_at) < rows;
}

template <int TYPE, int GC, int OP>
static hipError_t rows_mt(const W4Args &a, hipStream_t st) {
  float time;
  const int i = rows_tile(a, TYPE, OP, time);
  const bool pull = a.M > 4;       // 8192 x 8192, bfloat16: 11.7 us without and 12.1 with at 4 rows, 12.8 and 12.6 at 8
  if constexpr (OP == W4_LINEAR)
    if (i == 0) return pull ? rows_launch<TYPE, GC, 1, 1, OP, true>(a, st) : rows_launch<TYPE, GC, 1, 1, OP, false>(a, st);
  if (i == 1) return pull ? rows_launch<TYPE, GC, 1, 2, OP, true>(a, st) : rows_launch<TYPE, GC, 1, 2, OP, false>(a, st);
  if (i == 2) return rows_launch<TYPE, GC, 2, 2, OP, true>(a, st);
  if constexpr (TYPE != QC_TYPE_F32)
    if (i == 4) return rows_launch<TYPE, GC, 4, 4, OP, true>(a, st);
  return rows_launch<TYPE, GC, 4, 2, OP, true>(a, st);
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
