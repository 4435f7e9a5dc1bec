// Products with 4-bit weights of groups, many rows: linear layers, the gated block and its inner gradients.
//
// A workgroup makes 16 MI rows by 256 columns of weights (the gated block: 128 columns of each of its two), its four wavefronts side by
// side along the columns, so that no weight is expanded twice in a workgroup.  The weights go from memory to registers as
// packed codes, 128 inputs at a time and one chunk ahead, and are expanded there; the activations go through LDS, which all four
// wavefronts read.  The products of one group are summed apart and scaled in float32 as they are added: the codes are exact.
//
// What bounds it is the issue of vector instructions: a chunk of 80 rows and 64 columns in groups of 128 (bfloat16) is 80 matrix
// instructions of 16 clocks and 354 others of 4 (494 with zero points), most of them expansion (1.6 a weight; 2.7) and scaling (1 for each
// result and group), so two wavefronts a SIMD must share 1736 clocks each while the matrix unit needs 1280.  8192 x 8192 x 8192 bfloat16 runs at 960 TFLOP/s
// (the library's product of 16-bit matrices reaches 1140), 8-bit inputs at 1490 TOP/s (1715).  Scaling the weights first would save
// the second part and round every weight.  More row blocks a tile amortise the expansion, but a register in scratch memory makes the
// next wait one for every load in flight: 8 row blocks of 16-bit types spilled 11 registers and took 98 us at 4096 x 4608 x 1152 where 5
// take 65.
#include "w4_common.h"

namespace qc {

constexpr int TILE_N = 256, TILE_K = 128;

template <int TYPE>
constexpr int tile_row = TYPE == QC_TYPE_I8 ? 128 : 256;                 // bytes of a row of one plane of activations in LDS
template <int TYPE>
constexpr int tile_planes = TYPE == QC_TYPE_F32 ? 3 : 1;

// 16-byte unit u of row r: 16 rows of one unit lie in 16 different slots of 256 bytes
template <int TYPE>
__device__ __forceinline__ int tile_slot(int r, int u) {
  return TYPE == QC_TYPE_I8 ? r * 128 + ((u ^ ((r >> 1) & 7)) << 4) : r * 256 + ((u ^ (r & 15)) << 4);
}

// Activations of one chunk on their way from memory to LDS, in units of 16 bytes.  float32 goes through registers, where it is split;
// the other types go to LDS directly: a wavefront's load fills 1024 bytes in the order of its lanes, so the lane that fills a slot
// asks for the unit that belongs there.
template <int TYPE, int MI>
struct TileLoad {
  static constexpr int ES = TYPE == QC_TYPE_F32 ? 4 : TYPE == QC_TYPE_I8 ? 1 : 2;
  static constexpr int UR = TILE_K * ES / 16;                            // units a row
  static constexpr int NU = 16 * MI * UR / 256;
  static_assert(16 * MI * UR % 256 == 0, "whole loads");
  w4_u4 v[TYPE == QC_TYPE_F32 ? NU : 1];
  // x: the tile's first row; `last`: the last row of it that exists.  The offsets are formed again each time, not kept.
  __device__ __forceinline__ void load(const char *x, int row_bytes, int last, int k0, int K, char *lds) {
    asm volatile("" : "+s"(last));
    const bool whole = k0 + TILE_K <= K;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int t = threadIdx.x + 256 * i, r = t / UR;
      const int u = TYPE == QC_TYPE_F32 ? t % UR : t % UR ^ (TYPE == QC_TYPE_I8 ? (r >> 1) & 7 : r & 15);
      const int k = k0 + u * (16 / ES);
      const char *from = x + (unsigned)(min(r, last) * row_bytes + k * ES);
      if constexpr (TYPE == QC_TYPE_F32) {
        if (whole) {
          v[i] = *(const w4_u4 *)from;
        } else {
          v[i] = w4_u4{};
          if (k < K) v[i] = *(const w4_u4 *)from;
        }
      } else {
        char *to = lds + (threadIdx.x >> 6) * 1024 + i * 4096;
        if (whole || k < K)
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
        else
          *(w4_u4 *)(to + (threadIdx.x & 63) * 16) = w4_u4{};
      }
    }
  }
  __device__ __forceinline__ void store(char *lds) const {
    if constexpr (TYPE == QC_TYPE_F32) {
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        const int t = threadIdx.x + 256 * i, r = t / UR, u = t % UR;
        float p[4][3];                                                   // four values: half a unit of each plane
#pragma unroll
        for (int e = 0; e < 4; ++e) w4_split(__builtin_bit_cast(w4_f4, v[i])[e], p[e]);
#pragma unroll
        for (int s = 0; s < 3; ++s)
          *(w4_u2 *)(lds + s * 16 * MI * 256 + tile_slot<TYPE>(r, u >> 1) + (u & 1) * 8) = w4_u2{w4_pack_bf16(p[0][s], p[1][s]), w4_pack_bf16(p[2][s], p[3][s])};
      }
    }
  }
};

template <int TYPE, int MI>
constexpr int tile_buffer = 16 * MI * tile_row<TYPE> * tile_planes<TYPE>;
template <int TYPE, int MI>
constexpr int tile_lds = 2 * tile_buffer<TYPE, MI> > 4 * 16 * 68 * 4 ? 2 * tile_buffer<TYPE, MI> : 4 * 16 * 68 * 4;

// UK: inputs whose weights a wavefront holds expanded, a group or half of one
template <int TYPE, int GC, int MI, int OP, bool ASYM, int UK>
__global__ __launch_bounds__(256, 2) void w4_tile_kernel(W4Args a, int tm, int tn) {
  using F = FragOf<TYPE>;
  using T = typename W4Mem<TYPE>::T;
  constexpr int BUF = tile_buffer<TYPE, MI>, P = tile_planes<TYPE>;
  constexpr bool TWO = OP != W4_LINEAR;
  constexpr int LN = TWO ? 128 : 256, WN = LN / 4;                       // columns of the result: workgroup, wavefront
  constexpr bool K64 = TYPE == QC_TYPE_I8 && GC < 4;                     // matrix instructions of 64 inputs, not 32
  constexpr int UJ = UK / (K64 ? 64 : 32);                               // of them in a unit
  constexpr int U = 128 / UK, UG = U / GC;                               // units in a chunk, in a group
  extern __shared__ __align__(16) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, kb = lane >> 4;
  int mi, ni;
  tile_at(blockIdx.x, gridDim.x, tm, tn, 8, mi, ni);
  const int m0 = mi * 16 * MI, n0 = ni * LN + wave * WN;
  const int KB = a.K / 2, chunks = (a.K + 127) / 128;
  const int row_bytes = (int)a.ldx * TileLoad<TYPE, MI>::ES, last = a.M - 1 - m0;
  const char *x0 = (const char *)a.x + (int64_t)m0 * row_bytes;

  // block j of a wavefront: its matrix and its column in this lane.  Rows beyond the last read as zero.
  const auto wj = [&](int j) -> const W4Mat & { return a.w[TWO ? j >> 1 : 0]; };
  constexpr int MATS = TWO ? 2 : 1;
  __amdgpu_buffer_rsrc_t qb[MATS], sb[MATS], zb_[MATS];
  const int first = ni * LN, rest = a.N - first;
#pragma unroll
  for (int w = 0; w < MATS; ++w) {
    qb[w] = w4_buffer(a.w[w].q + (size_t)first * KB, (int64_t)rest * KB);
    sb[w] = w4_buffer(a.w[w].scale + (size_t)first * a.G, (int64_t)rest * a.G * 4);
    if (ASYM) zb_[w] = w4_buffer(a.w[w].zero + (size_t)first * a.G, (int64_t)rest * a.G);
  }
  const int nl = wave * WN + (lane >> 2), from = w4_from(lane), fromg = r16 * 16;

  w4_f4 y[MI][4] = {};
  TileLoad<TYPE, MI> next;
  w4_u4 q[4];
  unsigned s4[4], z4[4];                                                 // of four groups, in four neighbouring lanes
  constexpr int PER = 4 / GC;                                            // chunks to four groups
  const auto fetch = [&](int c) {
    int n = nl;
    asm volatile("" : "+v"(n));                                          // offsets are formed again each time, not kept
#pragma unroll
    for (int j = 0; j < 4; ++j)
      q[j] = __builtin_bit_cast(w4_u4, __builtin_amdgcn_raw_buffer_load_b128(qb[TWO ? j >> 1 : 0], (n + (TWO ? j & 1 : j) * 16) * KB + (lane & 3) * 16, c * 64, 0));
    if (c % PER == 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = (n + (TWO ? j & 1 : j) * 16) * a.G + (lane & 3);
        s4[j] = __builtin_amdgcn_raw_buffer_load_b32(sb[TWO ? j >> 1 : 0], at * 4, c * GC * 4, 0);
        if (ASYM) z4[j] = __builtin_amdgcn_raw_buffer_load_b8(zb_[TWO ? j >> 1 : 0], at, c * GC, 0);
      }
    }
  };
  next.load(x0, row_bytes, last, 0, a.K, lds);
  fetch(0);
  next.store(lds);
  __syncthreads();
  for (int c = 0; c < chunks; ++c) {
    const char *cur = lds + (c & 1) * BUF;
    float sc[4][GC], z16[4][GC];
    unsigned zb[4][GC];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int e = 0; e < 4; ++e) q[j][e] = w4_pull(q[j][e], from);
      if (!K64) w4_transpose(q[j]);
      else if (GC == 2) w4_swap32(q[j]);
#pragma unroll
      for (int g = 0; g < GC; ++g) {
        const int at = fromg + (c % PER * GC + g) * 4;
        const float s = __builtin_bit_cast(float, w4_pull(s4[j], at));
        // beyond the last group nothing is added, whatever was read there
        sc[j][g] = c * GC + g < a.G ? s * (TYPE == QC_TYPE_I8 ? 1.0f : 16.0f) : 0.0f;
        const int z = ASYM ? (int)w4_pull(z4[j], at) : 8;
        z16[j][g] = (float)(z - 8) * 0.0625f;
        zb[j][g] = (unsigned)z * 0x01010101u;
      }
    }
    if (c + 1 < chunks) next.load(x0, row_bytes, last, (c + 1) * 128, a.K, lds + ((c + 1) & 1) * BUF);
#pragma unroll
    for (int un = 0; un < U; ++un) {
      const int g = un / UG;
      w4_u4 wf[UJ][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(q[j]));         // nothing of a unit is expanded ahead of its turn
#pragma unroll
      for (int t = 0; t < UJ; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int jj = un * UJ + t;
          if constexpr (K64) {
            const w4_u2 lo = F::template weights<ASYM>(q[j][2 * jj], 0.0f, zb[j][g]), hi = F::template weights<ASYM>(q[j][2 * jj + 1], 0.0f, zb[j][g]);
            wf[t][j] = w4_u4{lo[0], lo[1], hi[0], hi[1]};
          } else if constexpr (TYPE == QC_TYPE_I8) {
            const w4_u2 v = F::template weights<ASYM>(q[j][jj], 0.0f, zb[j][g]);
            wf[t][j] = w4_u4{v[0], v[1], 0, 0};
          } else {
            wf[t][j] = __builtin_bit_cast(w4_u4, F::template weights<ASYM>(q[j][jj], z16[j][g], 0));
          }
        }
      // the next chunk's codes, now that this one's are expanded
      if (un == U - 1 && c + 1 < chunks) fetch(c + 1);
      // The products of one row block run while those of the one before are scaled; operands are read RING - 1 products ahead
      typedef typename std::conditional<K64, w4_i4, typename F::X>::type XF;
      constexpr int RING = TYPE == QC_TYPE_I8 ? 2 : 3;
      XF xf[RING][P];
      const auto read = [&](int step) {
        const int i = step / UJ, jj = un * UJ + step % UJ;
        const int u = !K64 ? (TYPE == QC_TYPE_I8 ? jj * 2 + (kb >> 1) : jj * 4 + kb) : GC == 1 ? kb * 2 + jj : jj * 4 + ((kb & 1) << 1 | kb >> 1);
#pragma unroll
        for (int p = 0; p < P; ++p)
          xf[step % RING][p] = *(const XF *)(cur + p * 16 * MI * 256 + tile_slot<TYPE>(16 * i + r16, u) + (TYPE == QC_TYPE_I8 && !K64 ? (kb & 1) * 8 : 0));
      };
      typename F::Acc acc[2][4];
#pragma unroll
      for (int t = 0; t + 1 < RING; ++t) read(t);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i <= MI; ++i) {
        if (i < MI) {
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i & 1][j] = typename F::Acc{};
#pragma unroll
          for (int t = 0; t < UJ; ++t) {
            const int step = i * UJ + t;
            if (step + RING - 1 < MI * UJ) read(step + RING - 1);
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const XF x = xf[step % RING][p];
                typename F::Acc &to = acc[i & 1][j];
                if constexpr (K64) to = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, __builtin_bit_cast(w4_i4, wf[t][j]), to, 0, 0, 0);
                else if constexpr (TYPE == QC_TYPE_I8) to = F::mma(x, w4_u2{wf[t][j][0], wf[t][j][1]}, to);
                else to = F::mma(x, __builtin_bit_cast(typename F::W, wf[t][j]), to);
              }
          }
        }
        if (i > 0) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) y[i - 1][j][e] += sc[j][g] * (float)acc[(i - 1) & 1][j][e];
#pragma unroll
          for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(y[i - 1][j]));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (c + 1 < chunks) next.store(lds + ((c + 1) & 1) * BUF);
    __syncthreads();
  }

  // Results of 16 rows at a time are turned through the wavefront's own part of LDS, so that a store covers neighbouring columns
  constexpr int SR = WN + 4, LR = WN / 4;                                // floats a staged row; lanes that store a row
  float *stage = (float *)lds + wave * (16 * 68);
  float bias[4], sum[4];
  int nj[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) nj[j] = min(n0 + (TWO ? j & 1 : j) * 16 + r16, a.N - 1);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    bias[j] = wj(j).bias ? wj(j).bias[nj[j]] : 0.0f;
    if (TYPE == QC_TYPE_I8) sum[j] = (float)a.zp * wj(j).sum[nj[j]];
  }
  const auto value = [&](int i, int j, int e) {
    float v = y[i][j][e];
    if (TYPE == QC_TYPE_I8) v = a.xs * (v - sum[j]);
    return v + bias[j];
  };
  const int col = n0 + lane % LR * 4;
  const auto put4 = [&](void *out, int64_t ld, int row, w4_f4 v) {
    T *o = (T *)out + (int64_t)row * ld + col;
    typedef T T4 __attribute__((ext_vector_type(4)));
    if (col + 4 <= a.N && (uintptr_t)o % sizeof(T4) == 0) {
      T4 t;
#pragma unroll
      for (int e = 0; e < 4; ++e) t[e] = W4Mem<TYPE>::put(v[e]);
      *(T4 *)o = t;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < a.N) o[e] = W4Mem<TYPE>::put(v[e]);
    }
  };
  const auto turn = [&]() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    constexpr int OUTS = OP == W4_GATED_GRAD ? 2 : 1;
    w4_f4 v[OUTS][WN / 16];
#pragma unroll
    for (int j = 0; j < WN / 16; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[0][j][e] = value(i, j, e);
        if constexpr (TWO) {
          float d;
          const float act = w4_act(a.act, v[0][j][e], d), up = value(i, j + 2, e);
          v[0][j][e] = OP == W4_GATED ? act * up : up * d;
          if constexpr (OP == W4_GATED_GRAD) v[1][j][e] = act;
        }
      }
#pragma unroll
    for (int o = 0; o < OUTS; ++o) {
#pragma unroll
      for (int j = 0; j < WN / 16; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) stage[(kb * 4 + e) * SR + j * 16 + r16] = v[o][j][e];
      turn();
#pragma unroll
      for (int rr = 0; rr < 16 * LR / 64; ++rr) {
        const int r = rr * (64 / LR) + lane / LR, row = m0 + i * 16 + r;
        w4_f4 t = *(const w4_f4 *)(stage + r * SR + lane % LR * 4);
        if (row < a.M) {
          if constexpr (OP == W4_GATED_GRAD) {
            const T *dh = (const T *)a.dh + (int64_t)row * a.lddh + col;
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] *= col + e < a.N ? W4Mem<TYPE>::get(dh[e]) : 0.0f;
          }
          put4(o ? a.y2 : a.y, a.ldy, row, t);
        }
      }
      turn();
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// row blocks of a tile: as many as 256 registers hold without spilling, float32 with zero points apart, which keeps 1 - 5 of them in scratch
// memory (seven kernels)
static constexpr int tile_mi_of(int type, int group) { return type == QC_TYPE_F32 ? 4 : type == QC_TYPE_I8 ? 8 : group == 128 ? 5 : 6; }
int w4_tile_rows(const W4Args &a, int type) { return 16 * tile_mi_of(type, a.group); }

template <int TYPE, int GC, int MI, int OP, bool ASYM>
static hipError_t tile_launch(const W4Args &a, hipStream_t st) {
  constexpr int lds = tile_lds<TYPE, MI>, UK = TYPE == QC_TYPE_F32 ? std::min(128 / GC, 64) : 128 / GC;
  const int tm = (a.M + 16 * MI - 1) / (16 * MI), tn = (a.N + (OP == W4_LINEAR ? 255 : 127)) / (OP == W4_LINEAR ? 256 : 128);
  static std::atomic<unsigned long long> done{0};
  auto kern = w4_tile_kernel<TYPE, GC, MI, OP, ASYM, UK>;
  if (lds > 65536) {
    hipError_t e = allow_lds((const void *)kern, lds, done);
    if (e != hipSuccess) return e;
  }
  kern<<<tm * tn, 256, lds, st>>>(a, tm, tn);
  return hipGetLastError();
}

template <int TYPE, int GC, int OP>
static hipError_t tile_mi(const W4Args &a, hipStream_t st) {
  constexpr int MI = tile_mi_of(TYPE, 128 / GC);
  return a.w[0].zero ? tile_launch<TYPE, GC, MI, OP, true>(a, st) : tile_launch<TYPE, GC, MI, OP, false>(a, st);
}

template <int TYPE, int OP>
static hipError_t tile_gc(const W4Args &a, hipStream_t st) {
  if (a.group == 128) return tile_mi<TYPE, 1, OP>(a, st);
  if (a.group == 64) return tile_mi<TYPE, 2, OP>(a, st);
  return tile_mi<TYPE, 4, OP>(a, st);
}

template <int TYPE>
static hipError_t tile_op(const W4Args &a, int op, hipStream_t st) {
  if (op == W4_LINEAR) return tile_gc<TYPE, W4_LINEAR>(a, st);
  if (op == W4_GATED) return tile_gc<TYPE, W4_GATED>(a, st);
  if constexpr (TYPE == QC_TYPE_I8) return hipErrorInvalidValue;
  else return tile_gc<TYPE, W4_GATED_GRAD>(a, st);
}

hipError_t launch_w4_tile(const W4Args &a, int type, int op, hipStream_t st) {
  if (type == QC_TYPE_F32) return tile_op<QC_TYPE_F32>(a, op, st);
  if (type == QC_TYPE_F16) return tile_op<QC_TYPE_F16>(a, op, st);
  if (type == QC_TYPE_BF16) return tile_op<QC_TYPE_BF16>(a, op, st);
  return tile_op<QC_TYPE_I8>(a, op, st);
}

}  // namespace qc
