// Products of the 8-bit layers with a scale for each token, many rows: y = x W^T and, on the byte planes of gradients, dx = dy W.
//
// A workgroup makes a tile of the result; slabs of BK bytes of the summed axis go from memory straight to LDS, ST of them in a ring, one
// barrier a slab.  Wavefronts read 16 x 64 operands of v_mfma_i32_16x16x64_i8 from there.  The weights' rows run along the summed axis in the
// forward product; in the gradient they run across it, and ds_read_b64_tr_b8 turns 8 rows x 16 bytes on their way to the registers.  Operands
// are exchanged (weights first), so that a lane holds four neighbouring columns of one row; the epilogue turns 16 rows at a time through the
// wavefront's own part of LDS and writes whole cache lines.
#include "t8_product.h"

namespace qc {

template <int BK, int ST, int WM, int WN, int MI, int NI>
struct T8Tile {
  static constexpr int W = WM * WN, TM = WM * MI * 16, TN = WN * NI * 16;
  static constexpr int ABYTES = TM * BK, BBYTES = TN * BK, STAGE = ABYTES + BBYTES;
  static constexpr int LA = ABYTES / 1024 / W, LB = BBYTES / 1024 / W;   // loads of a wavefront
  static constexpr int TURN = 16 * (NI * 16 * 4 + 16);                   // bytes of a wavefront's part in the epilogue
  static constexpr int LDS = ST * STAGE > W * TURN ? ST * STAGE : W * TURN;
  static_assert(ABYTES % (1024 * W) == 0 && BBYTES % (1024 * W) == 0, "whole loads");
};

// Four columns' values of 16 rows, turned through LDS, to rows of y
template <int TYPE, int NI>
__device__ __forceinline__ void t8_rows_out(char *turn, const w4_f4 v[NI], int lane, typename W4Mem<TYPE>::T *y, int64_t ldy, int rows, int cols) {
  using T = typename W4Mem<TYPE>::T;
  typedef T vec __attribute__((ext_vector_type(4)));
  constexpr int ES = sizeof(T), PITCH = NI * 16 * ES + 16, U = NI * ES, VE = 16 / ES;
  const int m = lane & 15, g = lane >> 4;
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    vec r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = W4Mem<TYPE>::put(v[j][e]);
    *(vec *)(turn + m * PITCH + (j * 16 + 4 * g) * ES) = r;
  }
#pragma unroll
  for (int t = 0; t < U / 4; ++t) {
    const int at = t * 64 + lane, row = at / U, u = at % U;
    const w4_u4 r = *(const w4_u4 *)(turn + row * PITCH + u * 16);
    T *to = y + row * ldy + u * VE;
    if (row < rows) {
      if (u * VE + VE <= cols) {
        *(t8_u4 *)to = r;
      } else {
        typedef T all __attribute__((ext_vector_type(VE)));
        const all q = __builtin_bit_cast(all, r);
#pragma unroll
        for (int i = 0; i < VE; ++i)
          if (u * VE + i < cols) to[i] = q[i];
      }
    }
  }
}

// P: 0 the forward product, else planes of a gradient.  PART: sums to the workspace.
template <int TYPE, int P, bool PART, int BK, int ST, int WM, int WN, int MI, int NI>
__global__ __launch_bounds__(64 * WM * WN, 2) void t8_tile_kernel(T8Product a) {
  using S = T8Tile<BK, ST, WM, WN, MI, NI>;
  constexpr int W = S::W, TM = S::TM, TN = S::TN, CH = BK / 16, RA = 1024 / BK;
  constexpr bool GRAD = P > 0;
  constexpr int CB = TN / 16, RB = 1024 / TN;              // gradient: chunks of a row of weights, rows of a load
  static_assert(P == 0 || MI % P == 0, "whole blocks of planes");
  extern __shared__ __align__(1024) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
  int tile = blockIdx.x, part = 0;
  const int total = a.tm * a.tn;
  if (PART) {
    part = tile / total;
    tile -= part * total;
  }
  int ti, tj;
  tile_at(tile, total, a.tm, a.tn, 8, ti, tj);
  const int m0 = __builtin_amdgcn_readfirstlane(ti * TM), n0 = __builtin_amdgcn_readfirstlane(tj * TN);
  const int cols = GRAD ? a.K : a.N, depth = GRAD ? (a.N + T8_SLAB - 1) / T8_SLAB * T8_SLAB : a.K;
  const int all = (depth + BK - 1) / BK, s0 = PART ? part * a.per : 0, ns = PART ? min(a.per, all - s0) : all;

  // this lane's places in a wavefront's loads: row and chunk of what belongs there
  const int lr = lane / CH, lc = (lane % CH) ^ t8_swz<BK>(lr);
  unsigned ao[S::LA], bo[S::LB];
#pragma unroll
  for (int i = 0; i < S::LA; ++i) ao[i] = (unsigned)(min(m0 + (wave * S::LA + i) * RA + lr, a.arows - 1) - m0) * (unsigned)a.lda + lc * 16;
#pragma unroll
  for (int i = 0; i < S::LB; ++i) {
    if constexpr (GRAD) {
      const int r = (wave * S::LB + i) * RB + lane / CB, c = (lane % CB) ^ (r & (CB - 1));
      bo[i] = (unsigned)min(n0 + c * 16, a.K - 16) - n0;
    } else {
      bo[i] = (unsigned)(min(n0 + (wave * S::LB + i) * RA + lr, a.N - 1) - n0) * (unsigned)a.ldw + lc * 16;
    }
  }
  // forward: chunks of the last slab beyond K re-read its end, and lie in LDS as zeros on the activations' side
  const unsigned back = GRAD ? 0u : (unsigned)max((all - 1) * BK + lc * 16 + 16 - a.K, 0);
  const int8_t *abase = a.a + (int64_t)m0 * a.lda, *bbase = a.w + (GRAD ? (int64_t)n0 : (int64_t)n0 * a.ldw);
  const unsigned lds0 = t8_lds_address(smem);
  const auto fetch = [&](int s, int stage) {               // s: slab of all
    const bool last = s == all - 1;
    const int row = min(s * BK, a.N - 1);                  // gradient: rows beyond the last meet zeros, and are the last
    const unsigned to = lds0 + stage * S::STAGE;
#pragma unroll
    for (int i = 0; i < S::LA; ++i) t8_to_lds(to + (wave * S::LA + i) * 1024, ao[i] - (last ? back : 0u), abase + (int64_t)s * BK);
#pragma unroll
    for (int i = 0; i < S::LB; ++i) {
      if constexpr (GRAD) {
        const int r = (wave * S::LB + i) * RB + lane / CB;
        t8_to_lds(to + S::ABYTES + (wave * S::LB + i) * 1024, bo[i] + (unsigned)min(r, a.N - 1 - row) * (unsigned)a.ldw, bbase + (int64_t)row * a.ldw);
      } else {
        t8_to_lds(to + S::ABYTES + (wave * S::LB + i) * 1024, bo[i] - (last ? back : 0u), bbase + (int64_t)s * BK);
      }
    }
  };

  t8_i4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = t8_i4{0, 0, 0, 0};
  const int wm = wave / WN * MI * 16, wn = wave % WN * NI * 16;

  constexpr int L = S::LA + S::LB;
#pragma unroll
  for (int i = 0; i < ST - 1; ++i)
    if (i < ns) fetch(s0 + i, i);
  int stage = 0;
  for (int s = 0; s < ns; ++s) {
    if (ST > 2 && s + 1 < ns) t8_wait_barrier<(ST - 2) * L>();
    else t8_wait_barrier<0>();
    if (s + ST - 1 < ns) fetch(s0 + s + ST - 1, stage == 0 ? ST - 1 : stage - 1);
    char *as = smem + stage * S::STAGE, *bs = as + S::ABYTES;
    if (!GRAD && s == ns - 1 && a.K % BK) {
      const int valid = a.K % BK / 16;
      for (int t = threadIdx.x; t < TM * CH; t += 64 * W) {
        const int r = t / CH, c = t % CH;
        if (c >= valid) *(w4_u4 *)(as + r * BK + ((c ^ t8_swz<BK>(r)) << 4)) = w4_u4{};
      }
      t8_barrier();
    }
#pragma unroll
    for (int kk = 0; kk < BK / 64; ++kk) {
      t8_i4 af[MI], bf[NI];
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int r = wm + i * 16 + r16;
        af[i] = *(const t8_i4 *)(as + r * BK + (((kk * 4 + g) ^ t8_swz<BK>(r)) << 4));
      }
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        if constexpr (GRAD) {
          // lane l of 16 gives the place of row l / 2, half l % 2 of 16 columns, and gets column l of 8 rows
          const int r = kk * 64 + g * 16 + (r16 >> 1), c = (wn >> 4) + j;
          typedef __attribute__((address_space(3))) t8_i2 lds_i2;
          const t8_i2 lo = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2 *)(bs + r * TN + ((c ^ (r & (CB - 1))) << 4) + (r16 & 1) * 8));
          const t8_i2 hi = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2 *)(bs + (r + 8) * TN + ((c ^ ((r + 8) & (CB - 1))) << 4) + (r16 & 1) * 8));
          bf[j] = t8_i4{lo[0], lo[1], hi[0], hi[1]};
        } else {
          const int r = wn + j * 16 + r16;
          bf[j] = *(const t8_i4 *)(bs + r * BK + (((kk * 4 + g) ^ t8_swz<BK>(r)) << 4));
        }
      }
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bf[j], af[i], acc[i][j], 0, 0, 0);
    }
    stage = stage == ST - 1 ? 0 : stage + 1;
  }

  const int col0 = n0 + wn;
  if constexpr (PART) {
    int32_t *to = a.part + (int64_t)part * a.arows * a.K;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int r = m0 + wm + i * 16 + r16;
#pragma unroll
      for (int j = 0; j < NI; ++j)
        if (r < a.arows && col0 + j * 16 < a.K) *(t8_i4 *)(to + (int64_t)r * a.K + col0 + j * 16 + 4 * g) = acc[i][j];
    }
    return;
  }
  t8_barrier();                                            // every wavefront has read its last operands
  if (col0 >= cols) return;
  using T = typename W4Mem<TYPE>::T;
  char *turn = smem + wave * S::TURN;
  w4_f4 v[NI];
  if constexpr (GRAD) {
    if constexpr (P > 0) {
#pragma unroll
      for (int q = 0; q < MI / P; ++q) {
        const int mb = ((m0 + wm) / 16 / P + q) * 16, m = mb + r16;
        const float scale = a.xs[min(m, a.M - 1)];
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            int s[P];
#pragma unroll
            for (int p = 0; p < P; ++p) s[p] = acc[q * P + p][j][e];
            v[j][e] = t8_join<P>(s, scale);
          }
        t8_rows_out<TYPE, NI>(turn, v, lane, (T *)a.y + (int64_t)mb * a.ldy + col0, a.ldy, a.M - mb, cols - col0);
      }
    }
  } else {
    w4_f4 ws[NI], bias[NI];
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = min(col0 + j * 16 + 4 * g + e, a.N - 1);
        ws[j][e] = a.ws[n];
        bias[j][e] = a.bias ? a.bias[n] : 0.0f;
      }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int mb = m0 + wm + i * 16;
      const float xs = a.xs[min(mb + r16, a.M - 1)];
#pragma unroll
      for (int j = 0; j < NI; ++j) v[j] = t8_finish(acc[i][j], ws[j], xs, bias[j]);
      t8_rows_out<TYPE, NI>(turn, v, lane, (T *)a.y + (int64_t)mb * a.ldy + col0, a.ldy, a.M - mb, cols - col0);
    }
  }
}

// Parts of the planes' sums to the gradient: four columns of a row a thread
template <int TYPE>
__global__ __launch_bounds__(256) void t8_join_kernel(T8Product a) {
  constexpr int P = t8_planes(TYPE);
  using T = typename W4Mem<TYPE>::T;
  const int quads = a.K / 4;
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= (int64_t)a.M * quads) return;
  const int m = (int)(t / quads), k = (int)(t % quads) * 4;
  t8_i4 s[P] = {};
  for (int z = 0; z < a.split; ++z)
#pragma unroll
    for (int p = 0; p < P; ++p) s[p] += *(const t8_i4 *)(a.part + ((int64_t)z * a.arows + t8_plane_row(m, p, P)) * a.K + k);
  const float scale = a.xs[m];
  T *to = (T *)a.y + (int64_t)m * a.ldy + k;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    int v[P];
#pragma unroll
    for (int p = 0; p < P; ++p) v[p] = s[p][e];
    to[e] = W4Mem<TYPE>::put(t8_join<P>(v, scale));
  }
}

template <int TYPE, int P, bool PART, int BK, int ST, int WM, int WN, int MI, int NI>
static hipError_t tile_launch(T8Product a, hipStream_t st) {
  using S = T8Tile<BK, ST, WM, WN, MI, NI>;
  a.tm = (a.arows + S::TM - 1) / S::TM;
  a.tn = ((P ? a.K : a.N) + S::TN - 1) / S::TN;
  static std::atomic<unsigned long long> done;
  const auto kern = t8_tile_kernel<TYPE, P, PART, BK, ST, WM, WN, MI, NI>;
  if (S::LDS > 65536) {
    const hipError_t e = allow_lds((const void *)kern, S::LDS, done);
    if (e != hipSuccess) return e;
  }
  kern<<<(unsigned)a.tm * (unsigned)a.tn * (unsigned)(PART ? a.split : 1), 64 * S::W, S::LDS, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_t8_tile(const T8Product &a, int type, hipStream_t st) {
  if (type == QC_TYPE_F32) return tile_launch<QC_TYPE_F32, 0, false, 64, 3, 1, 4, 8, 4>(a, st);
  if (type == QC_TYPE_F16) return tile_launch<QC_TYPE_F16, 0, false, 64, 3, 1, 4, 8, 4>(a, st);
  return tile_launch<QC_TYPE_BF16, 0, false, 64, 3, 1, 4, 8, 4>(a, st);
}

// ---- the gradient: tiles of 128 rows of planes by 256 columns; fewer than fill the chip split the summed axis
struct GradShape {
  int arows, split, per;
};
static GradShape grad_shape(int M, int N, int K, int type) {
  GradShape s;
  const int P = t8_planes(type), slabs = (N + T8_SLAB - 1) / T8_SLAB * (T8_SLAB / 64);
  s.arows = (M + 15) / 16 * 16 * P;
  const int64_t tiles = (int64_t)((s.arows + 127) / 128) * ((K + 255) / 256);
  int split = (int)std::max<int64_t>(1, std::min<int64_t>(512 / tiles, slabs / 4));
  s.per = (slabs + split - 1) / split;
  s.split = (slabs + s.per - 1) / s.per;
  return s;
}

int64_t t8_grad_part_bytes(int M, int N, int K, int type) {
  const GradShape s = grad_shape(M, N, K, type);
  return s.split > 1 ? (int64_t)s.split * s.arows * K * 4 : 0;
}

template <int TYPE>
static hipError_t grad_launch(T8Product a, hipStream_t st) {
  constexpr int P = t8_planes(TYPE);
  const GradShape s = grad_shape(a.M, a.N, a.K, TYPE);
  a.arows = s.arows;
  a.split = s.split;
  a.per = s.per;
  if (s.split == 1) return tile_launch<TYPE, P, false, 64, 3, 1, 4, 8, 4>(a, st);
  const hipError_t e = tile_launch<TYPE, P, true, 64, 3, 1, 4, 8, 4>(a, st);
  if (e != hipSuccess) return e;
  t8_join_kernel<TYPE><<<(unsigned)(((int64_t)a.M * (a.K / 4) + 255) / 256), 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_t8_grad(T8Product a, int type, hipStream_t st) {
  if (type == QC_TYPE_F32) return grad_launch<QC_TYPE_F32>(a, st);
  if (type == QC_TYPE_F16) return grad_launch<QC_TYPE_F16>(a, st);
  return grad_launch<QC_TYPE_BF16>(a, st);
}

}  // namespace qc
