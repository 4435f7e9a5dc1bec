// Products of the 8-bit layers with a scale for each token, many rows: y = x W^T and, on the byte planes of gradients, dx = dy W.
//
// Slabs of 128 bytes of the summed axis (whole cache lines: slabs of 64 made 4096 x 8192 x 8192 a quarter slower) go from memory straight to one of
// two or three places in LDS.  Wavefronts read 16 x 64 operands of v_mfma_i32_16x16x64_i8 from there half a slab ahead into registers: behind a
// slab's barrier its products start at once, the next operands come in under them, and the place of the slab that was read is filled again.
// The weights' rows run along the summed axis in the forward product; in the gradient they run across it, and ds_read_b64_tr_b8 turns 8 rows x
// 16 bytes on their way to the registers.
// Workgroups stay and walk over the tiles: the slabs of the next tile are on their way while the last of this one are multiplied.
// In the forward product a lane's columns are neighbours (of NI blocks, block j's lane l has weight row NI l + j), so that 16 lanes write whole lines of a
// row without any exchange: trading words between lanes took 16384 x 4608 x 1152 from 88 to 100 us.  The transposed reads of the gradient cannot
// permute columns; its operands are exchanged (weights first) and lanes trade words instead.
// What bounds it: 4096 x 8192 x 8192 takes 218 - 238 us, 2.3 - 2.5 POP/s (the spread is the cards': their clocks fall to 2.15 GHz under it; on codes of
// zero alone 198), where a loop of nothing but products runs at 4.1.  With every slab from the same lines of the caches it takes 8 % less, without any
// loads 20 %; fewer LDS clocks (the places of the weights' chunks, a quarter fewer) gave 1 %, a barrier later among the products nothing.  What ends a
// tile is not overlapped: 4.4 us of 20 at K = 1152.
#include "t8_product.h"

namespace qc {

constexpr int T8_BK = 128;

template <bool GRAD, int ST, int WM, int WN, int MI, int NI>
struct T8Tile {
  static constexpr int W = WM * WN, TM = WM * MI * 16, TN = WN * NI * 16;
  static constexpr int ABYTES = TM * T8_BK, BBYTES = TN * T8_BK, STAGE = ABYTES + BBYTES, RING = ST * STAGE;
  static constexpr int SCALES = GRAD ? 0 : (TM + 2 * TN) * 4, LDS = RING + 2 * SCALES;   // of two tiles: scales of rows and columns, biases
  static constexpr int LA = ABYTES / 1024 / W, LB = BBYTES / 1024 / W, L = LA + LB;      // loads of a wavefront
  static constexpr int PER_CU = 160 * 1024 / LDS < 2 ? 1 : 2;
  static_assert(ABYTES % (1024 * W) == 0 && BBYTES % (1024 * W) == 0, "whole loads");
};

// lanes m and m + 8 of 16 trade: afterwards lanes 0 - 7 hold the first words of rows 0 - 7 (a) and 8 - 15 (b), lanes 8 - 15 the second words
__device__ __forceinline__ void t8_trade8(unsigned &a, unsigned &b) {
  const unsigned first = (unsigned)__builtin_amdgcn_update_dpp((int)a, (int)b, 0x128, 0xF, 0xC, false);    // row_ror:8 to lanes 8 - 15
  b = (unsigned)__builtin_amdgcn_update_dpp((int)b, (int)a, 0x128, 0xF, 0x3, false);                       // to lanes 0 - 7
  a = first;
}

// 16 bytes of a row's columns from `col` on, of which `cols` exist
template <int TYPE, bool WHOLE>
__device__ __forceinline__ void t8_put16(typename W4Mem<TYPE>::T *row, int col, int cols, w4_u4 r) {
  using T = typename W4Mem<TYPE>::T;
  constexpr int VE = 16 / sizeof(T);
  if (WHOLE || col + VE <= cols) {
    *(t8_u4 *)(row + col) = r;
  } else {
    typedef T all __attribute__((ext_vector_type(VE)));
    const all q = __builtin_bit_cast(all, r);
#pragma unroll
    for (int i = 0; i < VE; ++i)
      if (col + i < cols) row[col + i] = q[i];
  }
}

// WHOLE: all of them exist.  16 rows' values, lane l's of row l % 16 and columns 16 j + 4 (l / 16) + e, to rows of y (its first row and column)
template <int TYPE, int NI, bool WHOLE>
__device__ __forceinline__ void t8_rows_out(const w4_f4 v[NI], int lane, typename W4Mem<TYPE>::T *y, int64_t ldy, int rows, int cols) {
  using T = typename W4Mem<TYPE>::T;
  typedef T four __attribute__((ext_vector_type(4)));
  static_assert(NI % 4 == 0, "whole lines");
  const int m = lane & 15, g = lane >> 4, low = m & 7, high = m >> 3;
  T *first = y + low * ldy, *second = first + 8 * ldy;
  if constexpr (sizeof(T) == 4) {
    // blocks 2 j and 2 j + 1: a line
#pragma unroll
    for (int j = 0; j < NI; j += 2) {
      w4_u4 a = __builtin_bit_cast(w4_u4, v[j]), b = __builtin_bit_cast(w4_u4, v[j + 1]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        unsigned p = a[e], q = b[e];
        t8_trade8(p, q);
        a[e] = p;
        b[e] = q;
      }
      const int col = (j + high) * 16 + 4 * g;
      if (WHOLE || low < rows) t8_put16<TYPE, WHOLE>(first, col, cols, a);
      if (WHOLE || low + 8 < rows) t8_put16<TYPE, WHOLE>(second, col, cols, b);
    }
  } else {
    // four blocks: a line.  Lanes of even g take a block's 8 columns from their neighbours 16 on, of odd g the next block's
    typedef unsigned u2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int j = 0; j < NI; j += 4) {
      w4_u4 u[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        four p, q;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[e] = W4Mem<TYPE>::put(v[j + 2 * h][e]);
          q[e] = W4Mem<TYPE>::put(v[j + 2 * h + 1][e]);
        }
        const u2 pw = __builtin_bit_cast(u2, p), qw = __builtin_bit_cast(u2, q);
        const u2 s0 = __builtin_amdgcn_permlane16_swap(pw[0], qw[0], false, false), s1 = __builtin_amdgcn_permlane16_swap(pw[1], qw[1], false, false);
        u[h] = w4_u4{s0[0], s1[0], s0[1], s1[1]};
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        unsigned p = u[0][e], q = u[1][e];
        t8_trade8(p, q);
        u[0][e] = p;
        u[1][e] = q;
      }
      const int col = j * 16 + 32 * high + 16 * (g & 1) + 8 * (g >> 1);
      if (WHOLE || low < rows) t8_put16<TYPE, WHOLE>(first, col, cols, u[0]);
      if (WHOLE || low + 8 < rows) t8_put16<TYPE, WHOLE>(second, col, cols, u[1]);
    }
  }
}

// P: 0 the forward product, else planes of a gradient.  PART: sums to the workspace.
template <int TYPE, int P, bool PART, int ST, int WM, int WN, int MI, int NI>
__global__ __launch_bounds__(64 * WM * WN, WM * WN > 4 ? 1 : 2) void t8_tile_kernel(T8Product a) {
  using S = T8Tile<(P > 0), ST, WM, WN, MI, NI>;
  constexpr int W = S::W, TM = S::TM, TN = S::TN, BK = T8_BK, L = S::L;
  static_assert(ST == 2 || ST == 3, "waits for the next of two or three slabs");
  constexpr bool GRAD = P > 0;
  constexpr int CB = TN / 16, RB = 1024 / TN;              // gradient: chunks of a row of weights, rows of a load
  static_assert(P == 0 || MI % P == 0, "whole blocks of planes");
  extern __shared__ __align__(1024) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
  const int wm = wave / WN * MI * 16, wn = wave % WN * NI * 16;
  const int cols = GRAD ? a.K : a.N, depth = GRAD ? (a.N + T8_SLAB - 1) / T8_SLAB * T8_SLAB : a.K;
  const int all = (depth + BK - 1) / BK, tiles = a.tm * a.tn;

  // The walk over the tiles: the workgroups of one XCD (every eighth) have a range of them, groups of 8 tile rows column by column, and take every
  // step-th.  (Not more than one division, but in the last rows.)
  struct At {
    int m0, n0, s0, ns, part;
  };
  struct Walk {
    int left, group, rows, in;                             // tiles of the range from this one on; group, its rows, place in it
  };
  const int step = ((int)gridDim.x + 7) >> 3;              // at least one, and no tile twice where the grid is the tiles
  const auto begin = [&]() {
    Walk w;
    int t = blockIdx.x;
    if (PART) {
      t %= tiles;                                          // one a workgroup
      w.left = 1;
    } else {
      const int x = t & 7, q = tiles >> 3, r = tiles & 7;
      w.left = q + (x < r) - (t >> 3);
      t = x * q + min(x, r) + (t >> 3);
    }
    w.group = t / (8 * a.tn);
    w.in = t - w.group * 8 * a.tn;
    w.rows = min(8, a.tm - w.group * 8);
    return w;
  };
  const auto advance = [&](Walk &w) {
    w.left -= step;
    w.in += step;
    if (w.left > 0)
      while (w.in >= w.rows * a.tn) {
        w.in -= w.rows * a.tn;
        ++w.group;
        w.rows = min(8, a.tm - w.group * 8);
      }
  };
  const auto at = [&](const Walk &w) {
    At r;
    const int nj = w.rows == 8 ? w.in >> 3 : w.in / w.rows, mi = w.in - nj * w.rows;
    r.m0 = __builtin_amdgcn_readfirstlane((w.group * 8 + mi) * TM);
    r.n0 = __builtin_amdgcn_readfirstlane(nj * TN);
    r.part = PART ? (int)blockIdx.x / tiles : 0;
    r.s0 = PART ? r.part * a.per : 0;
    r.ns = PART ? min(a.per, all - r.s0) : all;
    return r;
  };

  // ---- slabs to LDS: this lane's places in a wavefront's loads, row and chunk of what belongs there
  const int lr = lane / 8, lc = (lane % 8) ^ t8_swz(lr);
  // forward: chunks of the last slab beyond K re-read its end, and become zeros on the activations' side
  const auto back = [&](int c) { return (unsigned)max((all - 1) * BK + c * 16 + 16 - a.K, 0); };
  // of the forward product's weights, block j's lane l has row NI l + j, so that a lane's columns are neighbours; they lie in LDS block by block (as
  // they come, a read of every NI-th row met half of the banks)
  const auto wrow = [&](int p) { return p / (16 * NI) * (16 * NI) + p % 16 * NI + p / 16 % NI; };
  // of the gradient's, the chunks of rows 16 apart, which are read together, lie in different halves of the banks
  const auto turned = [&](int r) { return (r ^ (r >> 4 & 1) * (CB > 8 ? 8 : 1)) & (CB - 1); };
  const unsigned lds0 = t8_lds_address(smem);
  unsigned ao[S::LA], bo[S::LB];
  const int8_t *abase, *bbase;
  Walk fw = begin();                                       // tile, slab and place of the next load
  int fs = 0, fstage = 0, flying = 0;                      // and how many slabs have been asked for and not read
  At fat = at(fw);
  const auto aim = [&]() {
#pragma unroll
    for (int i = 0; i < S::LA; ++i) ao[i] = (unsigned)(min(fat.m0 + (wave * S::LA + i) * 8 + lr, a.arows - 1) - fat.m0) * (unsigned)a.lda + lc * 16;
#pragma unroll
    for (int i = 0; i < S::LB; ++i) {
      if constexpr (GRAD) {
        const int r = (wave * S::LB + i) * RB + lane / CB, c = (lane % CB) ^ turned(r);
        bo[i] = (unsigned)(min(fat.n0 + c * 16, a.K - 16) - fat.n0);
      } else {
        bo[i] = (unsigned)(min(fat.n0 + wrow((wave * S::LB + i) * 8 + lr), a.N - 1) - fat.n0) * (unsigned)a.ldw + lc * 16;
      }
    }
    abase = a.a + (int64_t)fat.m0 * a.lda;
    bbase = a.w + (GRAD ? (int64_t)fat.n0 : (int64_t)fat.n0 * a.ldw);
  };
  aim();
  const auto fetch = [&]() {
    if (fw.left <= 0) return;
    const int s = fat.s0 + fs;
    const bool last = !GRAD && s == all - 1;
    const int row = min(s * BK, a.N - 1);                  // gradient: rows beyond the last meet zeros, and are the last
    const unsigned to = lds0 + fstage * S::STAGE;
#pragma unroll
    for (int i = 0; i < S::LA; ++i) t8_to_lds(to + (wave * S::LA + i) * 1024, ao[i] - (last ? back(lc) : 0u), abase + (int64_t)s * BK);
#pragma unroll
    for (int i = 0; i < S::LB; ++i) {
      if constexpr (GRAD) {
        const int r = (wave * S::LB + i) * RB + lane / CB;
        t8_to_lds(to + S::ABYTES + (wave * S::LB + i) * 1024, bo[i] + (unsigned)min(r, a.N - 1 - row) * (unsigned)a.ldw, bbase + (int64_t)row * a.ldw);
      } else {
        t8_to_lds(to + S::ABYTES + (wave * S::LB + i) * 1024, bo[i] - (last ? back(lc) : 0u), bbase + (int64_t)s * BK);
      }
    }
    fstage = fstage == ST - 1 ? 0 : fstage + 1;
    ++flying;
    if (++fs == fat.ns) {
      fs = 0;
      advance(fw);
      if (fw.left > 0) {
        fat = at(fw);
        aim();
      }
    }
  };

  t8_i4 acc[MI][NI], af[MI], bf[2][NI];
  const auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = t8_i4{0, 0, 0, 0};
  };
  // the last slab of a K that is no whole slabs: zeros beyond it
  const auto blank = [&](int stage) {
    char *as = smem + stage * S::STAGE;
    const int valid = a.K % BK / 16;
    for (int t = threadIdx.x; t < TM * 8; t += 64 * W) {
      const int r = t / 8, c = t % 8;
      if (c >= valid) *(w4_u4 *)(as + r * BK + ((c ^ t8_swz(r)) << 4)) = w4_u4{};
    }
    t8_barrier();
  };
  // operands of half `kk` of the slab at `stage`
  const auto read_w = [&](t8_i4 (&w)[NI], int stage, int kk) {
    const char *bs = smem + stage * S::STAGE + S::ABYTES;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      if constexpr (GRAD) {
        // lane l of 16 gives the place of row l / 2, half l % 2 of 16 columns, and gets column l of 8 rows
        const int r = kk * 64 + g * 16 + (r16 >> 1), c = (wn >> 4) + j;
        typedef __attribute__((address_space(3))) t8_i2 lds_i2;
        const t8_i2 lo = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2 *)(bs + r * TN + ((c ^ turned(r)) << 4) + (r16 & 1) * 8));
        const t8_i2 hi = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2 *)(bs + (r + 8) * TN + ((c ^ turned(r + 8)) << 4) + (r16 & 1) * 8));
        w[j] = t8_i4{lo[0], lo[1], hi[0], hi[1]};
      } else {
        const int r = wn + j * 16 + r16;
        w[j] = *(const t8_i4 *)(bs + r * BK + (((kk * 4 + g) ^ t8_swz(r)) << 4));
      }
    }
  };
  const auto read_x = [&](int stage, int kk, int i) {
    const int r = wm + i * 16 + r16;
    return *(const t8_i4 *)(smem + stage * S::STAGE + r * BK + (((kk * 4 + g) ^ t8_swz(r)) << 4));
  };

  using T = typename W4Mem<TYPE>::T;
  // scales and biases of a tile, 4 bytes a lane; their place alternates from tile to tile
  const auto scales = [&](const At &p, int turn) {
    if constexpr (!GRAD) {
      const unsigned to = lds0 + S::RING + turn * S::SCALES;
      for (int t = wave; t < TM / 64; t += W) t8_word_to_lds(to + t * 256, (unsigned)min(t * 64 + lane, a.M - 1 - p.m0) * 4, a.xs + p.m0);
      for (int t = wave; t < TN / 64; t += W) {
        const unsigned off = (unsigned)min(t * 64 + lane, a.N - 1 - p.n0) * 4;
        t8_word_to_lds(to + TM * 4 + t * 256, off, a.ws + p.n0);
        if (a.bias) t8_word_to_lds(to + (TM + TN) * 4 + t * 256, off, a.bias + p.n0);
      }
    }
  };
  const auto rows_of = [&](const At &p, int turn, auto whole, auto stream) {
    constexpr bool WHOLE = decltype(whole)::value, STREAM = decltype(stream)::value;
    const int col0 = p.n0 + wn;
    w4_f4 v[NI];
    if constexpr (GRAD) {
#pragma unroll
      for (int q = 0; q < MI / (P ? P : 1); ++q) {
        const int mb = ((p.m0 + wm) / 16 / P + q) * 16;
        const float scale = a.xs[WHOLE ? mb + r16 : min(mb + r16, a.M - 1)];
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            int s[P ? P : 1];
#pragma unroll
            for (int b = 0; b < P; ++b) s[b] = acc[q * P + b][j][e];
            v[j][e] = t8_join<P>(s, scale);
          }
        t8_rows_out<TYPE, NI, WHOLE>(v, lane, (T *)a.y + (int64_t)mb * a.ldy + col0, a.ldy, a.M - mb, cols - col0);
      }
    } else {
      // a lane's rows 4 g + e of a block, and NI neighbouring columns: 16 lanes write whole lines
      typedef T some __attribute__((ext_vector_type(NI)));
      typedef some some_at __attribute__((aligned(sizeof(T))));
      const float *xs = (const float *)(smem + S::RING + turn * S::SCALES), *ws = xs + TM, *bias = ws + TN;
      float cs[NI], cb[NI];
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        cs[j] = ws[wn + r16 * NI + j];
        cb[j] = a.bias ? bias[wn + r16 * NI + j] : 0.0f;
      }
      const int mb = p.m0 + wm + 4 * g, col = col0 + r16 * NI;
      T *to = (T *)a.y + (int64_t)mb * a.ldy + col;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const w4_f4 scale = *(const w4_f4 *)(xs + wm + i * 16 + 4 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          some r;
#pragma unroll
          for (int j = 0; j < NI; ++j) r[j] = W4Mem<TYPE>::put(__builtin_fmaf((float)acc[i][j][e] * cs[j], scale[e], cb[j]));
          T *row = to + (int64_t)(i * 16 + e) * a.ldy;
          if (WHOLE) {
            if (STREAM) __builtin_nontemporal_store(r, (some_at *)row);
            else *(some_at *)row = r;
          } else if (mb + i * 16 + e < a.M) {
#pragma unroll
            for (int j = 0; j < NI; ++j)
              if (col + j < cols) row[j] = r[j];
          }
        }
      }
    }
  };
  const auto finish = [&](const At &p, int turn) {
    const int col0 = p.n0 + wn;
    if constexpr (PART) {
      // as they lie in the registers: 1024 bytes a store
      int32_t *to = a.part + (((int64_t)p.part * tiles + p.m0 / TM * a.tn + p.n0 / TN) * W + wave) * (MI * NI * 256) + lane * 4;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
          if (p.m0 + wm + i * 16 < a.arows && col0 + j * 16 < a.K) *(t8_i4 *)(to + (i * NI + j) * 256) = acc[i][j];
    } else if ((P ? (p.m0 + TM) / (P ? P : 1) : p.m0 + TM) <= a.M && p.n0 + TN <= cols) {
      if (!GRAD && a.stream) rows_of(p, turn, std::true_type(), std::true_type());
      else rows_of(p, turn, std::true_type(), std::false_type());
    } else if (col0 < cols) {
      rows_of(p, turn, std::false_type(), std::false_type());
    }
    clear();
  };

  // ---- slab after slab, tile after tile
  if (fw.left <= 0) return;
  const bool ragged = !GRAD && a.K % BK;
  Walk cw = fw;
  At cat = fat;
  int cs = 0, stage = 0, turn = 0;                         // slab of the tile, place, and place of the scales of what is multiplied
  // products of the operands in af and w, under which others come in: each row block's in the place of those just used
  const auto half = [&](const t8_i4 (&w)[NI], t8_i4 (&nw)[NI], int from, int kk) {
    read_w(nw, from, kk);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
#pragma unroll
      for (int j = 0; j < NI; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(GRAD ? w[j] : af[i], GRAD ? af[i] : w[j], acc[i][j], 0, 0, 0);
      af[i] = read_x(from, kk, i);
    }
    // in this order
    __builtin_amdgcn_sched_group_barrier(0x100, GRAD ? 2 * NI : NI, 0);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x8, NI, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
  };
  clear();
#pragma unroll
  for (int i = 0; i < ST; ++i) fetch();
  // the next slab, all loads but those of the slabs behind it (others that come in between make the wait longer)
  const auto arrive = [&]() {
    if (ST > 2 && flying >= 3) t8_wait_barrier<2 * (ST > 2) * L>();
    else if (flying >= 2) t8_wait_barrier<L>();
    else t8_wait_barrier<0>();
    --flying;
  };
  arrive();
  if (ragged && cat.ns == 1) blank(0);
  read_w(bf[0], 0, 0);
#pragma unroll
  for (int i = 0; i < MI; ++i) af[i] = read_x(0, 0, i);
  for (;;) {
    if (cs == 0) scales(cat, turn);
    half(bf[0], bf[1], stage, 1);
    const bool ends = cs + 1 == cat.ns;
    const At p = cat;
    if (ends) {
      cs = 0;
      advance(cw);
      if (cw.left > 0) cat = at(cw);
    } else {
      ++cs;
    }
    const bool more = cw.left > 0;
    // the next slab is there, and this one's operands are in registers
    if (ends) t8_wait_barrier<0>(), --flying;              // and the tile's scales
    else arrive();
    fetch();
    stage = stage == ST - 1 ? 0 : stage + 1;
    if (ragged && more && cs + 1 == cat.ns) blank(stage);
    half(bf[1], bf[0], stage, 0);                          // (behind the last slab: some operands that nothing uses)
    if (ends) {                                            // the epilogue takes the operands' registers: they are read again
      finish(p, turn);
      turn ^= 1;
      if (!more) break;
      read_w(bf[0], stage, 0);
#pragma unroll
      for (int i = 0; i < MI; ++i) af[i] = read_x(stage, 0, i);
    }
  }
}

// Parts of the planes' sums to the gradient.  A thread has what one lane of a tile's wavefront had of a row block's planes, four columns of a row; or 16
// threads share its parts where they are many
template <int TYPE, int Z, int WM, int WN, int MI, int NI>
__global__ __launch_bounds__(256) void t8_join_kernel(T8Product a) {
  constexpr int P = t8_planes(TYPE), ITEMS = 256 / Z, W = WM * WN, TILE = W * MI * NI * 256;
  using T = typename W4Mem<TYPE>::T;
  const int item = threadIdx.x % ITEMS, first = threadIdx.x / ITEMS;
  int64_t t = (int64_t)blockIdx.x * ITEMS + item;
  const int lane = (int)(t % 64), j = (int)(t / 64 % NI), q = (int)(t / (64 * NI) % (MI / P)), wave = (int)(t / (64 * NI * (MI / P)) % W);
  const int tile = (int)(t / (64 * NI * (MI / P) * W)), tm = tile / a.tn, tn = tile - tm * a.tn;
  const int m = ((tm * WM + wave / WN) * (MI / P) + q) * 16 + lane % 16, k = ((tn * WN + wave % WN) * NI + j) * 16 + lane / 16 * 4;
  const bool there = m < a.M && k < a.K;
  const int32_t *from = a.part + (int64_t)tile * TILE + (wave * MI + q * P) * (NI * 256) + j * 256 + lane * 4;
  t8_i4 s[P] = {};
  if (there)
    for (int z = first; z < a.split; z += Z)
#pragma unroll
      for (int p = 0; p < P; ++p) s[p] += *(const t8_i4 *)(from + (int64_t)z * a.tm * a.tn * TILE + p * (NI * 256));
  if constexpr (Z > 1) {
    __shared__ t8_i4 red[Z][P][ITEMS];
#pragma unroll
    for (int p = 0; p < P; ++p) red[first][p][item] = s[p];
    __syncthreads();
    if (first) return;
#pragma unroll
    for (int p = 0; p < P; ++p)
      for (int z = 1; z < Z; ++z) s[p] += red[z][p][item];
  }
  if (!there) return;
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

template <int TYPE, int P, bool PART, int ST, int WM, int WN, int MI, int NI>
static hipError_t tile_launch(T8Product a, hipStream_t st) {
  using S = T8Tile<(P > 0), ST, WM, WN, MI, NI>;
  a.tm = (a.arows + S::TM - 1) / S::TM;
  a.tn = ((P ? a.K : a.N) + S::TN - 1) / S::TN;
  // results of whole lines that outgrow the L2 caches stream past them (16384 x 4608 x 1152 bfloat16, 151 MB: 103 -> 97 us; 4096 rows, 38 MB: 32.7 ->
  // 28.7); pieces of lines meet there
  constexpr int ES = TYPE == QC_TYPE_F32 ? 4 : 2;
  a.stream = (int64_t)a.M * a.N * ES > (32 << 20) && a.ldy * ES % 128 == 0 && (uintptr_t)a.y % 128 == 0;
  static std::atomic<unsigned long long> done;
  const auto kern = t8_tile_kernel<TYPE, P, PART, ST, WM, WN, MI, NI>;
  if (S::LDS > 65536) {
    const hipError_t e = allow_lds((const void *)kern, S::LDS, done);
    if (e != hipSuccess) return e;
  }
  const int64_t tiles = (int64_t)a.tm * a.tn;
  kern<<<(unsigned)(PART ? tiles * a.split : std::min<int64_t>(tiles, 256 * S::PER_CU)), 64 * S::W, S::LDS, st>>>(a);
  return hipGetLastError();
}

// ---- Tiles: 256 x 256 by eight wavefronts, one workgroup a compute unit, or 128 x 128 by four, two.  The large one reads LDS half as often for a
// product, the small one leaves fewer compute units without a tile.  Where there is no tile for each compute unit, so that nothing works beside a
// workgroup while it waits for memory, 128 x 128 by eight with three slabs on their way (2048 x 1152 x 4608: 24.5 us, by four with two 26.7; 512 x 8192 x 8192
// 43.6 / 59; with more tiles than compute units it loses: 4096 x 4608 x 1152 33.7 / 28.2), and where there is none of half the size either, 64 x 128 by four
// with three (1000 x 1152 x 1152 8.1, 256 x 8192 x 4096 18.2; 128 x 128 10.0 / 11.4, 22.4 / 24.0).
// Three planes of a row need three row blocks, so that tiles have 192 or 96 rows of planes: 192 x 128 by four, two workgroups a compute unit (8192 x 1152
// from 4608: 129 us; 192 x 256 by eight 157, and at 2048 x 8192 from 8192 366 / 373), where they are few 96 x 128, two workgroups (1000 x 1152 from 4608:
// 31 us, 192 x 128 34), and where those are fewer than compute units one with three slabs on their way (128 x 8192 from 8192: 42 us, two 47).  Four need
// four: the first two.
// us of a slab and of a tile's ends, by how much of the chip is taken (measured at 16384 x 4608 x 128 - 4608, 16384 x 1152 x 4608 and 4096 x 8192 x 8192,
// and for LONE and HALF at those above; three planes: all slots and half of them, 1152 and 4608 deep, of LONE, which has 257 - 512 tiles, between 288 and
// 512):
struct TileCost {
  int rows, cols, slots;                                   // 0 rows: there is no such form
  float slab, ends, slab_rest, ends_rest;                  // all slots taken; half of them or fewer
};
enum { LARGE, SMALL, LONE, HALF };                         // the last two where no slot has more than one tile
struct TileCosts {
  TileCost form[4];
  int parts;                                               // the form of gradients' parts
};
constexpr TileCost LARGE_COST = {256, 256, 256, 1.72f, 4.4f, 1.3f, 4.0f}, SMALL_COST = {128, 128, 512, 0.93f, 3.2f, 0.68f, 4.5f};
constexpr TileCosts FORWARD = {{LARGE_COST, SMALL_COST, {128, 128, 256, 0.61f, 4.8f, 0.56f, 4.8f}, {64, 128, 256, 0.45f, 4.2f, 0.44f, 4.2f}}, 0},
                    THREE = {{{}, {192, 128, 512, 1.40f, 5.7f, 0.83f, 5.0f}, {96, 128, 512, 0.82f, 3.7f, 0.60f, 3.9f}, {96, 128, 256, 0.58f, 3.8f, 0.57f, 3.4f}}, LONE},
                    FOUR = {{LARGE_COST, SMALL_COST, {}, {}}, SMALL};
constexpr const TileCosts &tile_costs(int planes) { return planes == 0 ? FORWARD : planes == 3 ? THREE : FOUR; }

static float tile_time(const TileCost &c, int64_t rows, int cols, int slabs) {
  const int64_t tiles = ((rows + c.rows - 1) / c.rows) * ((cols + c.cols - 1) / c.cols), rest = tiles % c.slots;
  const float full = c.slab * slabs + c.ends, last = rest == 0 ? 0.0f : rest > c.slots / 2 ? full : c.slab_rest * slabs + c.ends_rest;
  return (float)(tiles / c.slots) * full + last;
}
// the form that is soonest
struct TileForm {
  int form;
  float time;
};
static TileForm tile_form(int64_t rows, int cols, int slabs, int planes) {
  const TileCosts &costs = tile_costs(planes);
  TileForm f{SMALL, tile_time(costs.form[SMALL], rows, cols, slabs)};
  for (const int form : {LARGE, LONE, HALF}) {
    const TileCost &c = costs.form[form];
    if (c.rows == 0 || (form != LARGE && ((rows + c.rows - 1) / c.rows) * ((cols + c.cols - 1) / c.cols) > c.slots)) continue;
    const float t = tile_time(c, rows, cols, slabs);
    if (t < f.time) f = {form, t};
  }
  return f;
}

float t8_tile_time(int M, int N, int K) {
  // weights that nothing else shares come at 3.7 TB/s (1 x 28672 x 8192: 63 us)
  return std::max(tile_form(M, N, (K + T8_BK - 1) / T8_BK, 0).time, (float)N * (float)K / 3.7e6f);
}

template <int TYPE, int P>
static hipError_t tile_of(const T8Product &a, hipStream_t st) {
  const int form = tile_form(a.arows, P ? a.K : a.N, ((P ? a.N : a.K) + T8_BK - 1) / T8_BK, P).form;
  if constexpr (P == 3) {
    if (form == LONE) return tile_launch<TYPE, P, false, 2, 2, 2, 3, 4>(a, st);
    if (form == HALF) return tile_launch<TYPE, P, false, 3, 2, 2, 3, 4>(a, st);
    return tile_launch<TYPE, P, false, 2, 2, 2, 6, 4>(a, st);
  } else {
    if (form == LARGE) {
      // 64 x 128 a wavefront instead of 128 x 64: 16-bit results go out in 256 bytes a row (8192 x 8192 x 1152 84 -> 81 us, 8192 x 8192 x 8192 438 -> 433;
      // float32 and the gradients, which spill, lose)
      if constexpr (P == 0 && TYPE != QC_TYPE_F32) return tile_launch<TYPE, P, false, 2, 4, 2, 4, 8>(a, st);
      else return tile_launch<TYPE, P, false, 2, 2, 4, 8, 4>(a, st);
    }
    if constexpr (P == 0) {
      if (form == LONE) return tile_launch<TYPE, P, false, 3, 4, 2, 2, 4>(a, st);
      if (form == HALF) return tile_launch<TYPE, P, false, 3, 2, 2, 2, 4>(a, st);
    }
    return tile_launch<TYPE, P, false, 2, 2, 2, 4, 4>(a, st);
  }
}

hipError_t launch_t8_tile(const T8Product &a, int type, hipStream_t st) {
  if (type == QC_TYPE_F32) return tile_of<QC_TYPE_F32, 0>(a, st);
  if (type == QC_TYPE_F16) return tile_of<QC_TYPE_F16, 0>(a, st);
  return tile_of<QC_TYPE_BF16, 0>(a, st);
}

// ---- The gradient: whole rounds of tiles first; the rows of what is left, or of a launch that makes no round, split the summed axis into parts
// whose sums a second kernel joins, where that is sooner.
struct GradPlan {
  int arows, whole;          // rows of planes, and of them those that are not split
  int split, per;            // parts, slabs of each
};
static GradPlan grad_plan(int M, int N, int K, int type) {
  const int P = t8_planes(type), slabs = (N + T8_BK - 1) / T8_BK;
  GradPlan best{(M + 15) / 16 * 16 * P, 0, 1, slabs};
  best.whole = best.arows;
  float time = tile_form(best.arows, K, slabs, P).time;
  const TileCosts &costs = tile_costs(P);
  const TileCost &part = costs.form[costs.parts];
  for (const int form : {LARGE, SMALL}) {
    const TileCost &c = costs.form[form];
    if (c.rows == 0) continue;
    const int64_t tn = (K + c.cols - 1) / c.cols, tiles = (best.arows + c.rows - 1) / c.rows * tn;
    const int whole = (int)(tiles / c.slots * c.slots / tn * c.rows), rest = best.arows - whole;
    const int64_t left = (int64_t)((rest + part.rows - 1) / part.rows) * ((K + part.cols - 1) / part.cols);
    if (left == 0 || left > part.slots / 2) continue;
    int split = (int)std::min<int64_t>(part.slots / left, std::max(1, slabs / 2));
    const int per = (slabs + split - 1) / split;
    split = (slabs + per - 1) / per;
    // a launch more, or two, and the sums' way to memory and back (kernels of 64 x 4096 from 14336 bfloat16 in 8 parts, 25 MB: 23.8 and 5.0 us; 100 x 1152 from
    // 8192 float32 in 13, 25 MB: 14.0 and 6.5; 15 x 2640 from 8838 bfloat16 in 24, 25 MB with what lies beyond row 15: 12.1 and 4.4)
    const float t = tile_time(c, whole, K, slabs) + part.slab * per + part.ends + 7.0f + (float)split * (float)rest * (float)K * 4.0f / 3.1e6f;
    if (split > 1 && t < time) {
      time = t;
      best.whole = whole;
      best.split = split;
      best.per = per;
    }
  }
  return best;
}

int64_t t8_grad_part_bytes(int M, int N, int K, int type) {
  const GradPlan p = grad_plan(M, N, K, type);
  const TileCosts &costs = tile_costs(t8_planes(type));
  const TileCost &part = costs.form[costs.parts];
  const int64_t tiles = (int64_t)((p.arows - p.whole + part.rows - 1) / part.rows) * ((K + part.cols - 1) / part.cols);
  return p.split > 1 ? p.split * tiles * part.rows * part.cols * 4 : 0;
}

template <int TYPE>
static hipError_t grad_launch(T8Product a, hipStream_t st) {
  constexpr int P = t8_planes(TYPE);
  const GradPlan p = grad_plan(a.M, a.N, a.K, TYPE);
  const int rows = p.whole / P;                            // of the result (a multiple of 16, or all)
  a.arows = p.whole;
  if (p.split == 1) return tile_of<TYPE, P>(a, st);
  if (p.whole) {
    T8Product w = a;
    w.M = rows;
    const hipError_t e = tile_of<TYPE, P>(w, st);
    if (e != hipSuccess) return e;
  }
  a.arows = p.arows - p.whole;
  a.split = p.split;
  a.per = p.per;
  a.M -= rows;
  a.a += (int64_t)p.whole * a.lda;
  a.xs += rows;
  a.y = (typename W4Mem<TYPE>::T *)a.y + (int64_t)rows * a.ldy;
  constexpr TileCost part = tile_costs(P).form[tile_costs(P).parts];
  constexpr int MI = part.rows / 32;
  const hipError_t e = tile_launch<TYPE, P, true, 2, 2, 2, MI, 4>(a, st);
  if (e != hipSuccess) return e;
  a.tm = (a.arows + part.rows - 1) / part.rows;
  a.tn = (a.K + part.cols - 1) / part.cols;
  const unsigned items = (unsigned)a.tm * a.tn * (part.rows * part.cols / 4 / P);
  if (a.split > 8) t8_join_kernel<TYPE, 16, 2, 2, MI, 4><<<items / 16, 256, 0, st>>>(a);
  else t8_join_kernel<TYPE, 1, 2, 2, MI, 4><<<items / 256, 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_t8_grad(T8Product a, int type, hipStream_t st) {
  if (type == QC_TYPE_F32) return grad_launch<QC_TYPE_F32>(a, st);
  if (type == QC_TYPE_F16) return grad_launch<QC_TYPE_F16>(a, st);
  return grad_launch<QC_TYPE_BF16>(a, st);
}

}  // namespace qc
