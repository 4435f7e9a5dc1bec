// y = x W^T of the 8-bit layers with a scale for each token, few rows: what counts is the stream of weights.
//
// A workgroup makes 16 MT rows by 16 NT columns; its wavefronts share the summed axis, each taking every W-th chunk of 128 bytes of all
// rows alone: chunks go from memory straight to the wavefront's own ring in LDS, ST of them on their way, without registers and without
// barriers.  A load covers 8 rows of 128 bytes, whole cache lines; operands are read back in the matrix instruction's order.  The integer
// sums of the wavefronts meet in LDS.  One row by 28672 x 8192 takes 41 us, 5.7 TB/s; the tiles' times stand beside the rule below.
#include "t8_product.h"

namespace qc {

template <int MT, int NT, int ST>
struct T8Few {
  static constexpr int STAGE = (MT + NT) * 16 * 128, RING = ST * STAGE, SUM = MT * NT * 1024;
  static constexpr int EACH = RING > SUM ? RING : SUM;                    // LDS of a wavefront
  static constexpr int MOST = 8 * EACH <= 160 * 1024 ? 8 : 4;             // wavefronts of a workgroup
  static_assert(MOST * EACH <= 160 * 1024, "LDS of a compute unit");
};

template <int TYPE, int MT, int NT, int ST>
__global__ __launch_bounds__((64 * T8Few<MT, NT, ST>::MOST)) void t8_few_kernel(T8Product a) {
  using S = T8Few<MT, NT, ST>;
  constexpr int L = 2 * (MT + NT);
  extern __shared__ __align__(1024) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int r16 = lane & 15, g = lane >> 4;
  const int ti = blockIdx.x / a.tn, tj = blockIdx.x % a.tn;
  const int m0 = ti * 16 * MT, n0 = tj * 16 * NT;
  const int chunks = (a.K + 127) / 128, mine = (chunks - wave + waves - 1) / waves;
  const int lr = lane >> 3, lc = (lane & 7) ^ lr;
  unsigned ao[2 * MT], bo[2 * NT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) ao[i] = (unsigned)(min(m0 + 8 * i + lr, a.M - 1) - m0) * (unsigned)a.lda + lc * 16;
#pragma unroll
  for (int i = 0; i < 2 * NT; ++i) bo[i] = (unsigned)(min(n0 + 8 * i + lr, a.N - 1) - n0) * (unsigned)a.ldw + lc * 16;
  const unsigned back = (unsigned)max((chunks - 1) * 128 + lc * 16 + 16 - a.K, 0);      // beyond K: the end again
  const int8_t *abase = a.a + (int64_t)m0 * a.lda, *bbase = a.w + (int64_t)n0 * a.ldw;
  char *ring = smem + wave * S::RING;
  const unsigned lds0 = t8_lds_address(ring);
  const auto fetch = [&](int i, int stage) {
    const int c = wave + i * waves;
    const unsigned less = c == chunks - 1 ? back : 0u, to = lds0 + stage * S::STAGE;
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) t8_to_lds(to + i * 1024, ao[i] - less, abase + (int64_t)c * 128);
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i) t8_to_lds(to + (2 * MT + i) * 1024, bo[i] - less, bbase + (int64_t)c * 128);
  };
  t8_i4 acc[MT][NT] = {};
#pragma unroll
  for (int i = 0; i < ST; ++i)
    if (i < mine) fetch(i, i);
  int stage = 0;
  for (int i = 0; i < mine; ++i) {
    const int behind = min(ST, mine - i) - 1;              // chunks that may still be on their way
    if (ST > 2 && behind == 2) t8_wait<2 * L>();
    else if (behind == 1) t8_wait<L>();
    else t8_wait<0>();
    const char *as = ring + stage * S::STAGE, *bs = as + MT * 2048;
    const int valid = min(8, (a.K - (wave + i * waves) * 128) / 16);
    t8_i4 af[2][MT], bf[2][NT];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const int place = ((kk * 4 + g) ^ (r16 & 7)) << 4;
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        af[kk][t] = *(const t8_i4 *)(as + (t * 16 + r16) * 128 + place);
        if (kk * 4 + g >= valid) af[kk][t] = t8_i4{0, 0, 0, 0};
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) bf[kk][t] = *(const t8_i4 *)(bs + (t * 16 + r16) * 128 + place);
    }
    if (i + ST < mine) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the operands have left the place that is filled next
      fetch(i + ST, stage);
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int u = 0; u < NT; ++u) acc[t][u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bf[kk][u], af[kk][t], acc[t][u], 0, 0, 0);
    stage = stage == ST - 1 ? 0 : stage + 1;
  }
  t8_barrier();                                            // the rings are read
  int *sums = (int *)smem;
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int u = 0; u < NT; ++u) *(t8_i4 *)(sums + ((wave * MT + t) * 16 + r16) * 16 * NT + u * 16 + 4 * g) = acc[t][u];
  t8_barrier();
  using T = typename W4Mem<TYPE>::T;
  for (int o = threadIdx.x; o < 256 * MT * NT; o += 64 * waves) {
    const int m = m0 + o / (16 * NT), n = n0 + o % (16 * NT);
    if (m >= a.M || n >= a.N) continue;
    int t = sums[o];
    for (int w = 1; w < waves; ++w) t += sums[w * 256 * MT * NT + o];
    const float v = __builtin_fmaf((float)t * a.ws[n], a.xs[m], a.bias ? a.bias[n] : 0.0f);
    ((T *)a.y)[(int64_t)m * a.ldy + n] = W4Mem<TYPE>::put(v);
  }
}

// More wavefronts where the workgroups are fewer than the compute units
template <int TYPE, int MT, int NT, int ST>
static hipError_t few_launch(T8Product a, hipStream_t st) {
  using S = T8Few<MT, NT, ST>;
  a.tm = (a.M + 16 * MT - 1) / (16 * MT);
  a.tn = (a.N + 16 * NT - 1) / (16 * NT);
  const int chunks = (a.K + 127) / 128;
  const int64_t groups = (int64_t)a.tm * a.tn;
  int waves = groups > 256 && MT * NT > 8 ? 2 : groups <= 128 && chunks >= 32 ? S::MOST : 4;
  while (waves > chunks) waves /= 2;
  const int lds = waves * S::EACH;
  static std::atomic<unsigned long long> done;
  const auto kern = t8_few_kernel<TYPE, MT, NT, ST>;
  if (lds > 65536) {
    const hipError_t e = allow_lds((const void *)kern, S::MOST * S::EACH, done);
    if (e != hipSuccess) return e;
  }
  kern<<<(unsigned)groups, 64 * waves, lds, st>>>(a);
  return hipGetLastError();
}

// us of a tile's launch: what its workgroups load, over the chip at 13 TB/s (from the L2 caches, mostly) and over one compute unit's share of them at
// 70 GB/s (50 where it has one workgroup of a large tile); the weights once, from memory, at 5.2 TB/s (3.9 where a compute unit has one workgroup of
// 32 x 32, too few loads on their way); and what a launch and the sum over the wavefronts take.  Measured (the best of these | the others | tiles of
// 64 x 128, t8_tile.hip): 1 x 28672 x 8192 40.7 with 16 x 16 | 44 with 16 x 64; 32 x 8192 x 8192 16.4 with 16 x 64 | 18.9 - 21.6; 64 x 8192 x 8192 19.5 with
// 32 x 64 | 22 - 24 | 33; 128 x 8192 x 8192 25.4 with 64 x 64 | | 32; 256 x 8192 x 8192 42 with 64 x 64 | 59 - 72 | 33; 256 x 1152 x 4608 10.5 with 32 x 32 |
// 10.6 - 16 | 20; 256 x 4608 x 1152 10.1 - 12 | 8.3.
static float few_time(const T8Product &a, int MT, int NT) {
  const int64_t groups = (int64_t)((a.M + 16 * MT - 1) / (16 * MT)) * ((a.N + 16 * NT - 1) / (16 * NT));
  const float each = (float)((a.K + 127) / 128) * (float)(MT + NT) * 2048.0f, memory = MT + NT == 4 && groups <= 256 ? 3.9e6f : 5.2e6f;
  const float load = std::max((float)groups * each / 13e6f, (float)((groups + 255) / 256) * each / (MT + NT > 4 ? 50e3f : 70e3f));
  return 4.0f + 0.25f * (float)(MT * NT) + std::max(load, (float)a.N * (float)a.K / memory);
}

template <int TYPE>
static hipError_t linear_launch(const T8Product &a, hipStream_t st) {
  constexpr int tiles[5][2] = {{1, 1}, {1, 4}, {2, 2}, {2, 4}, {4, 4}};
  float best = t8_tile_time(a.M, a.N, a.K);
  int at = -1;
  for (int i = 4; i >= 0; --i) {
    const float t = few_time(a, tiles[i][0], tiles[i][1]);
    if (t <= best) {
      best = t;
      at = i;
    }
  }
  switch (at) {
    case 0: return few_launch<TYPE, 1, 1, 3>(a, st);
    case 1: return few_launch<TYPE, 1, 4, 3>(a, st);
    case 2: return few_launch<TYPE, 2, 2, 2>(a, st);
    case 3: return few_launch<TYPE, 2, 4, 2>(a, st);
    case 4: return few_launch<TYPE, 4, 4, 2>(a, st);
  }
  return launch_t8_tile(a, TYPE, st);
}

hipError_t launch_t8_linear(T8Product a, int type, hipStream_t st) {
  a.arows = a.M;
  if (type == QC_TYPE_F32) return linear_launch<QC_TYPE_F32>(a, st);
  if (type == QC_TYPE_F16) return linear_launch<QC_TYPE_F16>(a, st);
  return linear_launch<QC_TYPE_BF16>(a, st);
}

}  // namespace qc
