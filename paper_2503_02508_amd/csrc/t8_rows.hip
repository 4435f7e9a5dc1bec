// Rows with a scale each: the quantiser of plain rows, of gated rows and of normalised rows, the planes of gradients, and the reading of codes.
//
// All of them move bytes: a row is read once, held in registers as float32 while its largest value is found, and written.  One wavefront
// takes a row of up to 256 vectors of 16 bytes, a workgroup of 2 - 16 wavefronts a longer one (or a short one where there are few rows:
// then nothing but latency counts), and rows beyond 16 wavefronts' registers are read again for each of the steps.
// Kernels alone: codes of 16384 x 4608 bfloat16 37.3 us, 6.1 TB/s; of its gated rows 70.9 us, 5.3 TB/s (the instructions take 60 of them); the norm of
// 16384 x 1152 bfloat16 with its residual 27.1 us, 4.9 TB/s; planes of 8192 x 4608 bfloat16 37.4 us, 5.1 TB/s; codes read back, 16384 x 4608 to
// bfloat16, 36 us, 6.3 TB/s.  One row of 8192 takes 3.6 us, 77 of 4608 float32 3.3: a read, two reductions, a write.
//
// Exact decisions.  The codes are those of the definition: float32 quotients, rounded half to even.  Each is formed as v (1 / scale), which is off by
// at most 1.2e-5 for quotients of up to 127, and where it is nearer than 2e-5 to a border the division decides.  The gated product is
// formed in float32 to 1.8e-6 of its value; where that is too near to a border, or to the row's largest value, float64 decides.
#include "t8_common.h"

namespace qc {

constexpr float T8_MAGIC = 12582912.0f;      // 1.5 2^23: a sum with it is rounded to an integer, which its low byte holds
constexpr float T8_NEAR = 2e-5f;
constexpr float T8_TINY = 0x1p-60f;          // gated rows with nothing above it are decided in float64 throughout
constexpr float T8_EMPTY = 0x1p-100f;        // gradients' rows with nothing above it are taken for zeros

__device__ __forceinline__ unsigned t8_code(float v, float scale) {
  const float n = fminf(fmaxf(__builtin_rintf(v / scale), -127.0f), 127.0f);
  return (unsigned)(int)n;
}

// One row's reductions over the wavefronts of a workgroup, a slot for each use.  Where a workgroup walks over rows the slots alternate from row to
// row: a wavefront that writes one again is at least one barrier behind the last that read it.
struct T8Across {
  double d[2][16];
  unsigned u[2][2][16];
};

// FULL: a workgroup a row (else a wavefront).  C: vectors a lane.
template <int TYPE, int SOURCE, bool FULL, int C>
__global__ __launch_bounds__(FULL ? 1024 : 256) void t8_rows_kernel(T8RowArgs a) {
  using T = typename W4Mem<TYPE>::T;
  constexpr int VL = t8_vl<TYPE>, ACT = SOURCE == T8_GELU ? QC_ACT_GELU : QC_ACT_SILU;
  constexpr bool GATED = SOURCE == T8_SILU || SOURCE == T8_GELU;
  __shared__ T8Across across;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves = FULL ? (int)blockDim.x >> 6 : 1, step = 64 * waves * VL, e0 = (FULL ? (int)threadIdx.x : lane) * VL;
  const int width = SOURCE == T8_PLANES ? a.pitch : a.K;
  // (one row a workgroup or wavefront: what does not depend on the row would be worked out ahead of a loop, in registers that then hold nothing else)
  const int64_t row = FULL ? blockIdx.x + (int64_t)blockIdx.y * gridDim.x : (blockIdx.x + (int64_t)blockIdx.y * gridDim.x) * 4 + wave;
  if (row >= a.M) return;
  const T *x = (const T *)a.x + row * a.ldx, *add = (const T *)a.add + row * a.lda;
  float v[C][VL], w[C][VL];
  w4_u4 first[C], second[C];
  // Gated rows: a wavefront whose elements all exist loads them without the masks, one behind the other (16384 x 4608 bfloat16 77 -> 73.6 us, 8192 x 14336
  // 114 -> 106; the other sources, whose instructions do not count, gain nothing: 16384 x 1152 float32 15.8 -> 17.3)
  if (GATED && ((FULL ? wave : 0) + 1) * 64 * VL + (C - 1) * step <= a.K) {
#pragma unroll
    for (int c = 0; c < C; ++c) first[c] = *(const t8_u4 *)((const char *)x + (unsigned)(e0 + c * step) * (unsigned)sizeof(T));
#pragma unroll
    for (int c = 0; c < C; ++c) second[c] = *(const t8_u4 *)((const char *)add + (unsigned)(e0 + c * step) * (unsigned)sizeof(T));
  } else {
#pragma unroll
    for (int c = 0; c < C; ++c) first[c] = t8_raw<TYPE>(x, e0 + c * step, a.K);
    if (GATED || (SOURCE == T8_NORM && a.add)) {
#pragma unroll
      for (int c = 0; c < C; ++c) second[c] = t8_raw<TYPE>(add, e0 + c * step, a.K);
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c) t8_values<TYPE>(first[c], v[c]);
  if constexpr (SOURCE == T8_PLANES) {
#pragma unroll
    for (int c = 0; c < C; ++c) t8_load_f32<VL>(a.w, e0 + c * step, a.K, w[c]);
  }
  if constexpr (SOURCE == T8_NORM) {
    if (a.add) {
      T *h = (T *)a.h + row * a.ldh;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float r[VL];
        t8_values<TYPE>(second[c], r);
#pragma unroll
        for (int i = 0; i < VL; ++i) v[c][i] = W4Mem<TYPE>::get(W4Mem<TYPE>::put(v[c][i] + r[i]));
        t8_store<TYPE>(h, e0 + c * step, a.K, v[c]);
      }
    }
    double ss = 0.0;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < VL; ++i) ss = __builtin_fma((double)v[c][i], (double)v[c][i], ss);
    ss = wave_sum_dpp(ss);
    if constexpr (FULL) {
      if (lane == 0) across.d[0][wave] = ss;
      t8_lds_barrier();
      ss = t8_across_sum(across.d[0], waves, lane);
    }
    const float rho = (float)t8_rsqrt(__builtin_fma(ss, a.share, (double)a.eps));
    asm volatile("" ::: "memory");                      // the weight is not loaded sooner: registers, and with them wavefronts
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int i = 0; i < VL; ++i) v[c][i] *= rho;
      if (a.w) {
        t8_load_f32<VL>(a.w, e0 + c * step, a.K, w[c]);
#pragma unroll
        for (int i = 0; i < VL; ++i) v[c][i] *= w[c][i];
      }
    }
    if (a.y) {
#pragma unroll
      for (int c = 0; c < C; ++c) t8_store<TYPE>((T *)a.y + row * a.ldy, e0 + c * step, a.K, v[c]);
    }
    if (!a.q) return;
  }
  uint32_t deep = 0;                                    // elements (c VL + i) whose gate is far below zero: float64 decides them
  if constexpr (GATED) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float g[VL], least = 0.0f;
      t8_values<TYPE>(second[c], g);
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        v[c][i] = t8_gate<ACT>(g[i], v[c][i]);
        least = fminf(least, g[i]);
      }
      if (least < T8_DEEP<ACT>) {
        // (until then they are nothing: a gate at its type's lowest value would be the row's largest.  What is not finite stays.)
        float f[VL];
        t8_values<TYPE>(first[c], f);
#pragma unroll
        for (int i = 0; i < VL; ++i)
          if (g[i] < T8_DEEP<ACT>) {
            deep |= 1u << (c * VL + i);
            if (t8_mag(g[i]) < 0x7F800000u && t8_mag(f[i]) < 0x7F800000u) v[c][i] = 0.0f;
          }
      }
    }
  }
  if constexpr (SOURCE == T8_PLANES) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < VL; ++i) v[c][i] *= w[c][i];
  }
  float tops[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    tops[c] = fabsf(v[c][0]);
#pragma unroll
    for (int i = 1; i < VL; ++i) tops[c] = t8_larger(tops[c], v[c][i]);
  }
  unsigned top = t8_mag(tops[0]);
#pragma unroll
  for (int c = 1; c < C; ++c) top = max(top, t8_mag(tops[c]));
  const auto over_row = [&](unsigned t, int use) {
    t = t8_wave_max(t);
    if constexpr (FULL) {
      if (lane == 0) across.u[0][use][wave] = t;
      t8_lds_barrier();
      t = t8_across_max(across.u[0][use], waves, lane);
    }
    return t;
  };
  top = over_row(top, 0);
  const bool lost = top >= 0x7F800000u;                 // an infinity or a NaN

  if constexpr (SOURCE == T8_PLANES) {
    constexpr int P = t8_planes(TYPE);
    const float most = __builtin_bit_cast(float, top);
    const bool empty = most < T8_EMPTY;
    const double full = P == 3 ? T8_PLANE_TOP : T8_PLANE_TOP * 256.0, mult = lost || empty ? 0.0 : full / (double)most;
    if (e0 == 0) a.scale[row] = lost ? __builtin_nanf("") : empty ? 0.0f : (float)((double)most / T8_PLANE_TOP);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      unsigned b[VL];
      int t[VL];
#pragma unroll
      for (int i = 0; i < VL; ++i) t[i] = lost ? 0 : (int)__builtin_rint((double)v[c][i] * mult);
#pragma unroll
      for (int p = 0; p < P; ++p) {
#pragma unroll
        for (int i = 0; i < VL; ++i) {
          b[i] = (unsigned)t[i];
          t[i] = (t[i] >> 8) + ((t[i] >> 7) & 1);       // what is left when a signed byte is taken away
        }
        t8_store_bytes<VL>(a.q + t8_plane_row((int)row, p, P) * a.pitch, e0 + c * step, a.pitch, b);
      }
    }
  } else {
    // elements that float64 or the division decides, as a word of bits (c VL + i), read again; few
    uint32_t flags = deep;
    const auto element = [&](int bit) { return e0 + bit / VL * step + bit % VL; };
    const auto exact = [&](int e) {
      const float g = W4Mem<TYPE>::get(add[e]), f = W4Mem<TYPE>::get(x[e]);
      return g == 0.0f || f == 0.0f || g < T8_GONE<ACT> ? 0.0f : (float)t8_gate_exact(ACT, g, f);      // rows of padding are zeros
    };
    const bool tiny = GATED && __builtin_bit_cast(float, top) < T8_TINY;
    if constexpr (GATED) {
      if (!lost) {
        const float near = __builtin_bit_cast(float, top) * (1.0f - 5e-6f);
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (tiny || tops[c] >= near) {
#pragma unroll
            for (int i = 0; i < VL; ++i) flags |= (tiny ? e0 + c * step + i < width : fabsf(v[c][i]) >= near) ? 1u << (c * VL + i) : 0u;
          }
        top = 0;
        while (flags) {
          const int bit = __builtin_ctz(flags);
          flags &= flags - 1;
          top = max(top, t8_mag(exact(element(bit))));
        }
        top = over_row(top, 1);
      }
      flags = deep;
    }
    float scale = __builtin_bit_cast(float, top) / 127.0f;
    if (scale == 0.0f) scale = 1.0f;
    const bool none = lost || top >= 0x7F800000u, all = tiny || scale < 0x1p-100f;
    if (e0 == 0) a.scale[row] = none ? __builtin_nanf("") : scale;
    const float inv = 1.0f / (all ? 1.0f : scale);
    int8_t *q = a.q + row * a.ldq;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      unsigned b[VL];
      float far = 0.0f;
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        const float m = __builtin_fmaf(v[c][i], inv, T8_MAGIC), n = m - T8_MAGIC, d = __builtin_fmaf(v[c][i], inv, -n);
        b[i] = __builtin_bit_cast(unsigned, m);
        if constexpr (GATED) far = fmaxf(far, __builtin_fmaf(fabsf(n), 2.5e-6f, fabsf(d)));
        else far = fmaxf(far, fabsf(d));
      }
      if (none) {
#pragma unroll
        for (int i = 0; i < VL; ++i) b[i] = 0;
      }
      t8_store_bytes<VL>(q, e0 + c * step, width, b);
      if (far > 0.5f - T8_NEAR) {
#pragma unroll
        for (int i = 0; i < VL; ++i) {
          const float n = __builtin_fmaf(v[c][i], inv, T8_MAGIC) - T8_MAGIC, d = fabsf(__builtin_fmaf(v[c][i], inv, -n));
          flags |= (GATED ? __builtin_fmaf(fabsf(n), 2.5e-6f, d) : d) > 0.5f - T8_NEAR ? 1u << (c * VL + i) : 0u;
        }
      }
    }
    if (all) flags = ~0u >> (32 - C * VL);
    if (none) flags = 0;
    while (flags) {                                     // a byte behind its vector, from the same lane: in this order
      const int bit = __builtin_ctz(flags), e = element(bit);
      flags &= flags - 1;
      if (e >= width) continue;
      float t;
      if constexpr (GATED) {
        t = exact(e);
      } else if constexpr (SOURCE == T8_NORM) {
        t = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < VL; ++i)
            if (bit == c * VL + i) t = v[c][i];
      } else {
        t = W4Mem<TYPE>::get(x[e]);
      }
      q[e] = (int8_t)t8_code(t, scale);
    }
  }
}

// Rows of any length, read again for each step; element after element, the gate in float64 twice: codes of 256 x 53248 bfloat16 35 us a call, of gated
// ones 70, where the bytes would take 8 and 14.
template <int TYPE, int SOURCE>
__global__ __launch_bounds__(1024) void t8_long_rows_kernel(T8RowArgs a) {
  using T = typename W4Mem<TYPE>::T;
  constexpr bool GATED = SOURCE == T8_SILU || SOURCE == T8_GELU;
  __shared__ T8Across across;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x, turn ^= 1) {
    const T *x = (const T *)a.x + row * a.ldx, *add = (const T *)a.add + row * a.lda;
    float rho = 1.0f;
    if constexpr (SOURCE == T8_NORM) {
      double ss = 0.0;
      T *h = (T *)a.h + row * a.ldh;
      for (int e = threadIdx.x; e < a.K; e += 1024) {
        float v = W4Mem<TYPE>::get(x[e]);
        if (a.add) {
          const T s = W4Mem<TYPE>::put(v + W4Mem<TYPE>::get(add[e]));
          v = W4Mem<TYPE>::get(s);
          h[e] = s;
        }
        ss = __builtin_fma((double)v, (double)v, ss);
      }
      ss = wave_sum_dpp(ss);
      if (lane == 0) across.d[turn][wave] = ss;
      __syncthreads();
      ss = t8_across_sum(across.d[turn], 16, lane);
      rho = (float)t8_rsqrt(__builtin_fma(ss, a.share, (double)a.eps));
      if (a.add) x = h;                                   // each thread reads what it wrote
    }
    const auto value = [&](int e) {
      float v = W4Mem<TYPE>::get(x[e]);
      if constexpr (GATED) v = (float)t8_gate_exact(SOURCE == T8_GELU ? QC_ACT_GELU : QC_ACT_SILU, W4Mem<TYPE>::get(add[e]), v);
      if constexpr (SOURCE == T8_PLANES) v *= a.w[e];
      if constexpr (SOURCE == T8_NORM) {
        v *= rho;
        if (a.w) v *= a.w[e];
      }
      return v;
    };
    unsigned top = 0;
    for (int e = threadIdx.x; e < a.K; e += 1024) {
      const float v = value(e);
      top = max(top, t8_mag(v));
      if constexpr (SOURCE == T8_NORM)
        if (a.y) ((T *)a.y)[row * a.ldy + e] = W4Mem<TYPE>::put(v);
    }
    if (SOURCE == T8_NORM && !a.q) continue;
    top = t8_wave_max(top);
    if (lane == 0) across.u[turn][0][wave] = top;
    __syncthreads();
    top = t8_across_max(across.u[turn][0], 16, lane);
    const bool lost = top >= 0x7F800000u;
    if constexpr (SOURCE == T8_PLANES) {
      constexpr int P = t8_planes(TYPE);
      const float most = __builtin_bit_cast(float, top);
      const bool empty = most < T8_EMPTY;
      const double full = P == 3 ? T8_PLANE_TOP : T8_PLANE_TOP * 256.0, mult = lost || empty ? 0.0 : full / (double)most;
      if (threadIdx.x == 0) a.scale[row] = lost ? __builtin_nanf("") : empty ? 0.0f : (float)((double)most / T8_PLANE_TOP);
      for (int e = threadIdx.x; e < a.pitch; e += 1024) {
        int t = 0;
        if (!lost && e < a.K) t = (int)__builtin_rint((double)value(e) * mult);
        for (int p = 0; p < P; ++p) {
          a.q[t8_plane_row((int)row, p, P) * a.pitch + e] = (int8_t)t;
          t = (t >> 8) + ((t >> 7) & 1);
        }
      }
    } else {
      float scale = __builtin_bit_cast(float, top) / 127.0f;
      if (scale == 0.0f) scale = 1.0f;
      if (threadIdx.x == 0) a.scale[row] = lost ? __builtin_nanf("") : scale;
      for (int e = threadIdx.x; e < a.K; e += 1024) a.q[row * a.ldq + e] = lost ? (int8_t)0 : (int8_t)t8_code(value(e), scale);
    }
  }
}

// Up to 4 vectors a lane: what a wavefront does once a row (its reductions, root and division) costs as much as one or two of them.
// Where the rows are fewer than the chip has wavefronts, one a lane.
template <int TYPE, int SOURCE>
static hipError_t rows_launch(const T8RowArgs &a, hipStream_t st) {
  constexpr int VL = t8_vl<TYPE>;
  const int vectors = ((SOURCE == T8_PLANES ? a.pitch : a.K) + VL - 1) / VL;
  if (vectors > 64 * 16 * 4 || a.K < VL) {
    t8_long_rows_kernel<TYPE, SOURCE><<<(unsigned)std::min(a.M, 1024), 1024, 0, st>>>(a);
    return hipGetLastError();
  }
  int waves = (vectors + 255) / 256;
  while (waves < 16 && vectors > 64 * waves && (int64_t)a.M * waves < 2048) ++waves;
  const int c = (vectors + 64 * waves - 1) / (64 * waves);
  const int groups = waves == 1 ? (a.M + 3) / 4 : a.M;
  const dim3 grid((unsigned)std::min(groups, 1 << 20), (unsigned)((groups + (1 << 20) - 1) >> 20));
  if (waves == 1) {
    if (c == 1) t8_rows_kernel<TYPE, SOURCE, false, 1><<<grid, 256, 0, st>>>(a);
    else if (c == 2) t8_rows_kernel<TYPE, SOURCE, false, 2><<<grid, 256, 0, st>>>(a);
    else if (c == 3) t8_rows_kernel<TYPE, SOURCE, false, 3><<<grid, 256, 0, st>>>(a);
    else t8_rows_kernel<TYPE, SOURCE, false, 4><<<grid, 256, 0, st>>>(a);
  } else {
    if (c == 1) t8_rows_kernel<TYPE, SOURCE, true, 1><<<grid, 64 * waves, 0, st>>>(a);
    else if (c == 2) t8_rows_kernel<TYPE, SOURCE, true, 2><<<grid, 64 * waves, 0, st>>>(a);
    else if (c == 3) t8_rows_kernel<TYPE, SOURCE, true, 3><<<grid, 64 * waves, 0, st>>>(a);
    else t8_rows_kernel<TYPE, SOURCE, true, 4><<<grid, 64 * waves, 0, st>>>(a);
  }
  return hipGetLastError();
}

template <int TYPE>
static hipError_t rows_source(const T8RowArgs &a, int source, hipStream_t st) {
  if (source == T8_PLAIN) return rows_launch<TYPE, T8_PLAIN>(a, st);
  if (source == T8_SILU) return rows_launch<TYPE, T8_SILU>(a, st);
  if (source == T8_GELU) return rows_launch<TYPE, T8_GELU>(a, st);
  if (source == T8_NORM) return rows_launch<TYPE, T8_NORM>(a, st);
  return rows_launch<TYPE, T8_PLANES>(a, st);
}

hipError_t launch_t8_rows(const T8RowArgs &a, int type, int source, hipStream_t st) {
  if (type == QC_TYPE_F32) return rows_source<QC_TYPE_F32>(a, source, st);
  if (type == QC_TYPE_F16) return rows_source<QC_TYPE_F16>(a, source, st);
  return rows_source<QC_TYPE_BF16>(a, source, st);
}

// ---------------------------------------------------------------- codes to values; the gates' gradient
// Elementwise: a workgroup takes `rows` whole rows (as many as make some thousand elements), or one a part of a row at a time.
template <int TYPE>
__global__ __launch_bounds__(256) void t8_expand_kernel(const int8_t *q, int64_t ldq, const float *scale, int M, int K, typename W4Mem<TYPE>::T *out, int64_t ldo,
                                                        int rows, int vectors) {
  constexpr int VL = t8_vl<TYPE>;                          // one store: 16 bytes beside 16 bytes, whole lines (two of float32 in turn: 151 us for 79)
  const int64_t first = (int64_t)blockIdx.x * rows;
  const int count = (int)min((int64_t)rows, M - first) * vectors;
  for (int t = blockIdx.y * 256 + threadIdx.x; t < count; t += gridDim.y * 256) {
    const int r = t / vectors, e = (t - r * vectors) * VL;
    const int64_t row = first + r;
    const float s = scale[row];
    const int8_t *from = q + row * ldq;
    typename W4Mem<TYPE>::T *to = out + row * ldo;
    float v[VL];
    if (e + VL <= K) {
      unsigned b[2];
      if constexpr (VL == 8) {
        const w4_u2 both = *(const t8_u2 *)(from + e);
        b[0] = both[0], b[1] = both[1];
      } else {
        b[0] = *(const t8_u1 *)(from + e);
      }
#pragma unroll
      for (int i = 0; i < VL; ++i) v[i] = (float)(int8_t)(b[i / 4] >> (8 * (i % 4))) * s;
    } else {
#pragma unroll
      for (int i = 0; i < VL; ++i) v[i] = e + i < K ? (float)from[e + i] * s : 0.0f;
    }
    t8_store<TYPE>(to, e, K, v);
  }
}

hipError_t launch_t8_expand(const int8_t *q, int64_t ldq, const float *scale, int M, int K, void *out, int type, int64_t ldo, hipStream_t st) {
  const int vl = type == QC_TYPE_F32 ? 4 : 8, vectors = (K + vl - 1) / vl, rows = std::max(1, 1024 / vectors);
  const dim3 grid((unsigned)((M + rows - 1) / rows), (unsigned)std::max(1, std::min(16, vectors / 1024)));
  if (type == QC_TYPE_F32) t8_expand_kernel<QC_TYPE_F32><<<grid, 256, 0, st>>>(q, ldq, scale, M, K, (float *)out, ldo, rows, vectors);
  else if (type == QC_TYPE_F16) t8_expand_kernel<QC_TYPE_F16><<<grid, 256, 0, st>>>(q, ldq, scale, M, K, (_Float16 *)out, ldo, rows, vectors);
  else t8_expand_kernel<QC_TYPE_BF16><<<grid, 256, 0, st>>>(q, ldq, scale, M, K, (__bf16 *)out, ldo, rows, vectors);
  return hipGetLastError();
}

// Every element is read before any of the same thread's results is written, so that results may take their inputs' place.
// Bytes bound it, and not far below them the instructions: 4096 x 4608 float16, GELU, 33.3 us a call among others, 5.7 TB/s (35.3 alone under a profiler).  When it
// was measured beside them, 32.7 against 35.3 with two vectors a thread and 37.8 with what far gates need in every element's way.
template <int TYPE, int ACT>
__global__ __launch_bounds__(256) void t8_gated_grad_kernel(const void *x, int64_t ldx, const void *g, int64_t ldg, const void *dv, int64_t lddv, int64_t M,
                                                            int K, void *dx, int64_t lddx, void *dg, int64_t lddg, int rows, int vectors) {
  using T = typename W4Mem<TYPE>::T;
  constexpr int VL = t8_vl<TYPE>;
  const int64_t first = (int64_t)blockIdx.x * rows;
  const int count = (int)min((int64_t)rows, M - first) * vectors;
  for (int t = blockIdx.y * 256 + threadIdx.x; t < count; t += gridDim.y * 256) {
    const int r = t / vectors, e = (t - r * vectors) * VL;
    const int64_t row = first + r;
    float xv[VL], gv[VL], d[VL], rx[VL], rg[VL];
    t8_load<TYPE>((const T *)x + row * ldx, e, K, xv);
    t8_load<TYPE>((const T *)g + row * ldg, e, K, gv);
    t8_load<TYPE>((const T *)dv + row * lddv, e, K, d);
    float most = fabsf(gv[0]);
#pragma unroll
    for (int i = 1; i < VL; ++i) most = t8_larger(most, gv[i]);
    if (most < T8_FAR<ACT>) {
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        rx[i] = d[i] * t8_act_near<ACT>(gv[i], rg[i]);
        rg[i] *= d[i] * xv[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        rx[i] = d[i] * t8_act(ACT, gv[i], rg[i]);
        rg[i] *= d[i] * xv[i];
      }
    }
    t8_store<TYPE>((T *)dx + row * lddx, e, K, rx);
    t8_store<TYPE>((T *)dg + row * lddg, e, K, rg);
  }
}

// rows that are shorter than a vector
template <int TYPE>
__global__ __launch_bounds__(256) void t8_gated_grad_narrow_kernel(const void *x, int64_t ldx, const void *g, int64_t ldg, const void *dv, int64_t lddv, int act,
                                                                   int64_t M, int K, void *dx, int64_t lddx, void *dg, int64_t lddg) {
  using T = typename W4Mem<TYPE>::T;
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, row = t / K, e = t % K;
  if (row >= M) return;
  const float xv = W4Mem<TYPE>::get(((const T *)x)[row * ldx + e]), gv = W4Mem<TYPE>::get(((const T *)g)[row * ldg + e]),
              d = W4Mem<TYPE>::get(((const T *)dv)[row * lddv + e]);
  float slope;
  const float rx = d * t8_act(act, gv, slope);
  ((T *)dx)[row * lddx + e] = W4Mem<TYPE>::put(rx);
  ((T *)dg)[row * lddg + e] = W4Mem<TYPE>::put(d * xv * slope);
}

template <int TYPE>
static void gated_grad(const void *x, int64_t ldx, const void *g, int64_t ldg, int act, const void *dv, int64_t lddv, int64_t M, int64_t K, void *dx, int64_t lddx,
                       void *dg, int64_t lddg, hipStream_t st) {
  constexpr int VL = t8_vl<TYPE>;
  // rows without anything between them are one row (of 32-bit offsets)
  if (M > 1 && ldx == K && ldg == K && lddv == K && lddx == K && lddg == K && M * K < (1ll << 30) - 4096) {
    K *= M;
    M = 1;
  }
  if (K < VL) {
    t8_gated_grad_narrow_kernel<TYPE><<<(unsigned)((M * K + 255) / 256), 256, 0, st>>>(x, ldx, g, ldg, dv, lddv, act, M, (int)K, dx, lddx, dg, lddg);
    return;
  }
  const int vectors = (int)((K + VL - 1) / VL), rows = std::max(1, 512 / vectors);
  const dim3 grid((unsigned)((M + rows - 1) / rows), (unsigned)std::max(1, std::min(M == 1 ? 16384 : 32, vectors / 256)));
  const auto kern = act == QC_ACT_SILU ? t8_gated_grad_kernel<TYPE, QC_ACT_SILU> : t8_gated_grad_kernel<TYPE, QC_ACT_GELU>;
  kern<<<grid, 256, 0, st>>>(x, ldx, g, ldg, dv, lddv, M, (int)K, dx, lddx, dg, lddg, rows, vectors);
}

hipError_t launch_t8_gated_grad(const void *x, int64_t ldx, const void *g, int64_t ldg, int act, const void *dv, int64_t lddv, int type, int M, int K, void *dx,
                                int64_t lddx, void *dg, int64_t lddg, hipStream_t st) {
  if (type == QC_TYPE_F32) gated_grad<QC_TYPE_F32>(x, ldx, g, ldg, act, dv, lddv, M, K, dx, lddx, dg, lddg, st);
  else if (type == QC_TYPE_F16) gated_grad<QC_TYPE_F16>(x, ldx, g, ldg, act, dv, lddv, M, K, dx, lddx, dg, lddg, st);
  else gated_grad<QC_TYPE_BF16>(x, ldx, g, ldg, act, dv, lddv, M, K, dx, lddx, dg, lddg, st);
  return hipGetLastError();
}

template <int TYPE>
__global__ __launch_bounds__(256) void t8_zero_kernel(typename W4Mem<TYPE>::T *x, int K, int64_t ld) {
  for (int k = threadIdx.x; k < K; k += 256) x[(int64_t)blockIdx.x * ld + k] = W4Mem<TYPE>::put(0.0f);
}

hipError_t launch_t8_zero(void *x, int type, int M, int K, int64_t ld, hipStream_t st) {
  if (type == QC_TYPE_F32) t8_zero_kernel<QC_TYPE_F32><<<M, 256, 0, st>>>((float *)x, K, ld);
  else if (type == QC_TYPE_F16) t8_zero_kernel<QC_TYPE_F16><<<M, 256, 0, st>>>((_Float16 *)x, K, ld);
  else t8_zero_kernel<QC_TYPE_BF16><<<M, 256, 0, st>>>((__bf16 *)x, K, ld);
  return hipGetLastError();
}

}  // namespace qc
