// Parts of the products of the 8-bit layers with a scale for each token.
#pragma once
#include "t8_common.h"

namespace qc {

typedef int t8_i4 __attribute__((ext_vector_type(4)));
typedef int t8_i2 __attribute__((ext_vector_type(2)));

// 1024 bytes from memory to LDS, 16 a lane: lane after lane from `lds` on.  (m0 is a reserved register, which a clobber list cannot name:
// nothing else in these kernels uses it, tests/test_codegen_t8_cpu.py)
__device__ __forceinline__ void t8_to_lds(unsigned lds, unsigned off, const void *base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base));
}
__device__ __forceinline__ void t8_word_to_lds(unsigned lds, unsigned off, const void *base) {      // 256 bytes, 4 a lane
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(off), "s"(base));
}
__device__ __forceinline__ unsigned t8_lds_address(const void *p) { return (unsigned)(size_t)(__attribute__((address_space(3))) const char *)p; }
// until at most N of this wavefront's loads are on their way (they end in order)
template <int N>
__device__ __forceinline__ void t8_wait() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
template <int N>
__device__ __forceinline__ void t8_wait_barrier() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }
__device__ __forceinline__ void t8_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A matrix instruction's 16 x 64 operand, rows of 128 bytes in LDS: row r's 16-byte chunk c lies at place c ^ swz(r), so that eight rows of one
// chunk lie in different banks
__device__ __forceinline__ int t8_swz(int r) { return r & 7; }

// Values of P planes of sums: plane p counts 256^(p + 3 - P) of the row's scale.  (float64: sums of two planes may cancel to less than either's float32
// rounding)
template <int P>
__device__ __forceinline__ float t8_join(const int s[P], float scale) {
  double v = (double)s[P - 1];
#pragma unroll
  for (int p = P - 2; p >= 0; --p) v = __builtin_fma(v, 256.0, (double)s[p]);
  return (float)(v * ((double)scale * (P == 4 ? 0x1p-8 : 1.0)));
}

}  // namespace qc
