// Arithmetic that the attention kernels share: packed fp32 pairs, three-input maxima, division by an invariant.
#pragma once
#include <stdint.h>

#include "internal.h"

namespace fvar {

// Softmax arithmetic on pairs of neighbouring keys: packed fp32, one instruction slot for two keys, and three-input
// maxima (a block took 576 issue slots a row, now 390).  Moving part of the exponentials from the special-function unit
// to a polynomial on the FMA pipe (degree 5, 1/8 to 1/2 of the keys) was measured and left out: 1144 TFLOP/s without,
// 1121 / 1089 / 1036 with 1/8, 1/4, 3/8 of them -- the chain through a tile's softmax bounds the kernel, not the unit.
__device__ __forceinline__ uint64_t pack_f2(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void unpack_f2(uint64_t v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma_f2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add_f2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// u / d by one multiplication where that is exact (see make_fast_div), else by a division (two in each role's way were 0.9 us
// of a 6 us launch).
__device__ __forceinline__ int fast_div(int u, const FastDiv &f) {
  return f.mul ? static_cast<int>(__umulhi(static_cast<unsigned>(u), f.mul)) : u / static_cast<int>(f.d);
}
inline FastDiv make_fast_div(unsigned d, unsigned long long max_u) {
  // ceil(2^32 / d) is exact for u with u * d < 2^32; d == 1 does not fit 32 bits
  return FastDiv{d, (d > 1 && max_u * d < (1ull << 32)) ? static_cast<unsigned>(((1ull << 32) + d - 1) / d) : 0u};
}

}  // namespace fvar
