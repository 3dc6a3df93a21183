// The format of the cache in 4 bits (include/fvar.h): decoding on the device.
#pragma once
#include <stdint.h>

#include "internal.h"

namespace fvar {

constexpr int kKv4Group = 32;                  // values a scale

// bf16 pair (s, s) of a scale byte: 8 e + m moved to exponent e - 20 + 127 and the top three mantissa bits.
__device__ __forceinline__ uint32_t kv4_scale2(uint32_t byte) { return byte * 0x00100010u + (107u << 7) * 0x00010001u; }
// The same for two bytes, one in each half; with 2^100 besides.
__device__ __forceinline__ uint32_t kv4_pairs(uint32_t bytes) { return bytes * 16u + (107u << 7) * 0x00010001u; }
__device__ __forceinline__ uint32_t kv4_pairs_p(uint32_t bytes) { return bytes * 16u + (207u << 7) * 0x00010001u; }
// The scale in byte g of four, as fp32.
__device__ __forceinline__ float kv4_scale_f32(uint32_t bytes, int g) {
  return __uint_as_float(__byte_perm(bytes, 0, 0x4440 + g) * 0x00100000u + (107u << 23));
}

__device__ __forceinline__ uint32_t fma_bf2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t mul_bf2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// -136 s: 136 = 17 * 8 and s has four significant bits, so the product has eight and is exact.
__device__ __forceinline__ uint32_t kv4_offset2(uint32_t s2) { return mul_bf2(s2, 0xC308C308u); }
// Two numbers of 4 bits in the low bits of both halves -> the two values.  0x4300 | u is 128 + u in bf16; (128 + u) s - 136 s =
// (u - 8) s has seven significant bits, so the one rounding of the fma changes nothing.  Mask and exponent in one three-input
// operation (written with & and |, it came out as two).
__device__ __forceinline__ uint32_t kv4_pair(uint32_t w, uint32_t s2, uint32_t off2) {
  uint32_t x;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(x) : "r"(w), "r"(0x000F000Fu), "r"(0x43004300u));      // (w & mask) | exponent
  return fma_bf2(x, s2, off2);
}
// A word of eight: values 2 p, 2 p + 1 in v[p].
__device__ __forceinline__ void kv4_word(uint32_t w, uint32_t s2, uint32_t off2, uint32_t (&v)[4]) {
#pragma unroll
  for (int p = 0; p < 4; ++p) v[p] = kv4_pair(w >> (4 * p), s2, off2);
}

}  // namespace fvar
