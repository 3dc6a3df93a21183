// Rows of keys and values quantised to 4 bits as they are written to the cache, and read back as bf16 (format: include/fvar.h).
//
// Both are bound by memory.  A lane holds 8 values (16 bytes of bf16, one 32-bit word of codes), a head's row is D / 8 lanes,
// the group's maximum is two shuffles over four lanes.  A warp takes kPasses x 32 / (D / 8) rows of one head, keys and values
// at once, all loads first; consecutive warps take consecutive heads of the same rows, which lie side by side in the input.
#include "kv4.cuh"
#include "ptx.cuh"

namespace fvar {

constexpr int kKv4Threads = 256;
constexpr int kPasses = 4;

// The least scale with 7.5 s >= top.  top / 7.5 has to be rounded up to four significant bits: exact quotients and all others
// are a relative 2^-9 apart from the next boundary (top has eight bits), so a product that is 2^-16 low decides as the quotient does.
__device__ __forceinline__ uint32_t kv4_scale_byte(float top) {
  const float t = top * ((1.0f - 1.0f / 65536.0f) / 7.5f);
  const int u = static_cast<int>((__float_as_uint(t) + 0x000FFFFFu) >> 20) - (107 << 3);      // exponent and three bits of mantissa
  return static_cast<uint32_t>(min(max(u, 0), 255));
}
// u = 8 + sign(x) min(7, floor(|x| / s + 1/2)).  |x| / s is a half-integer or at least 2^-9 away from one, so 2^-12 more than the
// half makes up for the rounding of 1 / s and of the product.  NaN: fminf and the comparison leave 0 of it (see below).
__device__ __forceinline__ uint32_t kv4_code(float x, float inv_s) {
  const float q = floorf(fmaf(fabsf(x), inv_s, 0.5f + 1.0f / 4096.0f));
  const int m = static_cast<int>(fminf(q, 7.0f));
  return static_cast<uint32_t>(x < 0.f ? 8 - m : 8 + m);
}
__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
// NaN -> 0 in both halves.
__device__ __forceinline__ uint32_t drop_nan2(uint32_t v) {
  const uint32_t lo = (v & 0x7FFFu) > 0x7F80u ? 0u : v & 0xFFFFu, hi = (v & 0x7FFF0000u) > 0x7F800000u ? 0u : v & 0xFFFF0000u;
  return lo | hi;
}

struct Kv4Place {
  int b, h, i0;                 // element, head, first row of the warp
  int n;                        // rows of the element
  int at;                       // cache row of row 0
};
template <int D>
__device__ __forceinline__ bool kv4_place(const Kv4Args &p, Kv4Place &w) {
  constexpr int kRows = kPasses * (32 / (D / 8));
  const long long unit = static_cast<long long>(blockIdx.x) * (kKv4Threads / 32) + (threadIdx.x >> 5);
  if (unit >= p.units) return false;
  const int blocks = (p.n + kRows - 1) / kRows;
  w.h = static_cast<int>(unit % p.H);
  const long long rest = unit / p.H;
  w.b = static_cast<int>(rest / blocks);
  w.i0 = static_cast<int>(rest - static_cast<long long>(w.b) * blocks) * kRows;
  w.n = p.count ? min(max(p.count[w.b], 0), p.n) : p.n;
  w.at = p.start ? p.start[w.b] : p.L0;
  return true;
}
// Cache row of row i of the element, -1 if there is none.
__device__ __forceinline__ long long kv4_row(const Kv4Args &p, const Kv4Place &w, int i, bool &bad) {
  if (i >= w.n) return -1;
  const long long pos = static_cast<long long>(w.at) + i;
  if (pos < 0 || pos >= p.L_cap) { bad = true; return -1; }
  return w.b * p.elem_stride + static_cast<long long>(w.h) * p.L_cap + pos;
}

template <int D>
__global__ void __launch_bounds__(kKv4Threads) kv4_write_kernel(const __grid_constant__ Kv4Args p) {
  constexpr int kLanes = D / 8, kStep = 32 / kLanes;
  pdl_wait();
  pdl_launch_dependents();
  Kv4Place w;
  if (!kv4_place<D>(p, w)) return;
  const int lane = threadIdx.x & 31, c = lane % kLanes, r0 = lane / kLanes;
  bool bad = false;
  uint4 x[2][kPasses];
  long long row[kPasses];
#pragma unroll
  for (int t = 0; t < kPasses; ++t) {
    const int i = w.i0 + t * kStep + r0;
    row[t] = kv4_row(p, w, i, bad);
    const long long src = (static_cast<long long>(w.b) * p.n + i) * p.ld + w.h * D + c * 8;
#pragma unroll
    for (int v = 0; v < 2; ++v)
      x[v][t] = row[t] >= 0 ? __ldcs(reinterpret_cast<const uint4 *>((v ? p.v_rows : p.k_rows) + src)) : make_uint4(0, 0, 0, 0);
  }
  if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(p.status, kStatusBadIndex);
#pragma unroll
  for (int t = 0; t < kPasses; ++t)
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      uint32_t e[4] = {x[v][t].x, x[v][t].y, x[v][t].z, x[v][t].w};
      uint32_t top2 = 0;                                             // maxima of the bit patterns: ordered as the magnitudes are
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        e[k] = drop_nan2(e[k]);
        top2 = __vmaxu2(top2, e[k] & 0x7FFF7FFFu);
      }
      top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 1));
      top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 2));
      const uint32_t byte = kv4_scale_byte(fmaxf(bf_lo(top2), bf_hi(top2)));
      const float inv_s = __frcp_rn(__uint_as_float((byte + (107u << 3)) << 20));
      uint32_t word = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) word |= kv4_code(bf_lo(e[k]), inv_s) << (4 * k) | kv4_code(bf_hi(e[k]), inv_s) << (16 + 4 * k);
      if (row[t] >= 0) {
        reinterpret_cast<uint32_t *>(v ? p.v_codes : p.k_codes)[row[t] * kLanes + c] = word;
        if ((c & 3) == 0) (v ? p.v_scales : p.k_scales)[row[t] * (D / kKv4Group) + c / 4] = static_cast<uint8_t>(byte);
      }
    }
}

template <int D>
__global__ void __launch_bounds__(kKv4Threads) kv4_read_kernel(const __grid_constant__ Kv4Args p) {
  constexpr int kLanes = D / 8, kStep = 32 / kLanes;
  pdl_wait();
  pdl_launch_dependents();
  Kv4Place w;
  if (!kv4_place<D>(p, w)) return;
  const int lane = threadIdx.x & 31, c = lane % kLanes, r0 = lane / kLanes;
  bool bad = false;
  uint32_t word[2][kPasses], byte[2][kPasses];
  bool there[kPasses];
#pragma unroll
  for (int t = 0; t < kPasses; ++t) {
    const long long row = kv4_row(p, w, w.i0 + t * kStep + r0, bad);
    there[t] = row >= 0;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      word[v][t] = there[t] ? __ldcs(reinterpret_cast<const uint32_t *>(v ? p.v_codes : p.k_codes) + row * kLanes + c) : 0u;
      byte[v][t] = there[t] ? (v ? p.v_scales : p.k_scales)[row * (D / kKv4Group) + c / 4] : 0u;
    }
  }
  if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(p.status, kStatusBadIndex);
#pragma unroll
  for (int t = 0; t < kPasses; ++t)
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      if (!there[t]) continue;
      const uint32_t s2 = kv4_scale2(byte[v][t]);
      uint32_t o[4];
      kv4_word(word[v][t], s2, kv4_offset2(s2), o);
      bf16 *dst = (v ? p.v_out : p.k_out) + w.b * p.out_elem + (w.i0 + t * kStep + r0) * p.out_row + w.h * p.out_head + c * 8;
      __stcs(reinterpret_cast<uint4 *>(dst), make_uint4(o[0], o[1], o[2], o[3]));
    }
}

cudaError_t launch_kv4_rows(bool write, Kv4Args a, cudaStream_t st) {
  const int rows = kPasses * (32 / (a.D / 8));
  a.units = static_cast<long long>(a.B) * a.H * ((a.n + rows - 1) / rows);
  const long long grid = (a.units + kKv4Threads / 32 - 1) / (kKv4Threads / 32);
  if (grid > 0x7FFFFFFF) return cudaErrorInvalidValue;
  const dim3 g(static_cast<unsigned>(grid)), b(kKv4Threads);
  if (a.D == 64) return write ? launch_pdl(kv4_write_kernel<64>, g, b, 0, st, a) : launch_pdl(kv4_read_kernel<64>, g, b, 0, st, a);
  return write ? launch_pdl(kv4_write_kernel<128>, g, b, 0, st, a) : launch_pdl(kv4_read_kernel<128>, g, b, 0, st, a);
}

}  // namespace fvar
