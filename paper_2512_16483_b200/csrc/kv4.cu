// Rows of keys and values quantised to 4 bits as they are written to the cache, and read back as bf16 (format: include/fvar.h).
//
// Both are bound by memory.  A lane holds 8 values (16 bytes of bf16, one 32-bit word of codes), a head's row is D / 8 lanes,
// the group's maximum is two shuffles over four lanes.  A warp takes kPasses x 32 / (D / 8) rows of one head, keys and values
// at once, all loads first; consecutive warps take consecutive heads of the same rows, which lie side by side in the input.
// 1600 rows of 2 x 16 heads, D = 128 (33 MB): write 10.4 us on its own with cold caches, read 7.4 behind it.  6425 rows of them read
// (133 MB): 20.7 us, 6.4 TB/s.  1 to 256 rows of 32 x 30 heads, D = 64: 12.2 and 9.7 us.  10521 rows of 37 x 8 heads (2.0 GB): 332 and 320 us,
// 6.1 and 6.3 TB/s (write: 422 us with comparisons and limits one value at a time).  Two passes a warp: 12 % slower writes at the large
// sizes; blocks of 128: 4 %.
#include "kv4.cuh"
#include "ptx.cuh"
#include "softmax.cuh"

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
// Magnitudes of two pairs: the greater ones (a NaN wins), the smaller ones with the first one's signs.
__device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t clamp_abs2(uint32_t x, uint32_t top) {
  uint32_t d;
  asm("min.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(x), "r"(top));
  return d;
}
// x / s rounded to the nearest integer, halves away from zero: x (1 / s) + 1.5 2^23 is rounded there.  |x| / s is a half-integer or at least
// 2^-9 away from one (x has eight bits, s four), so 1 / s taken larger by 2^-13 moves the halves, and nothing else, across; it also
// covers the error of 1 / s.  The four even and the four odd numbers are added up as fp32 integers, two at a time, in their places over
// 2^23 + 0x8888 (8 in each place), whose last 16 bits are then the half-word.
constexpr float kToInt = 12582912.0f, kCodeBase = 8388608.0f + 34952.0f;
__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
// NaN -> 0 in both halves.
__device__ __forceinline__ uint32_t drop_nan2(uint32_t v) {
  const uint32_t lo = (v & 0x7FFFu) > 0x7F80u ? 0u : v & 0xFFFFu, hi = (v & 0x7FFF0000u) > 0x7F800000u ? 0u : v & 0xFFFF0000u;
  return lo | hi;
}

// The rows of one warp: kRows rows from i0 on of head h of element b.
struct Kv4Place {
  int b, h, i0;
  int n;                        // rows of the element that there are
  int at;                       // cache row of row 0
  long long row0;               // row 0 of the head, in rows of the whole cache
};
template <int D>
__device__ __forceinline__ bool kv4_place(const Kv4Args &p, int b, Kv4Place &w) {
  constexpr int kRows = kPasses * (32 / (D / 8));
  const int unit = static_cast<int>(blockIdx.x) * (kKv4Threads / 32) + (threadIdx.x >> 5);
  if (unit >= p.units) return false;
  const int block = fast_div(unit, p.div_h);
  w.h = unit - block * p.H;
  w.i0 = block * kRows;
  w.b = b;
  w.n = p.count ? min(max(p.count[b], 0), p.n) : p.n;
  w.at = p.start ? p.start[b] : p.L0;
  w.row0 = b * p.elem_stride + static_cast<long long>(w.h) * p.L_cap;
  return w.i0 < w.n;
}
// Cache row of row i of the element, -1 if there is none.
__device__ __forceinline__ int kv4_row(const Kv4Args &p, const Kv4Place &w, int i, bool &bad) {
  if (i >= w.n) return -1;
  const long long pos = static_cast<long long>(w.at) + i;
  if (pos < 0 || pos >= p.L_cap) { bad = true; return -1; }
  return static_cast<int>(pos);
}

template <int D>
__device__ __forceinline__ void kv4_write_rows(const Kv4Args &p, const Kv4Place &w, int lane) {
  constexpr int kLanes = D / 8, kStep = 32 / kLanes, kGroups = D / kKv4Group;
  const int c = lane % kLanes, r0 = lane / kLanes;
  bool bad = false;
  uint4 x[2][kPasses];
  int row[kPasses];
  const long long src = (static_cast<long long>(w.b) * p.n + w.i0 + r0) * p.ld + w.h * D + c * 8;
#pragma unroll
  for (int t = 0; t < kPasses; ++t) {
    row[t] = kv4_row(p, w, w.i0 + t * kStep + r0, bad);
#pragma unroll
    for (int v = 0; v < 2; ++v)
      x[v][t] = row[t] >= 0 ? __ldcs(reinterpret_cast<const uint4 *>((v ? p.v_rows : p.k_rows) + src + t * kStep * p.ld)) : make_uint4(0, 0, 0, 0);
  }
  if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(p.status, kStatusBadIndex);
  // the row whose scales this lane writes: a row's are kGroups bytes
  const int srow = lane < kPasses * kStep ? kv4_row(p, w, w.i0 + lane, bad) : -1;
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    uint32_t bytes = 0;                                   // of the lane's group, a byte a pass
    uint32_t *codes = reinterpret_cast<uint32_t *>(v ? p.v_codes : p.k_codes) + w.row0 * kLanes + c;
#pragma unroll
    for (int t = 0; t < kPasses; ++t) {
      uint32_t e[4] = {x[v][t].x, x[v][t].y, x[v][t].z, x[v][t].w};
      uint32_t top2 = max_abs2(max_abs2(e[0], e[1]), max_abs2(e[2], e[3])) & 0x7FFF7FFFu;
      if (__any_sync(0xffffffffu, (top2 & 0xFFFFu) > 0x7F80u || top2 > 0x7F80FFFFu)) {       // a NaN in the warp: rarely
#pragma unroll
        for (int k = 0; k < 4; ++k) e[k] = drop_nan2(e[k]);
        top2 = max_abs2(max_abs2(e[0], e[1]), max_abs2(e[2], e[3])) & 0x7FFF7FFFu;
      }
      // bit patterns are ordered as the magnitudes are
      top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 1));
      top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 2));
      const uint32_t byte = kv4_scale_byte(fmaxf(bf_lo(top2), bf_hi(top2)));
      bytes |= byte << (8 * t);
      const uint32_t most = mul_bf2(kv4_scale2(byte), 0x40E040E0u);                          // 7 s: exact, and what is beyond it takes 7
      float inv_s;
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv_s) : "f"(__uint_as_float((byte + (107u << 3)) << 20)));
      inv_s *= 1.0f + 1.0f / 8192.0f;
      const uint64_t inv2 = pack_f2(inv_s, inv_s), up2 = pack_f2(kToInt, kToInt), down2 = pack_f2(-kToInt, -kToInt);
      uint64_t sum2 = pack_f2(kCodeBase, kCodeBase);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t x = clamp_abs2(e[k], most);
        const float place = static_cast<float>(1 << (4 * k));
        sum2 = fma_f2(add_f2(fma_f2(pack_f2(bf_lo(x), bf_hi(x)), inv2, up2), down2), pack_f2(place, place), sum2);
      }
      float even, odd;
      unpack_f2(sum2, even, odd);
      const uint32_t word = __byte_perm(__float_as_uint(even), __float_as_uint(odd), 0x5410);
      if (row[t] >= 0) codes[static_cast<long long>(row[t]) * kLanes] = word;
    }
    // Rows side by side have their scales side by side: a lane gathers those of one row, 32 bytes a warp.  (A byte a group and
    // pass, as they come, took 18.0 us for 1600 rows of 2 x 16 heads, with the slower arithmetic of that time.)
    const int from = lane / kStep * 8;                    // shift of the pass in which row i0 + lane was
    uint32_t mine = 0;
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
      mine |= ((__shfl_sync(0xffffffffu, bytes, (lane % kStep) * kLanes + g * 4) >> (from & 31)) & 255u) << (8 * g);
    uint8_t *dst = (v ? p.v_scales : p.k_scales) + (w.row0 + srow) * kGroups;
    if (srow >= 0) {
      if constexpr (kGroups == 4) *reinterpret_cast<uint32_t *>(dst) = mine;
      else *reinterpret_cast<uint16_t *>(dst) = static_cast<uint16_t>(mine);
    }
  }
}

template <int D>
__device__ __forceinline__ void kv4_read_rows(const Kv4Args &p, const Kv4Place &w, int lane) {
  constexpr int kLanes = D / 8, kStep = 32 / kLanes;
  const int c = lane % kLanes, r0 = lane / kLanes;
  bool bad = false;
  uint32_t word[2][kPasses], byte[2][kPasses];
  bool there[kPasses];
#pragma unroll
  for (int t = 0; t < kPasses; ++t) {
    const int pos = kv4_row(p, w, w.i0 + t * kStep + r0, bad);
    there[t] = pos >= 0;
    const long long row = w.row0 + pos;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      word[v][t] = there[t] ? __ldcs(reinterpret_cast<const uint32_t *>(v ? p.v_codes : p.k_codes) + row * kLanes + c) : 0u;
      byte[v][t] = there[t] ? (v ? p.v_scales : p.k_scales)[row * (D / kKv4Group) + c / 4] : 0u;
    }
  }
  if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(p.status, kStatusBadIndex);
  const long long dst = w.b * p.out_elem + (w.i0 + r0) * p.out_row + w.h * p.out_head + c * 8;
#pragma unroll
  for (int t = 0; t < kPasses; ++t)
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      if (!there[t]) continue;
      const uint32_t s2 = kv4_scale2(byte[v][t]);
      uint32_t o[4];
      kv4_word(word[v][t], s2, kv4_offset2(s2), o);
      *reinterpret_cast<uint4 *>((v ? p.v_out : p.k_out) + dst + t * kStep * p.out_row) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

template <int D, bool WRITE>
__global__ void __launch_bounds__(kKv4Threads) kv4_rows_kernel(const __grid_constant__ Kv4Args p) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  for (int b = blockIdx.y; b < p.B; b += gridDim.y) {
    Kv4Place w;
    if (!kv4_place<D>(p, b, w)) continue;
    if constexpr (WRITE) kv4_write_rows<D>(p, w, lane);
    else kv4_read_rows<D>(p, w, lane);
  }
}

cudaError_t launch_kv4_rows(bool write, Kv4Args a, cudaStream_t st) {
  const int rows = kPasses * (32 / (a.D / 8));
  const long long units = static_cast<long long>(a.H) * ((a.n + rows - 1) / rows);
  if (units > 0x7FFFFFF0) return cudaErrorInvalidValue;
  a.units = static_cast<int>(units);
  a.div_h = make_fast_div(a.H, units);
  const dim3 g(static_cast<unsigned>((units + kKv4Threads / 32 - 1) / (kKv4Threads / 32)), a.B < 65535 ? a.B : 65535), b(kKv4Threads);
  if (a.D == 64) return write ? launch_pdl(kv4_rows_kernel<64, true>, g, b, 0, st, a) : launch_pdl(kv4_rows_kernel<64, false>, g, b, 0, st, a);
  return write ? launch_pdl(kv4_rows_kernel<128, true>, g, b, 0, st, a) : launch_pdl(kv4_rows_kernel<128, false>, g, b, 0, st, a);
}

}  // namespace fvar
