// Attention of query rows over a cache in 4 bits (format and operator: include/fvar.h).
//
// Few rows (attention_kv4_few_kernel, 16 query rows a cache head at a time): bound by reading the cache, so the codes go from
// memory to the tensor cores without a stop on the way: TMA brings them to shared memory as they are, a warp takes the codes of 16
// keys into registers in the order in which mma.sync wants its operand, and decodes them there.  (Through tcgen05 they would have to
// be decoded into shared memory and read from there again: 2.5 times their bf16 size at 128 bytes a clock, 1.8 times what
// reading the codes from HBM takes.)  Keys and values are the operand of 16 rows, the query rows the one of 8:
//   S^T [16 keys][8 rows] = K Q^T,   O^T [16 of D][8 rows] += V^T P^T.
// What bounds it is the arithmetic of decoding, so little of it is left:
//   keys     A number u of 4 bits in a byte is u 2^-9 as e4m3, from 0 to 15 (below 8 a subnormal number, and the first binade above has
//            the same step).  So one mask makes four operand elements of a word's even half-bytes, a shift and a mask those of the odd
//            ones.  Queries are split into two e4m3 terms after scaling their row by a power of two to 128 .. 256: q = hi + lo, exact
//            for elements above 2^-10 of the row's greatest, and off by 2^-18 of it at most below.  A product covers one group, and is
//            scaled when it is added to the score: s += scale (acc - 8 sum q), the last term as the accumulator's first value.
//   values   (128 + u) s - 136 s in bf16 pairs (kv4_pair), two keys in a register.
#include <limits.h>
#include <cuda_fp16.h>
#include <math.h>

#include "kv4.cuh"
#include "ptx.cuh"

namespace fvar {

// D[16][8] += A[16][16] B[16][8], bf16, fp32 accumulator.
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// D[16][8] = A[16][32] B[32][8] + C, e4m3, fp32 accumulator.
__device__ __forceinline__ void mma_16832(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, float c0, float c1,
                                          float c2, float c3) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
// Four floats as e4m3, the first in the lowest byte, and what they became.
__device__ __forceinline__ uint32_t to_e4m3(const float (&x)[4], float (&back)[4]) {
  uint16_t lo, hi;
  uint32_t b0, b1;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x[1]), "f"(x[0]));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x[3]), "f"(x[2]));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(b0) : "h"(lo));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(b1) : "h"(hi));
  const float2 f0 = __half22float2(*reinterpret_cast<const __half2 *>(&b0)), f1 = __half22float2(*reinterpret_cast<const __half2 *>(&b1));
  back[0] = f0.x; back[1] = f0.y; back[2] = f1.x; back[3] = f1.y;
  return lo | static_cast<uint32_t>(hi) << 16;
}
// Transposes an 8 x 8 matrix of 16-bit elements that a warp holds two to a lane.
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
  return d;
}
__device__ __forceinline__ uint32_t pack_bf2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t ld_shared_u16(uint32_t addr) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint32_t ld_shared_u8(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ unsigned add_acq_rel(uint32_t addr, unsigned v) {
  unsigned old;
  asm volatile("atom.acq_rel.cta.shared::cta.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(addr), "r"(v) : "memory");
  return old;
}
template <int N>
__device__ __forceinline__ void ld_shared_words(uint32_t addr, uint32_t (&w)[N]) {
  if constexpr (N == 4) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr));
  if constexpr (N == 2) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(addr));
  if constexpr (N == 1) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(addr));
}

// Running maxima start here: finite, so that no difference of two of them is a NaN.
constexpr float kNoMax = -3.0e38f;
// What a query row's share of a range of keys weighs; maxima in units of log2.  A range without any key has l = 0.
__device__ __forceinline__ float range_weight(float m, float l, float m_all) { return l == 0.f ? 0.f : exp2f(m - m_all); }

constexpr int kFewMaxRanges = 8;

template <int D, int NB, int W>
struct FewCfg {
  static constexpr int kSets = NB == 1 ? 2 : 1;           // sets of 16 keys that a warp takes of a stage
  static constexpr int kStages = NB == 1 ? 3 : 4;
  static constexpr int kFewWarps = W, kFewThreads = 32 * W, kFewKeys = 16 * W, kFewStageKeys = kFewKeys * kSets;
  static constexpr int kRows = 8 * NB;                    // query rows of a unit
  static constexpr int kCodeBytes = kFewStageKeys * D / 2, kScaleBytes = kFewStageKeys * D / kKv4Group;
  static constexpr int kStageBytes = 2 * (kCodeBytes + kScaleBytes);          // K codes, V codes, K scales, V scales
  static constexpr int kPitch = (D + 4) * 4;              // bytes of a row in a warp's part
  static constexpr int kPartBytes = kFewWarps * kRows * kPitch;               // over the stages, when they are done with
  static constexpr int kQuads = kRows * D / 4;            // float4 of a unit
  static constexpr int kRecvBytes = (kQuads + kFewMaxRanges) * 16;            // what the ranges of a cluster push here
  static constexpr int kMlBytes = kFewMaxRanges * kRows * 8;
  static constexpr int kTailBytes = 64;                   // barriers, counters, the abort flag
  static constexpr int kQueryBytes = NB * (D / kKv4Group) * (32 * 16 + 8 * 4) + kRows * 4;   // e4m3 terms, first values, scales of the rows
  static constexpr int kStagesBytes = kStages * kStageBytes, kAllParts = (kPartBytes + kFewWarps * kRows * 8 + 127) / 128 * 128;
  static constexpr int kFrontBytes = kStagesBytes > kAllParts ? kStagesBytes : kAllParts;
  static constexpr int kSmemBytes = kFrontBytes + kRecvBytes + kMlBytes + kQueryBytes + kTailBytes;
  static_assert(kCodeBytes % (4 * D) == 0 && kStageBytes % (4 * D) == 0, "the swizzle repeats after eight rows of codes");
};

template <int D, int NB, int W>
__global__ void __launch_bounds__(32 * W, 16 / W)
attention_kv4_few_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Kv4AttnArgs p) {
  using Cfg = FewCfg<D, NB, W>;
  constexpr int kFewWarps = W, kFewThreads = 32 * W, kFewKeys = Cfg::kFewKeys, kFewStageKeys = Cfg::kFewStageKeys;
  constexpr int kSets = Cfg::kSets, kFewStages = Cfg::kStages, NG = D / kKv4Group, VW = D / 64;      // groups of a row, words a lane takes of a value row
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t stages = smem_u32(smem_raw);
  const uint32_t recv = stages + Cfg::kFrontBytes, recv_ml = recv + Cfg::kRecvBytes;
  const uint32_t q_terms = recv_ml + Cfg::kMlBytes, q_first = q_terms + NB * NG * 512, q_scale = q_first + NB * NG * 32;
  uint8_t *tail = smem_raw + Cfg::kSmemBytes - Cfg::kTailBytes;
  auto full = [&](int s) { return smem_u32(tail) + 8 * s; };
  unsigned *done = reinterpret_cast<unsigned *>(tail + 8 * kFewStages);        // warps that have finished with a slot, in all its uses
  volatile int &abort_flag = *reinterpret_cast<volatile int *>(tail + 12 * kFewStages);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  const long long wb = wait_budget(p.wait_cycles);
  if (stages & 1023) {                                    // the swizzle counts from 1024-byte boundaries
    if (threadIdx.x == 0) atomicOr(p.status, kStatusTimeout);
    return;
  }

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < kFewStages; ++s) {
      mbar_init(full(s), 1);
      done[s] = 0;
    }
    mbar_fence_init();
  }
  __syncthreads();
  pdl_wait();
  pdl_launch_dependents();
  const int splits = p.kv_splits, sp = static_cast<int>(blockIdx.x) % splits;
  if (splits > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // waited for before anything is pushed

  // The unit: query rows rho0 .. of one cache head of one element, rho = row * G + head of the group.
  const int G = p.H / p.Hkv, nrows = p.r * G;
  const int rho0 = static_cast<int>(blockIdx.x) / splits * Cfg::kRows, kv = blockIdx.y, b = blockIdx.z;
  auto limit_of = [&](int rho) {
    if (rho >= nrows) return 0;
    return p.limits ? min(max(p.limits[static_cast<long long>(b) * p.r + rho / G], 0), p.L) : p.L;
  };
  int kmax = p.L, kmin = p.L;                             // keys that some row sees, that every row sees
  if (p.limits) {
    const bool mine = lane < Cfg::kRows && rho0 + lane < nrows;
    const int lim = mine ? limit_of(rho0 + lane) : 0;
    kmax = __reduce_max_sync(0xffffffffu, lim);
    kmin = __reduce_min_sync(0xffffffffu, mine ? lim : INT_MAX);
  }
  // Its keys, in ranges of whole rounds: [k0, k1) here.
  const int rounds = (kmax + kFewKeys - 1) / kFewKeys, per = (rounds + splits - 1) / splits;
  const int k0 = min(sp * per * kFewKeys, kmax), k1 = min(k0 + per * kFewKeys, kmax);
  kmin = min(kmin, k1);
  const int nst = (k1 - k0 + kFewStageKeys - 1) / kFewStageKeys;
  const long long row0 = b * p.elem_stride + static_cast<long long>(kv) * p.L_cap;

  float o[NB][D / 16][4];
  float m[NB][2], l[NB][2];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k) o[nb][t][k] = 0.f;
    m[nb][0] = m[nb][1] = kNoMax;
    l[nb][0] = l[nb][1] = 0.f;
  }

  const int kend = (k1 + 7) & ~7;                         // whole 16 bytes of scales; within the cache (L_cap % 8 == 0)
  auto request = [&](int st) {
    const int slot = st % kFewStages, k = k0 + st * kFewStageKeys;
    const uint32_t n = min(kFewStageKeys, kend - k), dst = stages + slot * Cfg::kStageBytes;
    mbar_expect_tx(full(slot), 2 * Cfg::kCodeBytes + n * 2 * NG);
    tma_load_4d(dst, &tmK, full(slot), 0, k, kv, b);       // rows beyond L_cap become zeros, others nobody sees are masked
    bulk_load(dst + 2 * Cfg::kCodeBytes, p.k_scales + (row0 + k) * NG, n * NG, full(slot));
    tma_load_4d(dst + Cfg::kCodeBytes, &tmV, full(slot), 0, k, kv, b);
    bulk_load(dst + 2 * Cfg::kCodeBytes + Cfg::kScaleBytes, p.v_scales + (row0 + k) * NG, n * NG, full(slot));
  };
  if (threadIdx.x == 0)
    for (int st = 0; st < min(kFewStages, nst); ++st) request(st);
  // ------------------------------------------------------------------ queries
  // Warp nb prepares rows 8 nb ..: a lane's 8 values of each group become 4 + 4 bytes of the product's second operand, in the order
  // in which the masks leave the codes of a word (values 0, 4, 1, 5 and 2, 6, 3, 7).
  for (int nb = warp; nb < NB; nb += W) {
    const int rho = rho0 + nb * 8 + gid;
    const bool there = rho < nrows;
    const bf16 *src = p.q + (there ? (static_cast<long long>(b) * p.r + rho / G) * p.ldq + (kv * G + rho % G) * D + tig * 8 : 0);
    uint4 raw[NG];
    uint32_t top2 = 0;                                    // maxima of the bit patterns: ordered as the magnitudes are
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      raw[g] = there ? *reinterpret_cast<const uint4 *>(src + g * kKv4Group) : make_uint4(0, 0, 0, 0);
      top2 = __vmaxu2(top2, __vmaxu2(__vmaxu2(raw[g].x & 0x7FFF7FFFu, raw[g].y & 0x7FFF7FFFu), __vmaxu2(raw[g].z & 0x7FFF7FFFu, raw[g].w & 0x7FFF7FFFu)));
    }
    top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 1));
    top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 2));
    const int e = static_cast<int>(max(top2 & 0xFFFFu, top2 >> 16) >> 7);                    // biased exponent of the greatest; 255: infinite or NaN
    // q * 2^(134 - e) in two steps, as the factor may be beyond fp32; rows of denormal numbers only come out smaller than 128
    const int sh = 134 - max(e, 1);
    const float f1 = __uint_as_float(static_cast<uint32_t>(127 + (sh >> 1)) << 23), f2 = __uint_as_float(static_cast<uint32_t>(127 + sh - (sh >> 1)) << 23);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const uint32_t w[4] = {raw[g].x, raw[g].y, raw[g].z, raw[g].w};
      float x[8], sum = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[2 * k] = __uint_as_float(w[k] << 16) * f1 * f2;
        x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u) * f1 * f2;
      }
      uint32_t term[4];
#pragma unroll
      for (int half = 0; half < 2; ++half) {              // values 0, 4, 1, 5, then 2, 6, 3, 7
        const float y[4] = {x[2 * half], x[2 * half + 4], x[2 * half + 1], x[2 * half + 5]};
        float hi[4], rest[4], lo[4];
        term[half] = to_e4m3(y, hi);
#pragma unroll
        for (int k = 0; k < 4; ++k) rest[k] = y[k] - hi[k];
        term[2 + half] = to_e4m3(rest, lo);
#pragma unroll
        for (int k = 0; k < 4; ++k) sum += hi[k] + lo[k];
      }
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(q_terms + ((nb * NG + g) * 32 + lane) * 16), "r"(term[0]), "r"(term[1]), "r"(term[2]), "r"(term[3]) : "memory");
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      if (tig == 0) asm volatile("st.shared.f32 [%0], %1;" ::"r"(q_first + ((nb * NG + g) * 8 + gid) * 4), "f"(sum * (-8.f / 512.f)) : "memory");
    }
    // scores in units of log2: 2^9 for the codes, 2^-sh for the queries; a row with an infinity or a NaN is NaN
    const float f = e == 255 ? __uint_as_float(0x7FC00000u) : p.scale_log2 * 512.f / f1 / f2;
    if (tig == 0) asm volatile("st.shared.f32 [%0], %1;" ::"r"(q_scale + (nb * 8 + gid) * 4), "f"(f) : "memory");
  }
  __syncthreads();
  {
    // ------------------------------------------------------------------ products
    uint32_t qt[NB][NG][4];
    float2 first[NB][NG], c[NB];                          // of rows 2 tig and 2 tig + 1
    int lim[NB][2];
    auto load_terms = [&](int nb, int g) { ld_shared_words<4>(q_terms + ((nb * NG + g) * 32 + lane) * 16, qt[nb][g]); };
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        if (NB == 1) load_terms(nb, g);
        if (NB == 1) first[nb][g] = ld_shared_f2(q_first + ((nb * NG + g) * 8 + 2 * tig) * 4);
      }
      c[nb] = ld_shared_f2(q_scale + (nb * 8 + 2 * tig) * 4);
#pragma unroll
      for (int i = 0; i < 2; ++i) lim[nb][i] = min(limit_of(rho0 + nb * 8 + 2 * tig + i), k1);
    }
    // Which key of a set is row gid of the first operand, and which are the four whose values a lane takes (as k 2 tig, 2 tig + 1,
    // 2 tig + 8, 2 tig + 9 of the second product): free to choose as long as both agree, and such that the lanes of a load fall into
    // different banks of the swizzled tile.
    const int krow = D == 128 ? ((gid >> 1) & 1) + 4 * (gid >> 2) + 2 * (gid & 1) : (gid >> 1) + 4 * (gid & 1);
    auto vrow = [&](int i) { return (D == 128 ? (tig & 1) + 4 * (tig >> 1) + 2 * (i & 1) : tig + 4 * (i & 1)) + 8 * (i >> 1); };
    // 16-byte column of a row of codes in the swizzled tile
    auto column = [&](int row, int ch) { return D == 128 ? ch ^ ((row >> 1) & 3) : ch ^ ((row >> 2) & 1); };
    bool ok = true;
    for (int st = 0; st < nst; ++st) {
      const int slot = st % kFewStages;
      ok = __all_sync(0xffffffffu, mbar_wait(full(slot), (st / kFewStages) & 1, p.status, &abort_flag, wb));
      if (!ok) break;
      const uint32_t base = stages + slot * Cfg::kStageBytes, kbase = base, vbase = base + Cfg::kCodeBytes;
      const uint32_t ksbase = base + 2 * Cfg::kCodeBytes, vsbase = ksbase + Cfg::kScaleBytes;
      const int kr = warp * 16 * kSets, key = k0 + st * kFewStageKeys + kr;                  // the warp's keys
      if (key < k1) {
        uint32_t kw[kSets][2][NG], ks[kSets][2], vw[kSets][4][VW], vs[kSets][4];
#pragma unroll
        for (int x = 0; x < kSets; ++x)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = kr + 16 * x + krow + 8 * i;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              uint32_t one[1];
              ld_shared_words<1>(kbase + row * (D / 2) + column(row, g) * 16 + tig * 4, one);
              kw[x][i][g] = one[0];
            }
            if constexpr (NG == 4) {
              uint32_t one[1];
              ld_shared_words<1>(ksbase + row * NG, one);
              ks[x][i] = one[0];
            } else {
              ks[x][i] = ld_shared_u16(ksbase + row * NG);
            }
          }
#pragma unroll
        for (int x = 0; x < kSets; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int row = kr + 16 * x + vrow(i);
            ld_shared_words<VW>(vbase + row * (D / 2) + column(row, gid * (D / 16) / 16) * 16 + gid * (D / 16) % 16, vw[x][i]);
            vs[x][i] = ld_shared_u8(vsbase + row * NG + gid * (D / 8) / kKv4Group);
          }
        // S^T: lane (gid, tig) has scores of keys krow and krow + 8 and of rows 2 tig and 2 tig + 1
        float s[kSets][NB][4];
#pragma unroll
        for (int x = 0; x < kSets; ++x)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int k = 0; k < 4; ++k) s[x][nb][k] = 0.f;
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int x = 0; x < kSets; ++x) {
            const uint32_t a0 = kw[x][0][g] & 0x0F0F0F0Fu, a1 = kw[x][1][g] & 0x0F0F0F0Fu;
            const uint32_t a2 = kw[x][0][g] >> 4 & 0x0F0F0F0Fu, a3 = kw[x][1][g] >> 4 & 0x0F0F0F0Fu;
            const float sc0 = kv4_scale_f32(ks[x][0], g), sc1 = kv4_scale_f32(ks[x][1], g);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              if (NB > 1) load_terms(nb, g);
              const float2 f = NB == 1 ? first[nb][g] : ld_shared_f2(q_first + ((nb * NG + g) * 8 + 2 * tig) * 4);
              float acc[4];
              mma_16832(acc, a0, a1, a2, a3, qt[nb][g][0], qt[nb][g][1], f.x, f.y, f.x, f.y);
              mma_16832(acc, a0, a1, a2, a3, qt[nb][g][2], qt[nb][g][3], acc[0], acc[1], acc[2], acc[3]);
              s[x][nb][0] = fmaf(acc[0], sc0, s[x][nb][0]);
              s[x][nb][1] = fmaf(acc[1], sc0, s[x][nb][1]);
              s[x][nb][2] = fmaf(acc[2], sc1, s[x][nb][2]);
              s[x][nb][3] = fmaf(acc[3], sc1, s[x][nb][3]);
            }
          }
        // in units of log2
#pragma unroll
        for (int x = 0; x < kSets; ++x)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int k = 0; k < 4; ++k) s[x][nb][k] *= k & 1 ? c[nb].y : c[nb].x;
        if (key + 16 * kSets > kmin) {
#pragma unroll
          for (int x = 0; x < kSets; ++x)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (key + 16 * x + krow + 8 * (k >> 1) >= lim[nb][k & 1]) s[x][nb][k] = -INFINITY;
        }
        bool need = false;
        float top[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            top[nb][i] = fmaxf(s[0][nb][i], s[0][nb][i + 2]);
#pragma unroll
            for (int x = 1; x < kSets; ++x) top[nb][i] = fmaxf(top[nb][i], fmaxf(s[x][nb][i], s[x][nb][i + 2]));
            need = need || top[nb][i] > m[nb][i] + 8.f;
          }
        // the accumulators are scaled anew only when a maximum has grown by more than 2^8 (and at the first keys)
        if (__any_sync(0xffffffffu, need)) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float t2 = top[nb][i];
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) t2 = fmaxf(t2, __shfl_xor_sync(0xffffffffu, t2, d));
              const float m2 = fmaxf(m[nb][i], t2), a = exp2f(m[nb][i] - m2);
              m[nb][i] = m2;
              l[nb][i] *= a;
#pragma unroll
              for (int t = 0; t < D / 16; ++t) {
                o[nb][t][i] *= a;
                o[nb][t][i + 2] *= a;
              }
            }
        }
#pragma unroll
        for (int x = 0; x < kSets; ++x) {
          uint32_t pt[NB][2];                             // P^T of the set's two halves, as the second operand wants it
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            float e[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) e[k] = exp2f(s[x][nb][k] - m[nb][k & 1]);
            l[nb][0] += e[0] + e[2];
            l[nb][1] += e[1] + e[3];
            pt[nb][0] = transpose_8x8(pack_bf2(e[0], e[1]));
            pt[nb][1] = transpose_8x8(pack_bf2(e[2], e[3]));
          }
          // O^T += V^T P^T: lane (gid, tig) has values gid * D / 8 .. of four keys; a pair of keys makes an operand register
          const uint32_t v0 = kv4_scales(vs[x][0], vs[x][1]), v1 = kv4_scales(vs[x][2], vs[x][3]);
          const uint32_t g0 = kv4_offset2(v0), g1 = kv4_offset2(v1);
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            uint32_t even0[4], odd0[4], even1[4], odd1[4];  // values 2 p and 2 p + 1 of the word, of the first and the second two keys
            kv4_word(__byte_perm(vw[x][0][w], vw[x][1][w], 0x5410), v0, g0, even0);
            kv4_word(__byte_perm(vw[x][0][w], vw[x][1][w], 0x7632), v0, g0, odd0);
            kv4_word(__byte_perm(vw[x][2][w], vw[x][3][w], 0x5410), v1, g1, even1);
            kv4_word(__byte_perm(vw[x][2][w], vw[x][3][w], 0x7632), v1, g1, odd1);
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) mma_16816(o[nb][w * 4 + t], even0[t], odd0[t], even1[t], odd1[t], pt[nb][0], pt[nb][1]);
          }
        }
      }
      // The warp that is last to be done with the slot has it filled again: nobody waits for room.  (A ninth warp that did
      // spent a sixth of the issue slots on asking.)
      __syncwarp();
      if (lane == 0 && st + kFewStages < nst && add_acq_rel(smem_u32(&done[slot]), 1) % kFewWarps == kFewWarps - 1) request(st + kFewStages);
    }
    if (!ok && lane == 0) {                               // gave up: what was requested has to land before the memory is released
      const long long t0 = clock64();
      while (clock64() - t0 < kMinWaitCycles) {}
    }
  }

  // -------------------------------------------------------------------- the warps' parts meet, then those of the ranges
  __syncthreads();
  const uint32_t part = stages, part_ml = stages + Cfg::kPartBytes;
  {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float sum = l[nb][i];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const int row = nb * 8 + 2 * tig + i;
        if (gid == 0) asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(part_ml + (warp * Cfg::kRows + row) * 8), "f"(m[nb][i]), "f"(sum) : "memory");
        const uint32_t dst = part + (warp * Cfg::kRows + row) * Cfg::kPitch + gid * (D / 8) * 4;
#pragma unroll
        for (int t = 0; t < D / 16; t += 2)               // tile t: values 2 t and 2 t + 1 of the lane's
          asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dst + t * 8), "f"(o[nb][t][i]), "f"(o[nb][t][i + 2]), "f"(o[nb][t + 1][i]),
                       "f"(o[nb][t + 1][i + 2]) : "memory");
      }
  }
  __syncthreads();
  if (splits > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");                // every CTA of the cluster is there
  const int cnt = (Cfg::kQuads + splits - 1) / splits;    // float4 that a CTA of the cluster finishes
  for (int x = threadIdx.x; x < Cfg::kQuads; x += kFewThreads) {
    const int row = x * 4 / D, d = x * 4 % D;
    float2 ml[kFewWarps];
    float m_all = kNoMax, l_all = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      ml[w] = ld_shared_f2(part_ml + (w * Cfg::kRows + row) * 8);
      m_all = fmaxf(m_all, ml[w].x);
    }
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      const float a = range_weight(ml[w].x, ml[w].y, m_all);
      const float4 v = ld_shared_f4(part + (w * Cfg::kRows + row) * Cfg::kPitch + d * 4);
      acc.x = fmaf(a, v.x, acc.x); acc.y = fmaf(a, v.y, acc.y); acc.z = fmaf(a, v.z, acc.z); acc.w = fmaf(a, v.w, acc.w);
      l_all = fmaf(a, ml[w].y, l_all);
    }
    if (splits > 1) {
      const int owner = x / cnt;
      const uint32_t dst = mapa_shared(recv + (sp * cnt + x - owner * cnt) * 16, owner);
      asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "f"(acc.x), "f"(acc.y), "f"(acc.z), "f"(acc.w) : "memory");
      if (d == 0)
        for (int t = 0; t < splits; ++t)
          asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(mapa_shared(recv_ml + (sp * Cfg::kRows + row) * 8, t)), "f"(m_all), "f"(l_all) : "memory");
    } else if (rho0 + row < nrows && abort_flag == 0) {
      const float inv = l_all == 0.f ? 0.f : 1.0f / l_all;
      const int rho = rho0 + row;
      *reinterpret_cast<uint2 *>(p.out + ((static_cast<long long>(b) * p.r + rho / G) * p.H + kv * G + rho % G) * D + d) =
          make_uint2(pack_bf2(acc.x * inv, acc.y * inv), pack_bf2(acc.z * inv, acc.w * inv));
    }
  }
  if (splits > 1) {
    __syncwarp();
    cluster_sync_all();                                   // all parts have arrived; nobody touches a peer after this
    for (int y = threadIdx.x; y < cnt; y += kFewThreads) {
      const int x = sp * cnt + y;
      if (x >= Cfg::kQuads) break;
      const int row = x * 4 / D, d = x * 4 % D, rho = rho0 + row;
      float m_all = kNoMax, l_all = 0.f;
      for (int t = 0; t < splits; ++t) m_all = fmaxf(m_all, ld_shared_f2(recv_ml + (t * Cfg::kRows + row) * 8).x);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int t = 0; t < splits; ++t) {
        const float2 ml = ld_shared_f2(recv_ml + (t * Cfg::kRows + row) * 8);
        const float a = range_weight(ml.x, ml.y, m_all);
        const float4 v = ld_shared_f4(recv + (t * cnt + y) * 16);
        acc.x = fmaf(a, v.x, acc.x); acc.y = fmaf(a, v.y, acc.y); acc.z = fmaf(a, v.z, acc.z); acc.w = fmaf(a, v.w, acc.w);
        l_all = fmaf(a, ml.y, l_all);
      }
      if (rho >= nrows || abort_flag) continue;
      const float inv = l_all == 0.f ? 0.f : 1.0f / l_all;
      *reinterpret_cast<uint2 *>(p.out + ((static_cast<long long>(b) * p.r + rho / G) * p.H + kv * G + rho % G) * D + d) =
          make_uint2(pack_bf2(acc.x * inv, acc.y * inv), pack_bf2(acc.z * inv, acc.w * inv));
    }
  }
}

int g_few_force = 0;
template <int D, int NB, int W>
static cudaError_t launch_few(Kv4AttnArgs a, int num_sms, cudaStream_t st) {
  using Cfg = FewCfg<D, NB, W>;
  static unsigned long long prepared = 0;                 // a bit a device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !(prepared >> dev & 1)) {
    e = cudaFuncSetAttribute(attention_kv4_few_kernel<D, NB, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmemBytes);
    if (e != cudaSuccess) return e;
    if (dev < 64) prepared |= 1ull << dev;
  }
  CUtensorMap tk, tv;
  if (!tmap_codes(&tk, a.k_codes, a, Cfg::kFewStageKeys) || !tmap_codes(&tv, a.v_codes, a, Cfg::kFewStageKeys)) return cudaErrorInvalidValue;
  const int tiles = (a.r * (a.H / a.Hkv) + Cfg::kRows - 1) / Cfg::kRows;
  const long long units = static_cast<long long>(tiles) * a.Hkv * a.B;
  if (a.Hkv > 65535 || a.B > 65535) return cudaErrorInvalidConfiguration;
  const int rounds = (a.L + Cfg::kFewKeys - 1) / Cfg::kFewKeys;
  int s = 1;
  while (s < kFewMaxRanges && units * s < 2 * num_sms && rounds >= 2 * (s * 2)) s *= 2;
  if (g_few_force) s = g_few_force;
  a.kv_splits = s;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles * s, a.Hkv, a.B);
  cfg.blockDim = dim3(Cfg::kFewThreads);
  cfg.dynamicSmemBytes = Cfg::kSmemBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (s > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;     // the ranges of one unit
    attr[n].val.clusterDim.x = s;
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  if (one_predecessor(st)) attr[n++] = pdl_attribute();
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, attention_kv4_few_kernel<D, NB, W>, tk, tv, a);
}

int g_few_rows = 16;
cudaError_t launch_attention_kv4(const Kv4AttnArgs &a, void *workspace, size_t bytes, int num_sms, cudaStream_t st) {
  if (a.r * static_cast<long long>(a.H / a.Hkv) > g_few_rows) return launch_attention_kv4_many(a, workspace, bytes, num_sms, st);
  const bool one = a.r * static_cast<long long>(a.H / a.Hkv) <= 8;
  if (a.D == 64) return one ? launch_few<64, 1, 8>(a, num_sms, st) : launch_few<64, 2, 8>(a, num_sms, st);
  return one ? launch_few<128, 1, 8>(a, num_sms, st) : launch_few<128, 2, 8>(a, num_sms, st);
}

}  // namespace fvar
