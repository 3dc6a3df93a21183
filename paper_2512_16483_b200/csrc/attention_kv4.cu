// Attention of query rows over a cache in 4 bits (format and operator: include/fvar.h).
//
// Few rows (attention_kv4_few_kernel, 8 or 16 query rows a cache head at a time): the codes go from memory to the tensor cores without a
// stop on the way: TMA brings them to shared memory as they are, a warp takes the codes of 16 keys into registers by ldmatrix, and they
// become operands of mma.sync there.  (Through tcgen05 they would have to be decoded into shared memory and read from there again: 2.5
// times their bf16 size at 128 bytes a clock, 1.8 times what reading the codes from HBM takes.)  Keys and values are the operand of 16
// rows, the query rows the one of 8:
//   S^T [16 keys][8 rows] = K Q^T,   O^T [16 of D][8 rows] += V^T P^T.
// What bounds it is the issue of instructions (most of them hold an issue port for two cycles), so little is left of decoding: a number u of
// 4 bits, in bits 0 - 3 or 4 - 7 of a bf16 whose other bits are zero, is u 2^-133 or u 2^-129 -- a subnormal number, or one of the first
// binade, which has the same step -- and a product takes it as it is.  One mask makes an operand register, and one shift in eight of
// them.  The rest is done where there is less of it:
//   powers of two   the queries' elements carry 2^120 relative to their row's greatest and 2^-4 where they meet bits 4 - 7; P carries 2^100;
//                   the outputs' rows get 2^33 or 2^29 at the end.  All exact.
//   keys' scales    a product covers one group of D and is multiplied by the group's scale when it is added to the score;
//   values' scales  P is multiplied by the scales of a group before that group's product: one more rounding to bf16 of a weight;
//   u - 8           - 8 scale (sum of the group's queries) is a small product of its own, scales x sums in two bf16 terms, and what the
//                   scores begin with; 8 (sum of a group's P) is one more row of the second product, taken off at the end.
// ldmatrix gives a key's group as a row (K) and, transposed, pairs of keys in a register (V), so nothing is shuffled.
// One row of 37 x 8 heads over 10521 keys, D = 128 (424 MB): 82.3 us, 5.1 TB/s; 280 instructions for 16 keys, of which 156 on the ALU
// pipe (66 % busy, issue slots 59 %, tensor pipe 37 %).  4 rows of 64 x 8 heads over 0 - 8191 keys: 75.7 us, 3.8 TB/s.  One row of 2 x 16
// heads (46 MB): 17.2 us; 16 rows of 4 x 16 heads over 6441 keys: 26.1.
#include <limits.h>
#include <math.h>

#include "kv4.cuh"
#include "per_device.h"
#include "ptx.cuh"

namespace fvar {

// D[16][8] += A[16][16] B[16][8], bf16, fp32 accumulator.
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// D[16][8] = A[16][8] B[8][8].
__device__ __forceinline__ void mma_1688_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t b0) {
  asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5}, {%6}, {%7, %7, %7, %7};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(b0), "f"(0.f));
}
// D[16][8] = A[16][16] B[16][8].
__device__ __forceinline__ void mma_16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// Four 8 x 8 matrices of 16-bit elements, lane 8 m + r giving the address of row r of matrix m: a lane gets elements (lane / 4, 2 (lane mod 4))
// and the next one, or (TRANS) elements (2 (lane mod 4), lane / 4) and the one below.
template <bool TRANS>
__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
  if constexpr (TRANS)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
// Codes of 16 keys from row `row0` of a tile on, whose 16-byte columns are swizzled: w[eight keys][group] is word lane mod 4 of the group
// of key lane / 4 (K), or half-word lane / 4 of the group of keys 2 (lane mod 4) and the next (V: TRANS).
template <int D, bool TRANS>
__device__ __forceinline__ void load_codes(uint32_t tile, int row0, int lane, uint32_t (&w)[2][D / kKv4Group]) {
  const int m = lane >> 3, r = lane & 7;                  // matrix and row whose address the lane gives
  if constexpr (D == 128) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = row0 + 8 * h + r;
      ldmatrix_x4<TRANS>(tile + row * 64 + (m ^ ((row >> 1) & 3)) * 16, w[h]);
    }
  } else {
    const int row = row0 + 8 * (m >> 1) + r;
    uint32_t r4[4];
    ldmatrix_x4<TRANS>(tile + row * 32 + ((m & 1) ^ ((row >> 2) & 1)) * 16, r4);
    w[0][0] = r4[0]; w[0][1] = r4[1]; w[1][0] = r4[2]; w[1][1] = r4[3];
  }
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

constexpr uint32_t kLow = 0x000F000Fu, kHigh = 0x00F000F0u;       // u 2^-133, u 2^-129 in both halves
constexpr float k2p29 = 536870912.f, k2p33 = 16.f * k2p29, k2p66 = k2p33 * k2p33, k2m65 = 2.f / k2p66;
// Running maxima start here: finite, so that no difference of two of them is a NaN.
constexpr float kNoMax = -3.0e38f;
// What a query row's share of a range of keys weighs; maxima in units of log2.  A range without any key has l = 0.
__device__ __forceinline__ float range_weight(float m, float l, float m_all) { return l == 0.f ? 0.f : exp2f(m - m_all); }

constexpr int kFewWarps = 8, kFewThreads = 32 * kFewWarps;
constexpr int kFewSets = 2;                               // sets of 16 keys that a warp takes of a stage
constexpr int kFewKeys = 16 * kFewWarps, kFewStageKeys = kFewKeys * kFewSets;
constexpr int kFewStages = 3;
constexpr int kFewMaxRanges = 8;

template <int D, int NB>
struct FewCfg {
  static constexpr int kRows = 8 * NB;                    // query rows of a unit
  static constexpr int kCodeBytes = kFewStageKeys * D / 2, kScaleBytes = kFewStageKeys * D / kKv4Group;
  static constexpr int kStageBytes = 2 * (kCodeBytes + kScaleBytes);          // K codes, V codes, K scales, V scales
  static constexpr int kPitch = (D + 4) * 4;              // bytes of a row in a warp's part
  static constexpr int kPartBytes = kFewWarps * kRows * kPitch;               // over the stages, when they are done with
  static constexpr int kOcts = kRows * D / 8;             // eight values of a unit's result
  static constexpr int kRecvBytes = (kOcts + kFewMaxRanges) * 32;             // what the ranges of a cluster push here
  static constexpr int kMlBytes = kFewMaxRanges * kRows * 8;
  static constexpr int kStagesBytes = kFewStages * kStageBytes, kAllParts = (kPartBytes + kFewWarps * kRows * 8 + 127) / 128 * 128;
  static constexpr int kFrontBytes = kStagesBytes > kAllParts ? kStagesBytes : kAllParts;
  static constexpr int kTailBytes = 64;                   // barriers, counters, the abort flag
  static constexpr int kSmemBytes = kFrontBytes + kRecvBytes + kMlBytes + kTailBytes;
  static_assert(kCodeBytes % (4 * D) == 0 && kStageBytes % (4 * D) == 0, "the swizzle repeats after eight rows of codes");
};

template <int D, int NB>
__global__ void __launch_bounds__(kFewThreads, NB == 1 ? 2 : 1)
attention_kv4_few_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Kv4AttnArgs p) {
  using Cfg = FewCfg<D, NB>;
  constexpr int NG = D / kKv4Group;                       // groups of a row
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t stages = smem_u32(smem_raw);
  const uint32_t recv = stages + Cfg::kFrontBytes, recv_ml = recv + Cfg::kRecvBytes;
  uint8_t *tail = smem_raw + Cfg::kSmemBytes - Cfg::kTailBytes;
  auto full = [&](int s) { return smem_u32(tail) + 8 * s; };
  unsigned *done = reinterpret_cast<unsigned *>(tail + 8 * kFewStages);        // warps that have finished with a slot, in all its uses
  volatile int &abort_flag = *reinterpret_cast<volatile int *>(tail + 12 * kFewStages);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  const long long wb = wait_budget(p.wait_cycles);
  if (stages & 1023) {                                    // the swizzle counts from its own boundaries
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

  // Tiles 2 g and 2 g + 1: half-bytes 0, 2 and 1, 3 of group g.  o8: 8 x the sum of P of groups 2 t (its rows 0 - 7) and 2 t + 1 (8 - 15).
  float o[NB][2 * NG][4], o8[NB][NG / 2][4];
  float m[NB][2], l[NB][2];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
      for (int k = 0; k < 4; ++k) o[nb][t][k] = 0.f;
#pragma unroll
    for (int k = 0; k < 2 * NG; ++k) o8[nb][k / 4][k % 4] = 0.f;
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
  {
    // ------------------------------------------------------------------ queries
    // Lane (gid, tig) of a warp has word tig of every group of row gid: values 8 tig .. 8 tig + 7.  The row is multiplied by 2^sh so that
    // its greatest element is in [2^120, 2^121).
    uint32_t q[NB][NG][4], sums[NB];                      // [pair of values]; the groups' sums x -8 2^-133, two terms of them
    float c[NB][2];                                       // of rows 2 tig, 2 tig + 1: from the products' units to those of log2
    int lim[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int rho = rho0 + nb * 8 + gid;
      const bool there = rho < nrows;
      const bf16 *src = p.q + (there ? (static_cast<long long>(b) * p.r + rho / G) * p.ldq + (kv * G + rho % G) * D + tig * 8 : 0);
      uint4 raw[NG];
      uint32_t top2 = 0;                                  // maxima of the bit patterns: ordered as the magnitudes are
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        raw[g] = there ? *reinterpret_cast<const uint4 *>(src + g * kKv4Group) : make_uint4(0, 0, 0, 0);
        top2 = __vmaxu2(top2, __vmaxu2(__vmaxu2(raw[g].x & 0x7FFF7FFFu, raw[g].y & 0x7FFF7FFFu), __vmaxu2(raw[g].z & 0x7FFF7FFFu, raw[g].w & 0x7FFF7FFFu)));
      }
      top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 1));
      top2 = __vmaxu2(top2, __shfl_xor_sync(0xffffffffu, top2, 2));
      const int e = static_cast<int>(max(top2 & 0xFFFFu, top2 >> 16) >> 7);                  // biased exponent of the greatest; 255: infinite or NaN
      const int sh = 247 - max(e, 1);                     // in two steps: the factor may be beyond fp32
      const float f1 = __uint_as_float(static_cast<uint32_t>(127 + (sh >> 1)) << 23), f2 = __uint_as_float(static_cast<uint32_t>(127 + sh - (sh >> 1)) << 23);
      float sum[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const uint32_t w[4] = {raw[g].x, raw[g].y, raw[g].z, raw[g].w};
        sum[g] = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float lo = __uint_as_float(w[k] << 16) * f1 * f2, hi = __uint_as_float(w[k] & 0xFFFF0000u) * f1 * f2;
          sum[g] += lo + hi;
          const float odd = k & 1 ? 0.0625f : 1.0f;       // pairs 1 and 3 meet bits 4 - 7
          q[nb][g][k] = pack_bf2(lo * odd, hi * odd);     // exact
        }
        sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 1);
        sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 2);
        sum[g] = -sum[g] * k2m65 * k2m65;                 // - 8 2^-133 sum
      }
      // Two bf16 terms of each sum (16 bits; a score is off by 2^-14 of scale x sum |q| at most).  Row k of the small product's second operand:
      // groups 0, 1 and 2, 3 of term 0, of term 1 (D = 64: groups 0, 1 of terms 0 and 1, zeros).
      const float x = NG == 4 && (tig & 1) ? sum[NG - 2] : sum[0], y = NG == 4 && (tig & 1) ? sum[NG - 1] : sum[1];
      const float xt = __bfloat162float(__float2bfloat16_rn(x)), yt = __bfloat162float(__float2bfloat16_rn(y));
      const int term = NG == 4 ? tig >> 1 : tig;
      sums[nb] = term == 0 ? pack_bf2(x, y) : term == 1 ? pack_bf2(x - xt, y - yt) : 0u;
      // 2^133 for the codes, 2^-sh for the queries; a row with an infinity or a NaN is NaN.  What it multiplies is below 2^11.5 (23 x 128 terms of
      // 2^-12 and a scale of 3840), so up to 2^116 a score is finite; in a row that would need more (queries from 2^106 on)
      // the weights are 0 and 1 all the same, unless two scores agree to 2^-120 of the greatest possible.
      const float f = e == 255 ? __uint_as_float(0x7FC00000u) : fminf(p.scale_log2 * (k2p66 / f1) * ((2.f * k2p66) / f2), 0x1p116f);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        c[nb][i] = __shfl_sync(0xffffffffu, f, (2 * tig + i) * 4);
        lim[nb][i] = min(limit_of(rho0 + nb * 8 + 2 * tig + i), k1);
      }
    }
    // ------------------------------------------------------------------ products
    const uint32_t pair_sel = (NG == 4 && (tig & 1)) ? 0x4342u : 0x4140u;     // scales of groups 2, 3 or 0, 1
    // kept in registers: as constants they would be moved there again for every product
    uint32_t upper[4], lower[4];                          // u = 8 in rows 0 - 7, in rows 8 - 15
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      asm volatile("mov.u32 %0, %1;" : "=r"(upper[k]) : "r"(k & 1 ? 0u : 0x00080008u));
      asm volatile("mov.u32 %0, %1;" : "=r"(lower[k]) : "r"(k & 1 ? 0x00080008u : 0u));
    }
    bool ok = true;
    for (int st = 0; st < nst; ++st) {
      const int slot = st % kFewStages;
      ok = __all_sync(0xffffffffu, mbar_wait(full(slot), (st / kFewStages) & 1, p.status, &abort_flag, wb));
      if (!ok) break;
      const uint32_t kbase = stages + slot * Cfg::kStageBytes, vbase = kbase + Cfg::kCodeBytes, ksbase = kbase + 2 * Cfg::kCodeBytes, vsbase = ksbase + Cfg::kScaleBytes;
      const int kr = warp * 16 * kFewSets, key = k0 + st * kFewStageKeys + kr;               // the warp's keys
      if (key < k1) {
        // S^T: lane (gid, tig) has scores of keys gid and gid + 8 and of rows 2 tig and 2 tig + 1
        float s[kFewSets][NB][4];
#pragma unroll
        for (int x = 0; x < kFewSets; ++x) {
          uint32_t w[2][NG], ks[2];
          load_codes<D, false>(kbase, kr + 16 * x, lane, w);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t at = ksbase + (kr + 16 * x + 8 * h + gid) * NG;
            if constexpr (NG == 4) {
              uint32_t one[1];
              ld_shared_words<1>(at, one);
              ks[h] = one[0];
            } else {
              ks[h] = ld_shared_u16(at);
            }
          }
          const uint32_t a0 = kv4_pairs(__byte_perm(ks[0], 0, pair_sel)), a1 = kv4_pairs(__byte_perm(ks[1], 0, pair_sel));
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) mma_1688_first(s[x][nb], a0, a1, sums[nb]);
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const uint32_t w0 = w[0][g], w1 = w[1][g], v0 = w0 >> 8, v1 = w1 >> 8;
            const float sc0 = kv4_scale_f32(ks[0], g), sc1 = kv4_scale_f32(ks[1], g);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              float acc[4];
              mma_16816_first(acc, w0 & kLow, w1 & kLow, w0 & kHigh, w1 & kHigh, q[nb][g][0], q[nb][g][1]);
              mma_16816(acc, v0 & kLow, v1 & kLow, v0 & kHigh, v1 & kHigh, q[nb][g][2], q[nb][g][3]);
              s[x][nb][0] = fmaf(acc[0], sc0, s[x][nb][0]);
              s[x][nb][1] = fmaf(acc[1], sc0, s[x][nb][1]);
              s[x][nb][2] = fmaf(acc[2], sc1, s[x][nb][2]);
              s[x][nb][3] = fmaf(acc[3], sc1, s[x][nb][3]);
            }
          }
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int k = 0; k < 4; ++k) s[x][nb][k] *= c[nb][k & 1];          // in units of log2
        }
        if (key + 16 * kFewSets > kmin) {
#pragma unroll
          for (int x = 0; x < kFewSets; ++x)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (key + 16 * x + gid + 8 * (k >> 1) >= lim[nb][k & 1]) s[x][nb][k] = -INFINITY;
        }
        bool need = false;
        float top[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            top[nb][i] = fmaxf(s[0][nb][i], s[0][nb][i + 2]);
#pragma unroll
            for (int x = 1; x < kFewSets; ++x) top[nb][i] = fmaxf(top[nb][i], fmaxf(s[x][nb][i], s[x][nb][i + 2]));
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
              for (int t = 0; t < NG / 2; ++t) {
                o8[nb][t][i] *= a;
                o8[nb][t][i + 2] *= a;
              }
#pragma unroll
              for (int t = 0; t < 2 * NG; ++t) {
                o[nb][t][i] *= a;
                o[nb][t][i + 2] *= a;
              }
            }
        }
#pragma unroll
        for (int x = 0; x < kFewSets; ++x) {
          uint32_t w[2][NG], sv[2][NG];                   // sv: scales x 2^100 of the lane's two keys of eight
          load_codes<D, true>(vbase, kr + 16 * x, lane, w);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t at = vsbase + (kr + 16 * x + 8 * h + 2 * tig) * NG;
            if constexpr (NG == 4) {
              uint32_t b2[2];
              ld_shared_words<2>(at, b2);
              const uint32_t e0 = kv4_pairs_p(__byte_perm(b2[0], 0, 0x4240)), e1 = kv4_pairs_p(__byte_perm(b2[1], 0, 0x4240));   // groups 0, 2
              const uint32_t d0 = kv4_pairs_p(__byte_perm(b2[0], 0, 0x4341)), d1 = kv4_pairs_p(__byte_perm(b2[1], 0, 0x4341));   // groups 1, 3
              sv[h][0] = __byte_perm(e0, e1, 0x5410);
              sv[h][1] = __byte_perm(d0, d1, 0x5410);
              sv[h][2] = __byte_perm(e0, e1, 0x7632);
              sv[h][3] = __byte_perm(d0, d1, 0x7632);
            } else {
              uint32_t b1[1];
              ld_shared_words<1>(at, b1);
              sv[h][0] = kv4_pairs_p(__byte_perm(b1[0], 0, 0x4240));
              sv[h][1] = kv4_pairs_p(__byte_perm(b1[0], 0, 0x4341));
            }
          }
          uint32_t pt[NB][2];                             // P^T of keys 0 - 7 and 8 - 15, as the second operand wants it
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
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const uint32_t w0 = w[0][g], w1 = w[1][g], v0 = w0 >> 8, v1 = w1 >> 8;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              const uint32_t p0 = mul_bf2(pt[nb][0], sv[0][g]), p1 = mul_bf2(pt[nb][1], sv[1][g]);
              if (g & 1) mma_16816(o8[nb][g / 2], lower[0], lower[1], lower[2], lower[3], p0, p1);
              else mma_16816(o8[nb][g / 2], upper[0], upper[1], upper[2], upper[3], p0, p1);
              mma_16816(o[nb][2 * g], w0 & kLow, v0 & kLow, w1 & kLow, v1 & kLow, p0, p1);
              mma_16816(o[nb][2 * g + 1], w0 & kHigh, v0 & kHigh, w1 & kHigh, v1 & kHigh, p0, p1);
            }
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
        // the lane's values of a group: every other one of word gid / 2, its even or its odd ones
        const uint32_t dst = part + (warp * Cfg::kRows + row) * Cfg::kPitch + gid * 16;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const float off = o8[nb][g / 2][i + 2 * (g & 1)];
          asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dst + g * 128), "f"((o[nb][2 * g][i] - off) * k2p33),
                       "f"(fmaf(off, -16.f, o[nb][2 * g + 1][i]) * k2p29), "f"((o[nb][2 * g][i + 2] - off) * k2p33),
                       "f"(fmaf(off, -16.f, o[nb][2 * g + 1][i + 2]) * k2p29) : "memory");
        }
      }
  }
  __syncthreads();
  if (splits > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");                // every CTA of the cluster is there
  // Eight values of a row (a word of the format): four even ones, then four odd ones, in a part.
  const int cnt = (Cfg::kOcts + splits - 1) / splits;     // that a CTA of the cluster finishes
  auto store = [&](int row, int d, const float4 &even, const float4 &odd, float l_all) {
    const int rho = rho0 + row;
    if (rho >= nrows || abort_flag != 0) return;
    const float inv = l_all == 0.f ? 0.f : 1.0f / l_all;  // no weight at all: the row sees no key, since scores are finite or NaN
    *reinterpret_cast<uint4 *>(p.out + ((static_cast<long long>(b) * p.r + rho / G) * p.H + kv * G + rho % G) * D + d) =
        make_uint4(pack_bf2(even.x * inv, odd.x * inv), pack_bf2(even.y * inv, odd.y * inv), pack_bf2(even.z * inv, odd.z * inv), pack_bf2(even.w * inv, odd.w * inv));
  };
  auto add = [](float4 &acc, float a, const float4 &v) {
    acc.x = fmaf(a, v.x, acc.x); acc.y = fmaf(a, v.y, acc.y); acc.z = fmaf(a, v.z, acc.z); acc.w = fmaf(a, v.w, acc.w);
  };
  for (int x = threadIdx.x; x < Cfg::kOcts; x += kFewThreads) {
    const int row = x * 8 / D, d = x * 8 % D;
    float2 ml[kFewWarps];
    float m_all = kNoMax, l_all = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      ml[w] = ld_shared_f2(part_ml + (w * Cfg::kRows + row) * 8);
      m_all = fmaxf(m_all, ml[w].x);
    }
    float4 even = make_float4(0.f, 0.f, 0.f, 0.f), odd = even;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      const float a = range_weight(ml[w].x, ml[w].y, m_all);
      const uint32_t src = part + (w * Cfg::kRows + row) * Cfg::kPitch + d * 4;
      add(even, a, ld_shared_f4(src));
      add(odd, a, ld_shared_f4(src + 16));
      l_all = fmaf(a, ml[w].y, l_all);
    }
    if (splits > 1) {
      const int owner = x / cnt;
      const uint32_t dst = mapa_shared(recv + (sp * cnt + x - owner * cnt) * 32, owner);
      asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "f"(even.x), "f"(even.y), "f"(even.z), "f"(even.w) : "memory");
      asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dst + 16), "f"(odd.x), "f"(odd.y), "f"(odd.z), "f"(odd.w) : "memory");
      if (d == 0)
        for (int t = 0; t < splits; ++t)
          asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(mapa_shared(recv_ml + (sp * Cfg::kRows + row) * 8, t)), "f"(m_all), "f"(l_all) : "memory");
    } else {
      store(row, d, even, odd, l_all);
    }
  }
  if (splits > 1) {
    __syncwarp();
    cluster_sync_all();                                   // all parts have arrived; nobody touches a peer after this
    for (int y = threadIdx.x; y < cnt; y += kFewThreads) {
      const int x = sp * cnt + y;
      if (x >= Cfg::kOcts) break;
      const int row = x * 8 / D, d = x * 8 % D;
      float m_all = kNoMax, l_all = 0.f;
      for (int t = 0; t < splits; ++t) m_all = fmaxf(m_all, ld_shared_f2(recv_ml + (t * Cfg::kRows + row) * 8).x);
      float4 even = make_float4(0.f, 0.f, 0.f, 0.f), odd = even;
      for (int t = 0; t < splits; ++t) {
        const float2 ml = ld_shared_f2(recv_ml + (t * Cfg::kRows + row) * 8);
        const float a = range_weight(ml.x, ml.y, m_all);
        add(even, a, ld_shared_f4(recv + (t * cnt + y) * 32));
        add(odd, a, ld_shared_f4(recv + (t * cnt + y) * 32 + 16));
        l_all = fmaf(a, ml.y, l_all);
      }
      store(row, d, even, odd, l_all);
    }
  }
}

template <int D, int NB>
static cudaError_t launch_few(const Kv4AttnArgs &a, cudaStream_t st) {
  using Cfg = FewCfg<D, NB>;
  static PerDevice prepared;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess)
    e = prepared.once(dev, [] { return cudaFuncSetAttribute(attention_kv4_few_kernel<D, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmemBytes); });
  if (e != cudaSuccess) return e;
  CUtensorMap tk, tv;
  if (!tmap_codes(&tk, a.k_codes, a, kFewStageKeys) || !tmap_codes(&tv, a.v_codes, a, kFewStageKeys)) return cudaErrorInvalidValue;
  const int tiles = (a.r * (a.H / a.Hkv) + Cfg::kRows - 1) / Cfg::kRows, s = a.kv_splits;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles * s, a.Hkv, a.B);
  cfg.blockDim = dim3(kFewThreads);
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
  return cudaLaunchKernelEx(&cfg, attention_kv4_few_kernel<D, NB>, tk, tv, a);
}

// Waves of `ctas` blocks over `slots`: whole ones while there are fewer than `few`.
static double waves_of(double ctas, double slots, double few) {
  const double w = ctas / slots;
  return w <= 1.0 ? 1.0 : w < few ? ceil(w) : w;
}

// Form, tiles and key ranges of a launch: the least estimated time (microseconds).  The estimates are fitted to forced launches on B200,
// 10 shapes of few rows and 24 of many, 1 to 5000 rows over 77 to 10521 keys: what they pick of the forms of many rows is 1 % slower than the
// fastest on average and 7 % at worst.  Every element is taken to be L long, also where limits say less.
// Few rows: a block costs 5.5 and its keys 7.5 ns each at D = 128 with two blocks an SM, 4.1 with one (0.6 of that at D = 64);
// 9 to 16 rows at a time, one block an SM, 6.1.  Many rows: see attention_kv4_many_cost.  Where both can be taken they cross between 17 rows
// (8 units: 11.5 us against 21.8) and 64 (32 units over 8000 keys: 52 against 29).
Kv4Plan attention_kv4_plan(int B, int Hkv, int G, int r, int D, int L, int num_sms, const int *max_clusters) {
  const long long rows = static_cast<long long>(r) * G, groups = static_cast<long long>(Hkv) * B;
  Kv4Plan best = {kKv4Few, 1, 1, 0.f};
  auto take = [&](int form, int tiles, int splits, double cost) {
    if (best.us == 0.f || cost < best.us) best = Kv4Plan{form, tiles, splits, static_cast<float>(cost)};
  };
  if (rows <= 64) {
    const int nb = rows <= 8 ? 1 : 2, rounds = L > 0 ? (L + 127) / 128 : 1;
    const double units = static_cast<double>((rows + 8 * nb - 1) / (8 * nb)) * groups, d = D == 128 ? 1.0 : 0.6;
    for (int s = 1; s <= kFewMaxRanges; ++s) {
      const int per = (rounds + s - 1) / s;
      if (s > 1 && (rounds + per - 1) / per != s) continue;
      const double ctas = units * s;
      const double t = d * (nb == 2 ? 6.1e-3 : ctas <= num_sms / 2 ? 4.1e-3 : ctas <= num_sms ? 5.7e-3 : 7.5e-3);
      take(kKv4Few, nb, s, waves_of(ctas, nb == 2 ? num_sms : 2 * num_sms, nb == 2 ? 4.0 : 3.0) * (5.5 + 0.25 * (s - 1) + per * 128 * t));
    }
  }
  if (rows > 8)
    for (int tiles = rows > 128 ? 2 : 1; tiles >= 1; --tiles)
      for (int s = 1; s <= kKv4ManyMaxRanges; ++s) {
        const double cost = attention_kv4_many_cost(rows, groups, D, L, tiles, s, false, num_sms, max_clusters);
        if (cost > 0.0) take(kKv4Many, tiles, s, cost);
      }
  return best;
}

// Query tiles a block where decoding the cache once first is estimated to take a twentieth less time than `plan` does; else 0.
static int decode_once(const Kv4Plan &plan, int B, int Hkv, int G, int r, int D, int L, int num_sms, const int *max_clusters) {
  if (plan.form != kKv4Many || L <= 0) return 0;
  const long long rows = static_cast<long long>(r) * G, groups = static_cast<long long>(Hkv) * B;
  const double one = attention_kv4_many_cost(rows, groups, D, L, 1, 1, true, num_sms, max_clusters);
  const double two = rows > 128 ? attention_kv4_many_cost(rows, groups, D, L, 2, 1, true, num_sms, max_clusters) : one;
  return 1.05 * fmin(one, two) < plan.us ? (one <= two ? 1 : 2) : 0;
}

size_t attention_kv4_workspace(int B, int Hkv, int G, int r, int D, int L, int num_sms) {
  const int *clusters = attention_kv4_max_clusters();
  if (!clusters) return 0;
  return decode_once(attention_kv4_plan(B, Hkv, G, r, D, L, num_sms, clusters), B, Hkv, G, r, D, L, num_sms, clusters)
             ? static_cast<size_t>(B) * Hkv * L * D * 4 : 0;
}

cudaError_t launch_attention_kv4(Kv4AttnArgs a, void *workspace, size_t bytes, int num_sms, cudaStream_t st) {
  const int G = a.H / a.Hkv;
  const int *clusters = attention_kv4_max_clusters();
  if (!clusters) return cudaErrorInvalidConfiguration;
  const Kv4Plan plan = attention_kv4_plan(a.B, a.Hkv, G, a.r, a.D, a.L, num_sms, clusters);
  a.kv_splits = plan.splits;
  a.tiles_per_cta = plan.tiles;
  if (plan.form == kKv4Many) {
    if (workspace && bytes >= static_cast<size_t>(a.B) * a.Hkv * a.L * a.D * 4) {
      const int tiles = decode_once(plan, a.B, a.Hkv, G, a.r, a.D, a.L, num_sms, clusters);
      if (tiles) {
        a.kv_splits = 1;
        a.tiles_per_cta = tiles;
        return launch_attention_kv4_many(a, workspace, num_sms, st);
      }
    }
    return launch_attention_kv4_many(a, nullptr, num_sms, st);
  }
  if (a.D == 64) return plan.tiles == 1 ? launch_few<64, 1>(a, st) : launch_few<64, 2>(a, st);
  return plan.tiles == 1 ? launch_few<128, 1>(a, st) : launch_few<128, 2>(a, st);
}

}  // namespace fvar
