// Attention of query rows over a cache in 4 bits (format and operator: include/fvar.h).
//
// Few rows (attention_kv4_few_kernel, up to 16 query rows a cache head): bound by reading the cache, so the codes go from
// memory to the tensor cores without a stop on the way: bulk copies bring them to shared memory as they are, a warp takes the
// codes of 16 keys into registers in the order in which mma.sync wants its operand and decodes them there.  (Through tcgen05 they would
// have to be decoded into shared memory and read from there again: 2.5 times their bf16 size at 128 bytes a clock, 1.8 times
// what reading the codes from HBM takes.)  Keys and values are the operand of 16 rows, the query rows the one of 8:
//   S^T [16 keys][8 rows] = K Q^T,   O^T [16 of D][8 rows] += V^T P^T.
// The order of D within a product is free, so a lane takes whole words: of a key row the words of its own quarter of D (that is
// one group and one scale at D = 128), of four value rows one or two words each.
#include <limits.h>
#include <math.h>

#include "kv4.cuh"
#include "ptx.cuh"

namespace fvar {

// D[16][8] += A[16][16] B[16][8], bf16, fp32 accumulator.
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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
// What a query row's share of a range of keys weighs; m in units of the scores, c of log2.  A range without any key has l = 0.
__device__ __forceinline__ float range_weight(float m, float l, float m_all, float c) { return l == 0.f ? 0.f : exp2f((m - m_all) * c); }

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
  static constexpr int kQuads = kRows * D / 4;            // float4 of a unit
  static constexpr int kRecvBytes = (kQuads + kFewMaxRanges) * 16;            // what the ranges of a cluster push here
  static constexpr int kMlBytes = kFewMaxRanges * kRows * 8;
  static constexpr int kStagesBytes = kFewStages * kStageBytes, kAllParts = (kPartBytes + kFewWarps * kRows * 8 + 127) / 128 * 128;
  static constexpr int kFrontBytes = kStagesBytes > kAllParts ? kStagesBytes : kAllParts;
  static constexpr int kSmemBytes = kFrontBytes + kRecvBytes + kMlBytes + 128;
};

template <int D, int NB>
__global__ void __launch_bounds__(kFewThreads, NB == 1 ? 2 : 1) attention_kv4_few_kernel(const __grid_constant__ Kv4AttnArgs p) {
  using Cfg = FewCfg<D, NB>;
  constexpr int KW = D / 32, VW = D / 64;                 // words a lane takes of a key row, of a value row
  extern __shared__ __align__(128) uint8_t smem_raw[];
  __shared__ uint64_t bars[kFewStages];
  __shared__ unsigned done[kFewStages];                   // warps that have finished with a slot, in all its uses
  __shared__ volatile int abort_flag;
  const uint32_t stages = smem_u32(smem_raw);
  const uint32_t recv = stages + Cfg::kFrontBytes, recv_ml = recv + Cfg::kRecvBytes;
  auto full = [&](int s) { return smem_u32(&bars[s]); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  const long long wb = wait_budget(p.wait_cycles);

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

  const float c = p.scale_log2;
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
    mbar_expect_tx(full(slot), n * (D + 2 * (D / kKv4Group)));
    bulk_load(dst, p.k_codes + (row0 + k) * (D / 2), n * (D / 2), full(slot));
    bulk_load(dst + 2 * Cfg::kCodeBytes, p.k_scales + (row0 + k) * (D / kKv4Group), n * (D / kKv4Group), full(slot));
    bulk_load(dst + Cfg::kCodeBytes, p.v_codes + (row0 + k) * (D / 2), n * (D / 2), full(slot));
    bulk_load(dst + 2 * Cfg::kCodeBytes + Cfg::kScaleBytes, p.v_scales + (row0 + k) * (D / kKv4Group), n * (D / kKv4Group), full(slot));
  };
  if (threadIdx.x == 0)
    for (int st = 0; st < min(kFewStages, nst); ++st) request(st);
  {
    // ------------------------------------------------------------------ products
    uint32_t q[NB][KW][4];                                // [word][pair]: the lane's values of row rho0 + 8 nb + gid
    int lim[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int rho = rho0 + nb * 8 + gid;
      const bool there = rho < nrows;
      const bf16 *src = p.q + (static_cast<long long>(b) * p.r + rho / G) * p.ldq + (kv * G + rho % G) * D + tig * (D / 4);
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const uint4 v = there ? *reinterpret_cast<const uint4 *>(src + 8 * w) : make_uint4(0, 0, 0, 0);
        q[nb][w][0] = v.x; q[nb][w][1] = v.y; q[nb][w][2] = v.z; q[nb][w][3] = v.w;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) lim[nb][i] = min(limit_of(rho0 + nb * 8 + 2 * tig + i), k1);
    }
    const float grow = 8.f / c;
    bool ok = true;
    for (int st = 0; st < nst; ++st) {
      const int slot = st % kFewStages;
      ok = __all_sync(0xffffffffu, mbar_wait(full(slot), (st / kFewStages) & 1, p.status, &abort_flag, wb));
      if (!ok) break;
      const uint32_t base = stages + slot * Cfg::kStageBytes;
      const int kr = warp * 16 * kFewSets, key = k0 + st * kFewStageKeys + kr;               // the warp's keys
      if (key < k1) {
        uint32_t kw[kFewSets][2][KW], vw[kFewSets][4][VW], ks[kFewSets][2], vs[kFewSets][4];
#pragma unroll
        for (int x = 0; x < kFewSets; ++x) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = kr + 16 * x + gid + 8 * i;
            ld_shared_words<KW>(base + row * (D / 2) + tig * (D / 8), kw[x][i]);
            ks[x][i] = ld_shared_u8(base + 2 * Cfg::kCodeBytes + row * (D / kKv4Group) + tig * (D / 4) / kKv4Group);
          }
        }
        // S^T = K Q^T: lane (gid, tig) has quarter tig of keys gid and gid + 8 of a set
        float s[kFewSets][NB][4], s_odd[kFewSets][NB][4];
#pragma unroll
        for (int x = 0; x < kFewSets; ++x)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int k = 0; k < 4; ++k) s[x][nb][k] = s_odd[x][nb][k] = 0.f;
        uint32_t s0[kFewSets], s1[kFewSets], f0[kFewSets], f1[kFewSets];
#pragma unroll
        for (int x = 0; x < kFewSets; ++x) {
          s0[x] = kv4_scale2(ks[x][0]);
          s1[x] = kv4_scale2(ks[x][1]);
          f0[x] = kv4_offset2(s0[x]);
          f1[x] = kv4_offset2(s1[x]);
        }
#pragma unroll
        for (int w = 0; w < KW; ++w)
#pragma unroll
          for (int x = 0; x < kFewSets; ++x) {
            uint32_t a[4], a8[4];
            kv4_word(kw[x][0][w], s0[x], f0[x], a);
            kv4_word(kw[x][1][w], s1[x], f1[x], a8);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              mma_16816(s[x][nb], a[0], a8[0], a[1], a8[1], q[nb][w][0], q[nb][w][1]);
              mma_16816(s_odd[x][nb], a[2], a8[2], a[3], a8[3], q[nb][w][2], q[nb][w][3]);
            }
          }
#pragma unroll
        for (int x = 0; x < kFewSets; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) {                   // keys 2 tig, 2 tig + 1, 2 tig + 8, 2 tig + 9; values gid * D / 8 ...
            const int row = kr + 16 * x + 2 * tig + (i & 1) + 8 * (i >> 1);
            ld_shared_words<VW>(base + Cfg::kCodeBytes + row * (D / 2) + gid * (D / 16), vw[x][i]);
            vs[x][i] = ld_shared_u8(base + 2 * Cfg::kCodeBytes + Cfg::kScaleBytes + row * (D / kKv4Group) + gid * (D / 8) / kKv4Group);
          }
#pragma unroll
        for (int x = 0; x < kFewSets; ++x)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int k = 0; k < 4; ++k) s[x][nb][k] += s_odd[x][nb][k];          // two chains of products: 1.3 % of a launch
        // s[x][nb][0 .. 3]: (key gid, row 2 tig), (gid, 2 tig + 1), (gid + 8, 2 tig), (gid + 8, 2 tig + 1)
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
            need = need || top[nb][i] > m[nb][i] + grow;
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
              const float m2 = fmaxf(m[nb][i], t2), a = exp2f((m[nb][i] - m2) * c);
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
        for (int x = 0; x < kFewSets; ++x) {
          uint32_t pt[NB][2];                             // P^T of keys 0 - 7 and 8 - 15, as the second operand wants it
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            float e[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) e[k] = exp2f(fmaf(s[x][nb][k], c, -m[nb][k & 1] * c));
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
      const float a = range_weight(ml[w].x, ml[w].y, m_all, c);
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
        const float a = range_weight(ml.x, ml.y, m_all, c);
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

template <int D, int NB>
static cudaError_t launch_few(const Kv4AttnArgs &a, cudaStream_t st) {
  using Cfg = FewCfg<D, NB>;
  static unsigned long long prepared = 0;                 // a bit a device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !(prepared >> dev & 1)) {
    e = cudaFuncSetAttribute(attention_kv4_few_kernel<D, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmemBytes);
    if (e != cudaSuccess) return e;
    if (dev < 64) prepared |= 1ull << dev;
  }
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
  return cudaLaunchKernelEx(&cfg, attention_kv4_few_kernel<D, NB>, a);
}

// Waves of `ctas` blocks over `slots`: whole ones while there are fewer than `few`.
static double waves_of(double ctas, double slots, double few) {
  const double w = ctas / slots;
  return w <= 1.0 ? 1.0 : w < few ? ceil(w) : w;
}

// Form, tiles and key ranges of a launch: the least estimated time (microseconds).  The estimates are fitted to forced launches on B200,
// 10 shapes of few rows and 24 of many, 1 to 4096 rows over 77 to 10521 keys, which they rank as measured but for differences of a few
// per cent.  Few rows: a block costs 5.5 and its keys 8.25 ns each at D = 128 with two blocks an SM, 4.5 with one (4.8 and 2.7 at D = 64);
// 9 to 16 rows at a time, one block an SM, 5.8 (3.4).  Many rows: see attention_kv4_many_cost.  Where both can be taken they cross between 17 rows
// (8 units: 11.5 us against 21.8) and 64 (32 units over 8000 keys: 52 against 29).
Kv4Plan attention_kv4_plan(int B, int Hkv, int G, int r, int D, int L, int num_sms, const int *max_clusters) {
  const long long rows = static_cast<long long>(r) * G, groups = static_cast<long long>(Hkv) * B;
  Kv4Plan best = {kKv4Few, 1, 1};
  double best_cost = 0.0;
  auto take = [&](int form, int tiles, int splits, double cost) {
    if (best_cost == 0.0 || cost < best_cost) { best = Kv4Plan{form, tiles, splits}; best_cost = cost; }
  };
  if (rows <= 64) {
    const int nb = rows <= 8 ? 1 : 2, rounds = L > 0 ? (L + 127) / 128 : 1;
    const double units = static_cast<double>((rows + 8 * nb - 1) / (8 * nb)) * groups, d = D == 128 ? 1.0 : 0.58;
    for (int s = 1; s <= kFewMaxRanges; ++s) {
      const int per = (rounds + s - 1) / s;
      if (s > 1 && (rounds + per - 1) / per != s) continue;
      const double ctas = units * s;
      const double t = d * (nb == 2 ? 5.8e-3 : ctas <= num_sms / 2 ? 4.5e-3 : ctas <= num_sms ? 6.3e-3 : 8.25e-3);
      take(kKv4Few, nb, s, waves_of(ctas, nb == 2 ? num_sms : 2 * num_sms, nb == 2 ? 4.0 : 3.0) * (5.5 + 0.25 * (s - 1) + per * 128 * t));
    }
  }
  if (rows > 8)
    for (int tiles = rows > 128 ? 2 : 1; tiles >= 1; --tiles)
      for (int s = 1; s <= kKv4ManyMaxRanges; ++s) {
        const double cost = attention_kv4_many_cost(rows, groups, D, L, tiles, s, num_sms, max_clusters);
        if (cost > 0.0) take(kKv4Many, tiles, s, cost);
      }
  return best;
}

cudaError_t launch_attention_kv4(Kv4AttnArgs a, void *workspace, size_t bytes, int num_sms, cudaStream_t st) {
  const int G = a.H / a.Hkv;
  const int *clusters = attention_kv4_max_clusters();
  if (!clusters) return cudaErrorInvalidConfiguration;
  const Kv4Plan plan = attention_kv4_plan(a.B, a.Hkv, G, a.r, a.D, a.L, num_sms, clusters);
  a.kv_splits = plan.splits;
  a.tiles_per_cta = plan.tiles;
  if (plan.form == kKv4Many) return launch_attention_kv4_many(a, workspace, bytes, num_sms, st);
  if (a.D == 64) return plan.tiles == 1 ? launch_few<64, 1>(a, st) : launch_few<64, 2>(a, st);
  return plan.tiles == 1 ? launch_few<128, 1>(a, st) : launch_few<128, 2>(a, st);
}

}  // namespace fvar
