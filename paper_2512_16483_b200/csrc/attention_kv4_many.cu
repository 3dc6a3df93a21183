// Attention over a cache in 4 bits for many query rows (format and operator: include/fvar.h), on the fifth-generation tensor cores.
//
// A unit of work is up to 256 query rows (two tiles of 128) of one cache head of one element; with grouped heads the rows of all
// heads of the group, rho = row * G + head of the group.  One CTA of 16 warps:
//   warp 0             issues S_t = Q_t K^T and O_t += P_t V, accumulators in TMEM;
//   warp 7             requests the queries and, tile by tile, the codes and scales of 128 keys or their values (TMA);
//   warps 1-6          decode, two warps a tile: codes from shared memory to registers, and back as the bf16 operand tile, swizzled, in
//                      a ring of slots of its own;
//   warps 8-11, 12-15  softmax of stream 0 and 1, one query row a thread.
// The two streams are the two query tiles, out of phase, or with a lone tile the even and the odd blocks of keys.  A decoded
// tile serves both query tiles.  Keys and values have the same layout, rows of D: the keys are a K-major operand, the values an
// MN-major one, so neither is transposed.  The softmax is that of attention.cu (P in TMEM, two halves, rescaling only when a maximum has
// grown by 2^8).  Every wait is bounded.
//
// Few units over many keys: the key range is split over a cluster of up to 6 CTAs, whose rows are pushed to the CTA that merges them
// and added up in range order.
//
// Many query tiles a head: every unit would decode the same keys again, in issue slots that the softmax needs.  Then a pass of its
// own decodes the cache once into the caller's workspace, and the units (CODES false) request bf16 tiles by TMA.
//
// What bounds it is the issue of softmax and decoding together (410 rows of 2 x 16 heads over 2931 keys, D = 128: 35.3 us, 23 blocks of 1.3 us
// in 128 CTAs, tensor pipe 36 %, issue slots 39 % busy), at the largest size also the clock under load (4096 rows over 10521 keys: 570 to 580 us,
// 36 of them the pass, 1.22 PFLOP/s, in a short run, 690 to 705 in a long one).
#include <limits.h>
#include <math.h>

#include "kv4.cuh"
#include "per_device.h"
#include "ptx.cuh"
#include "softmax.cuh"

namespace fvar {

constexpr int kManyThreads = 512;
constexpr int kDecodeTeams = 3, kQueryWarp = 7, kManySoftmaxWarp = 8;      // teams of two warps
// Registers a thread after the split: 2 * 72 + 2 * 184 = 4 * 128.
constexpr int kRegsLaunch = 128, kRegsDecode = 72, kRegsRows = 184;
static_assert(2 * kRegsDecode + 2 * kRegsRows == 4 * kRegsLaunch, "what is given back is what is taken");
constexpr int kTileRows = 128, kBlockKeys = 128;
constexpr int kAtom = 128 * 128;              // [128 rows][64 bf16], swizzled
constexpr int kMaxOrdered = 128;              // elements of a batch that are taken by length
constexpr float kGrow = 8.0f;                 // log2 units
// Maxima beyond this (log2 units) are taken off the scores before these are multiplied, not in the same operation: the product with the
// maximum rounds by up to half a step, 2^-14 here, which all keys of a row share, but by any amount, up to an infinite weight, farther out.
constexpr float kLargeMax = 1024.0f;
constexpr float kNoRowMax = -3.0e38f;         // running maxima start here: finite, so that no difference of two of them is a NaN

template <int D, bool CODES>
struct ManyCfg {
  static constexpr int kTileBytes = 128 * D * 2;          // a query tile, a tile of 128 keys or of their values
  static constexpr int kRing = CODES ? (D == 64 ? 8 : 3) : (D == 64 ? 10 : 5);
  static constexpr int kCodeBytes = kBlockKeys * D / 2, kScaleBytes = kBlockKeys * D / kKv4Group;
  static constexpr int kRawBytes = kCodeBytes + kScaleBytes, kRaw = CODES ? (D == 64 ? 14 : 7) : 0;         // tiles of codes under way
  static constexpr int kQBytes = 2 * kTileBytes, kSwapBytes = 2 * kTileRows * 8, kOrderBytes = kMaxOrdered;
  static constexpr int kBars = 16 + 2 * kRing + 2 * kRaw;
  static constexpr int kSmemBytes = kQBytes + kRing * kTileBytes + kRaw * kRawBytes + kSwapBytes + kOrderBytes + 512;
  static constexpr int kTmemCols = 512;                   // S0, S1, O0, O1
  static_assert(kBars * 8 + 16 <= 512 && kSmemBytes <= 232448, "shared memory");
  static_assert(kSmemBytes > 116 * 1024, "one CTA per SM (the CTA allocates all of TMEM)");
  static_assert(kRawBytes % (4 * D) == 0, "the swizzle of codes repeats after eight rows");
};

// Elements of a batch by their last row's limit, the greatest first (equal ones in order): the units that come last in the walk are then short.
// order[0 .. B), in shared memory, for every thread of the block, which all call this; B <= kMaxOrdered.  Every warp has all limits in
// registers and ranks some of them by counting.  With limits between 0 and L in no order, 256 rows of 40 x 16 heads, L = 1000, D = 64, took 86.5 us
// without it and 65.7 with it, 300 rows of 16 x 8 heads, L = 3000, D = 128, 95.6 and 81.2; where all are equal it costs 0.7 to 1.3 us (2 % at most).
// In the kernel of few rows it cost as much as it gained (its blocks are more and shorter).
__device__ __forceinline__ void longest_first(uint8_t *order, const int *limits, int r, int B) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int key[kMaxOrdered / 32];                              // all different: limits in 24 bits, then the place
#pragma unroll
  for (int c = 0; c < kMaxOrdered / 32; ++c) {
    const int b = c * 32 + lane;
    key[c] = b < B ? min(max(limits[static_cast<long long>(b) * r + r - 1], 0), 0xFFFFFF) * 128 + (127 - b) : -1;
  }
#pragma unroll
  for (int c = 0; c < kMaxOrdered / 32; ++c)
    for (int i = warp; c * 32 + i < B && i < 32; i += kManyThreads / 32) {
      const int mine = __shfl_sync(0xffffffffu, key[c], i);
      int rank = 0;
#pragma unroll
      for (int d = 0; d < kMaxOrdered / 32; ++d) rank += __popc(__ballot_sync(0xffffffffu, key[d] > mine));
      if (lane == 0) order[rank] = static_cast<uint8_t>(c * 32 + i);
    }
  __syncthreads();
}

// 1 / l of a row that sees `limit` keys.  No weight at all: it sees none, or its scores are all minus infinity.
__device__ __forceinline__ float inverse_sum(float l, int limit) { return l != 0.f ? 1.0f / l : limit > 0 ? __uint_as_float(0x7FC00000u) : 0.f; }

template <int D, bool RANGES, bool CODES>
__global__ void __launch_bounds__(kManyThreads, 1)
attention_kv4_many_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Kv4AttnArgs p) {
  using Cfg = ManyCfg<D, CODES>;
  constexpr int NR = Cfg::kRing, NC = Cfg::kRaw;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t q_smem = smem_u32(smem_raw), ring_smem = q_smem + Cfg::kQBytes, raw_smem = ring_smem + NR * Cfg::kTileBytes;
  const uint32_t swap_smem = raw_smem + NC * Cfg::kRawBytes;
  const uint32_t bar_base = swap_smem + Cfg::kSwapBytes + Cfg::kOrderBytes;
  uint8_t *const order = smem_raw + (swap_smem - q_smem) + Cfg::kSwapBytes;
  uint8_t *tail = smem_raw + Cfg::kSmemBytes - 512 + 8 * Cfg::kBars;
  uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(tail);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tail + 4);
  auto q_full = [&](int s) { return bar_base + 8u * s; };
  auto q_empty = [&](int s) { return bar_base + 8u * (2 + s); };
  auto ring_full = [&](int s) { return bar_base + 8u * (4 + s); };
  auto ring_empty = [&](int s) { return bar_base + 8u * (4 + NR + s); };
  auto s_full = [&](int t) { return bar_base + 8u * (4 + 2 * NR + t); };
  auto p_half = [&](int t) { return bar_base + 8u * (6 + 2 * NR + t); };
  auto p_full = [&](int t) { return bar_base + 8u * (8 + 2 * NR + t); };
  auto o_full = [&](int t) { return bar_base + 8u * (10 + 2 * NR + t); };   // P V of a block that is not the stream's last
  auto o_last = [&](int t) { return bar_base + 8u * (12 + 2 * NR + t); };
  const uint32_t swap_full = bar_base + 8u * (14 + 2 * NR), swap_done = swap_full + 8;       // a lone tile's streams meet; both have stored their columns
  auto raw_full = [&](int s) { return bar_base + 8u * (16 + 2 * NR + s); };
  auto raw_empty = [&](int s) { return bar_base + 8u * (16 + 2 * NR + NC + s); };

  if (q_smem & 1023) {                                    // the swizzle counts from 1024-byte boundaries
    if (threadIdx.x == 0) atomicOr(p.status, kStatusTimeout);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long wb = wait_budget(p.wait_cycles);
  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int s = 0; s < 2; ++s) {
      mbar_init(q_full(s), 1);
      mbar_init(q_empty(s), 1);
    }
    for (int s = 0; s < NR; ++s) {
      mbar_init(ring_full(s), CODES ? 2 : 1);
      mbar_init(ring_empty(s), 1);
    }
    for (int s = 0; s < NC; ++s) {
      mbar_init(raw_full(s), 1);
      mbar_init(raw_empty(s), 2);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(s_full(t), 1);
      mbar_init(p_half(t), 128);
      mbar_init(p_full(t), 128);
      mbar_init(o_full(t), 1);
      mbar_init(o_last(t), 1);
    }
    mbar_init(swap_full, 256);
    mbar_init(swap_done, 256);
    mbar_fence_init();
  }
  if (warp == 0) {
    tmem_alloc(smem_u32(tmem_holder), Cfg::kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_holder;
  pdl_launch_dependents();
  pdl_wait();
  if (p.by_length) longest_first(order, p.limits, p.r, p.B);

  // Units: RANGES: the CTAs of a cluster take the key ranges of one; else a CTA walks the units blockIdx.x, + gridDim.x, ...
  const int splits = RANGES ? p.kv_splits : 1, sp = RANGES ? static_cast<int>(blockIdx.x) % splits : 0;
  const int unit0 = RANGES ? static_cast<int>(blockIdx.x) / splits : blockIdx.x, unit_step = RANGES ? p.units : gridDim.x;
  // Lone tiles have room for the queries of two units, pairs fill it with one's.
  const uint32_t qrooms = p.tiles_per_cta == 1 ? 2 : 1;
  const int G = p.H / p.Hkv, nrows = p.r * G;
  struct Unit {
    int rho0, h, e, ntiles, kb0, nkv, keys;               // keys: those that some row of the unit sees; blocks [kb0, kb0 + nkv) here
  };
  auto unit_at = [&](int u) {
    Unit x;
    const int g = fast_div(u, p.div_nqt), qt = u - g * static_cast<int>(p.div_nqt.d);       // neighbouring units share keys and values (L2)
    x.e = fast_div(g, p.div_h);
    x.h = g - x.e * p.Hkv;
    if (p.by_length) x.e = order[x.e];
    x.rho0 = qt * p.tiles_per_cta * kTileRows;
    x.ntiles = (p.tiles_per_cta == 2 && nrows - x.rho0 > kTileRows) ? 2 : 1;
    x.keys = p.L;
    if (p.limits) {
      const int i0 = fast_div(x.rho0, p.div_g), i1 = fast_div(min(nrows, x.rho0 + x.ntiles * kTileRows) - 1, p.div_g);
      int top = 0;
      for (int i = i0 + lane; i <= i1; i += 32) top = max(top, p.limits[static_cast<long long>(x.e) * p.r + i]);
      x.keys = min(__reduce_max_sync(0xffffffffu, top), p.L);
    }
    const int blocks = (x.keys + kBlockKeys - 1) / kBlockKeys, per = (blocks + splits - 1) / splits;
    x.kb0 = min(sp * per, blocks);
    x.nkv = min(per, blocks - x.kb0);
    return x;
  };
  // Tile i of a unit's stream: keys (v = 0) or values of which block.  A lone tile has two blocks under way.
  auto item_at = [](int i, int nkv, bool dual, int &j, int &v) {
    j = i >> 1, v = i & 1;                                // K 0, V 0, K 1, V 1, ...
    if (dual && nkv > 1) {                                // K 0, K 1, V 0, K 2, V 1, K 3, ... V nkv-2, V nkv-1
      const bool last = i == 2 * nkv - 1;
      v = last || (i > 0 && (i & 1) == 0);
      j = last ? nkv - 1 : v ? (i >> 1) - 1 : (i + 1) >> 1;
    }
  };
  float m_ref = kNoRowMax, l_run = 0.f;       // softmax threads: running maximum and sum of this thread's query row and stream
  bool final_ok = true, any_block = false;    // softmax threads: the stream's last P V has completed; there was one

  if (warp == 0) {
    setmaxnreg_dec<kRegsDecode>();
    // ---------------------------------------------------------------- MMA issuer: the whole warp walks, one lane issues
    constexpr uint32_t idesc_s = umma_idesc_bf16(kTileRows, kBlockKeys);
    constexpr uint32_t idesc_o = umma_idesc_bf16(kTileRows, D) | (1u << 16);       // bit 16: the values are MN-major
    const uint32_t leader = elect_one() ? 1u : 0u;
    auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, p.status, abort_flag, wb)) != 0; };
    const uint64_t q_desc = smem_desc_sw128(q_smem), k_desc = smem_desc_sw128(ring_smem), v_desc = smem_desc_sw128_mn(ring_smem, kAtom);
    auto issue_s = [&](int t, int qt, int slot) {       // S buffer t = Q_qt K^T
      const uint64_t dq = q_desc + static_cast<uint32_t>(qt * (Cfg::kTileBytes >> 4)), dk = k_desc + static_cast<uint32_t>(slot * (Cfg::kTileBytes >> 4));
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        constexpr uint32_t a = kAtom >> 4;
        umma_bf16_if(leader, tmem_base + t * kBlockKeys, dq + ((k / 4) * a + 2 * (k % 4)), dk + ((k / 4) * a + 2 * (k % 4)), idesc_s, k != 0);
      }
      umma_commit_if(leader, s_full(t));
    };
    auto issue_pv = [&](int t, int slot, int half, bool accumulate) {     // O_t (+)= P_t V over 64 keys
      const uint64_t dv = v_desc + static_cast<uint32_t>(slot * (Cfg::kTileBytes >> 4) + half * (64 * 128 >> 4));
      const uint32_t to = tmem_base + 256 + t * D, tp = tmem_base + t * kBlockKeys + half * 32;
#pragma unroll
      for (int k = 0; k < 4; ++k) umma_bf16_tmem_a_if(leader, to, tp + 8 * k, dv + k * (16 * 128 >> 4), idesc_o, (accumulate || k != 0) ? 1u : 0u);
    };
    bool ok = true;
    uint32_t qn = 0, p_par = 0, phase = 0;           // p_par: a bit a stream
    int slot = 0;
    auto take = [&]() {                                 // the next tile of the ring; its slot
      const int s = slot;
      ok = ok && wait(ring_full(s), phase);
      tc_fence_after();
      if (++slot == NR) { slot = 0; phase ^= 1u; }
      return s;
    };
    // P V of the next block of stream t over the values in slot `vs` (taken when first needed)
    auto pv = [&](int t, int &vs, bool accumulate, bool last) {
      ok = ok && wait(p_half(t), p_par >> t & 1u);
      if (vs < 0) vs = take();
      if (!ok) return;
      tc_fence_after();
      issue_pv(t, vs, 0, accumulate);
      ok = wait(p_full(t), p_par >> t & 1u);
      if (!ok) return;
      p_par ^= 1u << t;
      tc_fence_after();
      issue_pv(t, vs, 1, true);
      umma_commit_if(leader, last ? o_last(t) : o_full(t));
    };
    for (int u = unit0; ok && u < p.units; u += unit_step) {
      const Unit x = unit_at(u);
      const int nkv = x.nkv;
      if (nkv == 0) continue;
      const int room = qn % qrooms;
      ok = wait(q_full(room), qn / qrooms & 1u);
      ++qn;
      if (!ok) break;
      int ks = take();
      if (!ok) break;
      issue_s(0, room, ks);
      if (x.ntiles == 2) issue_s(1, 1, ks);
      umma_commit_if(leader, ring_empty(ks));
      if (nkv == 1) umma_commit_if(leader, q_empty(room));
      if (x.ntiles == 2) {
        for (int j = 0; ok && j < nkv; ++j) {
          int vs = -1;
          ks = -1;
          for (int t = 0; ok && t < 2; ++t) {
            pv(t, vs, j > 0, j + 1 == nkv);
            if (!ok) break;
            if (t == 1) umma_commit_if(leader, ring_empty(vs));
            if (j + 1 < nkv) {
              if (t == 0) ks = take();
              if (!ok) break;
              issue_s(t, t, ks);
              if (t == 1) {
                umma_commit_if(leader, ring_empty(ks));
                if (j + 2 == nkv) umma_commit_if(leader, q_empty(room));
              }
            }
          }
        }
      } else {
        if (nkv > 1) {
          ks = take();
          if (!ok) break;
          issue_s(1, room, ks);
          umma_commit_if(leader, ring_empty(ks));
          if (nkv == 2) umma_commit_if(leader, q_empty(room));
        }
        for (int j = 0; ok && j < nkv; ++j) {
          const int t = j & 1;
          int vs = -1;
          pv(t, vs, j > 1, j + 2 >= nkv);
          if (!ok) break;
          umma_commit_if(leader, ring_empty(vs));
          if (j + 2 < nkv) {
            ks = take();
            if (!ok) break;
            issue_s(t, room, ks);
            umma_commit_if(leader, ring_empty(ks));
            if (j + 3 == nkv) umma_commit_if(leader, q_empty(room));
          }
        }
      }
    }
  } else if (warp < kManySoftmaxWarp) {
    // ------------------------------------------------------------------ operand tiles
    setmaxnreg_dec<kRegsDecode>();
    const bool query_warp = warp == kQueryWarp;
    const int team = (warp - 1) >> 1, half = (warp - 1) & 1;
    // A lane decodes 32 values (one group) of a row at a time, eight neighbouring lanes eight neighbouring rows: the stores of a
    // quarter of a warp then fall into eight different 16-byte columns of the swizzled tile.  A warp has kStep rows at a time and 64
    // rows of a tile.  (All warps on every tile spent more issue slots on waiting and arriving than on decoding.)
    constexpr int kPieces = D / 32, kStep = 32 / kPieces, kReps = 64 / kStep;
    const int piece = (lane >> 3) % kPieces, lrow = half * 64 + (lane & 7) + 8 * ((lane >> 3) / kPieces);
    uint32_t column[4];                                   // where the lane's four words of a row go in the tile
#pragma unroll
    for (int n = 0; n < 4; ++n) column[n] = (piece >> 1) * kAtom + lrow * 128 + ((((piece & 1) * 4 + n) ^ (lane & 7)) * 16);
    // and where its codes and scales come from (16-byte columns of 64 bytes of codes are swizzled by row / 2, of 32 bytes by row / 4)
    const uint32_t code_at = lrow * (D / 2) + (piece ^ (D == 128 ? (lrow >> 1) & 3 : (lrow >> 2) & 1)) * 16, scale_at = Cfg::kCodeBytes + lrow * (D / kKv4Group) + piece;
    bool ok = true;
    unsigned base = 0;                                    // place of the unit's first tile among all that pass through the ring
    uint32_t q_units = 0, armed = 0, armed_par = 0, q_armed = 0, q_armed_par = 0;     // slots that a copy was requested into, and the parity of the last
    for (int u = unit0; ok && u < p.units; u += unit_step) {
      const Unit x = unit_at(u);
      if (x.nkv == 0) continue;
      const bool dual = x.ntiles == 1;
      const int tiles = 2 * x.nkv;
      if (query_warp) {
        const uint32_t room = q_units % qrooms;
        if (q_units >= qrooms) ok = __all_sync(0xffffffffu, mbar_wait(q_empty(room), (q_units / qrooms - 1) & 1u, p.status, abort_flag, wb));
        if (!ok) break;
        const uint32_t q_dst = q_smem + room * Cfg::kTileBytes;
        if (p.q_tma) {
          if (lane == 0) {
            mbar_expect_tx(q_full(room), x.ntiles * Cfg::kTileBytes);
            for (int t = 0; t < x.ntiles; ++t)
#pragma unroll
              for (int a = 0; a < D / 64; ++a)
                tma_load_4d(q_dst + t * Cfg::kTileBytes + a * kAtom, &tmQ, q_full(room), a * 64, x.h * G, fast_div(x.rho0 + t * kTileRows, p.div_g), x.e);
            q_armed |= 1u << room;
            q_armed_par = (q_armed_par & ~(1u << room)) | ((q_units / qrooms & 1u) << room);
          }
        } else {
          constexpr int kLanes = D / 8;                   // 16-byte pieces of a query row; rows that are not there become zeros
#pragma unroll 4
          for (int n = lane; n < x.ntiles * kTileRows * kLanes; n += 32) {
            const int row = n / kLanes, ch = n % kLanes, rho = x.rho0 + row;
            const bool there = rho < nrows;
            const int i = fast_div(rho, p.div_g);
            const bf16 *src = p.q + (there ? (static_cast<long long>(x.e) * p.r + i) * p.ldq + (x.h * G + rho - i * G) * D + ch * 8 : 0);
            const uint32_t dst = q_dst + (row >> 7) * Cfg::kTileBytes + (ch >> 3) * kAtom + (row & 127) * 128 + ((ch ^ row) & 7) * 16;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
          }
          asm volatile("cp.async.wait_all;" ::: "memory");
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(q_full(room));
        }
        ++q_units;
        if (CODES && lane == 0) {
          for (int i = 0; i < tiles; ++i) {
            int j, v;
            item_at(i, x.nkv, dual, j, v);
            const unsigned at = base + i;
            const int slot = at % (NC ? NC : 1);
            ok = mbar_wait(raw_empty(slot), ((at / (NC ? NC : 1)) & 1u) ^ 1u, p.status, abort_flag, wb);
            if (!ok) break;
            const int key = (x.kb0 + j) * kBlockKeys, n = min(kBlockKeys, ((x.keys + 7) & ~7) - key);     // rows of scales: whole 16 bytes; within the cache (L_cap % 8 == 0)
            const uint32_t dst = raw_smem + slot * Cfg::kRawBytes;
            mbar_expect_tx(raw_full(slot), Cfg::kCodeBytes + n * (D / kKv4Group));
            tma_load_4d(dst, v ? &tmV : &tmK, raw_full(slot), 0, key, x.h, x.e);      // rows beyond L_cap become zeros; what nobody sees is masked
            bulk_load(dst + Cfg::kCodeBytes, (v ? p.v_scales : p.k_scales) + (x.e * p.elem_stride + static_cast<long long>(x.h) * p.L_cap + key) * (D / kKv4Group),
                      n * (D / kKv4Group), raw_full(slot));
            armed |= 1u << slot;
            armed_par = (armed_par & ~(1u << slot)) | (((at / (NC ? NC : 1)) & 1u) << slot);
          }
        }
      } else if constexpr (CODES) {
        const int first = static_cast<int>((kDecodeTeams + team - base % kDecodeTeams) % kDecodeTeams);
        for (int i = first; i < tiles; i += kDecodeTeams) {
          const unsigned at = base + i;
          const int slot = at % NR, from = at % (NC ? NC : 1);
          ok = __all_sync(0xffffffffu, mbar_wait(raw_full(from), (at / (NC ? NC : 1)) & 1u, p.status, abort_flag, wb) &&
                                           mbar_wait(ring_empty(slot), ((at / NR) & 1u) ^ 1u, p.status, abort_flag, wb));
          if (!ok) break;
          const uint32_t tile = ring_smem + slot * Cfg::kTileBytes, raw = raw_smem + from * Cfg::kRawBytes;
#pragma unroll
          for (int k = 0; k < kReps; ++k) {
            const float4 c = ld_shared_f4(raw + code_at + k * kStep * (D / 2));
            const uint32_t s2 = kv4_scale2(ld_shared_u8(raw + scale_at + k * kStep * (D / kKv4Group))), f2 = kv4_offset2(s2);
            const uint32_t c4[4] = {__float_as_uint(c.x), __float_as_uint(c.y), __float_as_uint(c.z), __float_as_uint(c.w)};
#pragma unroll
            for (int n = 0; n < 4; ++n) {
              uint32_t o[4];
              kv4_word(c4[n], s2, f2, o);
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(tile + column[n] + k * kStep * 128), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
            }
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(ring_full(slot));
            mbar_arrive(raw_empty(from));
          }
        }
      } else if (threadIdx.x == 32) {
        for (int i = 0; ok && i < tiles; ++i) {
          int j, v;
          item_at(i, x.nkv, dual, j, v);
          const unsigned at = base + i;
          const int slot = at % NR;
          ok = mbar_wait(ring_empty(slot), ((at / NR) & 1u) ^ 1u, p.status, abort_flag, wb);
          if (!ok) break;
          mbar_expect_tx(ring_full(slot), Cfg::kTileBytes);
#pragma unroll
          for (int a = 0; a < D / 64; ++a)
            tma_load_3d(ring_smem + slot * Cfg::kTileBytes + a * kAtom, v ? &tmV : &tmK, ring_full(slot), a * 64, (x.kb0 + j) * kBlockKeys, x.e * p.Hkv + x.h);
          armed |= 1u << slot;
          armed_par = (armed_par & ~(1u << slot)) | (((at / NR) & 1u) << slot);
        }
      }
      ok = __all_sync(0xffffffffu, ok) != 0;              // one lane may have given up alone: a warp goes on together or not at all
      base += tiles;
    }
    if (!ok && (lane == 0) && (query_warp || (!CODES && warp == 1))) {      // let every copy that was requested land before the shared memory is released
      const long long t0 = clock64();
      for (int s = 0; s < 2; ++s)
        while ((q_armed >> s & 1u) && !mbar_try_wait(q_full(s), q_armed_par >> s & 1u) && clock64() - t0 < kWaitCycles) {}
      for (int s = 0; s < (CODES ? NC : NR); ++s)
        while ((armed >> s & 1u) && !mbar_try_wait(CODES ? raw_full(s) : ring_full(s), armed_par >> s & 1u) && clock64() - t0 < kWaitCycles) {}
    }
  } else {
    // ------------------------------------------------------------------ softmax
    setmaxnreg_inc<kRegsRows>();
    const int t = (warp - kManySoftmaxWarp) >> 2, quad = warp & 3, row_local = quad * 32 + lane;
    const uint32_t lane_addr = static_cast<uint32_t>(quad * 32) << 16;
    const uint32_t s_addr = tmem_base + lane_addr + t * kBlockKeys, o_addr = tmem_base + lane_addr + 256 + t * D;
    const float c = p.scale_log2;
    uint32_t s_par = 0, o_base = 0, last_par = 0, swap_par = 0;      // o_base: commits to o_full(t) so far; last_par: a bit a stream
    bool ok = true;
    for (int u = unit0; ok && u < p.units; u += unit_step) {
      const Unit x = unit_at(u);
      const bool dual = x.ntiles == 1;
      const int nblk = dual ? (x.nkv + 1 - t) >> 1 : x.nkv;
      const int rho = x.rho0 + (dual ? 0 : t * kTileRows) + row_local;
      const bool idle = rho - lane >= nrows;              // no row of this warp is there: nothing to compute, but the products wait for it
      m_ref = kNoRowMax;
      l_run = 0.f;
      any_block = nblk > 0;
      bool large = false;                                 // some row of the warp has a maximum beyond kLargeMax
      int limit = 0;
      if (rho < nrows) limit = p.limits ? min(p.limits[static_cast<long long>(x.e) * p.r + fast_div(rho, p.div_g)], x.keys) : x.keys;
      for (int j = 0; j < nblk; ++j) {
        ok = __all_sync(0xffffffffu, mbar_wait(s_full(t), s_par, p.status, abort_flag, wb));
        if (!ok) break;
        s_par ^= 1u;
        if (idle) {
          mbar_arrive(p_half(t));
          mbar_arrive(p_full(t));
          continue;
        }
        tc_fence_after();
        const int valid = limit - (x.kb0 + (dual ? 2 * j + t : j)) * kBlockKeys;       // keys of this block that the row sees (>= 128: all)
        uint32_t v[4][32];
#pragma unroll
        for (int cc = 0; cc < 4; ++cc) tmem_ld32(s_addr + cc * 32, v[cc]);
        tmem_ld_wait();
        if (__any_sync(0xffffffffu, valid < kBlockKeys)) {
#pragma unroll
          for (int cc = 0; cc < 4; ++cc)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (cc * 32 + i >= valid) v[cc][i] = 0xff800000u;   // -inf
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int cc = 0; cc < 4; ++cc)
#pragma unroll
          for (int i = 0; i < 32; i += 2) mx[(i >> 1) & 3] = max3(mx[(i >> 1) & 3], __uint_as_float(v[cc][i]), __uint_as_float(v[cc][i + 1]));
        const float m_cand = fmaxf(m_ref, fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]));
        const bool need = (m_cand - m_ref) * c > kGrow;
        if (__any_sync(0xffffffffu, need)) {
          if (j > 0) {                                    // O is about to be touched: P V of block j - 1 must be complete
            ok = __all_sync(0xffffffffu, mbar_wait(o_full(t), (o_base + j - 1) & 1u, p.status, abort_flag, wb));
            if (!ok) break;
            tc_fence_after();
          }
          const float alpha = need ? exp2f((m_ref - m_cand) * c) : 1.0f;
          if (need) m_ref = m_cand;
          large = __any_sync(0xffffffffu, fabsf(m_ref) * c > kLargeMax && m_ref != kNoRowMax);
          l_run *= alpha;
          if (j > 0) {
#pragma unroll 1
            for (int cc = 0; cc < D / 32; ++cc) {
              uint32_t o[32];
              tmem_ld32(o_addr + cc * 32, o);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
              tmem_st32(o_addr + cc * 32, o);
            }
            tmem_st_wait();
          }
        }
        float neg_mc = -m_ref * c;
        if (large) {
#pragma unroll
          for (int cc = 0; cc < 4; ++cc)
#pragma unroll
            for (int i = 0; i < 32; ++i) v[cc][i] = __float_as_uint(__uint_as_float(v[cc][i]) - m_ref);
          neg_mc = 0.f;
        }
        const uint64_t c2 = pack_f2(c, c), neg_mc2 = pack_f2(neg_mc, neg_mc);
        uint64_t ls[2] = {0ull, 0ull};
#pragma unroll
        for (int cc = 0; cc < 4; ++cc) {                  // keys 32 cc .. of this row, two a word, over the first columns of S
          uint32_t pk[16];
#pragma unroll
          for (int pr = 0; pr < 16; ++pr) {
            float p0, p1;
            unpack_f2(fma_f2(pack_f2(__uint_as_float(v[cc][2 * pr]), __uint_as_float(v[cc][2 * pr + 1])), c2, neg_mc2), p0, p1);
            p0 = exp2f(p0);
            p1 = exp2f(p1);
            ls[pr & 1] = add_f2(ls[pr & 1], pack_f2(p0, p1));
            const __nv_bfloat162 v2 = __floats2bfloat162_rn(p0, p1);
            pk[pr] = *reinterpret_cast<const uint32_t *>(&v2);
          }
          tmem_st16(s_addr + cc * 16, pk);
          if (cc & 1) {
            tmem_st_wait();
            tc_fence_before();
            mbar_arrive(cc == 1 ? p_half(t) : p_full(t));
          }
        }
        float l0, l1;
        unpack_f2(add_f2(ls[0], ls[1]), l0, l1);
        l_run += l0 + l1;
      }
      if (!ok) { final_ok = false; break; }               // the others run into the abort flag in their waits
      if (x.nkv == 0) {                                   // nobody of the unit sees a key (or no key of this range): no product has run
        if constexpr (!RANGES) {
          if (t < x.ntiles && rho < nrows) {
            const int i = fast_div(rho, p.div_g);
            uint4 *dst = reinterpret_cast<uint4 *>(p.out + ((static_cast<long long>(x.e) * p.r + i) * p.H + x.h * G + rho - i * G) * D);
            for (int k = 0; k < D / 8; ++k) dst[k] = make_uint4(0, 0, 0, 0);
          }
        }
        continue;
      }
      if (nblk > 0) {
        ok = __all_sync(0xffffffffu, mbar_wait(o_last(t), last_par >> t & 1u, p.status, abort_flag, wb));
        final_ok = ok;
        o_base += nblk - 1;
      }
      const bool both = dual && x.nkv > 1;                // the other stream has an accumulator too
      if constexpr (!RANGES) {
        // With a lone tile the two streams meet: maxima and sums change sides, and each warp-group finishes half of the columns.
        float norm = 0.f, other = 0.f;
        if (dual) {
          asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(swap_smem + (t * kTileRows + row_local) * 8), "f"(m_ref), "f"(l_run) : "memory");
          mbar_arrive(swap_full);
          if (t == 1 || both) ok = ok && __all_sync(0xffffffffu, mbar_wait(o_last(t ^ 1), last_par >> (t ^ 1) & 1u, p.status, abort_flag, wb));
          ok = ok && __all_sync(0xffffffffu, mbar_wait(swap_full, swap_par, p.status, abort_flag, wb));
        }
        if (ok && !idle) {
          tc_fence_after();
          if (dual) {
            const float2 ml = ld_shared_f2(swap_smem + ((t ^ 1) * kTileRows + row_local) * 8);
            const float m_all = fmaxf(m_ref, ml.x), w0 = exp2f((m_ref - m_all) * c), w1 = exp2f((ml.x - m_all) * c);
            const float l_all = t == 0 ? fmaf(l_run, w0, ml.y * w1) : fmaf(ml.y, w1, l_run * w0);   // the same sum on both sides
            const float inv = inverse_sum(l_all, limit);
            norm = w0 * inv;
            other = w1 * inv;
          } else {
            norm = inverse_sum(l_run, limit);
          }
          int u2 = u;                                     // decoded again: kept in registers through the loop, the unit spills
          asm volatile("" : "+r"(u2));
          const int g2 = fast_div(u2, p.div_nqt), n2 = fast_div(g2, p.div_h), h2 = g2 - n2 * p.Hkv, i2 = fast_div(rho, p.div_g);
          const int e2 = p.by_length ? order[n2] : n2;
          bf16 *dst = p.out + ((static_cast<long long>(e2) * p.r + i2) * p.H + h2 * G + rho - i2 * G) * D;
          const bool wide = (reinterpret_cast<uintptr_t>(p.out) & 31) == 0, there = rho < nrows;
          const int cc0 = dual ? t * (D / 64) : 0, cc1 = dual ? cc0 + D / 64 : D / 32;
#pragma unroll 1
          for (int cc = cc0; cc < cc1; ++cc) {
            uint32_t v[32];
            if (nblk > 0) {
              tmem_ld32(o_addr + cc * 32, v);
              tmem_ld_wait();
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = 0u;
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * norm);
            if (dual && (t == 1 || both)) {
              uint32_t v1[32];
              tmem_ld32(tmem_base + lane_addr + 256 + (t ^ 1) * D + cc * 32, v1);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(fmaf(__uint_as_float(v1[i]), other, __uint_as_float(v[i])));
            }
            if (there) {
              uint32_t w[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const __nv_bfloat162 v2 = __floats2bfloat162_rn(__uint_as_float(v[i * 2]), __uint_as_float(v[i * 2 + 1]));
                w[i] = *reinterpret_cast<const uint32_t *>(&v2);
              }
              if (wide) {
                st_global_32(dst + cc * 32, w);
                st_global_32(dst + cc * 32 + 16, w + 8);
              } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) reinterpret_cast<uint4 *>(dst + cc * 32)[k] = make_uint4(w[k * 4], w[k * 4 + 1], w[k * 4 + 2], w[k * 4 + 3]);
              }
            }
          }
          tc_fence_before();
        }
        // both halves are out before either warp-group hands over a P of the next unit and so lets an accumulator be overwritten
        if (dual) {
          mbar_arrive(swap_done);
          ok = ok && __all_sync(0xffffffffu, mbar_wait(swap_done, swap_par, p.status, abort_flag, wb));
          swap_par ^= 1u;
        }
        final_ok = ok;
      }
      last_par ^= dual ? (both ? 3u : 1u) : 3u;
    }
  }

  if constexpr (RANGES) {
    // ---------------------------------------------------------------- merge of the key ranges over the cluster
    // Row slice c of a tile is merged by CTA c.  Every CTA pushes its unnormalised rows (O, m, l) into the shared memory of the slices'
    // owners, over their rings.  A lone tile has two parts a CTA, one a stream.  All threads pass the same barriers.
    const Unit x = unit_at(unit0);
    const bool dual = x.ntiles == 1;
    const int parts = dual ? 2 * splits : splits;
    constexpr uint32_t kPitch = (D + 4) * 4;
    const int rpr0 = (min(kTileRows, nrows - x.rho0) + splits - 1) / splits;
    const int rpr1 = dual ? 0 : (min(kTileRows, nrows - x.rho0 - kTileRows) + splits - 1) / splits;
    const int total = parts * (rpr0 + rpr1);              // rows that arrive here, [tile][part][slice row]
    const uint32_t part_o = ring_smem, part_m = part_o + static_cast<uint32_t>(total) * kPitch;
    tc_fence_before();
    __syncwarp();
    cluster_sync_all();                                   // nobody's ring is in use any more
    if (warp >= kManySoftmaxWarp && final_ok) {
      tc_fence_after();
      const int wg = (warp - kManySoftmaxWarp) >> 2, tile = dual ? 0 : wg, part = dual ? 2 * sp + wg : sp, row = (warp & 3) * 32 + lane;
      const int rpr = tile == 0 ? rpr0 : rpr1;
      const uint32_t o_addr = tmem_base + 256 + wg * D + (static_cast<uint32_t>((warp & 3) * 32) << 16);
      const bool mine = x.rho0 + tile * kTileRows + row < nrows;
      const int owner = mine ? row / rpr : 0, at = (tile == 0 ? 0 : parts * rpr0) + part * rpr + row - owner * rpr;
      const uint32_t dst = mapa_shared(part_o + static_cast<uint32_t>(at) * kPitch, static_cast<uint32_t>(owner));
      const uint32_t dst_m = mapa_shared(part_m + static_cast<uint32_t>(at) * 8u, static_cast<uint32_t>(owner));
#pragma unroll 1
      for (int cc = 0; cc < D / 32; ++cc) {
        uint32_t v[32];
        if (any_block) {
          tmem_ld32(o_addr + cc * 32, v);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = 0u;
        }
        if (mine) {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + (cc * 32 + k * 4) * 4), "r"(v[k * 4]), "r"(v[k * 4 + 1]),
                         "r"(v[k * 4 + 2]), "r"(v[k * 4 + 3]) : "memory");
        }
      }
      if (mine) asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(dst_m), "f"(m_ref), "f"(l_run) : "memory");
    }
    tc_fence_before();
    __syncwarp();
    cluster_sync_all();                                   // all rows have arrived; nobody touches a peer after this
    if (warp >= kManySoftmaxWarp && *abort_flag == 0) {
      constexpr int kLanes = D / 4;                       // threads a row, one float4 each
      const int st = static_cast<int>(threadIdx.x) - 32 * kManySoftmaxWarp, d4 = (st % kLanes) * 4;
      const float c = p.scale_log2;
#pragma unroll 1
      for (int k0 = 0; k0 < rpr0 + rpr1; k0 += 256 / kLanes) {       // every lane of a warp goes round as often
        const bool there = k0 + st / kLanes < rpr0 + rpr1;
        const int k = there ? k0 + st / kLanes : 0;
        const int tile = k < rpr0 ? 0 : 1, lrow = tile == 0 ? k : k - rpr0, rpr = tile == 0 ? rpr0 : rpr1;
        const int rho = x.rho0 + tile * kTileRows + sp * rpr + lrow;
        const bool live = there && rho < nrows && sp * rpr + lrow < kTileRows;
        const uint32_t at0 = static_cast<uint32_t>((tile == 0 ? 0 : parts * rpr0) + lrow);
        // a lane takes one part's maximum and sum; the weights are formed side by side and handed round (12 parts at most)
        const int l16 = st & 15;
        const float2 ml = l16 < parts ? ld_shared_f2(part_m + (at0 + l16 * rpr) * 8u) : make_float2(kNoRowMax, 0.f);
        float m_all = ml.x;
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) m_all = fmaxf(m_all, __shfl_xor_sync(0xffffffffu, m_all, d));
        float w16 = ml.y == 0.f ? 0.f : exp2f((ml.x - m_all) * c), l_all = ml.y * w16;
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) l_all += __shfl_xor_sync(0xffffffffu, l_all, d);
        w16 *= inverse_sum(l_all, l_all != 0.f || !live ? 0 : p.limits ? p.limits[static_cast<long long>(x.e) * p.r + rho / G] : p.L);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int t2 = 0; t2 < parts; ++t2) {
          const float w = __shfl_sync(0xffffffffu, w16, t2, 16);
          const float4 v = ld_shared_f4(part_o + (at0 + t2 * rpr) * kPitch + d4 * 4);
          o.x = fmaf(w, v.x, o.x); o.y = fmaf(w, v.y, o.y); o.z = fmaf(w, v.z, o.z); o.w = fmaf(w, v.w, o.w);
        }
        if (!live) continue;
        const __nv_bfloat162 h0 = __floats2bfloat162_rn(o.x, o.y), h1 = __floats2bfloat162_rn(o.z, o.w);
        *reinterpret_cast<uint2 *>(p.out + ((static_cast<long long>(x.e) * p.r + rho / G) * p.H + x.h * G + rho % G) * D + d4) =
            make_uint2(*reinterpret_cast<const uint32_t *>(&h0), *reinterpret_cast<const uint32_t *>(&h1));
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem_base, Cfg::kTmemCols);
  }
}

template <int D, bool RANGES, bool CODES>
static cudaError_t many_prepare(int dev) {
  static PerDevice prepared;
  return prepared.once(dev, [] {
    // The register split draws on what the block was launched with: refuse a build whose kernel got fewer.
    cudaFuncAttributes fa;
    const cudaError_t e = cudaFuncGetAttributes(&fa, attention_kv4_many_kernel<D, RANGES, CODES>);
    if (e != cudaSuccess) return e;
    if (fa.numRegs < kRegsLaunch) return cudaErrorInvalidConfiguration;
    return cudaFuncSetAttribute(attention_kv4_many_kernel<D, RANGES, CODES>, cudaFuncAttributeMaxDynamicSharedMemorySize, ManyCfg<D, CODES>::kSmemBytes);
  });
}

// Estimated time in microseconds of a launch (0: not a launch): see attention_kv4_plan.  A block of 128 keys takes a lone tile 1.3 and a
// pair 2.3 (1.13 and 2.0 at D = 64), decoded ones 1.05 and 1.95 (0.92 and 1.85); a unit takes 3.5 or 4 more for its own first operands and
// store (0.5 less of decoded ones), the pass that decodes its bytes at 6.3 TB/s; ranges pay for their set-up, the barriers and the rows that
// cross the cluster.  Pairs, which decode once for two tiles, win where lone tiles make another wave (1024 rows of 2 x 16 heads over 4000
// keys: 70 us against 82), lone tiles elsewhere (410 rows over 2931 keys: 35 against 56).
double attention_kv4_many_cost(long long rows, long long groups, int D, int L, int tiles, int s, bool decoded, int num_sms, const int *max_clusters) {
  const int nkv = (L + kBlockKeys - 1) / kBlockKeys, per = (nkv + s - 1) / s;
  const double units = static_cast<double>((rows + tiles * kTileRows - 1) / (tiles * kTileRows)) * groups;
  const double t_block = decoded ? (tiles == 2 ? (D == 128 ? 1.95 : 1.85) : (D == 128 ? 1.05 : 0.92)) : (tiles == 2 ? (D == 128 ? 2.3 : 2.0) : (D == 128 ? 1.3 : 1.13));
  if (s == 1) {
    const double w = units / num_sms, pass = decoded ? 3.0 + 0.8e-6 * groups * L * D : 0.0;
    return 2.5 + pass + (w <= 1.0 ? 1.0 : w < 8.0 ? ceil(w) : w) * ((tiles == 2 ? 4.0 : 3.5) - (decoded ? 0.5 : 0.0) + per * t_block);
  }
  if (per < 2 || (nkv + per - 1) / per != s || max_clusters[s] <= 0) return 0.0;             // at least two key blocks a range
  const double part = (rows < tiles * kTileRows ? rows : tiles * kTileRows) / static_cast<double>(kTileRows);
  return ceil(units / max_clusters[s]) * (7.0 + 0.8 * s + 3.0 * part + per * t_block);
}

// Resident clusters of s CTAs on the current device (0: none), for both widths: one CTA an SM.
const int *attention_kv4_max_clusters() {
  static int resident[kMaxDevices][kKv4ManyMaxRanges + 1];
  static PerDevice asked;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev >= kMaxDevices) return nullptr;
  const cudaError_t e = asked.once(dev, [dev] {
    const cudaError_t e = many_prepare<128, true, true>(dev);
    if (e != cudaSuccess) return e;
    for (int s = 1; s <= kKv4ManyMaxRanges; ++s) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(s * 64);
      cfg.blockDim = dim3(kManyThreads);
      cfg.dynamicSmemBytes = ManyCfg<128, true>::kSmemBytes;
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = s;
      attr[0].val.clusterDim.y = 1;
      attr[0].val.clusterDim.z = 1;
      cfg.attrs = attr;
      cfg.numAttrs = 1;
      int n = 0;
      if (cudaOccupancyMaxActiveClusters(&n, attention_kv4_many_kernel<128, true, true>, &cfg) != cudaSuccess) {
        cudaGetLastError();
        n = 0;
      }
      resident[dev][s] = n;
    }
    return cudaSuccess;
  });
  return e == cudaSuccess ? resident[dev] : nullptr;
}

template <int D>
static cudaError_t launch_many_d(Kv4AttnArgs a, void *workspace, int num_sms, cudaStream_t st) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const int G = a.H / a.Hkv;
  const long long rows = static_cast<long long>(a.r) * G;
  if (rows > INT_MAX - 256) return cudaErrorInvalidValue;
  const long long nqt = (rows + a.tiles_per_cta * kTileRows - 1) / (a.tiles_per_cta * kTileRows), units = nqt * a.Hkv * a.B;
  if (units * kKv4ManyMaxRanges > INT_MAX) return cudaErrorInvalidValue;
  a.units = static_cast<int>(units);
  a.div_nqt = make_fast_div(static_cast<unsigned>(nqt), units);
  a.div_h = make_fast_div(a.Hkv, units);
  a.div_g = make_fast_div(G, rows + 256);
  CUtensorMap tq = {}, tk = {}, tv = {};
  a.by_length = a.limits && a.B > 1 && a.B <= kMaxOrdered && units * a.kv_splits > num_sms;
  a.q_tma = kTileRows % G == 0;                           // else the rows of a tile are no box
  if (a.q_tma && !tmap_queries(&tq, a, kTileRows / G)) return cudaErrorInvalidValue;
  if (workspace) {                                        // decode the whole cache once, in a pass of its own
    Kv4Args x = {};
    x.k_out = static_cast<bf16 *>(workspace);
    x.v_out = x.k_out + static_cast<size_t>(a.B) * a.Hkv * a.L * D;
    x.k_codes = const_cast<uint8_t *>(a.k_codes); x.v_codes = const_cast<uint8_t *>(a.v_codes);
    x.k_scales = const_cast<uint8_t *>(a.k_scales); x.v_scales = const_cast<uint8_t *>(a.v_scales);
    x.elem_stride = a.elem_stride;
    x.B = a.B; x.H = a.Hkv; x.D = D; x.L_cap = a.L_cap; x.n = a.L;
    x.out_row = D; x.out_head = static_cast<long long>(a.L) * D; x.out_elem = x.out_head * a.Hkv;
    x.status = a.status;
    const uint64_t heads = static_cast<uint64_t>(a.B) * a.Hkv;
    if (!tmap_3d(&tk, x.k_out, D, a.L, heads, D, static_cast<uint64_t>(a.L) * D, 64, 128) ||
        !tmap_3d(&tv, x.v_out, D, a.L, heads, D, static_cast<uint64_t>(a.L) * D, 64, 128))
      return cudaErrorInvalidValue;
    e = launch_kv4_rows(false, x, st);
    if (e == cudaSuccess) e = many_prepare<D, false, false>(dev);
    if (e != cudaSuccess) return e;
    return launch_pdl(attention_kv4_many_kernel<D, false, false>, dim3(a.units < num_sms ? a.units : num_sms), dim3(kManyThreads), ManyCfg<D, false>::kSmemBytes, st, tq, tk, tv, a);
  }
  if (!tmap_codes(&tk, a.k_codes, a, kBlockKeys) || !tmap_codes(&tv, a.v_codes, a, kBlockKeys)) return cudaErrorInvalidValue;
  if (a.kv_splits <= 1) {
    e = many_prepare<D, false, true>(dev);
    if (e != cudaSuccess) return e;
    return launch_pdl(attention_kv4_many_kernel<D, false, true>, dim3(a.units < num_sms ? a.units : num_sms), dim3(kManyThreads), ManyCfg<D, true>::kSmemBytes, st, tq, tk, tv, a);
  }
  e = many_prepare<D, true, true>(dev);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.units * a.kv_splits);
  cfg.blockDim = dim3(kManyThreads);
  cfg.dynamicSmemBytes = ManyCfg<D, true>::kSmemBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = a.kv_splits;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1] = pdl_attribute();
  cfg.attrs = attr;
  cfg.numAttrs = one_predecessor(st) ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, attention_kv4_many_kernel<D, true, true>, tq, tk, tv, a);
}

cudaError_t launch_attention_kv4_many(const Kv4AttnArgs &a, void *workspace, int num_sms, cudaStream_t st) {
  return a.D == 64 ? launch_many_d<64>(a, workspace, num_sms, st) : launch_many_d<128>(a, workspace, num_sms, st);
}

}  // namespace fvar
