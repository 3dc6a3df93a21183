// Attention of query rows over a cache in 4 bits (format and operator: include/fvar.h).
//
// A warp takes one query row of one head and walks its keys: four (or two) values a lane, one dot product at a time, a running
// maximum and sum.  fp32 throughout.
#include <math.h>

#include "kv4.cuh"
#include "ptx.cuh"

namespace fvar {

template <int D>
__global__ void __launch_bounds__(256) attention_kv4_rows_kernel(const __grid_constant__ Kv4AttnArgs p) {
  constexpr int V = D / 32;                                          // values a lane
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long unit = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  if (unit >= static_cast<long long>(p.B) * p.r * p.H) return;
  const int h = static_cast<int>(unit % p.H);
  const long long bi = unit / p.H;
  const int b = static_cast<int>(bi / p.r), kv = h / (p.H / p.Hkv);
  const int n = p.limits ? min(max(p.limits[bi], 0), p.L) : p.L;
  float q[V], o[V], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    q[k] = __bfloat162float(p.q[bi * p.ldq + h * D + lane * V + k]);
    o[k] = 0.f;
  }
  const long long row0 = b * p.elem_stride + static_cast<long long>(kv) * p.L_cap;
  const int first = (lane * V) % 8 / 2;                              // which pair of its word the lane's values begin with
  auto decode = [&](const uint8_t *codes, const uint8_t *scales, long long row, float (&x)[V]) {
    const uint32_t w = reinterpret_cast<const uint32_t *>(codes)[row * (D / 8) + lane * V / 8];
    const uint32_t s2 = kv4_scale2(scales[row * (D / kKv4Group) + lane * V / kKv4Group]);
#pragma unroll
    for (int k = 0; k < V / 2; ++k) {
      const uint32_t pr = kv4_pair(w >> (4 * (first + k)), s2, kv4_offset2(s2));
      x[2 * k] = __uint_as_float(pr << 16);
      x[2 * k + 1] = __uint_as_float(pr & 0xFFFF0000u);
    }
  };
  for (int j = 0; j < n; ++j) {
    float x[V], y[V], s = 0.f;
    decode(p.k_codes, p.k_scales, row0 + j, x);
    decode(p.v_codes, p.v_scales, row0 + j, y);
#pragma unroll
    for (int k = 0; k < V; ++k) s = fmaf(q[k], x[k], s);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    s *= p.scale_log2;
    const float m2 = fmaxf(m, s), a = exp2f(m - m2), e = exp2f(s - m2);
    l = fmaf(l, a, e);
#pragma unroll
    for (int k = 0; k < V; ++k) o[k] = fmaf(o[k], a, e * y[k]);
    m = m2;
  }
  const float inv = n > 0 ? 1.0f / l : 0.f;
#pragma unroll
  for (int k = 0; k < V; ++k) p.out[(bi * p.H + h) * D + lane * V + k] = __float2bfloat16_rn(o[k] * inv);
}

cudaError_t launch_attention_kv4(const Kv4AttnArgs &a, int, cudaStream_t st) {
  const long long units = static_cast<long long>(a.B) * a.r * a.H, grid = (units + 7) / 8;
  if (grid > 0x7FFFFFFF) return cudaErrorInvalidValue;
  const dim3 g(static_cast<unsigned>(grid));
  return a.D == 64 ? launch_pdl(attention_kv4_rows_kernel<64>, g, dim3(256), 0, st, a) : launch_pdl(attention_kv4_rows_kernel<128>, g, dim3(256), 0, st, a);
}

}  // namespace fvar
