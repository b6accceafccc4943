// Attention of new tokens over the paged cache, plainly: a wavefront per token and query head, fp32 throughout.
#include "cache.h"
#include "mfma_common.h"

namespace ssa {
namespace {

__device__ inline float wave_sum(float x) {
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ inline float code(const void* c, const float* s, int format, int64_t row, int D, int d) {
  if (d >= D) return 0.f;
  if (format == 0) return bf2f(((const uint16_t*)c)[row * D + d]);
  const uint8_t u = ((const uint8_t*)c)[row * D + d];
  return s[row] * (format == 1 ? __builtin_amdgcn_cvt_f32_fp8((int)u, 0) : (float)(int8_t)u);
}

__global__ __launch_bounds__(64) void cache_attn_kernel(CacheAttnP p) {
  const int t = blockIdx.x, h = blockIdx.y, hk = h / p.G, lane = threadIdx.x, D = p.c.D;
  const int b = packed_owner(p.cu, p.c.n_seq, t);
  if (b < 0) return;
  const int i = t - p.cu[b], n = min(p.cu[b + 1] - p.cu[b], p.max_new);
  if (i >= n) return;
  const int before = max(p.lens[b] - max(p.cu[b + 1] - p.cu[b], 0), 0);
  const int len = (int)min((int64_t)p.lens[b], (int64_t)p.c.max_pages << p.c.shift);
  const uint64_t mask = p.tree ? p.tree[t] : ~((~(uint64_t)1) << i);
  const uint16_t* q = (const uint16_t*)p.Q + t * p.q_st + h * p.q_sh;
  const float q0 = lane < D ? bf2f(q[lane]) : 0.f, q1 = lane + 64 < D ? bf2f(q[lane + 64]) : 0.f;
  float m = -INFINITY, l = 0.f, a0 = 0.f, a1 = 0.f;
  for (int j = 0; j < len; ++j) {
    if (j >= before && (j - before > 63 || !(mask >> (j - before) & 1))) continue;
    const int page = cache_page(p.c.table, p.c.n_pages, p.c.shift, p.c.max_pages, b, j);
    if (page < 0) continue;
    const int64_t row = cache_row(page, p.c.shift, p.c.HK, hk, j);
    const float x = p.scale * wave_sum(q0 * code(p.c.kc, p.c.ks, p.c.format, row, D, lane) + q1 * code(p.c.kc, p.c.ks, p.c.format, row, D, lane + 64));
    const float mn = fmaxf(m, x), alpha = expf(m - mn), e = expf(x - mn);
    m = mn;
    l = l * alpha + e;
    a0 = a0 * alpha + e * code(p.c.vc, p.c.vs, p.c.format, row, D, lane);
    a1 = a1 * alpha + e * code(p.c.vc, p.c.vs, p.c.format, row, D, lane + 64);
  }
  const float r = l > 0.f ? 1.f / l : 0.f;
  uint16_t* y = (uint16_t*)p.Y + t * p.y_st + h * p.y_sh;
  if (lane < D) y[lane] = f2bf(a0 * r);
  if (lane + 64 < D) y[lane + 64] = f2bf(a1 * r);
  if (lane == 0 && p.lse) p.lse[(int64_t)h * p.T + t] = l > 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace

size_t cache_attn_bytes(const CacheAttnP&) { return 0; }

hipError_t launch_cache_attn(const CacheAttnP& p, hipStream_t st) {
  cache_attn_kernel<<<dim3(p.T, p.H), 64, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace ssa
