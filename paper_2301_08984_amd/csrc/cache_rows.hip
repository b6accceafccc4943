// Rows into the paged cache and out of it (include/ss_cache.h): quantised as they are written, and read back.
//
// A row of D values is D / 8 lanes with 16 bytes each, so a wavefront takes 4 rows (D = 128) or 8 at a time, of one token:
// the K rows of its heads, then the V rows.  The largest magnitude goes round the row's lanes, every lane converts its
// own eight values.  Bound by memory: 4 D bytes in and 2 D + 8 out for a token and head, or the reverse.
#include "cache.h"
#include "mfma_common.h"

namespace ssa {
namespace {

__device__ inline float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
// the smallest power of two s >= 2^-126 with most <= 448 s = 1.75 2^8 s
__device__ inline float fp8_scale(float most) {
  const uint32_t u = __float_as_uint(most);
  return exp2_int(max((int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), -126));
}

// where a token's rows lie in the cache: its sequence's page, and the place in the pages' rows of head 0
struct Place {
  int page;  // -1: none
  int64_t pos;
};
__device__ inline Place place_of(const CacheRowsP& p, int t, int b) {
  Place a;
  a.pos = (int64_t)t - p.cu[b] + (p.start ? p.start[b] : 0);
  a.page = cache_page(p.c.table, p.c.n_pages, p.c.shift, p.c.max_pages, b, a.pos);
  return a;
}

template <int FMT, int D>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheRowsP p) {
  constexpr int LANES = D / 8, ROWS = 64 / LANES;
  const int lane = threadIdx.x & 63, c = lane % LANES;
  const int t = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (t >= p.T) return;
  const int b = packed_owner(p.cu, p.c.n_seq, t);
  if (b < 0) return;
  const Place at = place_of(p, t, b);
  if (at.page < 0) return;
  const int HK = p.c.HK;
  for (int r0 = 0; r0 < 2 * HK; r0 += ROWS) {
    const int r = r0 + lane / LANES;
    if (r >= 2 * HK) break;  // (whole rows of lanes leave)
    const bool v = r >= HK;
    const int h = v ? r - HK : r;
    const u32x4 x = *(const u32x4*)((const uint16_t*)(v ? p.V : p.K) + t * p.st + h * p.sh + 8 * c);
    const int64_t row = cache_row(at.page, p.c.shift, HK, h, at.pos);
    if (FMT == 0) {
      *(u32x4*)((uint16_t*)(v ? p.c.vc : p.c.kc) + row * D + 8 * c) = x;
      continue;
    }
    // the largest magnitude as an integer: bf16 without its sign is in order, with infinity and NaN on top
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) most = max(most, max(x[e] & 0x7fffu, x[e] >> 16 & 0x7fffu));
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
    const float amax = __uint_as_float(most << 16);
    const bool finite = most < 0x7f80u;
    float scale = FMT == 1 ? fp8_scale(amax) : fmaxf(amax / 127.f, 0x1p-126f);
    if (most == 0 || !finite) scale = 1.f;
    float f[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = __uint_as_float(x[e] << 16) / scale;
      f[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u) / scale;
    }
    uint32_t w[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      if (FMT == 1) {
        int o = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * g], f[4 * g + 1], 0, false);
        w[g] = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * g + 2], f[4 * g + 3], o, true);
      } else {
        w[g] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[g] |= ((uint32_t)(int)rintf(f[4 * g + e]) & 0xffu) << (8 * e);
      }
      if (!finite) w[g] = 0;
    }
    *(uint2*)((uint8_t*)(v ? p.c.vc : p.c.kc) + row * D + 8 * c) = uint2{w[0], w[1]};
    if (c == 0) (v ? p.c.vs : p.c.ks)[row] = finite ? scale : __uint_as_float(0x7fc00000u);
  }
}

template <int FMT, int D>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheRowsP p) {
  constexpr int LANES = D / 8, ROWS = 64 / LANES;
  const int lane = threadIdx.x & 63, c = lane % LANES;
  const int t = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (t >= p.T) return;
  const int b = packed_owner(p.cu, p.c.n_seq, t);
  if (b < 0) return;
  const Place at = place_of(p, t, b);
  const int HK = p.c.HK;
  for (int r0 = 0; r0 < 2 * HK; r0 += ROWS) {
    const int r = r0 + lane / LANES;
    if (r >= 2 * HK) break;
    const bool v = r >= HK;
    const int h = v ? r - HK : r;
    u32x4 x = {0, 0, 0, 0};
    if (at.page >= 0) {
      const int64_t row = cache_row(at.page, p.c.shift, HK, h, at.pos);
      if (FMT == 0) {
        x = *(const u32x4*)((const uint16_t*)(v ? p.c.vc : p.c.kc) + row * D + 8 * c);
      } else {
        const uint2 w = *(const uint2*)((const uint8_t*)(v ? p.c.vc : p.c.kc) + row * D + 8 * c);
        const float scale = (v ? p.c.vs : p.c.ks)[row];
        float f[8];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const uint32_t u = g ? w.y : w.x;
          if (FMT == 1) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, true);
            f[4 * g] = lo[0]; f[4 * g + 1] = lo[1]; f[4 * g + 2] = hi[0]; f[4 * g + 3] = hi[1];
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) f[4 * g + e] = (float)(int8_t)(u >> (8 * e));
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = pack2_bf16(f[2 * e] * scale, f[2 * e + 1] * scale);
      }
    }
    *(u32x4*)((uint16_t*)(v ? p.V : p.K) + t * p.st + h * p.sh + 8 * c) = x;
  }
}

template <typename F>
hipError_t with_format(const CacheP& c, F&& f) {
  auto by_size = [&](auto fmt) {
    if (c.D == 64) f(fmt, std::integral_constant<int, 64>{});
    else f(fmt, std::integral_constant<int, 128>{});
  };
  if (c.format == 0) by_size(std::integral_constant<int, 0>{});
  else if (c.format == 1) by_size(std::integral_constant<int, 1>{});
  else by_size(std::integral_constant<int, 2>{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const CacheRowsP& p, hipStream_t st) {
  return with_format(p.c, [&](auto fmt, auto d) { cache_write_kernel<fmt(), d()><<<(p.T + 3) / 4, 256, 0, st>>>(p); });
}
hipError_t launch_cache_read(const CacheRowsP& p, hipStream_t st) {
  return with_format(p.c, [&](auto fmt, auto d) { cache_read_kernel<fmt(), d()><<<(p.T + 3) / 4, 256, 0, st>>>(p); });
}

}  // namespace ssa
