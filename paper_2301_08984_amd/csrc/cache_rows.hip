// Rows into the paged cache and out of it (include/ss_cache.h): quantised as they are written, and read back.
//
// A row of D values is D / 8 lanes with 16 bytes each, so a wavefront takes 4 rows (D = 128) or 8, of one token (of
// its K rows, one a head, and V rows behind them).  The largest magnitude goes round the row's lanes, every lane converts its
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

// Where a token lies in the cache.
struct Place {
  int page;  // -1: none
  int64_t pos;
};
// The token's sequence (b = -1: none) and place: the offsets and starts of 64 sequences are asked for at once, so that the table's
// entry, which they name, is the second load in a row and not the third.
__device__ __forceinline__ int place_of(const CacheRowsP& p, int t, Place& at) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < p.c.n_seq; b0 += 64) {
    const int i = min(b0 + lane, p.c.n_seq - 1);
    const int from = max(p.cu[i], 0), to = p.cu[i + 1], start = p.start ? p.start[i] : 0;
    const uint64_t hit = __builtin_amdgcn_ballot_w64(b0 + lane < p.c.n_seq && from <= t && t < to);
    if (!hit) continue;
    const int l = 63 - __builtin_clzll(hit);
    at.pos = (int64_t)t - __builtin_amdgcn_readlane(from, l) + __builtin_amdgcn_readlane(start, l);
    at.page = cache_page(p.c.table, p.c.n_pages, p.c.shift, p.c.max_pages, b0 + l, at.pos);
    return b0 + l;
  }
  return -1;
}
// A wavefront's part of the launch: every p.groups-th ROWS of a token's 2 HK rows, from row r0 on.
template <int ROWS>
__device__ __forceinline__ bool rows_of(const CacheRowsP& p, int& t, int& r0) {
  const int u = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  t = u / p.groups;
  r0 = (u - t * p.groups) * ROWS;
  return t < p.T;
}

template <int FMT, int D>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheRowsP p) {
  constexpr int LANES = D / 8, ROWS = 64 / LANES;
  const int lane = threadIdx.x & 63, c = lane % LANES, HK = p.c.HK;
  int t, r0;
  if (!rows_of<ROWS>(p, t, r0)) return;
  auto load = [&](int r) {
    const bool v = r >= HK;
    return r < 2 * HK ? *(const u32x4*)((const uint16_t*)(v ? p.V : p.K) + t * p.st + (v ? r - HK : r) * p.sh + 8 * c) : u32x4{0, 0, 0, 0};
  };
  int r = r0 + lane / LANES;
  u32x4 next = load(r);
  Place at;
  if (place_of(p, t, at) < 0 || at.page < 0) return;
  for (; r < 2 * HK; r += p.groups * ROWS) {  // (whole rows of lanes leave)
    const u32x4 x = next;
    next = load(r + p.groups * ROWS);
    const bool v = r >= HK;
    const int h = v ? r - HK : r;
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
  const int lane = threadIdx.x & 63, c = lane % LANES, HK = p.c.HK;
  int t, r0;
  if (!rows_of<ROWS>(p, t, r0)) return;
  Place at;
  if (place_of(p, t, at) < 0) return;
#pragma unroll 2
  for (int r = r0 + lane / LANES; r < 2 * HK; r += p.groups * ROWS) {
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

// Wavefronts of a token, and work-groups of the launch: one wavefront for four (eight) rows while those are few, one for a token's rows
// where there are tokens enough.  One | several: 31200 tokens of 8 heads read back 32.0 | 36.9 us (6.05 TB/s with reads and writes together), one step's 64
// tokens written 7.9 | 5.1.
int cut(CacheRowsP& p) {
  const int rows = 512 / p.c.D;
  p.groups = p.T < 4096 ? (2 * p.c.HK + rows - 1) / rows : 1;
  return (int)(((int64_t)p.T * p.groups + 3) / 4);
}

}  // namespace

hipError_t launch_cache_write(const CacheRowsP& q, hipStream_t st) {
  CacheRowsP p = q;
  const int blocks = cut(p);
  return with_format(p.c, [&](auto fmt, auto d) { cache_write_kernel<fmt(), d()><<<blocks, 256, 0, st>>>(p); });
}
hipError_t launch_cache_read(const CacheRowsP& q, hipStream_t st) {
  CacheRowsP p = q;
  const int blocks = cut(p);
  return with_format(p.c, [&](auto fmt, auto d) { cache_read_kernel<fmt(), d()><<<blocks, 256, 0, st>>>(p); });
}

}  // namespace ssa
