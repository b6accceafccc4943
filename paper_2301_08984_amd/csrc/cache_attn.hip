// Attention of new tokens over the paged cache (include/ss_cache.h).
//
// Bound by reading the cache: 4 D bytes (2 D + 8 in 8 bits) a key and head for 4 D flops a row, so a key is read once for all rows that see
// it, the new tokens of a sequence times the G query heads of a key head, here up to 32 (more: cache_attn_rows.hip), and goes from memory into
// registers: nothing passes through LDS until the end.  The keys of all sequences are dealt out to the work-groups in equal pieces (cache_cut.h);
// the four wavefronts of a work-group take every fourth block of 32 keys of a piece each, with a running maximum and sum, and are
// joined through LDS.  A sequence within a piece is finished there; the parts of the others are joined by a second launch.
//
// Scores: S^T = K Q^T, a lane holding 16 (D = 128: of the row's 128) columns of its key, as they come; 8-bit codes become bf16
// exactly, and the key's scale multiplies the fp32 score.  O^T += V^T P^T: a lane holds D / 32 neighbouring columns of eight keys, which byte permutes turn
// into operands (eight keys of a column), so that V needs no transposed copy in LDS; the value's scale goes into P, which is
// rounded to bf16 as the matrix instructions take it.  Maxima, sums and O are fp32.
#include "cache_cut.h"

namespace ssa {
namespace {

// two bf16 of one register's 16-bit halves
__device__ __forceinline__ uint32_t lo_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t hi_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
template <int FMT, int D>
struct CacheTile {
  static constexpr int E = FMT == BF ? 2 : 1, ROW_B = D * E, KS = D / 16, NB = D / 32;
  static constexpr int KL = ROW_B / 32;      // 16-byte loads of a lane for K
  static constexpr int VW = NB * E;          // bytes of a lane and key of V: 2, 4 or 8
  static constexpr int VR = VW == 8 ? 2 : 1;  // registers
};

// One run (or part of one) of a piece: keys begin .. end of it; `all`: the whole of it.
template <int FMT, int D>
__device__ __forceinline__ void cache_attn_run(const CacheAttnP& p, char* smem, const Run& f, int hk, int begin, int end, bool all, int slot) {
  using T = CacheTile<FMT, D>;
  constexpr int KS = T::KS, NB = T::NB, ROW_B = T::ROW_B;
  int lane = threadIdx.x & 63;
  asm("" : "+v"(lane));  // (what follows from it is formed anew for every run: kept over the loop, it spills)
  const int r = lane & 31, hl = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const CacheSeq s = f.s;
  const int rows = s.n * p.G, shift = p.c.shift;  // up to 32 rows

  // pages of the part: a lane an entry, 64 of them and the 64 behind them
  const int32_t* line = p.c.table + (int64_t)f.b * p.c.max_pages;
  const int last_entry = (end - 1) >> shift;
  auto entries = [&](int from) {
    const int e = from + lane;
    return e <= last_entry ? line[e] : -1;  // (looked at when it is used, so that nothing waits for it here)
  };
  int window = (begin + 32 * w) >> shift;
  int win = entries(window), win_next = entries(window + 64);

  bf16x8 qf[KS];
  uint64_t bits;
  {
    const int R = min(r, rows - 1), tok = R / p.G, h = hk * p.G + R - tok * p.G;
    const uint16_t* Q = (const uint16_t*)p.Q + (int64_t)(s.q0 + tok) * p.q_st + (int64_t)h * p.q_sh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      // the columns of K's operands: as they lie in the 16 bytes that a lane loads
      const int col = FMT == BF ? 16 * ks + 8 * hl : 32 * (ks >> 1) + 16 * hl + 8 * (ks & 1);
      union { u32x4 u; bf16x8 v; } x;
      x.u = *(const u32x4*)(Q + col);
      const uint32_t flip = p.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
      for (int e = 0; e < 4; ++e) x.u[e] ^= flip;
      qf[ks] = x.v;
    }
    bits = p.tree ? p.tree[s.q0 + tok] : ~(~(uint64_t)1 << tok);
  }
  // (a factor of 0 would make NaN of a masked score)
  const float c1 = fmaxf(fabsf(p.scale) * LOG2E, 0x1p-120f);

  u32x4 kx[T::KL], vs4[4], ks4[4];
  uint32_t vx[16][T::VR];
  uint32_t live = 0, live_next = 0;  // keys of the block that are there
  const uint32_t k_lane = 16u * hl, v_lane = (uint32_t)(4 * hl) * ROW_B + (uint32_t)r * T::VW;
  int64_t row_of[4];  // rows of the pool: of keys 8 g ..
  auto locate = [&](int k0) {  // of the block that starts at k0
    if (((k0 + 24) >> shift) - window >= 64) {
      window += 64;
      win = win_next;
      win_next = entries(window + 64);
    }
    uint32_t there = end - k0 >= 32 ? ~0u : (1u << (end - k0)) - 1u;
    int64_t rk = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int pos = k0 + 8 * g, entry = __builtin_amdgcn_readlane(win, (pos >> shift) - window);
      const bool is = (uint32_t)entry < (uint32_t)p.c.n_pages;
      if (!is) there &= ~(0xffu << (8 * g));
      row_of[g] = cache_row(is ? entry : 0, shift, p.c.HK, hk, pos);
      if (r >> 3 == g) rk = row_of[g];
    }
    live_next = there;
    const char* K = (const char*)p.c.kc + (rk + (r & 7)) * ROW_B + k_lane;
#pragma unroll
    for (int j = 0; j < T::KL; ++j) kx[j] = *(const u32x4*)(K + 32 * j);
    if (FMT != BF) {
#pragma unroll
      for (int g = 0; g < 4; ++g) ks4[g] = *(const u32x4*)((const char*)(p.c.ks + row_of[g]) + 16 * hl);
    }
  };
  auto load_v = [&]() {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const char* V = (const char*)p.c.vc + row_of[g] * ROW_B;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const char* at = V + v_lane + i * ROW_B;
        if (T::VW == 8) {
          const uint2 x = *(const uint2*)at;
          vx[4 * g + i][0] = x.x;
          vx[4 * g + i][T::VR - 1] = x.y;
        } else if (T::VW == 4) {
          vx[4 * g + i][0] = *(const uint32_t*)at;
        } else {
          vx[4 * g + i][0] = *(const uint16_t*)at;
        }
      }
      if (FMT != BF) vs4[g] = *(const u32x4*)((const char*)(p.c.vs + row_of[g]) + 16 * hl);
    }
  };

  f32x16 acc[NB];
  float m = -1e30f, l = 0.f;
#pragma unroll
  for (int e = 0; e < NB; ++e)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[e][v] = 0.f;
  int k0 = begin + 32 * w;
  bool more = k0 < end;
  if (more) {
    locate(k0);
    load_v();
  }
  while (more) {  // (positions reach 2^31 - 9: none behind the end is formed)
    live = live_next;
    f32x16 sa;
#pragma unroll
      for (int v = 0; v < 16; ++v) sa[v] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      union { u32x4 u; bf16x8 v; } k;
      if (FMT == BF) {
        k.u = kx[ks % T::KL];
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t x = kx[ks >> 1][2 * (ks & 1) + h];
          k.u[2 * h] = two_codes<FMT, false>(x);
          k.u[2 * h + 1] = two_codes<FMT, true>(x);
        }
      }
      sa = mfma(k.v, qf[ks], sa);
    }
    float kc[16];  // what makes a score of a product, in base-2 units
#pragma unroll
    for (int v = 0; v < 16; ++v) kc[v] = FMT == BF ? c1 : c1 * __uint_as_float(ks4[v >> 2][v & 3]);
    more = end - k0 > 128;
    // all keys are there and none is a new token: nothing to mask
    const bool plain = live == ~0u && s.before - k0 >= 32;
    if (more) locate(k0 + 128);  // K of the next block starts on its way
    bf16x8 pf[2];
    {
      uint32_t seen = ~0u;  // keys of the block that this lane's row sees, from the half-wave's first on
#pragma unroll
      for (int v = 0; v < 16; ++v) sa[v] *= kc[v];
      if (!plain) {
        const int nb = s.before - k0;
        const uint32_t old = nb >= 32 ? ~0u : nb > 0 ? (1u << nb) - 1u : 0u;
        const uint32_t fresh = nb >= 32 ? 0u : nb >= 0 ? (uint32_t)(bits << nb) : nb > -64 ? (uint32_t)(bits >> -nb) : 0u;
        seen = (live & (old | fresh)) >> (4 * hl);
#pragma unroll
        for (int v = 0; v < 16; ++v) sa[v] = seen >> (8 * (v >> 2) + (v & 3)) & 1u ? sa[v] : -INFINITY;
      }
      float rmax = -INFINITY;
#pragma unroll
      for (int v = 0; v < 16; ++v) rmax = fmaxf(rmax, sa[v]);
      rmax = half_max(rmax);
      // the maximum is raised when exceeded by more than 2^8: probabilities stay below that
      if (__builtin_amdgcn_ballot_w64(rmax > m + 8.f) != 0) {
        const float mn = fmaxf(m, rmax), alpha = fast_exp2(m - mn);
        m = mn;
        l *= alpha;
#pragma unroll
        for (int e = 0; e < NB; ++e)
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[e][v] *= alpha;
      }
      float pr[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) pr[v] = fast_exp2(sa[v] - m);
      l += sum16(pr);
      if (FMT != BF) {
#pragma unroll
        for (int v = 0; v < 16; ++v) pr[v] *= __uint_as_float(vs4[v >> 2][v & 3]);
      }
      if (!plain) {  // (a slot where nothing lies may hold any scale)
#pragma unroll
        for (int v = 0; v < 16; ++v) pr[v] = seen >> (8 * (v >> 2) + (v & 3)) & 1u ? pr[v] : 0.f;
      }
      pf[0] = pack8(&pr[0]);
      pf[1] = pack8(&pr[8]);
    }
    if (live != ~0u) {  // ... and any code
#pragma unroll
      for (int v = 0; v < 16; ++v)
#pragma unroll
        for (int x = 0; x < T::VR; ++x) vx[v][x] = live >> (8 * (v >> 2) + (v & 3) + 4 * hl) & 1u ? vx[v][x] : 0u;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      u32x4 vf[NB];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint32_t(&a)[T::VR] = vx[8 * t + 2 * c], (&b)[T::VR] = vx[8 * t + 2 * c + 1];
        if (FMT == BF) {
#pragma unroll
          for (int x = 0; x < T::VR; ++x) {
            vf[2 * x][c] = lo_halves(a[x], b[x]);
            vf[2 * x + 1][c] = hi_halves(a[x], b[x]);
          }
        } else {
          const uint32_t x = __builtin_amdgcn_perm(b[0], a[0], 0x05010400u);  // bytes a0 b0 a1 b1
          vf[0][c] = two_codes<FMT, false>(x);
          vf[1][c] = two_codes<FMT, true>(x);
          if (NB == 4) {
            const uint32_t y = __builtin_amdgcn_perm(b[0], a[0], 0x07030602u);
            vf[NB - 2][c] = two_codes<FMT, false>(y);
            vf[NB - 1][c] = two_codes<FMT, true>(y);
          }
        }
      }
#pragma unroll
      for (int e = 0; e < NB; ++e) {
        union { u32x4 u; bf16x8 v; } a;
        a.u = vf[e];
        acc[e] = mfma(a.v, pf[t], acc[e]);
      }
    }
    if (more) {
      load_v();
      k0 += 128;
    }
  }

  // The wavefronts' parts: maxima and sums first, then O at the common maximum, quarter by quarter of the columns.  acc[e][v] is column
  // NB (8 (v / 4) + 4 hl + v % 4) + e: wavefront w adds up registers 4 w .. 4 w + 3, 4 NB neighbouring columns of each row.
  float* ml = (float*)smem;               // [wavefront][maximum, sum][32]
  float4* part = (float4*)(smem + 1024);  // [wavefront][e][quarter][lane]
  l = half_sum(l);
  __syncthreads();
  if (hl == 0) {
    ml[64 * w + r] = m;
    ml[64 * w + 32 + r] = l;
  }
  __syncthreads();
  float mg = -1e30f, sum = 0.f;
#pragma unroll
  for (int x = 0; x < 4; ++x) mg = fmaxf(mg, ml[64 * x + r]);
#pragma unroll
  for (int x = 0; x < 4; ++x) sum = fmaf(fast_exp2(ml[64 * x + r] - mg), ml[64 * x + 32 + r], sum);
  const float mine = fast_exp2(m - mg);
#pragma unroll
  for (int e = 0; e < NB; ++e)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      part[((w * NB + e) * 4 + g) * 64 + lane] = make_float4(acc[e][4 * g] * mine, acc[e][4 * g + 1] * mine, acc[e][4 * g + 2] * mine, acc[e][4 * g + 3] * mine);
  __syncthreads();
  float o[4 * NB];
#pragma unroll
  for (int e = 0; e < NB; ++e) {
    float4 x = part[((0 * NB + e) * 4 + w) * 64 + lane];
#pragma unroll
    for (int y = 1; y < 4; ++y) {
      const float4 z = part[((y * NB + e) * 4 + w) * 64 + lane];
      x.x += z.x; x.y += z.y; x.z += z.z; x.w += z.w;
    }
    o[e] = x.x; o[NB + e] = x.y; o[2 * NB + e] = x.z; o[3 * NB + e] = x.w;
  }
  const int R = r, col = NB * (8 * w + 4 * hl);
  if (R >= rows) return;
  if (all) {
    const int tok = R / p.G, h = hk * p.G + R - tok * p.G;
    const float inv = sum > 0.f ? 1.f / sum : sum;  // no key: 0; NaN stays
    uint16_t* y = (uint16_t*)p.Y + (int64_t)(s.q0 + tok) * p.y_st + (int64_t)h * p.y_sh + col;
#pragma unroll
    for (int x = 0; x < 4 * NB; x += 8)
      *(u32x4*)(y + x) = u32x4{pack2_bf16(o[x] * inv, o[x + 1] * inv), pack2_bf16(o[x + 2] * inv, o[x + 3] * inv),
                               pack2_bf16(o[x + 4] * inv, o[x + 5] * inv), pack2_bf16(o[x + 6] * inv, o[x + 7] * inv)};
    if (p.lse && w == 0 && hl == 0) p.lse[(int64_t)h * p.T + s.q0 + tok] = sum == 0.f ? -INFINITY : (mg + log2f(sum)) * LN2;
  } else {
    const int64_t at = part_row(p, slot, hk, R);
    float* y = (float*)p.ws + at * D + col;
#pragma unroll
    for (int x = 0; x < 4 * NB; x += 4) *(float4*)(y + x) = make_float4(o[x], o[x + 1], o[x + 2], o[x + 3]);
    if (w == 0 && hl == 0) *(float2*)((float*)p.ws + p.ml_at + 2 * at) = make_float2(mg, sum);
  }
}

template <int FMT, int D>
__global__ __launch_bounds__(256, 2) void cache_attn_kernel(CacheAttnP p) {
  __shared__ __attribute__((aligned(1024))) char smem[1024 + 4 * 32 * D * 4];
  const int piece = blockIdx.x / p.c.HK, hk = blockIdx.x - piece * p.c.HK;
  const Cut cut(p);
  for (int u = piece * cut.each, stop = min(u + cut.each, cut.total); u < stop;) {
    const Run f = cut.find(u);
    const int take = min(f.units - f.at, stop - u);
    const CacheSpan keys = cache_span(f.at, take, f.units, 7, f.s.len);
    u += take;
    cache_attn_run<FMT, D>(p, smem, f, hk, keys.begin, keys.end, take == f.units, part_slot(piece, cut.each, f.first));
  }
}

// Rows of sequences in more than one part: W wavefronts per token and head.  D / 4 lanes take a part's columns, each of 64 W / (D / 4) groups of lanes
// every so many parts, four at a time on their way, with a running maximum; then the groups are joined, in order.  Bound by
// the way of a few loads that follow each other (offsets, then the parts).
template <int D, int W>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnP p) {
  constexpr int LANES = D / 4, GROUPS = 64 / LANES, STRIDE = W * GROUPS;
  const int lane = threadIdx.x & 63, c = lane % LANES, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int unit = W == 4 ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave, t = unit / p.H, h = unit - t * p.H;
  if (t >= p.T) return;
  const Cut cut(p);
  const Run f = cut.owner(t);
  if (f.b < 0) return;
  const int hk = h / p.G, R = (t - f.s.q0) * p.G + h - hk * p.G, group = Cut::many(p, f.s.n) ? R >> 7 : 0;
  const int begin = f.first + group * f.units, piece = begin / cut.each, parts = (begin + f.units - 1) / cut.each - piece + 1;
  if (parts < 2) return;
  const float* ws = (const float*)p.ws;
  const int64_t first = part_row(p, part_slot(piece, cut.each, begin), hk, R - 128 * group);
  const int64_t second = part_row(p, part_slot(piece + 1, cut.each, begin), hk, R - 128 * group), step = part_row(p, 2, 0, 0);  // the first run of every piece to come
  float m = -1e30f, sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int x0 = (W == 4 ? wave * GROUPS : 0) + lane / LANES; x0 < parts; x0 += 4 * STRIDE) {
    float4 o[4];
    float2 s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = min(x0 + i * STRIDE, parts - 1);
      const int64_t at = x ? second + (x - 1) * step : first;
      s[i] = *(const float2*)(ws + p.ml_at + 2 * at);
      o[i] = *(const float4*)(ws + at * D + 4 * c);
    }
    float mn = m;
#pragma unroll
    for (int i = 0; i < 4; ++i) mn = fmaxf(mn, s[i].x);
    const float old = fast_exp2(m - mn);
    m = mn;
    sum *= old;
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] *= old;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (x0 + i * STRIDE >= parts) break;
      const float a = fast_exp2(s[i].x - m);
      sum = fmaf(a, s[i].y, sum);
      acc[0] = fmaf(a, o[i].x, acc[0]);
      acc[1] = fmaf(a, o[i].y, acc[1]);
      acc[2] = fmaf(a, o[i].z, acc[2]);
      acc[3] = fmaf(a, o[i].w, acc[3]);
    }
  }
  auto join = [&](float m1, float sum1, const float (&acc1)[4]) {
    const float mn = fmaxf(m, m1), a0 = fast_exp2(m - mn), a1 = fast_exp2(m1 - mn);
    m = mn;
    sum = fmaf(a1, sum1, a0 * sum);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = fmaf(a1, acc1[j], a0 * acc[j]);
  };
#pragma unroll
  for (int o = LANES; o < 64; o <<= 1) {
    float other[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) other[j] = __shfl_down(acc[j], o);  // (the first group's lanes are what counts)
    join(__shfl_down(m, o), __shfl_down(sum, o), other);
  }
  if (W == 4) {
    __shared__ float4 parts_of_waves[4][64];
    __shared__ float2 ml_of_waves[4];
    parts_of_waves[wave][lane] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    if (lane == 0) ml_of_waves[wave] = make_float2(m, sum);
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int x = 1; x < 4; ++x) {
      const float4 y = parts_of_waves[x][lane];
      const float other[4] = {y.x, y.y, y.z, y.w};
      join(ml_of_waves[x].x, ml_of_waves[x].y, other);
    }
  }
  if (lane >= LANES) return;
  const float inv = sum > 0.f ? 1.f / sum : sum;
  *(uint2*)((uint16_t*)p.Y + (int64_t)t * p.y_st + (int64_t)h * p.y_sh + 4 * c) = pack4_bf16(acc[0], acc[1], acc[2], acc[3], inv);
  if (p.lse && lane == 0) p.lse[(int64_t)h * p.T + t] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * LN2;
}

template <int FMT, int D>
void launch(const CacheAttnP& p, int blocks, hipStream_t st) {
  cache_attn_kernel<FMT, D><<<blocks, 256, 0, st>>>(p);
}
template <int D>
void launch_join(const CacheAttnP& p, hipStream_t st) {
  const int64_t units = (int64_t)p.T * p.H;
  if (units <= 1024) cache_join_kernel<D, 4><<<(int)units, 256, 0, st>>>(p);
  else cache_join_kernel<D, 1><<<(int)((units + 3) / 4), 256, 0, st>>>(p);
}

// How the work is cut (cache_cut.h): from the descriptors alone, so from the table's room, not from the lengths.
// Up to 512 keys of room one launch finishes every sequence; beyond that four wavefronts over a whole sequence take longer than pieces and the launch that joins
// them.  One launch | pieces and join, us, bf16, sequences as long as the table has room, heads of 128:
//   1 sequence, 4 key heads, 4 rows: 256 keys 7.7 | 9.5, 512 10.4 | 10.9, 1024 15.6 | 10.9, 4096 46 | 11; 64 rows: 256 10.3 | 12.1, 512 15.3 | 14.1, 1024 24.9 | 14.1
//   8 sequences, 8 key heads, 4 rows: 256 8.1 | 9.9, 512 10.7 | 11.2, 1024 16.7 | 12.5; 64 rows: 256 10.6 | 13.3, 512 15.8 | 15.7, 1024 26.3 | 18.7
//   64 sequences, 8 key heads, 4 rows: 256 15.0 | 17.8, 512 24.3 | 26.9, 1024 43.6 | 45.5 (equal lengths, as many runs as the chip holds)
// A piece has two units at least: one unit | two | four, us, 8 sequences of 8 key heads, 4 rows, room for 4096: 60 keys 8.3 | 12.1 | 19.8, 200 keys 9.7 | 9.9 | 15.2, 500 keys
// 10.2 | 11.4 | 12.7; but 32 sequences, 64 rows: 200 keys 25.6 | 19.3 | 27.7, and 4 sequences of 384 rows and 120 keys 22.7 | 14.8 | 21.6, where one unit has parts to join.
void cut(CacheAttnP& p) {
  p.max_rows = p.max_new * p.G;
  p.whole = ((int64_t)p.c.max_pages << p.c.shift) <= 512;
  const int runs = p.c.n_seq * (p.max_rows <= 64 ? 1 : (p.max_rows + 127) / 128);
  p.pieces = p.whole ? runs : p.c.HK < 512 ? 512 / p.c.HK : 1;  // two work-groups to a compute unit
  p.least = p.whole ? 1 : 2;
  p.part_rows = p.max_rows <= 64 ? p.max_rows : 128;
  p.ml_at = part_row(p, 2 * p.pieces, 0, 0) * p.c.D;
}

}  // namespace

size_t cache_attn_bytes(const CacheAttnP& q) {
  CacheAttnP p = q;
  cut(p);
  return p.whole ? 0 : (size_t)part_row(p, 2 * p.pieces, 0, 0) * (p.c.D + 2) * sizeof(float);
}

hipError_t launch_cache_attn(const CacheAttnP& q, hipStream_t st) {
  CacheAttnP p = q;
  cut(p);
  const int blocks = p.pieces * p.c.HK;
  auto by_size = [&](auto fmt) {
    if (p.c.D == 64) launch<fmt(), 64>(p, blocks, st);
    else launch<fmt(), 128>(p, blocks, st);
  };
  hipError_t e;
  if (p.max_rows > 32) {
    e = launch_cache_attn_rows(p, blocks, st);
  } else {
    if (p.c.format == BF) by_size(std::integral_constant<int, BF>{});
    else if (p.c.format == F8) by_size(std::integral_constant<int, F8>{});
    else by_size(std::integral_constant<int, I8>{});
    e = hipGetLastError();
  }
  if (e != hipSuccess || p.whole) return e;
  if (p.c.D == 64) launch_join<64>(p, st);
  else launch_join<128>(p, st);
  return hipGetLastError();
}

}  // namespace ssa
