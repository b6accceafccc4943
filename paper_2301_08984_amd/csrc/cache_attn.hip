// Attention of new tokens over the paged cache (include/ss_cache.h).
//
// Bound by reading the cache: 4 D bytes (2 D + 8 in 8 bits) a key and head for 4 D flops a row, so a key is read once for all rows that see
// it, the new tokens of a sequence times the G query heads of a key head, 32 or 64 (NQ = 2) to a wavefront, and goes from memory into
// registers: nothing passes through LDS until the end.  The keys of all sequences are cut into parts of about equal length, so that a long
// sequence does not keep the chip waiting; the four wavefronts of a work-group take every fourth block of 32 keys of a part each, with a
// running maximum and sum, and are joined through LDS.  A sequence in one part is finished there; the others' parts are joined by
// a second launch.
//
// Scores: S^T = K Q^T, a lane holding 16 (D = 128: of the row's 128) columns of its key, as they come; 8-bit codes become bf16
// exactly, and the key's scale multiplies the fp32 score.  O^T += V^T P^T: a lane holds D / 32 neighbouring columns of eight keys, which byte permutes turn
// into operands (eight keys of a column), so that V needs no transposed copy in LDS; the value's scale goes into P, which is
// rounded to bf16 as the matrix instructions take it.  Maxima, sums and O are fp32.
#include "cache.h"
#include "mfma_common.h"

namespace ssa {
namespace {

enum { BF = 0, F8 = 1, I8 = 2 };

// What one sequence has: its new tokens' rows, the keys before them and in all, and the parts of `chunk` keys.
struct CacheSeq {
  int q0, n, before, len;
};
__device__ __forceinline__ CacheSeq cache_seq(const CacheAttnP& p, int b) {
  CacheSeq s;
  s.q0 = min(max(p.cu[b], 0), p.T);
  const int n = max(min(p.cu[b + 1], p.T) - s.q0, 0), lens = max(p.lens[b], 0);
  s.n = min(n, p.max_new);
  s.before = max(lens - n, 0);
  s.len = (int)min((int64_t)lens, (int64_t)p.c.max_pages << p.c.shift);  // keys that the table has a place for
  return s;
}
__device__ __forceinline__ int parts_of(const CacheSeq& s, int chunk) { return s.n > 0 ? (s.len > 0 ? (s.len - 1) / chunk + 1 : 1) : 0; }

__device__ __forceinline__ int scan64(int x) {  // inclusive prefix sums over the wavefront
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}
__device__ __forceinline__ CacheSeq lane_seq(const CacheAttnP& p, int b) {
  CacheSeq s = cache_seq(p, min(b, p.c.n_seq - 1));
  if (b >= p.c.n_seq) s.n = s.len = 0;
  return s;
}
// keys of a part: enough parts to fill the chip (`p.parts` of them over all sequences), not shorter than p.least
__device__ __forceinline__ int chunk_of(const CacheAttnP& p) {
  int64_t total = 0;
  for (int b0 = 0; b0 < p.c.n_seq; b0 += 64) {
    const CacheSeq s = lane_seq(p, b0 + (int)(threadIdx.x & 63));
    // (in units of 128 keys: the sum of 64 sequences of 2^31 keys fits)
    total += __builtin_amdgcn_readlane(scan64(s.n > 0 ? (s.len >> 7) + 1 : 0), 63);
  }
  return (int)max((int64_t)p.least, min((total + p.parts - 1) / p.parts * 128, (int64_t)0x7fffff80));
}
// the sequence of slot `slot`, and its part there; b = -1: fewer slots than that
struct Slot {
  CacheSeq s;
  int b, part, parts;
};
__device__ __forceinline__ Slot find_slot(const CacheAttnP& p, int chunk, int slot) {
  const int lane = threadIdx.x & 63;
  Slot f;
  f.b = -1;
  for (int b0 = 0; b0 < p.c.n_seq; b0 += 64) {
    const CacheSeq s = lane_seq(p, b0 + lane);
    const int mine = parts_of(s, chunk), upto = scan64(mine), all = __builtin_amdgcn_readlane(upto, 63);
    if (slot >= all) {
      slot -= all;
      continue;
    }
    const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > slot));
    f.s.q0 = __builtin_amdgcn_readlane(s.q0, l);
    f.s.n = __builtin_amdgcn_readlane(s.n, l);
    f.s.before = __builtin_amdgcn_readlane(s.before, l);
    f.s.len = __builtin_amdgcn_readlane(s.len, l);
    f.b = b0 + l;
    f.parts = __builtin_amdgcn_readlane(mine, l);
    f.part = slot - (__builtin_amdgcn_readlane(upto, l) - f.parts);
    return f;
  }
  return f;
}

// two bf16 of one register's 16-bit halves
__device__ __forceinline__ uint32_t lo_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t hi_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
// two 8-bit codes (bytes 2 HI and 2 HI + 1) as packed bf16, exactly
template <int FMT, bool HI>
__device__ __forceinline__ uint32_t two_codes(uint32_t x) {
  if (FMT == F8) {
    union { bf16x2 v; uint32_t u; } o;
    o.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, HI);
    return o.u;
  }
  return pack2_bf16((float)(int8_t)(x >> (HI ? 16 : 0)), (float)(int8_t)(x >> (HI ? 24 : 8)));
}

template <int FMT, int D>
struct CacheTile {
  static constexpr int E = FMT == BF ? 2 : 1, ROW_B = D * E, KS = D / 16, NB = D / 32;
  static constexpr int KL = ROW_B / 32;      // 16-byte loads of a lane for K
  static constexpr int VW = NB * E;          // bytes of a lane and key of V: 2, 4 or 8
  static constexpr int VR = VW == 8 ? 2 : 1;  // registers
};

template <int FMT, int D, int NQ>
__device__ __forceinline__ void cache_attn_part(const CacheAttnP& p, char* smem) {
  using T = CacheTile<FMT, D>;
  constexpr int KS = T::KS, NB = T::NB, ROW_B = T::ROW_B;
  const int lane = threadIdx.x & 63, r = lane & 31, hl = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // row groups of one part next to each other on one XCD: all but the first find its keys in that XCD's L2
  const int idx = blockIdx.x >> 3, unit = idx / p.groups * 8 + (int)(blockIdx.x & 7), rg = idx % p.groups;
  const int slot = unit / p.c.HK, hk = unit - slot * p.c.HK;
  if (slot >= p.slots) return;
  const int chunk = chunk_of(p);
  const Slot f = find_slot(p, chunk, slot);
  if (f.b < 0) return;
  const CacheSeq s = f.s;
  const int rows = s.n * p.G, row0 = 32 * NQ * rg;
  if (row0 >= rows) return;
  const int begin = f.part * chunk, end = begin + min(chunk, s.len - begin);
  const int shift = p.c.shift;

  // pages of the part: a lane an entry, 64 of them and the 64 behind them
  const int32_t* line = p.c.table + (int64_t)f.b * p.c.max_pages;
  const int last_entry = (end - 1) >> shift;
  auto entries = [&](int from) {
    const int e = from + lane;
    const int page = e <= last_entry ? line[e] : -1;
    return page >= 0 && page < p.c.n_pages ? page : -1;
  };
  int window = (begin + 32 * w) >> shift;
  int win = entries(window), win_next = entries(window + 64);

  bf16x8 qf[NQ][KS];
  uint64_t bits[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int R = min(row0 + 32 * q + r, rows - 1), tok = R / p.G, h = hk * p.G + R - tok * p.G;
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
      qf[q][ks] = x.v;
    }
    bits[q] = p.tree ? p.tree[s.q0 + tok] : ~(~(uint64_t)1 << tok);
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
      const int pos = k0 + 8 * g, page = __builtin_amdgcn_readlane(win, (pos >> shift) - window);
      if (page < 0) there &= ~(0xffu << (8 * g));
      row_of[g] = cache_row(max(page, 0), shift, p.c.HK, hk, pos);
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

  f32x16 acc[NQ][NB];
  float m[NQ], l[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    m[q] = -1e30f;
    l[q] = 0.f;
#pragma unroll
    for (int e = 0; e < NB; ++e)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[q][e][v] = 0.f;
  }
  int k0 = begin + 32 * w;
  if (k0 < end) {
    locate(k0);
    load_v();
  }
  for (; k0 < end; k0 += 128) {
    live = live_next;
    f32x16 sa[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int v = 0; v < 16; ++v) sa[q][v] = 0.f;
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
#pragma unroll
      for (int q = 0; q < NQ; ++q) sa[q] = mfma(k.v, qf[q][ks], sa[q]);
    }
    float kc[16];  // what makes a score of a product, in base-2 units
#pragma unroll
    for (int v = 0; v < 16; ++v) kc[v] = FMT == BF ? c1 : c1 * __uint_as_float(ks4[v >> 2][v & 3]);
    const bool more = k0 + 128 < end;
    // all keys are there and none is a new token: nothing to mask
    const bool plain = live == ~0u && k0 + 32 <= s.before;
    if (more) locate(k0 + 128);  // K of the next block starts on its way
    bf16x8 pf[NQ][2];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      uint32_t seen = ~0u;  // keys of the block that this lane's row sees, from the half-wave's first on
#pragma unroll
      for (int v = 0; v < 16; ++v) sa[q][v] *= kc[v];
      if (!plain) {
        const int nb = s.before - k0;
        const uint32_t old = nb >= 32 ? ~0u : nb > 0 ? (1u << nb) - 1u : 0u;
        const uint32_t fresh = nb >= 32 ? 0u : nb >= 0 ? (uint32_t)(bits[q] << nb) : nb > -64 ? (uint32_t)(bits[q] >> -nb) : 0u;
        seen = (live & (old | fresh)) >> (4 * hl);
#pragma unroll
        for (int v = 0; v < 16; ++v) sa[q][v] = seen >> (8 * (v >> 2) + (v & 3)) & 1u ? sa[q][v] : -INFINITY;
      }
      float rmax = -INFINITY;
#pragma unroll
      for (int v = 0; v < 16; ++v) rmax = fmaxf(rmax, sa[q][v]);
      rmax = half_max(rmax);
      // the maximum is raised when exceeded by more than 2^8: probabilities stay below that
      if (__builtin_amdgcn_ballot_w64(rmax > m[q] + 8.f) != 0) {
        const float mn = fmaxf(m[q], rmax), alpha = fast_exp2(m[q] - mn);
        m[q] = mn;
        l[q] *= alpha;
#pragma unroll
        for (int e = 0; e < NB; ++e)
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[q][e][v] *= alpha;
      }
      float pr[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) pr[v] = fast_exp2(sa[q][v] - m[q]);
      l[q] += sum16(pr);
      if (FMT != BF) {
#pragma unroll
        for (int v = 0; v < 16; ++v) pr[v] *= __uint_as_float(vs4[v >> 2][v & 3]);
      }
      if (!plain) {  // (a slot where nothing lies may hold any scale)
#pragma unroll
        for (int v = 0; v < 16; ++v) pr[v] = seen >> (8 * (v >> 2) + (v & 3)) & 1u ? pr[v] : 0.f;
      }
      pf[q][0] = pack8(&pr[0]);
      pf[q][1] = pack8(&pr[8]);
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
#pragma unroll
        for (int q = 0; q < NQ; ++q) acc[q][e] = mfma(a.v, pf[q][t], acc[q][e]);
      }
    }
    if (more) load_v();
  }

  // The wavefronts' parts: maxima and sums first, then O at the common maximum, quarter by quarter of the columns.  acc[e][v] is column
  // NB (8 (v / 4) + 4 hl + v % 4) + e: wavefront w adds up registers 4 w .. 4 w + 3, 4 NB neighbouring columns of each row.
  float* ml = (float*)smem;               // [wavefront][maximum, sum][32]
  float4* part = (float4*)(smem + 1024);  // [wavefront][e][quarter][lane]
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    l[q] = half_sum(l[q]);
    __syncthreads();
    if (hl == 0) {
      ml[64 * w + r] = m[q];
      ml[64 * w + 32 + r] = l[q];
    }
    __syncthreads();
    float mg = -1e30f, sum = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) mg = fmaxf(mg, ml[64 * x + r]);
#pragma unroll
    for (int x = 0; x < 4; ++x) sum = fmaf(fast_exp2(ml[64 * x + r] - mg), ml[64 * x + 32 + r], sum);
    const float mine = fast_exp2(m[q] - mg);
#pragma unroll
    for (int e = 0; e < NB; ++e)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        part[((w * NB + e) * 4 + g) * 64 + lane] = make_float4(acc[q][e][4 * g] * mine, acc[q][e][4 * g + 1] * mine, acc[q][e][4 * g + 2] * mine, acc[q][e][4 * g + 3] * mine);
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
    const int R = row0 + 32 * q + r, col = NB * (8 * w + 4 * hl);
    if (R >= rows) continue;  // (no barrier is left out: `continue` leaves a lane's stores only)
    if (f.parts == 1) {
      const int tok = R / p.G, h = hk * p.G + R - tok * p.G;
      const float inv = sum > 0.f ? 1.f / sum : sum;  // no key: 0; NaN stays
      uint16_t* y = (uint16_t*)p.Y + (int64_t)(s.q0 + tok) * p.y_st + (int64_t)h * p.y_sh + col;
#pragma unroll
      for (int x = 0; x < 4 * NB; x += 8)
        *(u32x4*)(y + x) = u32x4{pack2_bf16(o[x] * inv, o[x + 1] * inv), pack2_bf16(o[x + 2] * inv, o[x + 3] * inv),
                                 pack2_bf16(o[x + 4] * inv, o[x + 5] * inv), pack2_bf16(o[x + 6] * inv, o[x + 7] * inv)};
      if (p.lse && w == 0 && hl == 0) p.lse[(int64_t)h * p.T + s.q0 + tok] = sum == 0.f ? -INFINITY : (mg + log2f(sum)) * LN2;
    } else {
      const int64_t at = ((int64_t)slot * p.c.HK + hk) * p.max_rows + R;
      float* y = (float*)p.ws + at * D + col;
#pragma unroll
      for (int x = 0; x < 4 * NB; x += 4) *(float4*)(y + x) = make_float4(o[x], o[x + 1], o[x + 2], o[x + 3]);
      if (w == 0 && hl == 0) *(float2*)((float*)p.ws + p.ml_at + 2 * at) = make_float2(mg, sum);
    }
  }
}

template <int FMT, int D, int NQ>
__global__ __launch_bounds__(256, NQ == 1 ? 2 : 1) void cache_attn_kernel(CacheAttnP p) {
  __shared__ __attribute__((aligned(1024))) char smem[1024 + 4 * 32 * D * 4];
  cache_attn_part<FMT, D, NQ>(p, smem);
}

// Rows of sequences in more than one part: a wavefront per token and head, the parts in order.
template <int D>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnP p) {
  constexpr int C = D / 64;  // columns of a lane
  const int lane = threadIdx.x & 63;
  const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), t = unit / p.H, h = unit - t * p.H;
  if (t >= p.T) return;
  const int chunk = chunk_of(p);
  const int b = packed_owner(p.cu, p.c.n_seq, t);
  if (b < 0) return;
  const CacheSeq s = cache_seq(p, b);
  const int parts = parts_of(s, chunk), tok = t - s.q0;
  if (parts < 2 || tok >= s.n) return;
  int slot = 0;  // the sequence's first
  for (int b0 = 0; b0 < b; b0 += 64) {
    const int i = b0 + lane;
    slot += __builtin_amdgcn_readlane(scan64(i < b ? parts_of(cache_seq(p, i), chunk) : 0), 63);
  }
  const int hk = h / p.G, R = tok * p.G + h - hk * p.G;
  const float* ws = (const float*)p.ws;
  const int64_t first = ((int64_t)slot * p.c.HK + hk) * p.max_rows + R, step = (int64_t)p.c.HK * p.max_rows;
  float mg = -1e30f;
  for (int x = lane; x < parts; x += 64) mg = fmaxf(mg, ws[p.ml_at + 2 * (first + x * step)]);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) mg = fmaxf(mg, __shfl_xor(mg, o));
  float sum = 0.f, acc[C];
#pragma unroll
  for (int c = 0; c < C; ++c) acc[c] = 0.f;
  for (int x = 0; x < parts; ++x) {
    const int64_t at = first + x * step;
    const float2 ml = *(const float2*)(ws + p.ml_at + 2 * at);
    const float a = fast_exp2(ml.x - mg);
    sum = fmaf(a, ml.y, sum);
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] = fmaf(a, ws[at * D + C * lane + c], acc[c]);
  }
  const float inv = sum > 0.f ? 1.f / sum : sum;
  uint16_t* y = (uint16_t*)p.Y + (int64_t)t * p.y_st + (int64_t)h * p.y_sh + C * lane;
  if (C == 2) *(uint32_t*)y = pack2_bf16(acc[0] * inv, acc[C - 1] * inv);
  else *y = f2bf(acc[0] * inv);
  if (p.lse && lane == 0) p.lse[(int64_t)h * p.T + t] = sum == 0.f ? -INFINITY : (mg + log2f(sum)) * LN2;
}

template <int FMT, int D>
void launch(const CacheAttnP& p, int blocks, hipStream_t st) {
  if (p.max_rows <= 32) cache_attn_kernel<FMT, D, 1><<<blocks, 256, 0, st>>>(p);
  else cache_attn_kernel<FMT, D, 2><<<blocks, 256, 0, st>>>(p);
}

// How the work is cut: from the descriptors alone.
void cut(CacheAttnP& p) {
  p.max_rows = p.max_new * p.G;
  p.groups = p.max_rows <= 32 ? 1 : (p.max_rows + 63) / 64;
  const int64_t most = (int64_t)p.c.max_pages << p.c.shift;  // keys of a sequence
  // two work-groups to a compute unit (one with 64 rows a wavefront); a context that fits 512 keys is one part
  const int64_t want = (p.max_rows <= 32 ? 512 : 256) / ((int64_t)p.c.HK * p.groups);
  p.parts = (int)(want > 1 ? want : 1);
  p.least = most <= 512 ? 512 : 256;
  p.slots = p.parts + p.c.n_seq;
  p.ml_at = (int64_t)p.slots * p.c.HK * p.max_rows * p.c.D;
}
bool one_part(const CacheAttnP& p) { return ((int64_t)p.c.max_pages << p.c.shift) <= p.least; }

}  // namespace

size_t cache_attn_bytes(const CacheAttnP& q) {
  CacheAttnP p = q;
  cut(p);
  return one_part(p) ? 0 : (size_t)p.slots * p.c.HK * p.max_rows * (p.c.D + 2) * sizeof(float);
}

hipError_t launch_cache_attn(const CacheAttnP& q, hipStream_t st) {
  CacheAttnP p = q;
  cut(p);
  const int blocks = (int)((((int64_t)p.slots * p.c.HK + 7) / 8) * 8 * p.groups);
  auto by_size = [&](auto fmt) {
    if (p.c.D == 64) launch<fmt(), 64>(p, blocks, st);
    else launch<fmt(), 128>(p, blocks, st);
  };
  if (p.c.format == BF) by_size(std::integral_constant<int, BF>{});
  else if (p.c.format == F8) by_size(std::integral_constant<int, F8>{});
  else by_size(std::integral_constant<int, I8>{});
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || one_part(p)) return e;
  const int units = (int)(((int64_t)p.T * p.H + 3) / 4);
  if (p.c.D == 64) cache_join_kernel<64><<<units, 256, 0, st>>>(p);
  else cache_join_kernel<128><<<units, 256, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace ssa
