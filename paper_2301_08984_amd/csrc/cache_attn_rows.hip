// Attention over the cache where a sequence and key head have more than 32 rows (trees of drafts, groups of many query heads).
//
// Here the products count: 4 D flops for each of 33 and more rows a key, whose codes cost the vector ALUs 1.5 instructions each to become operands.
// So a block of keys is converted once, by all wavefronts of a work-group, into a bf16 tile in LDS (the images of packed_tile.h), from
// which every wavefront's 32 rows read it as packed_fwd.hip does: K along the rows, V transposed.  Four wavefronts of 32 rows share tiles of
// 64 keys; with up to 64 rows two of them share tiles of 32 keys, and the two pairs, with every other tile, are joined through LDS at the
// end.  The codes of the next tile travel into registers while a tile is at work, and are converted into the other buffer after it.
// With these rows in the registers of one wavefront instead (64 of them, every wavefront converting its own keys): 343 drafts
// of 16 trees over 48000 keys, 8 key heads, e4m3: 84 us against 64; 24 sequences of 8 tokens, groups of eight heads of 64, over 36000 keys, int8: 17 against 14.
#include "cache_cut.h"
#include "packed_tile.h"

#include <type_traits>

namespace ssa {
namespace {

template <int FMT, int D, int RB>
struct RowsLds {
  static constexpr int KG = 4 / RB, KEYS = 64 / KG, NKB = KEYS / 32;     // key groups; keys of a tile, blocks of 32
  static constexpr int TILE_B = 2 * KEYS * 2 * D, SCALES = 2 * KG * TILE_B;  // K and V; two buffers a group, then [group][buffer][K, V][64]
  static constexpr int BYTES = SCALES + KG * 2 * 512;
};

// One run (or part of one) of a piece (as in cache_attn.hip), for 32 RB rows.
template <int FMT, int D, int RB>
__device__ __forceinline__ void cache_rows_run(const CacheAttnP& p, char* smem, const Run& f, int hk, int begin, int end, bool all, int slot) {
  using T = PTile<D>;
  using L = RowsLds<FMT, D, RB>;
  constexpr int KS = T::KS, DB = T::DB, KG = L::KG, KEYS = L::KEYS, NKB = L::NKB;
  constexpr int ROW_B = D * (FMT == BF ? 2 : 1), LPR = ROW_B / 16, NL = ROW_B / 64, RPL = 64 / LPR;  // lanes of a row; loads of 16 rows; rows of one
  int lane = threadIdx.x & 63;
  asm("" : "+v"(lane));  // (what follows from it is formed anew for every run: kept over the loop, it spills)
  const int r = lane & 31, hl = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rb = w % RB, kg = w / RB;
  const CacheSeq s = f.s;
  const int rows = s.n * p.G, row0 = 128 * f.group, shift = p.c.shift;
  const int steps = end > begin ? ((end - begin - 1) >> 6) + 1 : 0;  // of 64 keys

  const int32_t* line = p.c.table + (int64_t)f.b * p.c.max_pages;
  const int last_entry = (end - 1) >> shift;
  auto entries = [&](int from) {
    const int e = from + lane;
    return e <= last_entry ? line[e] : -1;  // (looked at when it is used, so that nothing waits for it here)
  };
  int window = begin >> shift;
  int win = entries(window), win_next = entries(window + 64);

  const int R = min(row0 + 32 * rb + r, rows - 1), tok = R / p.G, h = hk * p.G + R - tok * p.G;
  const bool live_row = row0 + 32 * rb + r < rows, at_work = row0 + 32 * rb < rows;
  bf16x8 qf[KS];
  {
    const uint16_t* Q = (const uint16_t*)p.Q + (int64_t)(s.q0 + tok) * p.q_st + (int64_t)h * p.q_sh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = w_frag(p_signed(*(const u32x4*)(Q + 16 * ks + 8 * hl), p.scale));
  }
  const uint64_t bits = p.tree ? p.tree[s.q0 + tok] : ~(~(uint64_t)1 << tok);
  const float c1 = p_factor(p.scale);

  char* mine = smem + kg * 2 * L::TILE_B;
  uint32_t ka[KS], va[2][DB];
  p_nat_addr<D>(ka, mine, r, hl);
  p_tr_addr<D>(va, mine, lane);
  uint32_t live_next = 0, live_hi_next = 0;
  u32x4 kx[NL], vx[NL];
  float scale = 0.f;
  uint32_t here = 0;  // of these 16 keys, those that are there (looked at when the loads have arrived)
  // asks for the tile of step i
  auto load = [&](int i) {
    const int k0 = begin + 64 * i + KEYS * kg;
    if (((k0 + KEYS - 8) >> shift) - window >= 64) {
      window += 64;
      win = win_next;
      win_next = entries(window + 64);
    }
    uint64_t there = end - k0 >= 64 ? ~0ull : end - k0 > 0 ? (1ull << (end - k0)) - 1 : 0;
    // the entries of the tile's pages; one that is none takes its keys out
    const int e0 = (k0 >> shift) - window, e1 = ((k0 + KEYS - 8) >> shift) - window;
    const uint64_t need = ((2ull << (e1 - e0)) - 1) << e0, ok = __builtin_amdgcn_ballot_w64((uint32_t)win < (uint32_t)p.c.n_pages);
    if ((ok & need) != need)
      for (int g = 0; g < KEYS / 8; ++g)
        if (!(ok >> (((k0 + 8 * g) >> shift) - window) & 1)) there &= ~(0xffull << (8 * g));
    const int pos = k0 + 16 * rb;
    const int page_a = __builtin_amdgcn_readlane(win, (pos >> shift) - window), page_b = __builtin_amdgcn_readlane(win, ((pos + 8) >> shift) - window);
    auto page = [&](int entry) { return (uint32_t)entry < (uint32_t)p.c.n_pages ? entry : 0; };
    live_next = (uint32_t)there;
    live_hi_next = NKB == 2 ? (uint32_t)(there >> 32) : 0u;
    const int64_t row_a = cache_row(page(page_a), shift, p.c.HK, hk, pos), row_b = cache_row(page(page_b), shift, p.c.HK, hk, pos + 8);
    here = (uint32_t)(there >> (16 * rb)) & 0xffffu;
#pragma unroll
    for (int u = 0; u < NL; ++u) {
      const int x = RPL * u + lane / LPR;
      const int64_t row = (x < 8 ? row_a : row_b) + (x & 7);
      kx[u] = *(const u32x4*)((const char*)p.c.kc + row * ROW_B + 16 * (lane % LPR));
      vx[u] = *(const u32x4*)((const char*)p.c.vc + row * ROW_B + 16 * (lane % LPR));
    }
    if (FMT != BF) {
      const int x = lane & 15;
      scale = ((lane & 16) ? p.c.vs : p.c.ks)[(x < 8 ? row_a : row_b) + (x & 7)];
    }
  };
  // ... and puts it into buffer `to`
  auto stage = [&](int to) {
    char* tile = mine + to * L::TILE_B;
    int lane = threadIdx.x & 63;
    asm("" : "+v"(lane));  // (as above)
    uint32_t put[NL];  // this wavefront's 16 rows of a tile: where lanes put them
#pragma unroll
    for (int u = 0; u < NL; ++u) {
      const int row = 16 * rb + RPL * u + lane / LPR, c = (lane % LPR) * (FMT == BF ? 1 : 2);
      put[u] = (uint32_t)(row & 31) * (2 * D) + (uint32_t)(row >> 5) * T::SUB_B + (uint32_t)((c ^ p_sw<D>(row & 31)) << 4);
    }
    if (here != 0xffffu) {  // what lies in other slots may be anything
#pragma unroll
      for (int u = 0; u < NL; ++u) {
        const bool is = here >> (RPL * u + lane / LPR) & 1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          kx[u][e] = is ? kx[u][e] : 0u;
          vx[u][e] = is ? vx[u][e] : 0u;
        }
      }
      scale = here >> (lane & 15) & 1 ? scale : 0.f;
    }
#pragma unroll
    for (int u = 0; u < NL; ++u)
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const u32x4& x = kv ? vx[u] : kx[u];
        char* at = tile + kv * NKB * T::SUB_B;
        if (FMT == BF) {
          *(u32x4*)(at + put[u]) = x;
        } else {
          *(u32x4*)(at + put[u]) = u32x4{two_codes<FMT, false>(x[0]), two_codes<FMT, true>(x[0]), two_codes<FMT, false>(x[1]), two_codes<FMT, true>(x[1])};
          *(u32x4*)(at + (put[u] ^ 16u)) = u32x4{two_codes<FMT, false>(x[2]), two_codes<FMT, true>(x[2]), two_codes<FMT, false>(x[3]), two_codes<FMT, true>(x[3])};
          __builtin_amdgcn_sched_barrier(0);  // (16 codes at a time: all of them at once spill)
        }
      }
    if (FMT != BF && lane < 32) ((float*)(smem + L::SCALES + (2 * kg + to) * 512))[(lane & 16 ? 64 : 0) + 16 * rb + (lane & 15)] = lane & 16 ? scale : scale * c1;
  };

  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;
  float m = -1e30f, l = 0.f;

  auto tile = [&](auto buffer, int k0, uint64_t there) {
    constexpr int SB = decltype(buffer)::value * L::TILE_B;
    f32x16 sa[NKB];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) {
#pragma unroll
      for (int v = 0; v < 16; ++v) sa[kb][v] = 0.f;
    }
    auto scores = [&](auto kb) {
      u32x4 fk[KS];
      p_nat_issue<SB + decltype(kb)::value * T::SUB_B>(fk, ka);
      p_nat_wait(fk);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sa[decltype(kb)::value] = mfma(w_frag(fk[ks]), qf[ks], sa[decltype(kb)::value]);
    };
    scores(std::integral_constant<int, 0>{});
    if constexpr (NKB == 2) scores(std::integral_constant<int, NKB - 1>{});
    const float* sc = (const float*)(smem + L::SCALES + (2 * kg + decltype(buffer)::value) * 512) + 4 * hl;
    const bool plain = there == (NKB == 2 ? ~0ull : 0xffffffffull) && s.before - k0 >= KEYS;
    uint32_t seen[NKB];
    float rmax = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 x = FMT == BF ? make_float4(c1, c1, c1, c1) : *(const float4*)(sc + 32 * kb + 8 * g);  // (the factor is in the scale)
        sa[kb][4 * g] *= x.x;
        sa[kb][4 * g + 1] *= x.y;
        sa[kb][4 * g + 2] *= x.z;
        sa[kb][4 * g + 3] *= x.w;
      }
      if (!plain) {
        const int nb = s.before - k0 - 32 * kb;
        const uint32_t old = nb >= 32 ? ~0u : nb > 0 ? (1u << nb) - 1u : 0u;
        const uint32_t fresh = nb >= 32 ? 0u : nb >= 0 ? (uint32_t)(bits << nb) : nb > -64 ? (uint32_t)(bits >> -nb) : 0u;
        seen[kb] = ((uint32_t)(there >> (32 * kb)) & (old | fresh)) >> (4 * hl);
#pragma unroll
        for (int v = 0; v < 16; ++v) sa[kb][v] = seen[kb] >> (8 * (v >> 2) + (v & 3)) & 1u ? sa[kb][v] : -INFINITY;
      }
#pragma unroll
      for (int v = 0; v < 16; ++v) rmax = fmaxf(rmax, sa[kb][v]);
    }
    rmax = half_max(rmax);
    // the maximum is raised when exceeded by more than 2^8: probabilities stay below that
    if (__builtin_amdgcn_ballot_w64(rmax > m + 8.f) != 0) {
      const float mn = fmaxf(m, rmax), alpha = fast_exp2(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[db][v] *= alpha;
    }
    bf16x8 pf[2 * NKB];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) {
      float pr[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) pr[v] = fast_exp2(sa[kb][v] - m);
      l += sum16(pr);
      if (FMT != BF) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float4 x = *(const float4*)(sc + 64 + 32 * kb + 8 * g);
          pr[4 * g] *= x.x;
          pr[4 * g + 1] *= x.y;
          pr[4 * g + 2] *= x.z;
          pr[4 * g + 3] *= x.w;
        }
      }
      if (!plain) {  // (a new token that is not seen may have any scale)
#pragma unroll
        for (int v = 0; v < 16; ++v) pr[v] = seen[kb] >> (8 * (v >> 2) + (v & 3)) & 1u ? pr[v] : 0.f;
      }
      pf[2 * kb] = pack8(&pr[0]);
      pf[2 * kb + 1] = pack8(&pr[8]);
    }
    u32x2 vt[2][2 * DB];
    p_tr_issue<SB + NKB * T::SUB_B>(vt, va);
    p_tr_wait(vt);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] = mfma(w_frag2(vt[t][2 * db], vt[t][2 * db + 1]), pf[t], acc[db]);
    if constexpr (NKB == 2) {
      p_tr_issue<SB + 3 * T::SUB_B>(vt, va);
      p_tr_wait(vt);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] = mfma(w_frag2(vt[t][2 * db], vt[t][2 * db + 1]), pf[2 * NKB - 2 + t], acc[db]);
    }
  };
  if (steps > 0) load(0);
  // step i: its tile, in registers, goes into buffer i % 2, which everybody has left since the last barrier
  auto step = [&](auto buffer, int i) {
    const uint64_t there = (uint64_t)live_hi_next << 32 | live_next;
    stage(decltype(buffer)::value);
    if (i + 1 < steps) load(i + 1);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (at_work && there) tile(buffer, begin + 64 * i + KEYS * kg, there);
  };
  for (int i = 0; i < steps; i += 2) {
    step(std::integral_constant<int, 0>{}, i);
    if (i + 1 < steps) step(std::integral_constant<int, 1>{}, i + 1);
  }

  l = half_sum(l);
  float sum = l;
  if (KG == 2) {  // the second pair's part
    float* ml = (float*)smem + rb * 64;
    float4* part = (float4*)(smem + 1024) + rb * DB * 4 * 64 + lane;
    __syncthreads();
    if (kg == 1) {
      if (hl == 0) {
        ml[r] = m;
        ml[32 + r] = l;
      }
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) part[(4 * db + g) * 64] = make_float4(acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]);
    }
    __syncthreads();
    const float m1 = ml[r], mg = fmaxf(m, m1), a0 = fast_exp2(m - mg), a1 = fast_exp2(m1 - mg);
    sum = fmaf(a1, ml[32 + r], a0 * l);
    m = mg;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 x = part[(4 * db + g) * 64];
        acc[db][4 * g] = fmaf(a1, x.x, a0 * acc[db][4 * g]);
        acc[db][4 * g + 1] = fmaf(a1, x.y, a0 * acc[db][4 * g + 1]);
        acc[db][4 * g + 2] = fmaf(a1, x.z, a0 * acc[db][4 * g + 2]);
        acc[db][4 * g + 3] = fmaf(a1, x.w, a0 * acc[db][4 * g + 3]);
      }
  }
  if (kg == 0 && all) {
    const float inv = sum > 0.f ? 1.f / sum : sum;  // no key: 0; NaN stays
    uint16_t* y = (uint16_t*)p.Y + (int64_t)(s.q0 + tok) * p.y_st + (int64_t)h * p.y_sh;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      uint2 o[4];
#pragma unroll
      for (int g = 0; g < 4; ++g) o[g] = pack4_bf16(acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3], inv);
      store_row32(y + 32 * db, o, hl, live_row);
    }
    if (live_row && p.lse && hl == 0) p.lse[(int64_t)h * p.T + s.q0 + tok] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * LN2;
  } else if (kg == 0 && live_row) {
    const int64_t at = part_row(p, slot, hk, R - row0);
    float* y = (float*)p.ws + at * D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(float4*)(y + 32 * db + 8 * g + 4 * hl) = make_float4(acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]);
    if (hl == 0) *(float2*)((float*)p.ws + p.ml_at + 2 * at) = make_float2(m, sum);
  }
  __syncthreads();  // the next run's tiles come where this one's lay
}

template <int FMT, int D>
__global__ __launch_bounds__(256, 2) void cache_attn_rows_kernel(CacheAttnP p) {
  __shared__ __attribute__((aligned(1024))) char smem[RowsLds<FMT, D, 2>::BYTES];
  static_assert(RowsLds<FMT, D, 2>::BYTES >= RowsLds<FMT, D, 4>::BYTES && RowsLds<FMT, D, 2>::BYTES >= 1024 + 2 * 32 * D * 4, "both forms and the second pair's part");
  const int piece = blockIdx.x / p.c.HK, hk = blockIdx.x - piece * p.c.HK;
  const Cut cut(p);
  for (int u = piece * cut.each, stop = min(u + cut.each, cut.total); u < stop;) {
    const Run f = cut.find(u);
    const int sh = Cut::many(p, f.s.n) ? 6 : 7, take = min(f.units - f.at, stop - u);
    const CacheSpan keys = cache_span(f.at, take, f.units, sh, f.s.len);
    u += take;
    const int slot = part_slot(piece, cut.each, f.first);
    if (sh == 6) cache_rows_run<FMT, D, 4>(p, smem, f, hk, keys.begin, keys.end, take == f.units, slot);
    else cache_rows_run<FMT, D, 2>(p, smem, f, hk, keys.begin, keys.end, take == f.units, slot);
  }
}

template <int FMT, int D>
void launch(const CacheAttnP& p, int blocks, hipStream_t st) {
  cache_attn_rows_kernel<FMT, D><<<blocks, 256, 0, st>>>(p);
}

}  // namespace

hipError_t launch_cache_attn_rows(const CacheAttnP& p, int blocks, hipStream_t st) {
  auto by_size = [&](auto fmt) {
    if (p.c.D == 64) launch<fmt(), 64>(p, blocks, st);
    else launch<fmt(), 128>(p, blocks, st);
  };
  if (p.c.format == BF) by_size(std::integral_constant<int, BF>{});
  else if (p.c.format == F8) by_size(std::integral_constant<int, F8>{});
  else by_size(std::integral_constant<int, I8>{});
  return hipGetLastError();
}

}  // namespace ssa
