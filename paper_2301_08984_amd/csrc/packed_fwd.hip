// Forward of attention over packed sequences.
//
// A work-group of four wavefronts owns a tile of 128 rows (packed_tile.h), a wavefront 32 of them, and walks the keys in blocks of 64
// with the running maximum and sum of a softmax; K / V tiles travel from memory straight into two LDS buffers, one barrier a
// block (as in fast_fwd128.hip, whose arithmetic this is).  KG = 2: two groups of four wavefronts take every other block of keys (p_two_groups) and are
// joined at the end.  P is rounded to bf16 for the product with V, which is what the matrix
// instructions take; scores, maxima, sums and O are fp32.
//
// Measured: one document of 16384 tokens, 12 heads of 128, 786 us, 1050 TFLOP/s (a large library product of bf16 matrices: 1216), bound by the matrix
// and vector instructions of a block of keys.  19 prompts, 9001 tokens, 32 heads in groups of four: 82 us, 590 TFLOP/s; a tile there has
// 6 blocks on average, and finding it, the first loads and the epilogue (4000 cycles each) are as long as four of them.
#include "packed_tile.h"

#include <type_traits>

namespace ssa {
namespace {

template <int D, int KG>
__device__ __forceinline__ void packed_fwd_tile(const PackedP& p, char* smem) {
  using T = PTile<D>;
  constexpr int KS = T::KS, DB = T::DB, U = T::LOADS / 4, STAGE_B = 4 * T::SUB_B;
  const int lane = threadIdx.x & 63, r = lane & 31, hl = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = KG == 2 ? wave & 3 : wave, kg = KG == 2 ? wave >> 2 : 0;
  char* mine = smem + kg * 2 * STAGE_B;
  const PPlace at = p_place(p.h1 - p.h0);
  const PFound f = p_find<false, 7>(p, at.rank);
  if (f.t < 0) return;
  const PackedSeq s = f.s;
  const int hk = p.h0 + at.head, rows = s.n * p.G, more = s.m - s.n;
  const int first = 128 * f.t + 32 * w;  // this wavefront's rows
  const int R = min(first + r, rows - 1), tok = R / p.G, h = hk * p.G + R - tok * p.G, pos = tok + more;  // sees keys 0 .. pos
  const bool live = first + r < rows;
  auto blocks = [&](int row) { return (max(min(row, rows - 1) / p.G + more + 1, 0) + 63) >> 6; };  // of 64 keys that rows up to `row` see
  const int ntiles = blocks(128 * f.t + 127), wtiles = first < rows ? blocks(first + 31) : 0;
  const int first_pos = min(first, rows - 1) / p.G + more;
  const float c1 = p_factor(p.scale);

  // this wavefront's share of a tile: U load instructions of each of its four sub-tiles
  const uint32_t ks2 = (uint32_t)p.k_st * 2u;
  uint32_t goff[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int rho = T::ROWS * (U * w + u) + lane / T::CHUNKS, c = (lane % T::CHUNKS) ^ p_sw<D>(rho);
    goff[u] = 8 * c < p.D ? (uint32_t)rho * ks2 + 16u * (uint32_t)c : P_NOWHERE;
  }
  const int64_t kbase = (int64_t)s.k0 * p.k_st + (int64_t)hk * p.k_sh;
  auto fetch_tile = [&](char* stage, int kt) {
#pragma unroll
    for (int sub = 0; sub < 4; ++sub) {
      const int row0 = kt * 64 + 32 * (sub & 1), left = min(s.m - row0, 32);  // rows of this sub-tile; those behind the last arrive as zeros
      const uint16_t* from = (const uint16_t*)(sub < 2 ? p.K : p.V) + kbase + (left > 0 ? (int64_t)row0 * p.k_st : 0);
      const __amdgpu_buffer_rsrc_t rs =
          __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, left > 0 ? (int)((uint32_t)(left - 1) * ks2 + 2u * p.D) : 0, 0x00020000);
#pragma unroll
      for (int u = 0; u < U; ++u)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (w_lds_void*)(stage + sub * T::SUB_B + (U * w + u) * 1024), 16, goff[u], 0, 0, 0);
    }
  };
  uint32_t ka[KS], va[2][DB];
  p_nat_addr<D>(ka, mine, r, hl);
  p_tr_addr<D>(va, mine, lane);

  const int steps = (ntiles + KG - 1) / KG;  // a group's step i is key tile KG i + kg
  if (steps > 0) fetch_tile(mine, kg);
  bf16x8 qf[KS];
  {
    const uint16_t* q = (const uint16_t*)p.Q + (int64_t)(s.q0 + tok) * p.q_st + (int64_t)h * p.q_sh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = w_frag(p_signed(p_load8(q, 16 * ks + 8 * hl, p.D), p.scale));
  }
  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) oacc[db][v] = 0.f;
  float m = -1e30f, l = 0.f;

  // one key tile in the stage buffer SB bytes into LDS: scores, online softmax, value product
  auto tile = [&](auto sb, int k0) {
    constexpr int SB = decltype(sb)::value;
    f32x16 sa[2];
    {
      u32x4 fa[KS], fb[KS];
      p_nat_issue<SB>(fa, ka);
      p_nat_issue<SB + T::SUB_B>(fb, ka);
      p_nat_wait(fa);
      p_nat_wait(fb);
#pragma unroll
      for (int v = 0; v < 16; ++v) { sa[0][v] = 0.f; sa[1][v] = 0.f; }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        sa[0] = mfma(w_frag(fa[ks]), qf[ks], sa[0]);
        sa[1] = mfma(w_frag(fb[ks]), qf[ks], sa[1]);
      }
    }
    u32x2 vt[2][2 * DB];
    p_tr_issue<SB + 2 * T::SUB_B>(vt, va);
    if (k0 + 63 > first_pos) {  // (a row's keys end inside the sequence: this covers the keys behind its last, too)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v) sa[kb][v] = k0 + 32 * kb + key_of(v, hl) > pos ? -INFINITY : sa[kb][v];
    }
    float rmax = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) rmax = fmaxf(rmax, sa[kb][v]);
    rmax = half_max(rmax * c1);
    // the maximum is raised when exceeded by more than 2^8: probabilities stay below that, harmless in fp32 and bf16
    if (__builtin_amdgcn_ballot_w64(rmax > m + 8.f) != 0) {
      const float mn = fmaxf(m, rmax), alpha = fast_exp2(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) oacc[db][v] *= alpha;
    }
    float lsum = 0.f;
    bf16x8 pf[4];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      float pr[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        pr[v] = fast_exp2(fmaf(sa[kb][v], c1, -m));
        lsum += pr[v];
      }
      pf[2 * kb] = pack8(&pr[0]);
      pf[2 * kb + 1] = pack8(&pr[8]);
    }
    l += lsum;
    p_tr_wait(vt);
    u32x2 vu[2][2 * DB];
    p_tr_issue<SB + 3 * T::SUB_B>(vu, va);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db] = mfma(w_frag2(vt[t][2 * db], vt[t][2 * db + 1]), pf[t], oacc[db]);
    p_tr_wait(vu);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db] = mfma(w_frag2(vu[t][2 * db], vu[t][2 * db + 1]), pf[2 + t], oacc[db]);
  };
  auto step = [&](auto sb, int i) {
    constexpr int SB = decltype(sb)::value;
    const int kt = KG * i + kg;
    W_VMCNT(0);  // this wavefront's part of the tile has landed
    __builtin_amdgcn_s_barrier();  // ... everybody's; and everybody is done with the other buffer
    asm volatile("" ::: "memory");
    if (i + 1 < steps) fetch_tile(mine + (STAGE_B - SB), kt + KG);
    if (kt < wtiles) tile(sb, kt * 64);
  };
  int i = 0;
  for (; i + 1 < steps; i += 2) {
    step(std::integral_constant<int, 0>{}, i);
    step(std::integral_constant<int, STAGE_B>{}, i + 1);
  }
  if (i < steps) step(std::integral_constant<int, 0>{}, i);

  if (KG == 2) {  // the second group's part, through LDS
    float* ml = (float*)smem + 128 * w;
    float4* part = (float4*)(smem + 2048) + w * DB * 4 * 64 + lane;
    __syncthreads();
    if (kg == 1) {
      ml[lane] = l;
      ml[64 + lane] = m;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) part[(4 * db + g) * 64] = make_float4(oacc[db][4 * g], oacc[db][4 * g + 1], oacc[db][4 * g + 2], oacc[db][4 * g + 3]);
    }
    __syncthreads();
    if (kg == 1) return;
    const float m1 = ml[64 + lane], mg = fmaxf(m, m1), a0 = fast_exp2(m - mg), a1 = fast_exp2(m1 - mg);
    l = fmaf(a1, ml[lane], a0 * l);
    m = mg;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 x = part[(4 * db + g) * 64];
        oacc[db][4 * g] = fmaf(a1, x.x, a0 * oacc[db][4 * g]);
        oacc[db][4 * g + 1] = fmaf(a1, x.y, a0 * oacc[db][4 * g + 1]);
        oacc[db][4 * g + 2] = fmaf(a1, x.z, a0 * oacc[db][4 * g + 2]);
        oacc[db][4 * g + 3] = fmaf(a1, x.w, a0 * oacc[db][4 * g + 3]);
      }
  }
  const float sum = half_sum(l), inv = sum > 0.f ? 1.f / sum : sum;  // no key: 0; NaN stays
  const float lse = sum == 0.f ? -INFINITY : (m + log2f(sum)) * LN2;
  if (live && hl == 0 && p.lse_out) p.lse_out[(int64_t)h * p.Tq + s.q0 + tok] = lse;
  uint16_t* y = (uint16_t*)p.Yo + (int64_t)(s.q0 + tok) * p.y_st + (int64_t)h * p.y_sh;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    uint2 o[4];
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4)
      o[g4] = pack4_bf16(oacc[db][4 * g4], oacc[db][4 * g4 + 1], oacc[db][4 * g4 + 2], oacc[db][4 * g4 + 3], inv);
    p_store_row32(y, o, 32 * db, hl, live, p.D);
  }
}

template <int D, int KG>
__global__ __launch_bounds__(256 * KG, D == 128 ? 2 : 4) void packed_fwd_kernel(PackedP p) {
  __shared__ __attribute__((aligned(1024))) char smem[KG * 2 * 4 * PTile<D>::SUB_B];
  static_assert(KG == 1 || sizeof(smem) >= 2048 + 4 * 32 * D * 4, "the second group's part fits");
  packed_fwd_tile<D, KG>(p, smem);
}

}  // namespace

hipError_t launch_packed_fwd(const PackedP& p, hipStream_t st) {
  const int g = (int)p_blocks(p_most_tiles(p, false, 7), p.h1 - p.h0);
  auto by_groups = [&](auto d) {
    if (p_two_groups(p)) packed_fwd_kernel<d(), 2><<<g, 512, 0, st>>>(p);
    else packed_fwd_kernel<d(), 1><<<g, 256, 0, st>>>(p);
  };
  if (p.D <= 64) by_groups(std::integral_constant<int, 64>{});
  else by_groups(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace ssa
