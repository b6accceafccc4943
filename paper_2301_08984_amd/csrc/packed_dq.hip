// dQ of attention over packed sequences.
//
// The tiles of 128 rows and the buffers of packed_fwd.hip.  Q and dY fragments stay in registers; per block of 32 keys the scores and dP
// come from the matrix instructions, dS = P (dP - Delta) from the vector ALUs (rounded to bf16, the type of the last product's operands), and
// dQ^T += K^T dS^T reads the same K sub-tile transposed.
//
// Measured: one document of 16384 tokens, 12 heads of 128, 1071 us, 1155 TFLOP/s; 23 documents, 8192 tokens, 12 heads in groups of three: 40 us, bound by
// what a tile does before and after its blocks of keys.
#include "packed_tile.h"

#include <type_traits>

namespace ssa {
namespace {

template <int D, int KG>
__device__ __forceinline__ void packed_dq_tile(const PackedP& p, char* smem) {
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
  const int first = 128 * f.t + 32 * w;
  const int R = min(first + r, rows - 1), tok = R / p.G, h = hk * p.G + R - tok * p.G, pos = tok + more;
  const bool live = first + r < rows;
  auto blocks = [&](int row) { return (max(min(row, rows - 1) / p.G + more + 1, 0) + 63) >> 6; };
  const int ntiles = blocks(128 * f.t + 127), wtiles = first < rows ? blocks(first + 31) : 0;
  const int first_pos = min(first, rows - 1) / p.G + more;
  const float c1 = p_factor(p.scale);

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
      const int row0 = kt * 64 + 32 * (sub & 1), left = min(s.m - row0, 32);  // rows behind the last arrive as zeros
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
  const int64_t qrow = (int64_t)(s.q0 + tok) * p.q_st + (int64_t)h * p.q_sh, yrow = (int64_t)(s.q0 + tok) * p.y_st + (int64_t)h * p.y_sh;
  bf16x8 qf[KS], gf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    qf[ks] = w_frag(p_signed(p_load8((const uint16_t*)p.Q + qrow, 16 * ks + 8 * hl, p.D), p.scale));
    gf[ks] = w_frag(p_load8((const uint16_t*)p.dY + yrow, 16 * ks + 8 * hl, pos >= 0 ? p.D : 0));  // (a row that sees no key may hold anything)
  }
  const float lse = p.lse[(int64_t)(h - p.lse_h0) * p.Tq + s.q0 + tok];
  const float nlse2 = lse == -INFINITY ? lse : -lse * LOG2E;  // no key: every probability is 0
  const float delta = p.delta[(int64_t)(h - p.delta_h0) * p.Tq + s.q0 + tok];
  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;

  // one 32-key half (K sub-tile KO bytes, V sub-tile VO bytes into LDS) of a tile
  auto half = [&](auto ko, auto vo, int k0, bool edge) {
    constexpr int KO = decltype(ko)::value, VO = decltype(vo)::value;
    f32x16 sa, pa;
    {
      u32x4 fk[KS], fv[KS];
      p_nat_issue<KO>(fk, ka);
      p_nat_issue<VO>(fv, ka);
      p_nat_wait(fk);
      p_nat_wait(fv);
#pragma unroll
      for (int v = 0; v < 16; ++v) { sa[v] = 0.f; pa[v] = 0.f; }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        sa = mfma(w_frag(fk[ks]), qf[ks], sa);
        pa = mfma(w_frag(fv[ks]), gf[ks], pa);
      }
    }
    u32x2 kt_[2][2 * DB];
    p_tr_issue<KO>(kt_, va);
    if (edge) {
#pragma unroll
      for (int v = 0; v < 16; ++v) sa[v] = k0 + key_of(v, hl) > pos ? -INFINITY : sa[v];
    }
    bf16x8 df[2];
    {
      float ds[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) ds[v] = fast_exp2(fmaf(sa[v], c1, nlse2)) * (pa[v] - delta);
      df[0] = pack8(&ds[0]);
      df[1] = pack8(&ds[8]);
    }
    p_tr_wait(kt_);
#pragma unroll
    for (int hb = 0; hb < 2; ++hb)
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] = mfma(w_frag2(kt_[hb][2 * db], kt_[hb][2 * db + 1]), df[hb], acc[db]);
  };
  auto step = [&](auto sb, int i) {
    constexpr int SB = decltype(sb)::value;
    const int kt = KG * i + kg;
    W_VMCNT(0);  // this wavefront's part of the tile has landed
    __builtin_amdgcn_s_barrier();  // ... everybody's; and everybody is done with the other buffer
    asm volatile("" ::: "memory");
    if (i + 1 < steps) fetch_tile(mine + (STAGE_B - SB), kt + KG);
    if (kt < wtiles) {
      const int k0 = kt * 64;
      const bool edge = k0 + 63 > first_pos;
      half(std::integral_constant<int, SB>{}, std::integral_constant<int, SB + 2 * T::SUB_B>{}, k0, edge);
      half(std::integral_constant<int, SB + T::SUB_B>{}, std::integral_constant<int, SB + 3 * T::SUB_B>{}, k0 + 32, edge);
    }
  };
  int i = 0;
  for (; i + 1 < steps; i += 2) {
    step(std::integral_constant<int, 0>{}, i);
    step(std::integral_constant<int, STAGE_B>{}, i + 1);
  }
  if (i < steps) step(std::integral_constant<int, 0>{}, i);
  if (KG == 2) {  // the second group's sums, through LDS
    float4* part = (float4*)smem + w * DB * 4 * 64 + lane;
    __syncthreads();
    if (kg == 1) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) part[(4 * db + g) * 64] = make_float4(acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]);
    }
    __syncthreads();
    if (kg == 1) return;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 x = part[(4 * db + g) * 64];
        acc[db][4 * g] += x.x;
        acc[db][4 * g + 1] += x.y;
        acc[db][4 * g + 2] += x.z;
        acc[db][4 * g + 3] += x.w;
      }
  }
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    uint2 o[4];
#pragma unroll
    for (int g = 0; g < 4; ++g)
      o[g] = pack4_bf16(acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3], p.scale);
    p_store_row32((uint16_t*)p.dQ + qrow, o, 32 * db, hl, live, p.D);
  }
}

template <int D, int KG>
__global__ __launch_bounds__(256 * KG, KG == 1 && D == 64 ? 3 : 2) void packed_dq_kernel(PackedP p) {
  __shared__ __attribute__((aligned(1024))) char smem[KG * 2 * 4 * PTile<D>::SUB_B];
  packed_dq_tile<D, KG>(p, smem);
}

}  // namespace

hipError_t launch_packed_dq(const PackedP& p, hipStream_t st) {
  const int g = (int)p_blocks(p_most_tiles(p, false, 7), p.h1 - p.h0);
  auto by_groups = [&](auto d) {
    if (p_two_groups(p)) packed_dq_kernel<d(), 2><<<g, 512, 0, st>>>(p);
    else packed_dq_kernel<d(), 1><<<g, 256, 0, st>>>(p);
  };
  if (p.D <= 64) by_groups(std::integral_constant<int, 64>{});
  else by_groups(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace ssa
