// Delta of attention over packed sequences, for its backward: Delta_i = sum_j P_ij dP_ij, and LSE too where the forward's was not kept.
//
// Delta_i is dY_i . Y_i as well, but Y is kept in bf16 (and P is rounded on its way into the product that makes it), and an error e of Delta_i is
// scale e sum_j P_ij k_j in dQ_i.  That does not shrink with the number of keys where K has a mean, and where one key has nearly all of a row's
// probability dS is small while its key is not: with 1 channel of 20 at a mean of 4 in K and 16 in V, rows of 512 keys, dQ was off by 8 % of its
// size, and with a first key that takes most of every row by 20 - 40 %, against 0.25 % from rounding dS.  So Delta comes from the scores and dP, in
// fp32 as the kernels that use it form them, one more walk over the keys; it is divided by the sum of the same probabilities, so that sum_j dS_ij is 0 to fp32.
//
// The tiles of 128 rows and the buffers of packed_fwd.hip, and its running maximum where LSE is not known; no product needs K or V
// transposed, and a row keeps three numbers in place of its output.
//
// Measured: one document of 16384 tokens, 12 heads of 128, 759 us, 1085 TFLOP/s (a large library product: 1216), bound by the matrix instructions of two
// products; 23 documents, 8192 tokens, 12 heads in groups of three, 30 us; 11 documents, 6007 tokens, 16 heads of 64 in groups of eight, with LSE, 57 us.
#include "packed_tile.h"

#include <type_traits>

namespace ssa {
namespace {

template <int D, bool KEPT, int KG>
__device__ __forceinline__ void packed_delta_tile(const PackedP& p, char* smem) {
  using T = PTile<D>;
  constexpr int KS = T::KS, U = T::LOADS / 4, STAGE_B = 4 * T::SUB_B;
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
  uint32_t ka[KS];
  p_nat_addr<D>(ka, mine, r, hl);

  const int steps = (ntiles + KG - 1) / KG;  // a group's step i is key tile KG i + kg
  if (steps > 0) fetch_tile(mine, kg);
  const int64_t qrow = (int64_t)(s.q0 + tok) * p.q_st + (int64_t)h * p.q_sh, yrow = (int64_t)(s.q0 + tok) * p.y_st + (int64_t)h * p.y_sh;
  bf16x8 qf[KS], gf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    qf[ks] = w_frag(p_signed(p_load8((const uint16_t*)p.Q + qrow, 16 * ks + 8 * hl, p.D), p.scale));
    gf[ks] = w_frag(p_load8((const uint16_t*)p.dY + yrow, 16 * ks + 8 * hl, p.D));
  }
  // exponents are taken from -off: the kept statistics, or this lane's maximum so far
  float off = 1e30f, l = 0.f, sum = 0.f;
  if (KEPT) {
    const float lse = p.lse[(int64_t)(h - p.lse_h0) * p.Tq + s.q0 + tok];
    off = lse == -INFINITY ? lse : -lse * LOG2E;  // no key: every probability is 0
  }

  auto arithmetic = [&](f32x16& sa, const f32x16& pa, int k0, bool edge) {
    if (edge) {
#pragma unroll
      for (int v = 0; v < 16; ++v) sa[v] = k0 + key_of(v, hl) > pos ? -INFINITY : sa[v];
    }
    if (!KEPT) {
      float rmax = sa[0];
#pragma unroll
      for (int v = 1; v < 16; ++v) rmax = fmaxf(rmax, sa[v]);
      const float now = fminf(off, -rmax * c1), alpha = fast_exp2(now - off);
      off = now;
      l *= alpha;
      sum *= alpha;
    }
    float pr[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) pr[v] = fast_exp2(fmaf(sa[v], c1, off));
    l += sum16(pr);
#pragma unroll
    for (int v = 0; v < 16; ++v) pr[v] *= pa[v];
    sum += sum16(pr);
  };
  auto products = [&](const u32x4 (&fk)[KS], const u32x4 (&fv)[KS], f32x16& sa, f32x16& pa) {
#pragma unroll
    for (int v = 0; v < 16; ++v) { sa[v] = 0.f; pa[v] = 0.f; }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      sa = mfma(w_frag(fk[ks]), qf[ks], sa);
      pa = mfma(w_frag(fv[ks]), gf[ks], pa);
    }
  };
  auto tile = [&](auto sb, int k0) {
    constexpr int SB = decltype(sb)::value;
    const bool edge = k0 + 63 > first_pos;  // (a row's keys end inside the sequence: this covers the keys behind its last, too)
    f32x16 sa, pa;
    u32x4 fk[KS], fv[KS];
    p_nat_issue<SB>(fk, ka);
    p_nat_issue<SB + 2 * T::SUB_B>(fv, ka);
    p_nat_wait(fk);
    p_nat_wait(fv);
    products(fk, fv, sa, pa);
    p_nat_issue<SB + T::SUB_B>(fk, ka);
    p_nat_issue<SB + 3 * T::SUB_B>(fv, ka);
    arithmetic(sa, pa, k0, edge);
    p_nat_wait(fk);
    p_nat_wait(fv);
    products(fk, fv, sa, pa);
    arithmetic(sa, pa, k0 + 32, edge);
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

  // the two halves of a wavefront have every other four keys of a row each, with a maximum of their own
  auto join = [&](float off1, float l1, float sum1) {
    const float both = fminf(off, off1), a0 = KEPT ? 1.f : fast_exp2(both - off), a1 = KEPT ? 1.f : fast_exp2(both - off1);
    off = both;
    l = fmaf(a1, l1, a0 * l);
    sum = fmaf(a1, sum1, a0 * sum);
  };
  join(__shfl_xor(off, 32), __shfl_xor(l, 32), __shfl_xor(sum, 32));
  if (KG == 2) {  // the second group's part, through LDS
    float* part = (float*)smem + 96 * w + r;
    __syncthreads();
    if (kg == 1 && hl == 0) {
      part[0] = off;
      part[32] = l;
      part[64] = sum;
    }
    __syncthreads();
    if (kg == 1) return;
    join(part[0], part[32], part[64]);
  }
  if (!live || hl) return;
  const int64_t stat = (int64_t)(s.q0 + tok);
  if (!KEPT) p.lse_out[(int64_t)(h - p.lse_h0) * p.Tq + stat] = l == 0.f ? -INFINITY : (log2f(l) - off) * LN2;
  p.delta_out[(int64_t)(h - p.delta_h0) * p.Tq + stat] = l == 0.f ? 0.f : sum / l;  // no key: 0; NaN stays
}

template <int D, bool KEPT, int KG>
__global__ __launch_bounds__(256 * KG, KG == 1 && D == 64 ? 3 : 2) void packed_delta_kernel(PackedP p) {
  __shared__ __attribute__((aligned(1024))) char smem[KG * 2 * 4 * PTile<D>::SUB_B];
  packed_delta_tile<D, KEPT, KG>(p, smem);
}

template <bool KEPT>
hipError_t launch(const PackedP& p, hipStream_t st) {
  const int g = (int)p_blocks(p_most_tiles(p, false, 7), p.h1 - p.h0);
  auto by_groups = [&](auto d) {
    if (p_two_groups(p)) packed_delta_kernel<d(), KEPT, 2><<<g, 512, 0, st>>>(p);
    else packed_delta_kernel<d(), KEPT, 1><<<g, 256, 0, st>>>(p);
  };
  if (p.D <= 64) by_groups(std::integral_constant<int, 64>{});
  else by_groups(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_delta(const PackedP& p, bool kept, hipStream_t st) { return kept ? launch<true>(p, st) : launch<false>(p, st); }

}  // namespace ssa
