// dK and dV of attention over packed sequences: a wavefront for each gradient, the probabilities handed over through LDS (the scheme
// of fast_kv128.hip).
//
// A work-group of eight wavefronts owns 128 keys of one key head.  Of the two wavefronts of a 32-key block the first forms S = Q K^T and P, hands P
// over in fp32 and adds dY^T P to dV; the second forms dP = dY V^T, takes P a step later, forms dS and adds Q^T dS to dK.
// The rows that see the keys go by in steps of 32 (token, head) pairs, all G heads of a token one after the other, so that the sums over the heads
// are the accumulators' own, without atomics and in a fixed order.  Q and dY rows travel straight into a ring of four LDS slots, two
// steps ahead, one barrier a step; the second wavefronts are a step behind the first ones.
#include "packed_tile.h"

#include <type_traits>

namespace ssa {
namespace {

template <int D>
struct KvLds {
  static constexpr int SLOTS = 4, SLOT_B = 2 * PTile<D>::SUB_B;  // Q and dY rows of a step
  static constexpr int P_AT = SLOTS * SLOT_B;                    // two slots of P: 32 x 32 fp32 for each of the four key blocks
  static constexpr int STAT = P_AT + 2 * 4 * 4096;               // of a step: -LSE (base 2) [32], Delta [32], last key seen [32]
  static constexpr int BYTES = STAT + SLOTS * 384;
};

// rows of (token, head) pairs, 32 further on with every step
struct RowWalk {
  int tok, g;
  __device__ __forceinline__ void init(int row, int G) {
    tok = row / G;
    g = row - tok * G;
  }
  __device__ __forceinline__ void step(int G, int dtok, int dg) {
    tok += dtok;
    g += dg;
    if (g >= G) {
      g -= G;
      ++tok;
    }
  }
};

template <int OFF, int STRIDE>
__device__ __forceinline__ void quads_issue(u32x4 (&f)[4], uint32_t at) {
  asm volatile("ds_read_b128 %0, %4 offset:%5\n\tds_read_b128 %1, %4 offset:%6\n\tds_read_b128 %2, %4 offset:%7\n\tds_read_b128 %3, %4 offset:%8"
               : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
               : "v"(at), "n"(OFF), "n"(OFF + STRIDE), "n"(OFF + 2 * STRIDE), "n"(OFF + 3 * STRIDE)
               : "memory");
}

template <int D, bool DK>  // DK: the second wavefront of a key block
__device__ __forceinline__ void packed_kv_wave(const PackedP& p, char* smem, const PackedSeq& s, int tile, int hk) {
  using T = PTile<D>;
  using L = KvLds<D>;
  constexpr int KS = T::KS, DB = T::DB, NF = D == 128 ? 2 : 1;  // load instructions of a wavefront and step
  const int lane = threadIdx.x & 63, r = lane & 31, hl = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kblock = w & 3;
  const int G = p.G, rows = s.n * G, more = s.m - s.n;
  const int k0 = tile * 128 + 32 * kblock, key = k0 + r;
  const float c1 = p_factor(p.scale);
  const int tok0 = max(tile * 128 - more, 0);  // the first token that sees the tile's first key
  const int first = tok0 < s.n ? tok0 * G / 32 : 0, n = tok0 < s.n ? (rows + 31) / 32 - first : 0;  // steps
  const int dtok = 32 / G, dg = 32 % G;

  // this wavefront's share of a step: D = 128: rows 4w .. 4w + 3 of Q and of dY; D = 64: rows 8 kblock .. + 7 of Q (first kind) or dY
  const uint32_t qs2 = (uint32_t)p.q_st * 2u, qh2 = (uint32_t)p.q_sh * 2u, ys2 = (uint32_t)p.y_st * 2u, yh2 = (uint32_t)p.y_sh * 2u;
  const int rho = T::ROWS * (D == 128 ? w : kblock) + lane / T::CHUNKS, chunk = (lane % T::CHUNKS) ^ p_sw<D>(rho);
  const bool column = 8 * chunk < p.D;
  const int64_t qbase = (int64_t)s.q0 * p.q_st + (int64_t)hk * G * p.q_sh, ybase = (int64_t)s.q0 * p.y_st + (int64_t)hk * G * p.y_sh;
  RowWalk base, mine, own;  // the step's first row (uniform), the row this lane fetches, the row whose statistics it fetches
  base.init(32 * first, G);
  mine.init(32 * first + rho, G);
  own.init(32 * first + r, G);
  float pstat = 0.f;
  int pseen = 0;
  // step t into its slot, in order (past the last step and the last row: zeros arrive); the statistics travel through registers of one
  // wavefront of each kind, asked for before the rows so that waiting for them leaves those under way
  auto fetch = [&](char* slot, int t) {
    const int left = rows - 32 * (first + t);
    if (kblock == 0) {
      const bool there = r < left;
      const int64_t at = (int64_t)(hk * G + own.g - (DK ? p.delta_h0 : p.lse_h0)) * p.Tq + s.q0 + own.tok;
      pstat = there ? (DK ? p.delta : p.lse)[at] : (DK ? 0.f : -INFINITY);
      pseen = there ? own.tok + more : -1;
      own.step(G, dtok, dg);
    }
    const uint32_t dt = (uint32_t)(mine.tok - base.tok);
    const bool there = column && rho < left;
    if (D == 128 || !DK) {
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint16_t*)p.Q + qbase + (int64_t)base.tok * p.q_st), 0, 0x7e000000, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (w_lds_void*)(slot + (D == 128 ? w : kblock) * 1024), 16,
                                               there ? dt * qs2 + (uint32_t)mine.g * qh2 + 16u * (uint32_t)chunk : P_NOWHERE, 0, 0, 0);
    }
    if (D == 128 || DK) {
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint16_t*)p.dY + ybase + (int64_t)base.tok * p.y_st), 0, 0x7e000000, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (w_lds_void*)(slot + T::SUB_B + (D == 128 ? w : kblock) * 1024), 16,
                                               there ? dt * ys2 + (uint32_t)mine.g * yh2 + 16u * (uint32_t)chunk : P_NOWHERE, 0, 0, 0);
    }
    base.step(G, dtok, dg);
    mine.step(G, dtok, dg);
  };
  const uint32_t lds0 = (uint32_t)(size_t)(w_lds_void*)smem;
  uint32_t ka[KS], va[2][DB];
  p_nat_addr<D>(ka, smem, r, hl);
  p_tr_addr<D>(va, smem, lane);
  const uint32_t pa_ = lds0 + L::P_AT + 4096u * kblock + 16u * lane;
  const uint32_t st_w = lds0 + L::STAT + (DK ? 128u : 0u) + 4u * r, st_r = lds0 + L::STAT + (DK ? 128u : 0u) + 16u * hl;
  auto put_stat = [&](auto slot) {
    constexpr int TO = 384 * decltype(slot)::value;
    const float x = DK || pstat == -INFINITY ? pstat : -pstat * LOG2E;  // a row without a key, or behind the last: its probabilities are 0
    const uint32_t to = st_w;
    const int last = pseen;
    if (kblock == 0) {
      asm volatile("ds_write_b32 %0, %1 offset:%2" ::"v"(to), "v"(x), "n"(TO) : "memory");
      if (!DK) asm volatile("ds_write_b32 %0, %1 offset:%2" ::"v"(to), "v"(last), "n"(TO + 256) : "memory");
    }
  };

  u32x4 kr[KS];  // of K, of V
  {
    const uint16_t* x = (const uint16_t*)(DK ? p.V : p.K) + (int64_t)(s.k0 + min(key, s.m - 1)) * p.k_st + (int64_t)hk * p.k_sh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4 y = p_load8(x, 16 * ks + 8 * hl, p.D);
      kr[ks] = DK ? y : p_signed(y, p.scale);
    }
  }
  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = 0.f;

  RowWalk a, e;  // the first and the last row of the step at work (uniform)
  a.init(32 * first, G);
  e.init(32 * first + 31, G);
  // step t: S and dV, or dP and dK of the step before
  auto work = [&](auto slot) {
    constexpr int SL = decltype(slot)::value, SO = SL * L::SLOT_B, PO = 16384 * (SL & 1), TO = 384 * SL;
    const int begin = a.tok + more, end = e.tok + more;
    const uint32_t pp = pa_;
    a.step(G, dtok, dg);
    e.step(G, dtok, dg);
    if (k0 >= s.m || end < k0) return;  // no visible pair for this key block
    f32x16 x;
#pragma unroll
    for (int v = 0; v < 16; ++v) x[v] = 0.f;
    u32x4 l4[4], pr[4];
    {
      u32x4 fr[KS];
      p_nat_issue<SO + (DK ? T::SUB_B : 0)>(fr, ka);
      quads_issue<TO, 32>(l4, st_r);
      if (DK) quads_issue<PO, 1024>(pr, pa_);
      p_nat_wait(fr);
      asm volatile("" : "+v"(l4[0]), "+v"(l4[1]), "+v"(l4[2]), "+v"(l4[3]));
      if (DK) asm volatile("" : "+v"(pr[0]), "+v"(pr[1]), "+v"(pr[2]), "+v"(pr[3]));
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) x = mfma(w_frag(fr[ks]), w_frag(kr[ks]), x);
    }
    if (!DK && begin < k0 + 31) {  // the diagonal
      u32x4 seen[4];
      quads_issue<TO + 256, 32>(seen, st_r);
      asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(seen[0]), "+v"(seen[1]), "+v"(seen[2]), "+v"(seen[3]) : : "memory");
#pragma unroll
      for (int v = 0; v < 16; ++v) x[v] = key > (int)seen[v >> 2][v & 3] ? -INFINITY : x[v];
    }
    // the transposed fragments of the second product arrive under the arithmetic
    u32x2 tf[2][2 * DB];
    p_tr_issue<SO + (DK ? 0 : T::SUB_B)>(tf, va);
    bf16x8 of[2];  // P or dS as packed operands
    float y[16];
    if (DK) {
#pragma unroll
      for (int v = 0; v < 16; ++v) y[v] = __uint_as_float(pr[v >> 2][v & 3]) * (x[v] - __uint_as_float(l4[v >> 2][v & 3]));
    } else {
#pragma unroll
      for (int v = 0; v < 16; ++v) y[v] = fast_exp2(fmaf(x[v], c1, __uint_as_float(l4[v >> 2][v & 3])));
#pragma unroll
      for (int g = 0; g < 4; ++g) pr[g] = u32x4{__float_as_uint(y[4 * g]), __float_as_uint(y[4 * g + 1]), __float_as_uint(y[4 * g + 2]), __float_as_uint(y[4 * g + 3])};
      asm volatile("ds_write_b128 %4, %0 offset:%5\n\tds_write_b128 %4, %1 offset:%6\n\tds_write_b128 %4, %2 offset:%7\n\t"
                   "ds_write_b128 %4, %3 offset:%8"
                   : : "v"(pr[0]), "v"(pr[1]), "v"(pr[2]), "v"(pr[3]), "v"(pp), "n"(PO), "n"(PO + 1024), "n"(PO + 2048), "n"(PO + 3072)
                   : "memory");
    }
    of[0] = pack8(&y[0]);
    of[1] = pack8(&y[8]);
    p_tr_wait(tf);
#pragma unroll
    for (int hb = 0; hb < 2; ++hb)
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] = mfma(w_frag2(tf[hb][2 * db], tf[hb][2 * db + 1]), of[hb], acc[db]);
  };
  // step t of the work-group: rows t have landed for everybody, P of step t - 1 is there, and slot t + 2 and P's slot t are free
  auto step = [&](auto slot, int t) {
    constexpr int SL = decltype(slot)::value;
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(NF) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    put_stat(std::integral_constant<int, (SL + 1) & 3>{});
    fetch(smem + ((SL + 2) & 3) * L::SLOT_B, t + 2);
    if (DK) {
      if (t > 0) work(std::integral_constant<int, (SL + 3) & 3>{});
    } else {
      if (t < n) work(slot);
    }
  };
  if (n > 0) {
    fetch(smem, 0);
    put_stat(std::integral_constant<int, 0>{});
    fetch(smem + L::SLOT_B, 1);
    // (used here, so that the loop holds no wait for them)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(kr[ks]));
    for (int t = 0; t <= n; t += 4) {
      step(std::integral_constant<int, 0>{}, t);
      if (t + 1 <= n) step(std::integral_constant<int, 1>{}, t + 1);
      if (t + 2 <= n) step(std::integral_constant<int, 2>{}, t + 2);
      if (t + 3 <= n) step(std::integral_constant<int, 3>{}, t + 3);
    }
    W_VMCNT(0);  // nothing may still be on its way into LDS when the work-group ends
  }
  uint16_t* out = (uint16_t*)(DK ? p.dK : p.dV) + (int64_t)(s.k0 + min(key, s.m - 1)) * p.k_st + (int64_t)hk * p.k_sh;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    uint2 o[4];
#pragma unroll
    for (int g = 0; g < 4; ++g)
      o[g] = pack4_bf16(acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3], DK ? p.scale : 1.f);
    p_store_row32(out, o, 32 * db, hl, key < s.m, p.D);
  }
}

template <int D>
__global__ __launch_bounds__(512, 2) void packed_dkdv_kernel(PackedP p) {
  __shared__ __attribute__((aligned(1024))) char smem[KvLds<D>::BYTES];
  const PPlace at = p_place(p.h1 - p.h0);
  const PFound f = p_find<true>(p, at.rank);
  if (f.t < 0) return;
  if (__builtin_amdgcn_readfirstlane(threadIdx.x >> 8)) packed_kv_wave<D, true>(p, smem, f.s, f.t, p.h0 + at.head);
  else packed_kv_wave<D, false>(p, smem, f.s, f.t, p.h0 + at.head);
}

}  // namespace

hipError_t launch_packed_dkdv(const PackedP& p, hipStream_t st) {
  const int g = (int)p_blocks(p_most_tiles(p, true), p.h1 - p.h0);
  if (p.D <= 64) packed_dkdv_kernel<64><<<g, 512, 0, st>>>(p);
  else packed_dkdv_kernel<128><<<g, 512, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace ssa
