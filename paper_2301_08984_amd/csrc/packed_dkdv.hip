// dK and dV of attention over packed sequences: a wavefront for each gradient, the probabilities handed over through LDS (the scheme
// of fast_kv128.hip).
//
// A work-group has eight wavefronts, four pairs.  The first of a pair forms S = Q K^T and P for 32 keys and 32 rows, hands P over in fp32 and
// adds dY^T P to dV; the second forms dP = dY V^T, takes P a step later, forms dS and adds Q^T dS to dK.  The rows that
// see the keys go by in steps of 32 (token, head) pairs, all G heads of a token one after the other, so that the sums over the heads
// are the accumulators' own, without atomics and in a fixed order.  Q and dY rows travel straight into a ring of LDS slots, one
// or two steps ahead, one barrier a step; the second wavefronts are a step behind the first ones.
//
// KB x RG: the pairs take KB blocks of 32 keys, and RG groups of them every RG-th step each; the groups' sums are added up
// through LDS at the end, in order.  With few keys and key heads a work-group of 128 keys walks far more rows than there are
// work-groups to fill the chip; the rows are then read by more work-groups.
//
// Measured: one document of 16384 tokens, 12 heads of 128, 1886 us, 870 TFLOP/s, bound by LDS and vector instructions between the products;
// 23 documents, 8192 tokens, 12 heads in groups of three: 60 us; 11 documents, 6007 tokens, 16 heads of 64 in groups of eight: 134 us,
// bound by the rows that a work-group walks one after the other.
#include "packed_tile.h"

#include <type_traits>

namespace ssa {
namespace {

template <int D, int RG>
struct KvLds {
  static constexpr int SLOTS = D * RG == 256 ? 3 : 4, AHEAD = SLOTS - 2;  // three where four do not fit
  static constexpr int PERIOD = SLOTS == 3 ? 6 : 4;                       // steps after which slots and P's two slots come round
  static constexpr int SLOT_B = 2 * PTile<D>::SUB_B, RING_B = SLOTS * SLOT_B;  // Q and dY rows of a step; of a group
  static constexpr int P_AT = RG * RING_B;         // two slots of P: 32 x 32 fp32 for each of the four pairs
  static constexpr int STAT = P_AT + 2 * 4 * 4096;  // of a group and step: -LSE (base 2) [32], Delta [32], last key seen [32]
  static constexpr int BYTES = STAT + RG * SLOTS * 384;
};

// rows of (token, head) pairs, a fixed number further on with every step
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

template <int D, int RG, bool DK>  // DK: the second wavefront of a pair
__device__ __forceinline__ void packed_kv_wave(const PackedP& p, char* smem, const PackedSeq& s, int tile, int hk, int part) {
  using T = PTile<D>;
  using L = KvLds<D, RG>;
  constexpr int KS = T::KS, DB = T::DB, KB = 4 / RG, TK = 32 * KB;
  constexpr int MATES = 8 / RG, NF = 2 * T::LOADS / MATES;  // wavefronts of a group; load instructions of one in a step
  constexpr int NR = NF > 1 ? NF / 2 : 1;                   // ... of Q and of dY (D = 64, one group: of one of them)
  const int lane = threadIdx.x & 63, r = lane & 31, hl = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kblock = (w & 3) % KB, group = (w & 3) / KB, mate = (DK ? KB : 0) + kblock;
  const int G = p.G, rows = s.n * G, more = s.m - s.n;
  const int k0 = tile * TK + 32 * kblock, key = k0 + r;
  const float c1 = p_factor(p.scale);
  const int tok0 = max(tile * TK - more, 0);  // the first token that sees the tile's first key
  const int from = tok0 < s.n ? tok0 * G / 32 : 0, all = tok0 < s.n ? (rows + 31) / 32 - from : 0;
  const int first = from + (int)((int64_t)all * part / p.parts), steps = from + (int)((int64_t)all * (part + 1) / p.parts) - first;  // this part's
  const int stop = min(rows, 32 * (first + steps));  // this part's rows end here
  const int n = (steps + RG - 1) / RG, row0 = 32 * (first + group);  // of a group; a group's step t begins at row row0 + 32 RG t
  const int dtok = 32 * RG / G, dg = 32 * RG % G;
  char* ring = smem + group * L::RING_B;

  const uint32_t qs2 = (uint32_t)p.q_st * 2u, qh2 = (uint32_t)p.q_sh * 2u, ys2 = (uint32_t)p.y_st * 2u, yh2 = (uint32_t)p.y_sh * 2u;
  const int64_t qbase = (int64_t)s.q0 * p.q_st + (int64_t)hk * G * p.q_sh, ybase = (int64_t)s.q0 * p.y_st + (int64_t)hk * G * p.y_sh;
  // this wavefront's load instructions: the group's instructions mate, mate + MATES, .., Q's before dY's
  RowWalk base, mine[NR], own;  // the step's first row (uniform), the rows this lane fetches, the row whose statistics it fetches
  uint32_t c16[NR];
  base.init(row0, G);
  own.init(row0 + r, G);
#pragma unroll
  for (int u = 0; u < NR; ++u) {
    const int rho = T::ROWS * ((mate + MATES * u) % T::LOADS) + lane / T::CHUNKS, chunk = (lane % T::CHUNKS) ^ p_sw<D>(rho);
    mine[u].init(row0 + rho, G);
    c16[u] = 8 * chunk < p.D ? 16u * (uint32_t)chunk : P_NOWHERE;
  }
  float pstat = 0.f;
  int pseen = 0;
  // the group's step t into its slot, in order (past the last step and the last row: zeros arrive); the statistics travel through registers of
  // one wavefront of each kind, asked for before the rows so that waiting for them leaves those under way
  auto fetch = [&](char* slot, int t) {
    const int left = stop - (row0 + 32 * RG * t);
    if (kblock == 0) {
      const bool there = r < left;
      const int64_t at = (int64_t)(hk * G + own.g - (DK ? p.delta_h0 : p.lse_h0)) * p.Tq + s.q0 + own.tok;
      pstat = there ? (DK ? p.delta : p.lse)[at] : (DK ? 0.f : -INFINITY);
      pseen = there ? own.tok + more : -1;
      own.step(G, dtok, dg);
    }
    const __amdgpu_buffer_rsrc_t rq = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint16_t*)p.Q + qbase + (int64_t)base.tok * p.q_st), 0, 0x7e000000, 0x00020000);
    const __amdgpu_buffer_rsrc_t ry = __builtin_amdgcn_make_buffer_rsrc((void*)((const uint16_t*)p.dY + ybase + (int64_t)base.tok * p.y_st), 0, 0x7e000000, 0x00020000);
    uint32_t oq[NR], oy[NR];
#pragma unroll
    for (int u = 0; u < NR; ++u) {
      const int rho = T::ROWS * ((mate + MATES * u) % T::LOADS) + lane / T::CHUNKS;
      const uint32_t dt = (uint32_t)(mine[u].tok - base.tok), g = (uint32_t)mine[u].g;
      const bool there = rho < left && mine[u].tok + more >= 0 && c16[u] != P_NOWHERE;  // (a row that sees no key may hold anything)
      oq[u] = there ? dt * qs2 + g * qh2 + c16[u] : P_NOWHERE;
      oy[u] = there ? dt * ys2 + g * yh2 + c16[u] : P_NOWHERE;
      mine[u].step(G, dtok, dg);
    }
    base.step(G, dtok, dg);
#pragma unroll
    for (int u = 0; u < NR; ++u)
      if (NF > 1 || !DK)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, (w_lds_void*)(slot + ((mate + MATES * u) % T::LOADS) * 1024), 16, oq[u], 0, 0, 0);
#pragma unroll
    for (int u = 0; u < NR; ++u)
      if (NF > 1 || DK)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ry, (w_lds_void*)(slot + T::SUB_B + ((mate + MATES * u) % T::LOADS) * 1024), 16, oy[u], 0, 0, 0);
  };
  const uint32_t lds0 = (uint32_t)(size_t)(w_lds_void*)smem;
  uint32_t ka[KS], va[2][DB];
  p_nat_addr<D>(ka, ring, r, hl);
  p_tr_addr<D>(va, ring, lane);
  const uint32_t pa_ = lds0 + L::P_AT + 4096u * (w & 3) + 16u * lane;
  const uint32_t stat0 = lds0 + L::STAT + (uint32_t)group * (L::SLOTS * 384) + (DK ? 128u : 0u);
  const uint32_t st_w = stat0 + 4u * r, st_r = stat0 + 16u * hl;
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
  a.init(row0, G);
  e.init(row0 + 31, G);
  // a step in slot SL, P in slot PS: S and dV, or dP and dK
  auto work = [&](auto slot, auto pslot) {
    constexpr int SL = decltype(slot)::value, SO = SL * L::SLOT_B, PO = 16384 * decltype(pslot)::value, TO = 384 * SL;
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
      if (DK) quads_issue<PO, 1024>(pr, pp);
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
                   : : "v"(pr[0]), "v"(pr[1]), "v"(pr[2]), "v"(pr[3]), "v"(pp), "n"(PO), "n"(PO + 1024), "n"(PO + 2048), "n"(PO + 3 * 1024)
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
  // Step t: its rows have landed for everybody and P of step t - 1 is there; the slots of step t + AHEAD and of P t are free.
  // The statistics of step t are in LDS: written a step before, or, if they were asked for one step ahead only, before the barrier.
  auto step = [&](auto number, int t) {
    constexpr int I = decltype(number)::value, SL = I % L::SLOTS;
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NF * (L::AHEAD - 1)) : "memory");
    if (L::AHEAD == 1) put_stat(std::integral_constant<int, SL>{});
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (L::AHEAD == 2) put_stat(std::integral_constant<int, (SL + 1) % L::SLOTS>{});
    fetch(ring + ((SL + L::AHEAD) % L::SLOTS) * L::SLOT_B, t + L::AHEAD);
    if (DK) {
      if (t > 0) work(std::integral_constant<int, (SL + L::SLOTS - 1) % L::SLOTS>{}, std::integral_constant<int, (I + 1) & 1>{});
    } else {
      if (t < n) work(std::integral_constant<int, SL>{}, std::integral_constant<int, I & 1>{});
    }
  };
  if (n > 0) {
    fetch(ring, 0);
    if (L::AHEAD == 2) {
      put_stat(std::integral_constant<int, 0>{});
      fetch(ring + L::SLOT_B, 1);
    }
    // (used here, so that the loop holds no wait for them)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(kr[ks]));
    for (int t = 0; t <= n; t += L::PERIOD) {
      step(std::integral_constant<int, 0>{}, t);
      if (t + 1 <= n) step(std::integral_constant<int, 1>{}, t + 1);
      if (t + 2 <= n) step(std::integral_constant<int, 2>{}, t + 2);
      if (t + 3 <= n) step(std::integral_constant<int, 3>{}, t + 3);
      if (L::PERIOD == 6) {
        if (t + 4 <= n) step(std::integral_constant<int, 4>{}, t + 4);
        if (t + 5 <= n) step(std::integral_constant<int, 5>{}, t + 5);
      }
    }
    W_VMCNT(0);  // nothing may still be on its way into LDS
    if (RG > 1) {
      // the other groups' sums, in the rings' place: a quarter of a block is 64 lanes x 16 bytes
      float4* part = (float4*)smem + ((((DK ? 1 : 0) * KB + kblock) * RG + group) * DB * 4) * 64 + lane;
      __syncthreads();
      if (group > 0) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g) part[(4 * db + g) * 64] = make_float4(acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]);
      }
      __syncthreads();
      if (group == 0) {
#pragma unroll
        for (int o = 1; o < RG; ++o)
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const float4 x = part[((o * DB + db) * 4 + g) * 64];
              acc[db][4 * g] += x.x;
              acc[db][4 * g + 1] += x.y;
              acc[db][4 * g + 2] += x.z;
              acc[db][4 * g + 3] += x.w;
            }
      }
    }
  }
  if (group > 0) return;
  if (p.parts > 1) {
    float* out = p.dkdv_parts + (((int64_t)(2 * part + (DK ? 1 : 0)) * p.Tk + s.k0 + min(key, s.m - 1)) * (p.h1 - p.h0) + hk - p.h0) * p.D;
    const float scale = DK ? p.scale : 1.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int col = 32 * db + 8 * g + 4 * hl;
        if (key < s.m && col < p.D)
          *(float4*)(out + col) = make_float4(acc[db][4 * g] * scale, acc[db][4 * g + 1] * scale, acc[db][4 * g + 2] * scale, acc[db][4 * g + 3] * scale);
      }
    return;
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

template <int D, int RG>
__global__ __launch_bounds__(512, 2) void packed_dkdv_kernel(PackedP p) {
  __shared__ __attribute__((aligned(1024))) char smem[KvLds<D, RG>::BYTES];
  static_assert(sizeof(smem) <= 160 * 1024 && (RG == 1 || 8 * 32 * D * 4 <= KvLds<D, RG>::STAT), "the groups' sums fit, too");
  const PPlace at = p_place((p.h1 - p.h0) * p.parts);
  const PFound f = p_find<true, RG == 1 ? 7 : RG == 2 ? 6 : 5>(p, at.rank);
  if (f.t < 0) return;
  const int head = at.head / p.parts, part = at.head - head * p.parts;
  if (__builtin_amdgcn_readfirstlane(threadIdx.x >> 8)) packed_kv_wave<D, RG, true>(p, smem, f.s, f.t, p.h0 + head, part);
  else packed_kv_wave<D, RG, false>(p, smem, f.s, f.t, p.h0 + head, part);
}

// The parts of dK and dV, added up in order: a wavefront per key row (of a sequence: other rows stay as they were).
__global__ __launch_bounds__(256) void packed_join_kernel(PackedP p) {
  const int lane = threadIdx.x & 63, t = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (t >= p.Tk || packed_owner(p.cu_k, p.n_seq, t) < 0) return;
  const int heads = p.h1 - p.h0, row = heads * p.D;  // values
  for (int i = 4 * lane; i < 2 * row; i += 256) {
    const bool dk = i >= row;
    const int at = dk ? i - row : i, h = at / p.D;
    const float* from = p.dkdv_parts + ((int64_t)(dk ? 1 : 0) * p.Tk + t) * row + at;
    float4 x = *(const float4*)from;
    for (int part = 1; part < p.parts; ++part) {
      const float4 y = *(const float4*)(from + (int64_t)2 * part * p.Tk * row);
      x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
    }
    *(uint2*)((uint16_t*)(dk ? p.dK : p.dV) + (int64_t)t * p.k_st + (int64_t)(p.h0 + h) * p.k_sh + (at - h * p.D)) = pack4_bf16(x.x, x.y, x.z, x.w, 1.f);
  }
}

template <int D, int RG>
hipError_t launch(const PackedP& p, hipStream_t st) {
  packed_dkdv_kernel<D, RG><<<(int)p_blocks(p_most_tiles(p, true, RG == 1 ? 7 : RG == 2 ? 6 : 5), (p.h1 - p.h0) * p.parts), 512, 0, st>>>(p);
  if (p.parts > 1) packed_join_kernel<<<(p.Tk + 3) / 4, 256, 0, st>>>(p);
  return hipGetLastError();
}

// Row groups of a work-group: more where there are few tiles of keys.  One | two | four, us: 8192 tokens, 23 documents, 12 heads in groups of three of 128,
// 86 | 60; one document of 16384, 12 heads, 1886 | 2147; 6007 tokens, 11 documents, 16 heads of 64 in groups of eight, 293 | 190 | 134.
// (Heads of 128 in four groups do not fit LDS.)
int row_groups(const PackedP& p) {
  const int64_t tiles = (int64_t)(p.Tk >> 7) * p.share_heads;
  if (p.D > 64) return tiles < 512 ? 2 : 1;
  return tiles < 256 ? 4 : tiles < 512 ? 2 : 1;
}

}  // namespace

// Where a launch has few work-groups and sequences are long, the longest of them, which walk most rows, keep the chip waiting: their rows
// are then cut into two parts, and into four or eight where the work-groups still leave most of the chip idle and a part has some ten steps.
// One part | two | four | eight, us, the backward: 6007 tokens x 16 heads of 64 in groups of eight, 11 documents (dK and dV alone) 214 | 138 | 158 | -;
// one sequence of 3000, 8 heads of 128 in one group, 484 | 284 | 182 | 134; 688 tokens, 16 heads in groups of four, 79 | 63 | 56 | 62; 1401 tokens,
// 16 heads in pairs, 93 | 81 | 96 | 131; 8 of 700 tokens, 12 heads in groups of three (45 MiB of sums), 104 | 125 | 156 | 217.
int packed_dkdv_parts(const PackedP& p) {
  const int rg = row_groups(p);
  const int64_t groups = ((int64_t)p.Tk * rg >> 7) * p.share_heads, rows = (int64_t)p.Tq * p.G / p.n_seq;
  auto fit = [&](int parts) { return (int64_t)2 * parts * p.Tk * p.share_heads * p.D * 4 <= (24 << 20); };  // (what their sums may add to the workspace; it keeps out, too, where the sums cost more than the parts give, as the last example above)
  if (groups >= 768 || rows < 2048 || !fit(2)) return 1;
  int parts = 2;
  while (parts < 8 && groups * parts < 256 && rows >= 1280 * parts && fit(2 * parts)) parts *= 2;
  return parts;
}

hipError_t launch_packed_dkdv(const PackedP& p, hipStream_t st) {
  const int rg = row_groups(p);
  if (p.D > 64) return rg == 2 ? launch<128, 2>(p, st) : launch<128, 1>(p, st);
  return rg == 4 ? launch<64, 4>(p, st) : rg == 2 ? launch<64, 2>(p, st) : launch<64, 1>(p, st);
}

}  // namespace ssa
