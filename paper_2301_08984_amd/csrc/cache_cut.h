// What the kernels of attention over the cache share: which sequence and which of its parts a work-group takes, and codes as bf16.
#pragma once
#include "cache.h"
#include "mfma_common.h"
#include "wave_scan.h"

namespace ssa {
namespace {

enum { BF = 0, F8 = 1, I8 = 2 };

// What one sequence has: its new tokens' rows, the keys before them and in all.
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

// How the work is cut.  All keys of all sequences, for one key head, are one line of units, a unit being 128 keys (64 where a sequence has
// more than 64 rows, which take twice as long; those go over the keys once for every 128 rows).  The line is dealt out in equal pieces of
// `each` units to as many work-groups as the chip holds: they all end at the same time, however the lengths are spread.  A piece
// may end in the middle of a sequence, whose parts are then joined by a second launch, and may hold several sequences one after the
// other.  (Equal parts of every sequence, with as many work-groups, against this, us: 64 conversations, 256000 keys, 8 key
// heads, e4m3, 125 | 112; 4 of 400012 keys together, int8, 172 | 162; 16 trees over 48016 keys 95 | 75.)
// Where no sequence has room for more than 512 keys, every run over the keys is a piece and nothing is joined.
struct Run {  // over the keys of one sequence, for its rows of group `group`
  CacheSeq s;
  int b, group, first, units, at;  // `first`: its first unit on the line; `units` it has; `at`: the unit asked for, from there
};
__host__ __device__ __forceinline__ bool cut_many(int n, int G) { return n * G > 64; }
// units of one run of a sequence with n new tokens and len keys, and its runs
__host__ __device__ __forceinline__ int cut_units(bool whole, int n, int G, int len) {
  return whole || len <= 0 ? 1 : ((len - 1) >> (cut_many(n, G) ? 6 : 7)) + 1;
}
__host__ __device__ __forceinline__ int cut_runs(int n, int G) { return n <= 0 ? 0 : cut_many(n, G) ? (n * G + 127) >> 7 : 1; }
__host__ __device__ __forceinline__ int cut_each(int least, int total, int pieces) {
  const int even = (total + pieces - 1) / pieces;
  return even > least ? even : least;
}
struct Cut {
  const CacheAttnP& p;
  CacheSeq mine;     // of the first 64 sequences, a lane each
  int total, each;
  __device__ __forceinline__ Cut(const CacheAttnP& q) : p(q), total(0) {
    const int lane = threadIdx.x & 63;
    mine = at_lane(lane);
    for (int b0 = 0; b0 < p.c.n_seq; b0 += 64) total += __builtin_amdgcn_readlane(scan64(line(b0 ? at_lane(b0 + lane) : mine)), 63);
    each = cut_each(p.least, total, p.pieces);
  }
  __device__ __forceinline__ static bool many(const CacheAttnP& p, int n) { return cut_many(n, p.G); }
  __device__ __forceinline__ int units(const CacheSeq& s) const { return cut_units(p.whole, s.n, p.G, s.len); }  // of one run
  __device__ __forceinline__ int line(const CacheSeq& s) const { return units(s) * cut_runs(s.n, p.G); }
  __device__ __forceinline__ CacheSeq at_lane(int b) const {
    CacheSeq s = cache_seq(p, min(b, p.c.n_seq - 1));
    if (b >= p.c.n_seq) s.n = s.len = 0;
    return s;
  }
  // the run that holds unit `u` < total of the line
  __device__ __forceinline__ Run find(int u) const {
    Run f;
    f.b = -1;
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int b0 = 0; b0 < p.c.n_seq; b0 += 64) {
      const CacheSeq s = b0 ? at_lane(b0 + lane) : mine;
      const int n = line(s), upto = scan64(n);
      const uint64_t hit = __builtin_amdgcn_ballot_w64(u - before < upto);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        take(f, s, b0, l);
        const int off = u - before - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(n, l));
        f.group = off / f.units;
        f.at = off - f.group * f.units;
        f.first = u - f.at;
        return f;
      }
      before += __builtin_amdgcn_readlane(upto, 63);
    }
    return f;
  }
  // the first run of token t's sequence; b = -1: a token of none, or behind the last that counts
  __device__ __forceinline__ Run owner(int t) const {
    Run f;
    f.b = -1;
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int b0 = 0; b0 < p.c.n_seq; b0 += 64) {
      const CacheSeq s = b0 ? at_lane(b0 + lane) : mine;
      const int upto = scan64(line(s));
      const uint64_t hit = __builtin_amdgcn_ballot_w64(s.q0 <= t && t - s.q0 < s.n);
      if (hit) {
        take(f, s, b0, __builtin_ctzll(hit));
        f.first = before + __builtin_amdgcn_readlane(upto, __builtin_ctzll(hit)) - line(f.s);
        return f;
      }
      before += __builtin_amdgcn_readlane(upto, 63);
    }
    return f;
  }

 private:
  __device__ __forceinline__ void take(Run& f, const CacheSeq& s, int b0, int l) const {
    f.s.q0 = __builtin_amdgcn_readlane(s.q0, l);
    f.s.n = __builtin_amdgcn_readlane(s.n, l);
    f.s.before = __builtin_amdgcn_readlane(s.before, l);
    f.s.len = __builtin_amdgcn_readlane(s.len, l);
    f.b = b0 + l;
    f.units = units(f.s);
    f.group = f.at = 0;
  }
};
// A piece's first run may have begun in an earlier piece, its last one may go on in the next: two slots for parts a piece.
__host__ __device__ __forceinline__ int part_slot(int piece, int each, int first) { return 2 * piece + (first > piece * each ? 1 : 0); }
// where a part's row lies in the workspace, in rows
__host__ __device__ __forceinline__ int64_t part_row(const CacheAttnP& p, int slot, int hk, int row) {
  return ((int64_t)slot * p.c.HK + hk) * p.part_rows + row;
}

// two 8-bit codes (bytes 2 HI and 2 HI + 1) as packed bf16, exactly
template <int FMT, bool HI>
__device__ __forceinline__ uint32_t two_codes(uint32_t x) {
  if (FMT == F8) {
    union { bf16x2 v; uint32_t u; } o;
    o.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, HI);
    return o.u;
  }
  const uint32_t u = x ^ 0x80808080u;
  return pack2_bf16((float)(uint8_t)(u >> (HI ? 16 : 0)) - 128.f, (float)(uint8_t)(u >> (HI ? 24 : 8)) - 128.f);
}

}  // namespace
}  // namespace ssa
