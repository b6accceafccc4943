// What the kernels of attention over the cache share: which sequence and which of its parts a work-group takes, and codes as bf16.
#pragma once
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
// The parts of all sequences: a lane holds one, 64 at a time (up to 64 sequences: loaded once).
struct Slot {
  CacheSeq s;
  int b, part, parts;
};
struct Cut {
  const CacheAttnP& p;
  CacheSeq mine;  // of the first 64
  int chunk;      // keys of a part
  __device__ __forceinline__ Cut(const CacheAttnP& q) : p(q) {
    const int lane = threadIdx.x & 63;
    mine = lane_seq(p, lane);
    // Parts enough to fill the chip once (`p.parts` over all sequences), of p.least keys or more; where they would be long, half as long, down to
    // 1024 keys: the sequences' last parts then leave less of the chip idle than the second round's starts cost.  One round | two |
    // four, us: 64 sequences x 4000, 8 heads, e4m3, 137.6 | 125.6 | 124.5; 4 x 100000, int8, 227.0 | 173.0 | 190.8; 24 x 1500, 2 heads of 64 21.0 | 27.3 | 27.3.
    int64_t total = 0;  // in units of 128 keys: the sum of 64 sequences of 2^31 keys fits an int
    for (int b0 = 0; b0 < p.c.n_seq; b0 += 64) {
      const CacheSeq s = b0 ? lane_seq(p, b0 + lane) : mine;
      total += __builtin_amdgcn_readlane(scan64(s.n > 0 ? (s.len >> 7) + 1 : 0), 63);
    }
    const int64_t once = (total + p.parts - 1) / p.parts * 128;
    chunk = (int)max((int64_t)p.least, min(min(once, max((once + 255) / 256 * 128, (int64_t)1024)), (int64_t)0x7fffff80));
  }
  // the sequence of slot `slot`, and its part there; b = -1: fewer slots than that
  __device__ __forceinline__ Slot find(int slot) const {
    const int lane = threadIdx.x & 63;
    Slot f;
    f.b = -1;
    for (int b0 = 0; b0 < p.c.n_seq; b0 += 64) {
      const CacheSeq s = b0 ? lane_seq(p, b0 + lane) : mine;
      const int n = parts_of(s, chunk), upto = scan64(n), all = __builtin_amdgcn_readlane(upto, 63);
      if (slot >= all) {
        slot -= all;
        continue;
      }
      const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > slot));
      take(f, s, b0, l, n);
      f.part = slot - (__builtin_amdgcn_readlane(upto, l) - f.parts);
      return f;
    }
    return f;
  }
  // the sequence of token t; `part`: the first of its slots
  __device__ __forceinline__ Slot owner(int t) const {
    const int lane = threadIdx.x & 63;
    Slot f;
    f.b = -1;
    int before = 0;
    for (int b0 = 0; b0 < p.c.n_seq; b0 += 64) {
      const CacheSeq s = b0 ? lane_seq(p, b0 + lane) : mine;
      const int n = parts_of(s, chunk), upto = scan64(n);
      const uint64_t hit = __builtin_amdgcn_ballot_w64(s.q0 <= t && t - s.q0 < s.n);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        take(f, s, b0, l, n);
        f.part = before + __builtin_amdgcn_readlane(upto, l) - f.parts;
        return f;
      }
      before += __builtin_amdgcn_readlane(upto, 63);
    }
    return f;
  }

 private:
  __device__ __forceinline__ static void take(Slot& f, const CacheSeq& s, int b0, int l, int n) {
    f.s.q0 = __builtin_amdgcn_readlane(s.q0, l);
    f.s.n = __builtin_amdgcn_readlane(s.n, l);
    f.s.before = __builtin_amdgcn_readlane(s.before, l);
    f.s.len = __builtin_amdgcn_readlane(s.len, l);
    f.b = b0 + l;
    f.parts = __builtin_amdgcn_readlane(n, l);
  }
};

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
