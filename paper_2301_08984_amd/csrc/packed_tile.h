// What the kernels of attention over packed sequences share: LDS images for head sizes of up to 64 and 128, and the
// order in which work-groups take tiles.
//
// Rows.  The G query heads of a key head see the same keys, so a tile is 128 consecutive rows of (token, head) pairs, row
// R of a sequence being head R % G of token R / G: any G fills the matrix instructions, a K / V tile is shared by
// 128 rows whatever G is, and the rows of a tile, spanning 128 / G tokens, end at nearly the same key (with a tile of 128 tokens of
// one head half of the diagonal's tiles are wasted).
//
// LDS images are those of wave_dma.h, with rows of 2 D bytes: chunk c (16 bytes) of row rho sits at position c ^ sw(rho), so that 16
// consecutive rows put one chunk, and 4 consecutive rows a 64-byte group of chunks, into different banks.  Two rows of 128 bytes
// fill the banks once, hence another swizzle for D = 64.  A head size between the two is padded with zeros: its missing
// chunks are fetched from behind the end of the buffer.
#pragma once
#include "packed.h"
#include "wave_dma.h"
#include "wave_scan.h"

namespace ssa {
namespace {

constexpr uint32_t P_NOWHERE = 0x7f000000u;  // a lane offset behind the end of every buffer: zeros arrive

template <int D>
__device__ __forceinline__ int p_sw(int row) {
  return D == 128 ? w_sw(row) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
}
template <int D>
struct PTile {
  static constexpr int ROW_B = 2 * D, SUB_B = 32 * ROW_B;  // bytes of a row and of a sub-tile of 32 rows
  static constexpr int LOADS = SUB_B / 1024, CHUNKS = D / 8, ROWS = 32 / LOADS;  // load instructions of a sub-tile, rows of one
  static constexpr int KS = D / 16, DB = D / 32;
};
template <int D>
__device__ __forceinline__ void p_nat_addr(uint32_t (&ka)[D / 16], const char* tile0, int r, int hl) {
  const uint32_t a0 = (uint32_t)(size_t)(w_lds_void*)tile0 + (uint32_t)r * (2 * D) + (uint32_t)((hl ^ p_sw<D>(r)) << 4);
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) ka[ks] = a0 ^ (uint32_t)(ks << 5);
}
// see w_tr_addr: va[half][db] for rows 0 .. 15, rows 16 .. 31 are 16 rows further on
template <int D>
__device__ __forceinline__ void p_tr_addr(uint32_t (&va)[2][D / 32], const char* tile0, int lane) {
  const int i = lane & 15, bk = lane >> 4;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int row = 8 * half + 4 * (bk >> 1) + (i >> 2);
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
      va[half][db] = (uint32_t)(size_t)(w_lds_void*)tile0 + (uint32_t)row * (2 * D) +
                     (uint32_t)(((4 * db + 2 * (bk & 1) + ((i & 3) >> 1)) ^ p_sw<D>(row)) << 4) + 8u * (i & 1);
  }
}
template <int OFF>
__device__ __forceinline__ void p_nat_issue(u32x4 (&f)[8], const uint32_t (&ka)[8]) { w_nat_issue<OFF>(f, ka); }
template <int OFF>
__device__ __forceinline__ void p_nat_issue(u32x4 (&f)[4], const uint32_t (&ka)[4]) {
  asm volatile("ds_read_b128 %0, %4 offset:%8\n\tds_read_b128 %1, %5 offset:%8\n\tds_read_b128 %2, %6 offset:%8\n\tds_read_b128 %3, %7 offset:%8"
               : "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
               : "v"(ka[0]), "v"(ka[1]), "v"(ka[2]), "v"(ka[3]), "n"(OFF)
               : "memory");
}
__device__ __forceinline__ void p_nat_wait(u32x4 (&f)[8]) { w_nat_wait(f); }
__device__ __forceinline__ void p_nat_wait(u32x4 (&f)[4]) {
  asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3]) : : "memory");
}
template <int OFF>
__device__ __forceinline__ void p_tr_issue(u32x2 (&f)[2][8], const uint32_t (&va)[2][4]) { w_tr_issue<OFF>(f, va); }
template <int OFF>
__device__ __forceinline__ void p_tr_issue(u32x2 (&f)[2][4], const uint32_t (&va)[2][2]) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    if (t == 0)
      asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%8\n\tds_read_b64_tr_b16 %1, %5 offset:%8\n\tds_read_b64_tr_b16 %2, %6 offset:%8\n\t"
                   "ds_read_b64_tr_b16 %3, %7 offset:%8"
                   : "=&v"(f[0][0]), "=&v"(f[0][1]), "=&v"(f[0][2]), "=&v"(f[0][3])
                   : "v"(va[0][0]), "v"(va[1][0]), "v"(va[0][1]), "v"(va[1][1]), "n"(OFF)
                   : "memory");
    else
      asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%8\n\tds_read_b64_tr_b16 %1, %5 offset:%8\n\tds_read_b64_tr_b16 %2, %6 offset:%8\n\t"
                   "ds_read_b64_tr_b16 %3, %7 offset:%8"
                   : "=&v"(f[1][0]), "=&v"(f[1][1]), "=&v"(f[1][2]), "=&v"(f[1][3])
                   : "v"(va[0][0]), "v"(va[1][0]), "v"(va[0][1]), "v"(va[1][1]), "n"(OFF + 2048)
                   : "memory");
  }
}
__device__ __forceinline__ void p_tr_wait(u32x2 (&f)[2][8]) { w_tr_wait(f); }
__device__ __forceinline__ void p_tr_wait(u32x2 (&f)[2][4]) {
  asm volatile("s_waitcnt lgkmcnt(0)"
               : "+v"(f[0][0]), "+v"(f[0][1]), "+v"(f[0][2]), "+v"(f[0][3]), "+v"(f[1][0]), "+v"(f[1][1]), "+v"(f[1][2]), "+v"(f[1][3])
               :
               : "memory");
}
// store_row32 of the columns below D
__device__ __forceinline__ void p_store_row32(uint16_t* row_ptr, const uint2 (&a)[4], int col, int hl, bool live, int D) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    auto s = __builtin_amdgcn_permlane32_swap(a[2 * j].x, a[2 * j + 1].x, false, false);
    auto t = __builtin_amdgcn_permlane32_swap(a[2 * j].y, a[2 * j + 1].y, false, false);
    const int at = col + 8 * (2 * j + hl);
    if (live && at < D) *(u32x4*)(row_ptr + at) = u32x4{s[0], t[0], s[1], t[1]};
  }
}
// eight columns from `col` on of a row, zeros behind its D columns
__device__ __forceinline__ u32x4 p_load8(const uint16_t* row_ptr, int col, int D) {
  return col < D ? *(const u32x4*)(row_ptr + col) : u32x4{0, 0, 0, 0};
}

__device__ __forceinline__ int p_max(int x) {  // of the wavefront's non-negative numbers
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ int p_total(int x) { return __builtin_amdgcn_readlane(scan64(x), 63); }

// A launch's work-groups: 8 XCDs with an L2 each are dealt them in turn.  Every XCD gets HK / 8 whole key heads, whose K and V
// stay in its L2; of the heads left over 4, 2 and 1 at a time are spread over 2, 4 or 8 XCDs by the rank of their tiles.  Tiles go
// by rank (the heaviest first), the heads of one rank next to each other.
struct PPlace { int rank, head; };
__host__ __device__ __forceinline__ PPlace p_place_of(int block, int HK) {
  const int x = block & 7, idx = block >> 3, q = idx / HK, a = HK >> 3;
  int rem = idx - q * HK;
  PPlace o;
  if (rem < 8 * a) {
    o.rank = rem / a;
    o.head = x * a + (rem - o.rank * a);
    o.rank += 8 * q;
    return o;
  }
  rem -= 8 * a;
  int first = 8 * a;
  if (HK & 4) {
    if (rem < 4) return PPlace{8 * q + 2 * rem + (x & 1), first + (x >> 1)};
    rem -= 4;
    first += 4;
  }
  if (HK & 2) {
    if (rem < 2) return PPlace{8 * q + 4 * rem + (x & 3), first + (x >> 2)};
    first += 2;
  }
  return PPlace{8 * q + x, first};
}
__device__ __forceinline__ PPlace p_place(int HK) { return p_place_of((int)blockIdx.x, HK); }
inline int64_t p_blocks(int64_t tiles, int HK) { return (tiles + 7) / 8 * 8 * HK; }

// The tile of rank `rank`: its sequence, and its number in it (-1: fewer tiles than that).  KEYS: tiles of 1 << SH keys, else of 1 << SH
// rows.  What a tile costs is the number of its steps: blocks of 64 keys that a tile of rows walks, or of 32 rows that a tile of
// keys walks.  Up to 64 sequences (a lane each) the tiles are ranked by it, the longest first, so that the chip does not wait for a long one
// that started last: the number of tiles with at least L steps has a closed form for a sequence, and L is found by
// bisection.  With more sequences tiles are in the order of the sequences.
struct PFound { PackedSeq s; int t; };
template <bool KEYS, int SH>
__host__ __device__ __forceinline__ int p_tiles(const PackedSeq& s, int G) { return ((KEYS ? s.m : s.n * G) + (1 << SH) - 1) >> SH; }
template <bool KEYS, int SH>
__host__ __device__ __forceinline__ int p_steps(const PackedSeq& s, int G) {  // of the sequence's heaviest tile
  return KEYS ? (s.n * G + 31) >> 5 : (s.m + 63) >> 6;
}
template <bool KEYS, int SH>
__host__ __device__ __forceinline__ int p_at_least(const PackedSeq& s, int G, int L) {  // tiles with L steps or more
  const int tiles = p_tiles<KEYS, SH>(s, G), more = s.m - s.n;
  if (L <= 0) return tiles;
  if (KEYS) {
    const int z = s.n - 1 - (32 * (L - 1)) / G;  // the last first token that leaves as many rows
    return z < 0 || z + more < 0 ? 0 : min(tiles, ((z + more) >> SH) + 1);
  }
  const int y = 64 * (L - 1) - more;  // the first token that sees as many keys
  return y >= s.n ? 0 : tiles - ((max(y, 0) * G) >> SH);
}
// The steps of the tile of rank `rank` when they are in order of their steps, at most `most` (count(L): tiles with L steps or more): more than `rank` tiles
// have that many or more, not as many have more.
template <typename Count>
__host__ __device__ __forceinline__ int p_level(int rank, int most, Count&& count) {
  int lo = 0, hi = most + 1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (count(mid) > rank) lo = mid;
    else hi = mid;
  }
  return lo;
}
// The number in its sequence of `tiles` tiles of the i-th tile with exactly some number of steps, when `above` have more: a sequence's first tiles of
// keys, and its last tiles of rows, have most steps.
template <bool KEYS>
__host__ __device__ __forceinline__ int p_number(int tiles, int above, int i) { return KEYS ? above + i : tiles - 1 - above - i; }
template <bool KEYS, int SH>
__device__ __forceinline__ PFound p_find(const PackedP& p, int rank) {
  const int lane = threadIdx.x & 63, G = p.G;
  PFound f;
  f.t = -1;
  auto of_lane = [&](int b0) {
    PackedSeq s = packed_seq(p, min(b0 + lane, p.n_seq - 1));
    if (b0 + lane >= p.n_seq) s.n = s.m = 0;
    return s;
  };
  auto from = [&](const PackedSeq& s, int l) {
    f.s.q0 = __builtin_amdgcn_readlane(s.q0, l);
    f.s.n = __builtin_amdgcn_readlane(s.n, l);
    f.s.k0 = __builtin_amdgcn_readlane(s.k0, l);
    f.s.m = __builtin_amdgcn_readlane(s.m, l);
  };
  if (p.n_seq <= 64) {
    const PackedSeq s = of_lane(0);
    if (rank >= p_total(p_tiles<KEYS, SH>(s, G))) return f;
    const int level = p_level(rank, p_max(p_steps<KEYS, SH>(s, G)), [&](int L) { return p_total(p_at_least<KEYS, SH>(s, G, L)); });
    const int above = p_at_least<KEYS, SH>(s, G, level + 1), mine = p_at_least<KEYS, SH>(s, G, level) - above;
    const int left = rank - p_total(above), upto = scan64(mine);
    const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > left));
    from(s, l);
    const int i = left - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l)), ab = __builtin_amdgcn_readlane(above, l);
    f.t = p_number<KEYS>(p_tiles<KEYS, SH>(f.s, G), ab, i);
    return f;
  }
  for (int b0 = 0; b0 < p.n_seq; b0 += 64) {
    const PackedSeq s = of_lane(b0);
    const int mine = p_tiles<KEYS, SH>(s, G), upto = scan64(mine), all = __builtin_amdgcn_readlane(upto, 63);
    if (rank >= all) {
      rank -= all;
      continue;
    }
    const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > rank));
    from(s, l);
    const int i = rank - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l));
    f.t = p_number<KEYS>(p_tiles<KEYS, SH>(f.s, G), 0, i);
    return f;
  }
  return f;
}
// (row tiles: 128 * tiles <= Tq * G + 127 * n_seq; key tiles alike)
inline int64_t p_most_tiles(const PackedP& p, bool keys, int sh) { return ((keys ? (int64_t)p.Tk : (int64_t)p.Tq * p.G) >> sh) + p.n_seq; }

// Two groups of wavefronts share a tile of rows where the longest tile is what a launch lasts: it then takes half as long.  They cost a join at the end,
// and one work-group fits a compute unit where two of one group do, so there have to be at most as many tiles as the chip holds of one group (512; heads of 64:
// more, but their backward has the registers of 256 to 768), and tiles have to be long, which is known of the mean sequence only.  One group | two, us, the forward (the
// backward and heads of 64 turn at the same places), 32 heads in groups of four unless said otherwise, tiles x heads first:
//   64: 2 sequences of 128 tokens 8.4 | 9.4, 1 of 512 (16 heads on 2) 15.2 | 14.2; 200: 5 of 160 10.1 | 11.4, 2 of 400 13.5 | 13.3, 1 of 1600 (16 on 2) 33.7 | 28.1
//   256: 3 of 341 13.6 | 17.2, 1 of 1024 24.6 | 21.9; 320: 2 of 640 19.7 | 20.1, 1 of 1280 30.2 | 25.3; 400: 2 of 800 23.8 | 25.0, 1 of 1600 37.4 | 33.5
//   512: 3 of 682 23.6 | 33.7, 1 of 2048 49.5 | 45.7; 600: 2 of 2400 (16 on 2) 59.8 | 65.8; 768: 2 of 1536 51.5 | 58.8
// (11 documents of up to 3300 tokens, 16 heads of 64 in groups of eight, 750 tiles, one group by this rule: Delta 57.7 | 58.2, dQ 67.5 | 66.5; of up to 2300: forward 38.0 | 31.2.)
inline bool p_two_groups(const PackedP& p) {
  const int64_t tiles = (((int64_t)p.Tq * p.G) >> 7) * p.share_heads, keys = p.Tk / p.n_seq;
  return tiles < 256 ? keys >= 400 : tiles <= 512 && keys >= 3 * tiles;
}

// 1 / ln 2 times the scale, never zero: a factor of 0 would make NaN of a masked score; any score times 2^-120 is 0
// next to the exponents that matter.  Its sign goes into Q.
__device__ __forceinline__ float p_factor(float scale) { return fmaxf(fabsf(scale) * LOG2E, 0x1p-120f); }
__device__ __forceinline__ u32x4 p_signed(u32x4 x, float scale) {
  const uint32_t flip = scale < 0.f ? 0x80008000u : 0u;
  return u32x4{x[0] ^ flip, x[1] ^ flip, x[2] ^ flip, x[3] ^ flip};
}

}  // namespace
}  // namespace ssa
