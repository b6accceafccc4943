// The order of tiles and the cutting of keys as the kernels' own functions have them (packed_tile.h, cache_cut.h), on the host.  What the kernels do
// with a lane for each sequence is a loop over the sequences here.  Reads questions from stdin, one a line.
#include <cstdio>
#include <vector>

#include "packed_tile.h"
#include "cache_cut.h"

using ssa::PackedSeq;

template <bool KEYS, int SH>
static void tiles(const std::vector<PackedSeq>& s, int G) {
  int total = 0, most = 0;
  for (auto& x : s) {
    total += ssa::p_tiles<KEYS, SH>(x, G);
    const int steps = ssa::p_steps<KEYS, SH>(x, G);
    if (steps > most) most = steps;
  }
  for (int rank = 0; rank < total; ++rank) {
    const int level = ssa::p_level(rank, most, [&](int L) {
      int n = 0;
      for (auto& x : s) n += ssa::p_at_least<KEYS, SH>(x, G, L);
      return n;
    });
    int left = rank;
    for (auto& x : s) left -= ssa::p_at_least<KEYS, SH>(x, G, level + 1);
    for (size_t b = 0; b < s.size(); ++b) {
      const int above = ssa::p_at_least<KEYS, SH>(s[b], G, level + 1), mine = ssa::p_at_least<KEYS, SH>(s[b], G, level) - above;
      if (left < mine) {
        std::printf("%zu %d ", b, ssa::p_number<KEYS>(ssa::p_tiles<KEYS, SH>(s[b], G), above, left));
        break;
      }
      left -= mine;
    }
  }
  std::printf("\n");
}

int main() {
  char what;
  while (std::scanf(" %c", &what) == 1) {
    if (what == 'p') {  // place: blocks, heads
      int blocks, HK;
      if (std::scanf("%d %d", &blocks, &HK) != 2) return 1;
      for (int b = 0; b < blocks; ++b) {
        const ssa::PPlace o = ssa::p_place_of(b, HK);
        std::printf("%d %d ", o.rank, o.head);
      }
      std::printf("\n");
    } else if (what == 't') {  // tiles: keys or rows, shift, group, sequences, n and m of each
      int keys, sh, G, n;
      if (std::scanf("%d %d %d %d", &keys, &sh, &G, &n) != 4) return 1;
      std::vector<PackedSeq> s(n);
      for (auto& x : s)
        if (std::scanf("%d %d", &x.n, &x.m) != 2) return 1;
      if (!keys) tiles<false, 7>(s, G);
      else if (sh == 5) tiles<true, 5>(s, G);
      else if (sh == 6) tiles<true, 6>(s, G);
      else tiles<true, 7>(s, G);
    } else if (what == 'c') {  // cut: whole, new tokens, group, keys -> rows need two kinds of units, units, runs
      int whole, n, G, len;
      if (std::scanf("%d %d %d %d", &whole, &n, &G, &len) != 4) return 1;
      std::printf("%d %d %d\n", (int)ssa::cut_many(n, G), ssa::cut_units(whole, n, G, len), ssa::cut_runs(n, G));
    } else if (what == 'e') {
      int least, total, pieces;
      if (std::scanf("%d %d %d", &least, &total, &pieces) != 3) return 1;
      std::printf("%d\n", ssa::cut_each(least, total, pieces));
    } else if (what == 's') {
      int piece, each, first;
      if (std::scanf("%d %d %d", &piece, &each, &first) != 3) return 1;
      std::printf("%d\n", ssa::part_slot(piece, each, first));
    }
  }
  return 0;
}
