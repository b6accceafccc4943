// Kernel-side view of the paged cache (include/ss_cache.h), the rule that finds a row in it, and the launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ssa {

struct CacheP {
  void *kc, *vc;    // codes [n_pages][HK][page][D]
  float *ks, *vs;   // scales [n_pages][HK][page]; NULL: bf16
  const int32_t* table;
  int n_pages, page, shift, HK, D, format, n_seq, max_pages;  // page = 1 << shift
};

// The pool's page that holds position `pos` of sequence b; -1: none.
#ifdef __HIPCC__
__host__ __device__
#endif
inline int cache_page(const int32_t* table, int n_pages, int shift, int max_pages, int b, int64_t pos) {
  if (pos < 0 || pos >> shift >= max_pages) return -1;
  const int page = table[(int64_t)b * max_pages + (pos >> shift)];
  return page >= 0 && page < n_pages ? page : -1;
}
// The row (of D codes, and of one scale) of head h and position `pos` in page `page`.
#ifdef __HIPCC__
__host__ __device__
#endif
inline int64_t cache_row(int page, int shift, int HK, int h, int64_t pos) {
  return (((int64_t)page * HK + h) << shift) + (pos & ((1 << shift) - 1));
}

// The keys of units at .. at + take - 1 of a run of `units` units of 1 << sh keys over `len` keys.  (The end of the last unit is not formed
// from the unit's number: at 2^31 - 1 keys it does not fit.)
struct CacheSpan { int begin, end; };
#ifdef __HIPCC__
__host__ __device__
#endif
inline CacheSpan cache_span(int at, int take, int units, int sh, int len) {
  return CacheSpan{at << sh, at + take == units ? len : (at + take) << sh};
}

struct CacheRowsP {  // write, read
  CacheP c;
  void *K, *V;  // bf16, packed tokens
  int64_t st, sh;
  const int32_t *cu, *start;
  int T;
  int groups;  // wavefronts of a token (cache_rows.hip)
};
hipError_t launch_cache_write(const CacheRowsP& p, hipStream_t st);
hipError_t launch_cache_read(const CacheRowsP& p, hipStream_t st);

struct CacheAttnP {
  CacheP c;
  const void* Q;
  void* Y;
  float* lse;
  const int32_t *cu, *lens;
  const uint64_t* tree;
  int64_t q_st, q_sh, y_st, y_sh;
  float scale;
  int T, H, G, max_new;
  char* ws;
  // how the work is cut (cache_cut.h): rows of a sequence and key head at most, and of a part; pieces, the shortest one, whether every run
  // is one; and where in the workspace, in floats, the parts' maxima and sums begin
  int max_rows, part_rows, pieces, least;
  bool whole;
  int64_t ml_at;
};
size_t cache_attn_bytes(const CacheAttnP& p);
hipError_t launch_cache_attn(const CacheAttnP& p, hipStream_t st);
hipError_t launch_cache_attn_rows(const CacheAttnP& p, int blocks, hipStream_t st);  // more than 32 rows

}  // namespace ssa
