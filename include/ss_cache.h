/* ss_cache.h -- C ABI of a paged cache of keys and values, and of attention over it, for MI355X (gfx950).
 *
 * The cache of one layer is a pool of pages of `page` tokens for HK key / value heads.  The table says which pages
 * hold a sequence: token `pos` of sequence b lies in slot pos % page of page table[b][pos / page].  A row (one token
 * of one head, D values) is kept as bf16, or in 8 bits with one fp32 scale, K and V apart:
 *
 *   SS_CACHE_FP8  codes in e4m3 (finite, largest 448); scale = the smallest power of two s >= 2^-126 with
 *                 max |x| <= 448 s.  A power of two, so that neither x / s nor the product that is read back is
 *                 rounded: what the format loses is the code's own rounding, at most max(2^-4 |x|, 2^-10 scale) (below
 *                 2^-6 scale codes are subnormal: steps of 2^-9 scale).
 *   SS_CACHE_INT8 codes -127 .. 127; scale = max(max |x| / 127, 2^-126).
 *   code = round to nearest even of x / scale (the quotient in fp32); value = code * scale.
 *   A row of zeros has scale 1.  A row that holds a NaN or an infinity gets a scale of NaN, so that it shows.
 *
 * Layout: codes [n_pages][HK][page][D] in the format's element, scales float [n_pages][HK][page].
 *
 * The table and the lengths are DEVICE memory and may change from call to call without the host's knowledge (a
 * captured step replays over longer and longer contexts).  A table entry outside 0 .. n_pages-1, and a position outside
 * 0 .. max_pages*page-1, stand for rows that are not there: they are not written, are read back as zeros, and no
 * query sees them.  All pointers are DEVICE pointers, descriptors and size outputs HOST memory; no call allocates,
 * synchronises or keeps state.  Error codes are those of ss_attn.h.
 */
#ifndef SS_CACHE_H
#define SS_CACHE_H

#include <stddef.h>
#include <stdint.h>

#include "ss_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SS_CACHE_BF16 = 0, SS_CACHE_FP8 = 1, SS_CACHE_INT8 = 2 } ss_cache_format;

typedef struct {
  int32_t n_pages;   /* pages of the pool                                  */
  int32_t page;      /* tokens of a page: a power of two, 8 .. 1024        */
  int32_t HK, D;     /* key / value heads, head size (64 or 128)           */
  int32_t format;    /* ss_cache_format                                    */
  int32_t n_seq;     /* sequences of the table                             */
  int32_t max_pages; /* entries of a line of the table; max_pages*page < 2^31 */
} ss_cache_desc;

/* Bytes of one code array and of one scale array (0 for SS_CACHE_BF16); K and V have one of each.  Codes are
 * 16-byte aligned. */
int ss_cache_bytes(const ss_cache_desc* desc, size_t* codes, size_t* scales);

/* Writes the packed tokens K, V [T tokens, HK heads, D] (bf16; element (t,h,d) at t*stride_t + h*stride_h + d, strides
 * multiples of 8 and at least D, pointers 16-byte aligned) into the cache.
 *   cu    in : int32 [n_seq+1]: the tokens of sequence b are rows cu[b] .. cu[b+1]-1 (clamped to 0 .. T)
 *   start in : int32 [n_seq]: the position of the first of them; NULL: 0
 *   table in : int32 [n_seq][max_pages]
 * A page that is written belongs to one sequence of the call: if two tokens name one slot, what it then holds may be of
 * either.  Drafted tokens that were not accepted are simply written over. */
int ss_cache_write(const ss_cache_desc* desc, int32_t T, const void* K, const void* V, int64_t stride_t, int64_t stride_h,
                   const int32_t* cu, const int32_t* start, const int32_t* table, void* k_codes, float* k_scales,
                   void* v_codes, float* v_scales, void* hip_stream);

/* Reads rows back as bf16 (rounded once), packed as ss_packed_fwd takes its keys: row cu[b] + i of K and V is position
 * start[b] + i (start NULL: 0) of sequence b (cu clamped to 0 .. T).  Rows outside cu[0] .. cu[n_seq]-1 are left as they were. */
int ss_cache_read(const ss_cache_desc* desc, int32_t T, const int32_t* cu, const int32_t* start, const int32_t* table,
                  const void* k_codes, const float* k_scales, const void* v_codes, const float* v_scales, void* K, void* V,
                  int64_t stride_t, int64_t stride_h, void* hip_stream);

/* New tokens: Q and Y are packed [T tokens, H heads, D] (bf16; strides as above), sequence b has rows cu[b] ..
 * cu[b+1]-1, at most max_new of them. */
typedef struct {
  int32_t T, H;      /* new tokens of all sequences; query heads, a multiple of HK           */
  int32_t max_new;   /* the most new tokens of a sequence, 1 .. 64                           */
  float scale;       /* multiplies <q,k>; finite                                             */
  int64_t q_stride_t, q_stride_h;
  int64_t y_stride_t, y_stride_h;
} ss_cache_attn_desc;

/* Workspace bytes of ss_cache_attn (host output). */
int ss_cache_attn_workspace_bytes(const ss_cache_desc* desc, const ss_cache_attn_desc* attn, size_t* bytes);

/* Attention of the new tokens over the cache, which holds their own keys and values already (ss_cache_write).
 *   lens in : int32 [n_seq]: tokens of sequence b in the cache, the n = cu[b+1]-cu[b] new ones, its last, among them.
 *   tree in : uint64 [T], or NULL.  New token i of a sequence sees every token before the new ones, and of the new
 *             ones token j where bit j of its entry is set (itself only if its own bit is).  NULL: j <= i, a row of
 *             tokens (one new token: plain decoding).
 *   Y    out: the rows of the sequences; a row that sees nothing is 0.   lse out: float [H, T], or NULL; -inf for such a row.
 *             Rows of no sequence, and a sequence's rows from max_new on, are left as they were.
 * The keys of all sequences together are cut into pieces of equal length, which run side by side; where a sequence lies in
 * more than one, its parts are joined by a second launch, in a fixed order: the same call gives the same bits.  (Where the cuts
 * fall depends on the other sequences of the call, and with it the last bits of a row.)
 *   workspace : 256-byte aligned, need not start at zero.
 * What lies in slots behind a sequence's end has no influence.  In SS_CACHE_BF16 the V of a new token that another new
 * token does not see has to be finite (it is multiplied by a probability of zero); in 8 bits it may be anything. */
int ss_cache_attn(const ss_cache_desc* desc, const ss_cache_attn_desc* attn, const void* Q, const int32_t* cu,
                  const int32_t* lens, const uint64_t* tree, const int32_t* table, const void* k_codes,
                  const float* k_scales, const void* v_codes, const float* v_scales, void* Y, float* lse, void* workspace,
                  size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SS_CACHE_H */
