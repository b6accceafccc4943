/* ss_packed.h -- C ABI of co-sharded attention over packed sequences with grouped heads, for MI355X (gfx950).
 *
 * Sequences of different lengths lie one behind the other in one tensor of tokens (documents packed into a
 * training sample, the prompts of a serving batch), and H query heads share HK key / value heads: query head h
 * reads key head h / (H / HK).  The mask is causal inside a sequence, and nothing is seen across sequences.
 * A sequence may have more keys than queries: its queries are then its last tokens (the new turn of a
 * conversation whose past was read back from a cache, ss_cache.h).  For sequence b with n queries and m keys
 *
 *     s_ij = scale * <q_i, k_j>  for  j <= i + (m - n);   P = softmax over j;   Y_i = sum_j P_ij v_j
 *     lse_i = log sum_j exp s_ij  (natural)
 *
 * and the backward produces, for dY:  dV_j = sum P_ij dY_i,  dS_ij = P_ij (<dY_i, v_j> - Delta_i),
 * Delta_i = <dY_i, Y_i>,  dQ_i = scale sum_j dS_ij k_j,  dK_j = scale sum dS_ij q_i, where the sums over i
 * run over all H / HK query heads of a key head.  A query that sees no key (n > m) has Y = 0, lse = -inf and
 * passes no gradient on; a key that no query sees has dK = dV = 0.
 *
 * One call runs one GPU's share, the key heads [lo,hi) with their query heads, as k sub-operators along that
 * axis (op-trans, op-order; ss_attn.h): the scratch of the backward is that of one chunk and shrinks as 1/k, and the
 * results are the same bits for every k.  (Chunks run together where their scratch fits the workspace at hand, or the buffer that
 * the library holds on each GPU, unless another stream is using it or the call is being captured into a graph.)  All pointers
 * are DEVICE pointers, the descriptor and size outputs HOST memory; no call allocates or synchronises, and that buffer is the
 * only state.  Error codes are those of ss_attn.h.
 */
#ifndef SS_PACKED_H
#define SS_PACKED_H

#include <stddef.h>
#include <stdint.h>

#include "ss_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element (t, h, d) of Q and dQ is at t*q_stride_t + h*q_stride_h + d, of K, V, dK and dV at
 * t*k_stride_t + h*k_stride_h + d, of Y and dY at t*y_stride_t + h*y_stride_h + d (in elements, d contiguous), so
 * that Q, K and V may be slices of one buffer.  Strides are multiples of 8 elements, at least D and below 2^24;
 * base pointers 16-byte aligned; D a multiple of 8 up to 128 (64 and 128 waste nothing).  A step's rows lie within a lane's reach:
 * H/HK * stride_h + 33 * stride_t < 10^9, of Q and of Y; rows are counted in 30 bits: Tk at most and Tq * H/HK below 2^30. */
typedef struct {
  int32_t Tq, Tk;    /* tokens (rows) of Q, Y, dY, dQ, and of K, V, dK, dV           */
  int32_t n_seq;     /* sequences, up to 65535                                       */
  int32_t H, HK, D;  /* query heads, key / value heads (a divisor of H), head size   */
  int32_t dtype;     /* SS_BF16                                                      */
  float scale;       /* multiplies <q,k>; finite                                     */
  int64_t q_stride_t, q_stride_h;
  int64_t k_stride_t, k_stride_h;
  int64_t y_stride_t, y_stride_h;
  int32_t lo, hi;    /* this GPU's key heads                                         */
  int32_t k;         /* co-shard factor, 1 <= k <= hi-lo                             */
  uint32_t flags;    /* 0                                                            */
} ss_packed_desc;

/* Workspace bytes (host outputs, either may be NULL).  Forward: 0.  Backward: one chunk's statistics (LSE and Delta)
 * and, where the work of dK and dV is cut into parts because it is little, one chunk's share of up to 24 MiB for the parts' sums. */
int ss_packed_workspace_bytes(const ss_packed_desc* desc, size_t* fwd_bytes, size_t* bwd_bytes);

/* The key heads of chunk c (0 <= c < k): lo + floor(c*n/k) .. lo + floor((c+1)*n/k), n = hi-lo. */
int ss_packed_chunk_range(const ss_packed_desc* desc, int32_t c, int32_t* lo, int32_t* hi);

/* Forward.
 *   cu_q   in : int32 [n_seq+1], on the device: the queries of sequence b are rows cu_q[b] .. cu_q[b+1]-1.
 *               Ascending; values are clamped to 0 .. Tq, and a sequence that would end before it begins
 *               is empty.  (Overlapping sequences are the caller's mistake: no access leaves the tensors, but some
 *               rows may be left out.)
 *   cu_k   in : the same for the keys, or NULL: the keys are as many as the queries, cu_q (Tk = Tq then).
 *   Y      out: the rows of the sequences, heads of the share; other rows are left as they were.
 *   lse    out: float [H, Tq], the same entries; may be NULL.
 *   workspace : unused, may be NULL.
 * Values in rows of other sequences, and in rows of no sequence, have no influence, whatever they are.  Inside a
 * sequence the K and V of a masked key have to be finite (they are multiplied by a probability of zero). */
int ss_packed_fwd(const ss_packed_desc* desc, const void* Q, const void* K, const void* V, const int32_t* cu_q,
                  const int32_t* cu_k, void* Y, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Backward.
 *   Y, lse in : as the forward wrote them, or both NULL: recomputed chunk by chunk (one without the other:
 *               SS_ERR_NULL).  What is used is lse: Delta is formed from the products that dS is formed from, sum_j P_ij <dY_i, v_j>,
 *               not from the rounded Y, whose error would show in dQ wherever the keys have a mean or one key has most of a row.
 *   Q, dY  in : in rows of other sequences, of no sequence, and of queries that see no key they may be anything.  Inside a
 *               sequence those of a query that sees a key have to be finite (for the keys that it does not see they are multiplied by
 *               a probability of zero).
 *   dQ, dK, dV out: the rows of the sequences, heads of the share; other rows are left as they were.
 *   workspace : at least bwd_bytes, 256-byte aligned; need not start at zero. */
int ss_packed_bwd(const ss_packed_desc* desc, const void* Q, const void* K, const void* V, const int32_t* cu_q,
                  const int32_t* cu_k, const void* Y, const void* dY, const float* lse, void* dQ, void* dK, void* dV,
                  void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SS_PACKED_H */
