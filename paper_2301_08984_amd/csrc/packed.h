// Kernel-side view of one chunk of key heads of attention over packed sequences (include/ss_packed.h), and the
// launchers.  Filled by packed_api.hip, passed by value to every kernel.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ssa {

struct PackedP {
  const void *Q, *K, *V, *dY;
  void *Yo, *dQ, *dK, *dV;  // Yo: the forward's output
  const int32_t *cu_q, *cu_k;
  int64_t q_st, q_sh, k_st, k_sh, y_st, y_sh;  // strides of (Q, dQ), (K, V, dK, dV), (Y, dY)
  // softmax statistics, query head h and row t at (h - s_h0) * Tq + t; `lse_out` may be NULL
  float *lse_out, *delta_out;
  const float *lse, *delta;
  int lse_h0, delta_h0;
  float scale;
  int Tq, Tk, n_seq, H, HK, D, G;  // G = H / HK
  int h0, h1;                      // the chunk's key heads
  int parts;                       // of the rows that a work-group of dK and dV takes; more than one: the parts' sums in dkdv_parts, [part][dV, dK][Tk][heads][D]
  float* dkdv_parts;
  int share_heads;                 // key heads of the whole share: kernel-shape choices go by it, never by the chunk
};

hipError_t launch_packed_fwd(const PackedP& p, hipStream_t st);    // Yo, and lse_out if given
hipError_t launch_packed_delta(const PackedP& p, bool kept, hipStream_t st);  // delta_out; from lse where it was kept, else lse_out too
hipError_t launch_packed_dq(const PackedP& p, hipStream_t st);
hipError_t launch_packed_dkdv(const PackedP& p, hipStream_t st);
int packed_dkdv_parts(const PackedP& p);  // from the share, never from the chunk

#ifdef __HIPCC__
// The sequence whose packed tokens, by the n_seq + 1 offsets `cu`, hold row t (the same in all lanes of the wavefront);
// -1: none.  64 offsets at a time: those that are at most t come first.
__device__ inline int packed_owner(const int32_t* cu, int n_seq, int t) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < n_seq; b0 += 64) {
    const int i = b0 + lane;
    const uint64_t before = __builtin_amdgcn_ballot_w64(i < n_seq && cu[min(i, n_seq - 1)] <= t && t < cu[min(i, n_seq - 1) + 1]);
    if (before) return b0 + 63 - __builtin_clzll(before);
  }
  return -1;
}

// One sequence: its first query row and queries, its first key row and keys.  Offsets are clamped, so that no row
// outside the tensors is named whatever the array holds.
struct PackedSeq { int q0, n, k0, m; };
__device__ inline PackedSeq packed_seq(const PackedP& p, int b) {
  PackedSeq s;
  s.q0 = min(max(p.cu_q[b], 0), p.Tq);
  s.n = max(min(p.cu_q[b + 1], p.Tq) - s.q0, 0);
  s.k0 = min(max(p.cu_k[b], 0), p.Tk);
  s.m = max(min(p.cu_k[b + 1], p.Tk) - s.k0, 0);
  return s;
}
#endif

}  // namespace ssa
