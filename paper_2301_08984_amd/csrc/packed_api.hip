// C ABI of attention over packed sequences with grouped heads: validation, chunk plan, workspace layout and the
// sequence of kernel launches per chunk of key heads (include/ss_packed.h).
#include "../../include/ss_packed.h"

#include <cmath>
#include <cstdio>

#include "packed.h"
#include "shared_scratch.h"

namespace {

using ssa::PackedP;

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

bool bad_stride(int64_t st, int64_t sh, int D) { return st < D || sh < D || (st & 7) || (sh & 7); }

int validate(const ss_packed_desc* d) {
  if (!d) return SS_ERR_NULL;
  if (d->Tq < 1 || d->Tk < 1 || d->n_seq < 1 || d->H < 1 || d->HK < 1 || d->D < 1 || d->H % d->HK || (d->D & 7)) return SS_ERR_BAD_SHAPE;
  if (bad_stride(d->q_stride_t, d->q_stride_h, d->D) || bad_stride(d->k_stride_t, d->k_stride_h, d->D) ||
      bad_stride(d->y_stride_t, d->y_stride_h, d->D))
    return SS_ERR_BAD_SHAPE;
  if (!std::isfinite(d->scale)) return SS_ERR_BAD_SHAPE;
  if (d->dtype != SS_BF16 || d->D > 128 || d->flags || d->n_seq > 65535 || d->H > 65535) return SS_ERR_UNSUPPORTED;
  // lanes address the 32 rows of a tile with 32-bit byte offsets
  const int64_t lim = (int64_t)1 << 24;
  if (d->q_stride_t >= lim || d->q_stride_h >= lim || d->k_stride_t >= lim || d->k_stride_h >= lim || d->y_stride_t >= lim || d->y_stride_h >= lim)
    return SS_ERR_UNSUPPORTED;
  // ... and a step's 32 rows of (token, head) pairs too, whose buffer descriptors end at 0x7e000000 bytes; rows and work-groups are counted in 31 bits
  const int64_t G = d->H / d->HK;
  if (G * d->q_stride_h + 33 * d->q_stride_t >= 1000000000ll || G * d->y_stride_h + 33 * d->y_stride_t >= 1000000000ll) return SS_ERR_UNSUPPORTED;
  if (d->Tq > (1 << 30) || d->Tk > (1 << 30) || d->Tq * G >= (1 << 30)) return SS_ERR_UNSUPPORTED;
  if ((((d->Tq * G > 4ll * d->Tk ? d->Tq * G : 4ll * d->Tk) >> 7) + d->n_seq + 8) * 8 * d->HK >= (int64_t)1 << 31) return SS_ERR_UNSUPPORTED;
  if (d->lo < 0 || d->lo >= d->hi || d->hi > d->HK) return SS_ERR_BAD_RANGE;
  if (d->k < 1 || d->k > d->hi - d->lo) return SS_ERR_BAD_K;
  return SS_OK;
}

void chunk(const ss_packed_desc* d, int k, int c, int* a, int* b) {
  const int64_t n = d->hi - d->lo;
  *a = d->lo + (int)((c * n) / k);
  *b = d->lo + (int)(((c + 1) * n) / k);
}

PackedP params(const ss_packed_desc* d) {
  PackedP p{};
  p.q_st = d->q_stride_t; p.q_sh = d->q_stride_h;
  p.k_st = d->k_stride_t; p.k_sh = d->k_stride_h;
  p.y_st = d->y_stride_t; p.y_sh = d->y_stride_h;
  p.scale = d->scale;
  p.Tq = d->Tq; p.Tk = d->Tk; p.n_seq = d->n_seq;
  p.H = d->H; p.HK = d->HK; p.D = d->D; p.G = d->H / d->HK;
  p.h0 = d->lo; p.h1 = d->hi;
  p.share_heads = d->hi - d->lo;
  return p;
}

// The scratch of one chunk: LSE (unless the caller kept it) and Delta of its query heads, and the parts of dK and dV.
struct Ws {
  size_t lse, parts, total;
};
Ws layout(const ss_packed_desc* d, int k, bool kept) {
  const int64_t n = d->hi - d->lo, most = (n + k - 1) / k;  // key heads of the largest chunk
  const size_t stat = align256((size_t)(most * (d->H / d->HK)) * d->Tq * 4);
  const int parts = ssa::packed_dkdv_parts(params(d));
  Ws w{stat, kept ? stat : 2 * stat, 0};
  w.total = w.parts + (parts > 1 ? align256((size_t)parts * 2 * d->Tk * most * d->D * 4) : 0);
  return w;
}
// The fewest chunks, at most d->k, whose scratch fits `bytes`: 1, 2, 4, .. (every number gives the same results).
int fewest_chunks(const ss_packed_desc* d, bool kept, size_t bytes) {
  for (int k = 1; k < d->k; k *= 2)
    if (layout(d, k, kept).total <= bytes) return k;
  return d->k;
}

int hip_fail(hipError_t e, const char* what) {
  std::fprintf(stderr, "ss_packed: %s: %s\n", what, hipGetErrorString(e));
  return SS_ERR_HIP;
}
#define PK_LAUNCH(expr, what)                        \
  do {                                               \
    const hipError_t e_ = (expr);                    \
    if (e_ != hipSuccess) return hip_fail(e_, what); \
  } while (0)

bool misaligned(const void* p) { return (uintptr_t)p & 15; }

}  // namespace

extern "C" {

int ss_packed_workspace_bytes(const ss_packed_desc* d, size_t* fwd_bytes, size_t* bwd_bytes) {
  const int rc = validate(d);
  if (rc != SS_OK) return rc;
  if (fwd_bytes) *fwd_bytes = 0;
  if (bwd_bytes) *bwd_bytes = layout(d, d->k, false).total;
  return SS_OK;
}

int ss_packed_chunk_range(const ss_packed_desc* d, int32_t c, int32_t* lo, int32_t* hi) {
  const int rc = validate(d);
  if (rc != SS_OK) return rc;
  if (!lo || !hi) return SS_ERR_NULL;
  if (c < 0 || c >= d->k) return SS_ERR_BAD_K;
  int a, b;
  chunk(d, d->k, c, &a, &b);
  *lo = a; *hi = b;
  return SS_OK;
}

int ss_packed_fwd(const ss_packed_desc* d, const void* Q, const void* K, const void* V, const int32_t* cu_q,
                  const int32_t* cu_k, void* Y, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  (void)workspace; (void)workspace_bytes;
  const int rc = validate(d);
  if (rc != SS_OK) return rc;
  if (!Q || !K || !V || !cu_q || !Y) return SS_ERR_NULL;
  if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(Y) || (!cu_k && d->Tk != d->Tq)) return SS_ERR_BAD_SHAPE;
  hipStream_t st = (hipStream_t)hip_stream;
  PackedP p = params(d);
  p.Q = Q; p.K = K; p.V = V; p.Yo = Y; p.cu_q = cu_q; p.cu_k = cu_k ? cu_k : cu_q;
  p.lse_out = lse;
  PK_LAUNCH(ssa::launch_packed_fwd(p, st), "forward");
  return SS_OK;
}

int ss_packed_bwd(const ss_packed_desc* d, const void* Q, const void* K, const void* V, const int32_t* cu_q,
                  const int32_t* cu_k, const void* Y, const void* dY, const float* lse, void* dQ, void* dK, void* dV,
                  void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = validate(d);
  if (rc != SS_OK) return rc;
  if (!Q || !K || !V || !cu_q || !dY || !dQ || !dK || !dV || !Y != !lse) return SS_ERR_NULL;
  if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(Y) || misaligned(dY) || misaligned(dQ) || misaligned(dK) || misaligned(dV) ||
      (!cu_k && d->Tk != d->Tq))
    return SS_ERR_BAD_SHAPE;
  if (!workspace || workspace_bytes < layout(d, d->k, false).total || ((uintptr_t)workspace & 255)) return SS_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)hip_stream;
  // A chunk of few heads leaves most of the chip idle, and what keeps chunks apart is only that they reuse one chunk's scratch:
  // run the fewest whose scratch fits the caller's workspace, or else half of the library's buffer if nobody is using it.
  // One chunk | two | four | eight as asked, then the same merged, us: 9 documents, 4496 tokens, 32 heads of 128 in groups of four,
  // recomputed, 261 | 408 | 755 | 1484, 261 | 269 | 250 | 244; one document of 8192, one | eight, 2447 | 10669, 2438 | 2415.
  const bool kept = lse != nullptr;
  char* ws = (char*)workspace;
  int k = fewest_chunks(d, kept, workspace_bytes);
  const int ks = k > 1 ? fewest_chunks(d, kept, ssa::SHARED_HALF) : k;
  ssa::SharedUse shared;
  if (ks < k) {
    char* own = shared.take(st, ssa::SHARED_FIRST);
    if (!own) own = shared.take(st, ssa::SHARED_SECOND);
    if (own) {
      ws = own;
      k = ks;
    }
  }
  const Ws w = layout(d, k, kept);
  PackedP p = params(d);
  p.Q = Q; p.K = K; p.V = V; p.dY = dY; p.dQ = dQ; p.dK = dK; p.dV = dV;
  p.cu_q = cu_q; p.cu_k = cu_k ? cu_k : cu_q;
  p.parts = ssa::packed_dkdv_parts(p);
  p.dkdv_parts = (float*)(ws + w.parts);
  for (int c = 0; c < k; ++c) {
    chunk(d, k, c, &p.h0, &p.h1);
    p.delta_h0 = p.h0 * p.G;
    p.delta_out = (float*)ws;
    p.delta = p.delta_out;
    if (kept) {
      p.lse = lse;
    } else {
      p.lse_h0 = p.h0 * p.G;
      p.lse_out = (float*)(ws + w.lse);
      p.lse = p.lse_out;
    }
    PK_LAUNCH(ssa::launch_packed_delta(p, kept, st), "Delta");
    PK_LAUNCH(ssa::launch_packed_dq(p, st), "dQ");
    PK_LAUNCH(ssa::launch_packed_dkdv(p, st), "dK, dV");
  }
  return SS_OK;
}

}  // extern "C"
