// C ABI of the paged cache and of attention over it: validation and launches (include/ss_cache.h).
#include "../../include/ss_cache.h"

#include <cmath>
#include <cstdio>

#include "cache.h"

namespace {

using ssa::CacheAttnP;
using ssa::CacheP;
using ssa::CacheRowsP;

int validate(const ss_cache_desc* d) {
  if (!d) return SS_ERR_NULL;
  if (d->n_pages < 1 || d->page < 1 || d->HK < 1 || d->D < 1 || d->n_seq < 1 || d->max_pages < 1) return SS_ERR_BAD_SHAPE;
  if (d->format < SS_CACHE_BF16 || d->format > SS_CACHE_INT8) return SS_ERR_UNSUPPORTED;
  if ((d->D != 64 && d->D != 128) || (d->page & (d->page - 1)) || d->page < 8 || d->page > 1024) return SS_ERR_UNSUPPORTED;
  if (d->HK > 65535 || d->n_seq > 65535 || (int64_t)d->max_pages * d->page >= (int64_t)1 << 31) return SS_ERR_UNSUPPORTED;
  // (row numbers times the bytes of a row stay far below 2^63)
  if ((int64_t)d->n_pages * d->HK * d->page >= (int64_t)1 << 48) return SS_ERR_UNSUPPORTED;
  return SS_OK;
}

bool bad_stride(int64_t st, int64_t sh, int D) {
  return st < D || sh < D || (st & 7) || (sh & 7) || st >= (int64_t)1 << 31 || sh >= (int64_t)1 << 31;
}
bool misaligned(const void* p) { return (uintptr_t)p & 15; }

int validate(const ss_cache_desc* d, const ss_cache_attn_desc* a) {
  const int rc = validate(d);
  if (rc != SS_OK) return rc;
  if (!a) return SS_ERR_NULL;
  if (a->T < 1 || a->H < 1 || a->H % d->HK || a->max_new < 1 || !std::isfinite(a->scale)) return SS_ERR_BAD_SHAPE;
  if (bad_stride(a->q_stride_t, a->q_stride_h, d->D) || bad_stride(a->y_stride_t, a->y_stride_h, d->D)) return SS_ERR_BAD_SHAPE;
  if (a->max_new > 64 || a->H > 65535 || (int64_t)a->T * a->H >= (int64_t)1 << 31) return SS_ERR_UNSUPPORTED;
  // (all sequences' keys, 64 at a time, once for every 128 rows, and work-groups are counted in 31 bits)
  const int64_t runs = (int64_t)d->n_seq * ((a->max_new * (a->H / d->HK) + 127) / 128);
  if (runs * ((((int64_t)d->max_pages * d->page) >> 6) + 1) >= (int64_t)1 << 30 || runs * d->HK >= (int64_t)1 << 31) return SS_ERR_UNSUPPORTED;
  return SS_OK;
}

// the arrays that a cache of this format has
int check_store(const ss_cache_desc* d, const void* kc, const float* ks, const void* vc, const float* vs) {
  if (!kc || !vc || (d->format != SS_CACHE_BF16 && (!ks || !vs))) return SS_ERR_NULL;
  return misaligned(kc) || misaligned(vc) ? SS_ERR_BAD_SHAPE : SS_OK;
}

CacheP store(const ss_cache_desc* d, const int32_t* table, const void* kc, const float* ks, const void* vc, const float* vs) {
  CacheP c{};
  c.kc = const_cast<void*>(kc); c.vc = const_cast<void*>(vc);
  c.ks = const_cast<float*>(ks); c.vs = const_cast<float*>(vs);
  c.table = table;
  c.n_pages = d->n_pages; c.page = d->page; c.shift = __builtin_ctz(d->page);
  c.HK = d->HK; c.D = d->D; c.format = d->format; c.n_seq = d->n_seq; c.max_pages = d->max_pages;
  return c;
}

int done(hipError_t e, const char* what) {
  if (e == hipSuccess) return SS_OK;
  std::fprintf(stderr, "ss_cache: %s: %s\n", what, hipGetErrorString(e));
  return SS_ERR_HIP;
}

CacheAttnP params(const ss_cache_desc* d, const ss_cache_attn_desc* a) {
  CacheAttnP p{};
  p.c = store(d, nullptr, nullptr, nullptr, nullptr, nullptr);
  p.q_st = a->q_stride_t; p.q_sh = a->q_stride_h;
  p.y_st = a->y_stride_t; p.y_sh = a->y_stride_h;
  p.scale = a->scale;
  p.T = a->T; p.H = a->H; p.G = a->H / d->HK; p.max_new = a->max_new;
  return p;
}

int check_rows(const ss_cache_desc* d, int T, const void* K, const void* V, int64_t st, int64_t sh, const int32_t* cu, const int32_t* table) {
  const int rc = validate(d);
  if (rc != SS_OK) return rc;
  if (T < 1 || bad_stride(st, sh, d->D)) return SS_ERR_BAD_SHAPE;
  if ((int64_t)T * (d->HK / 2 + 1) >= (int64_t)1 << 31) return SS_ERR_UNSUPPORTED;  // (wavefronts are counted in 31 bits)
  if (!K || !V || !cu || !table) return SS_ERR_NULL;
  return misaligned(K) || misaligned(V) ? SS_ERR_BAD_SHAPE : SS_OK;
}

}  // namespace

extern "C" {

int ss_cache_bytes(const ss_cache_desc* d, size_t* codes, size_t* scales) {
  const int rc = validate(d);
  if (rc != SS_OK) return rc;
  const size_t rows = (size_t)d->n_pages * d->HK * d->page;
  if (codes) *codes = rows * d->D * (d->format == SS_CACHE_BF16 ? 2 : 1);
  if (scales) *scales = d->format == SS_CACHE_BF16 ? 0 : rows * 4;
  return SS_OK;
}

int ss_cache_write(const ss_cache_desc* d, int32_t T, const void* K, const void* V, int64_t stride_t, int64_t stride_h,
                   const int32_t* cu, const int32_t* start, const int32_t* table, void* k_codes, float* k_scales,
                   void* v_codes, float* v_scales, void* hip_stream) {
  int rc = check_rows(d, T, K, V, stride_t, stride_h, cu, table);
  if (rc == SS_OK) rc = check_store(d, k_codes, k_scales, v_codes, v_scales);
  if (rc != SS_OK) return rc;
  const CacheRowsP p{store(d, table, k_codes, k_scales, v_codes, v_scales), const_cast<void*>(K), const_cast<void*>(V), stride_t, stride_h, cu, start, T, 0};
  return done(ssa::launch_cache_write(p, (hipStream_t)hip_stream), "write");
}

int ss_cache_read(const ss_cache_desc* d, int32_t T, const int32_t* cu, const int32_t* start, const int32_t* table,
                  const void* k_codes, const float* k_scales, const void* v_codes, const float* v_scales, void* K, void* V,
                  int64_t stride_t, int64_t stride_h, void* hip_stream) {
  int rc = check_rows(d, T, K, V, stride_t, stride_h, cu, table);
  if (rc == SS_OK) rc = check_store(d, k_codes, k_scales, v_codes, v_scales);
  if (rc != SS_OK) return rc;
  const CacheRowsP p{store(d, table, k_codes, k_scales, v_codes, v_scales), K, V, stride_t, stride_h, cu, start, T, 0};
  return done(ssa::launch_cache_read(p, (hipStream_t)hip_stream), "read");
}

int ss_cache_attn_workspace_bytes(const ss_cache_desc* d, const ss_cache_attn_desc* a, size_t* bytes) {
  const int rc = validate(d, a);
  if (rc != SS_OK) return rc;
  if (bytes) *bytes = ssa::cache_attn_bytes(params(d, a));
  return SS_OK;
}

int ss_cache_attn(const ss_cache_desc* d, const ss_cache_attn_desc* a, const void* Q, const int32_t* cu,
                  const int32_t* lens, const uint64_t* tree, const int32_t* table, const void* k_codes,
                  const float* k_scales, const void* v_codes, const float* v_scales, void* Y, float* lse, void* workspace,
                  size_t workspace_bytes, void* hip_stream) {
  int rc = validate(d, a);
  if (rc != SS_OK) return rc;
  if (!Q || !cu || !lens || !table || !Y) return SS_ERR_NULL;
  if (misaligned(Q) || misaligned(Y)) return SS_ERR_BAD_SHAPE;
  rc = check_store(d, k_codes, k_scales, v_codes, v_scales);
  if (rc != SS_OK) return rc;
  CacheAttnP p = params(d, a);
  const size_t need = ssa::cache_attn_bytes(p);
  if (need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))) return SS_ERR_WORKSPACE;
  p.c = store(d, table, k_codes, k_scales, v_codes, v_scales);
  p.Q = Q; p.Y = Y; p.lse = lse; p.cu = cu; p.lens = lens; p.tree = tree;
  p.ws = (char*)workspace;
  return done(ssa::launch_cache_attn(p, (hipStream_t)hip_stream), "attention");
}

}  // extern "C"
