// Host-only driver for an AddressSanitizer + UndefinedBehaviorSanitizer build of the host code of packed attention and of the cache
// (include/ss_packed.h, include/ss_cache.h): seeded random and boundary descriptors through every entry point.  The launchers are stubbed out and
// look at what a launch would be given: a backward's chunks follow each other over the share's key heads, their scratch lies inside the workspace.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "ss_cache.h"
#include "ss_packed.h"
#include "../../paper_2301_08984_amd/csrc/cache.h"
#include "../../paper_2301_08984_amd/csrc/packed.h"
#include "../../paper_2301_08984_amd/csrc/shared_scratch.h"

#define CHECK(c) do { if (!(c)) { std::fprintf(stderr, "check failed line %d: %s\n", __LINE__, #c); std::exit(1); } } while (0)

static uint64_t rng_state = 0x9e3779b97f4a7c15ull;
static uint64_t rnd() {
  rng_state ^= rng_state << 13; rng_state ^= rng_state >> 7; rng_state ^= rng_state << 17;
  return rng_state;
}
static int pick(int lo, int hi) { return lo + (int)(rnd() % (uint64_t)((int64_t)hi - lo + 1)); }
static int wide() {  // any size of number, boundaries among them
  const int s = pick(0, 31);
  const int64_t x = ((int64_t)1 << s) + pick(-2, 2);
  return (int)std::min<int64_t>(std::max<int64_t>(x, -2), 2147483647);
}

static int next_head, chunks, parts_now, forwards, deltas, dqs;
static bool shared_there, kept_now;
static char *ws_begin, *ws_end;

namespace ssa {
char* SharedUse::take(hipStream_t, int) { return shared_there ? (char*)0x70000000ull : nullptr; }
SharedUse::~SharedUse() {}
int packed_dkdv_parts(const PackedP& p) { return (int64_t)2 * parts_now * p.Tk * p.share_heads * p.D * 4 <= (24 << 20) ? parts_now : 1; }

static void inside(const void* at, size_t bytes) {
  const char* p = (const char*)at;
  const bool shared = p >= (char*)0x70000000ull && p < (char*)0x70000000ull + SHARED_HALF;
  if (shared) CHECK(p + bytes <= (char*)0x70000000ull + SHARED_HALF);
  else CHECK(p >= ws_begin && p + bytes <= ws_end);
}
hipError_t launch_packed_fwd(const PackedP& p, hipStream_t) {
  ++forwards;
  CHECK(p.h0 >= 0 && p.h0 < p.h1 && p.h1 <= p.HK && p.share_heads == p.h1 - p.h0 && p.cu_k && p.Yo);
  return hipSuccess;
}
hipError_t launch_packed_delta(const PackedP& p, bool kept, hipStream_t) {
  ++deltas;
  CHECK(kept == kept_now && p.h0 == next_head && p.h1 > p.h0);
  const size_t stat = (size_t)(p.h1 - p.h0) * p.G * p.Tq * 4;
  CHECK(p.delta_h0 == p.h0 * p.G);
  inside(p.delta_out, stat);
  if (!kept) {
    CHECK(p.lse_h0 == p.delta_h0 && p.lse == p.lse_out);
    inside(p.lse_out, stat);
    CHECK((char*)p.lse_out >= (char*)p.delta_out + stat);
  } else {
    CHECK(p.lse_h0 == 0);
  }
  return hipSuccess;
}
hipError_t launch_packed_dq(const PackedP& p, hipStream_t) {
  ++dqs;
  CHECK(p.delta == p.delta_out);
  return hipSuccess;
}
hipError_t launch_packed_dkdv(const PackedP& p, hipStream_t) {
  ++chunks;
  next_head = p.h1;
  if (p.parts > 1) {
    inside(p.dkdv_parts, (size_t)p.parts * 2 * p.Tk * (p.h1 - p.h0) * p.D * 4);
    const char* stats_end = kept_now ? (char*)p.delta_out : (char*)p.lse_out;
    CHECK((char*)p.dkdv_parts >= stats_end + (size_t)(p.h1 - p.h0) * p.G * p.Tq * 4);
  }
  return hipSuccess;
}
size_t cache_attn_bytes(const CacheAttnP& p) { return p.max_new > 8 ? 4096 : 0; }
static int cache_launches;
hipError_t launch_cache_write(const CacheRowsP& p, hipStream_t) { ++cache_launches; CHECK(p.T > 0 && 1 << p.c.shift == p.c.page); return hipSuccess; }
hipError_t launch_cache_read(const CacheRowsP& p, hipStream_t) { ++cache_launches; CHECK(p.T > 0); return hipSuccess; }
hipError_t launch_cache_attn(const CacheAttnP& p, hipStream_t) {
  ++cache_launches;
  CHECK(p.T > 0 && p.G >= 1 && p.G * p.c.HK == p.H && p.max_new >= 1 && p.max_new <= 64 && p.c.table && p.cu && p.lens && p.Q && p.Y);
  return hipSuccess;
}
}  // namespace ssa

static int packed() {
  long ok = 0, bad = 0, in_chunks = 0;
  for (int it = 0; it < 40000; ++it) {
    ss_packed_desc d;
    std::memset(&d, 0, sizeof d);
    const bool any = it % 3 == 0;
    d.Tq = any ? wide() : pick(1, 3000); d.Tk = any ? wide() : pick(1, 3000); d.n_seq = any ? wide() : pick(1, 90);
    d.HK = any ? wide() : pick(1, 9); d.H = any && it % 2 ? wide() : (int)std::min<int64_t>((int64_t)d.HK * pick(1, 8), 2147483647);
    d.D = it % 5 ? 8 * pick(1, 16) : pick(-1, 300);
    d.dtype = it % 17 ? SS_BF16 : pick(-1, 2); d.scale = 0.1f; d.flags = it % 19 ? 0 : (uint32_t)rnd();
    d.q_stride_h = d.y_stride_h = d.k_stride_h = d.D;
    d.q_stride_t = d.y_stride_t = (int64_t)d.H * d.D; d.k_stride_t = (int64_t)d.HK * d.D;
    if (any) d.q_stride_t = (int64_t)(rnd() >> pick(1, 60)) & ~7ll;
    if (it % 6 == 0) d.y_stride_h = (int64_t)(rnd() >> pick(1, 60)) & ~7ll;
    const int top = d.HK > 0 ? d.HK : 1;
    d.lo = pick(-1, top > 100000 ? 100000 : top); d.hi = any ? wide() : pick(d.lo, top);
    d.k = pick(0, 9);
    size_t f = 1, b = 0;
    const int rc = ss_packed_workspace_bytes(&d, &f, &b);
    if (rc != SS_OK) {
      ++bad;
      CHECK(ss_packed_fwd(&d, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0) == rc);
      CHECK(ss_packed_bwd(&d, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0) == rc);
      continue;
    }
    ++ok;
    CHECK(f == 0 && b % 256 == 0);
    parts_now = 1 << pick(0, 3);
    CHECK(ss_packed_workspace_bytes(&d, nullptr, &b) == SS_OK);
    int last = d.lo;
    for (int c = 0; c < std::min(d.k, 20); ++c) {
      int lo, hi;
      CHECK(ss_packed_chunk_range(&d, c, &lo, &hi) == SS_OK);
      CHECK(lo == last && hi > lo);
      last = hi;
    }
    CHECK(d.k > 20 || last == d.hi);
    void* a = (void*)256;
    const int32_t* cu = (const int32_t*)256;
    forwards = 0;
    CHECK(ss_packed_fwd(&d, a, a, a, cu, cu, a, (float*)a, nullptr, 0, nullptr) == SS_OK && forwards == 1);
    const size_t extra = it % 2 ? 0 : (size_t)(rnd() >> pick(30, 60));
    ws_begin = (char*)0x100000000000ull;
    ws_end = ws_begin + b + extra;
    for (int kept = 0; kept < 2; ++kept) {
      kept_now = kept;
      shared_there = it % 4 == 0;
      next_head = d.lo; chunks = deltas = dqs = 0;
      CHECK(ss_packed_bwd(&d, a, a, a, cu, cu, kept ? a : nullptr, a, kept ? (const float*)a : nullptr, a, a, a, ws_begin, b + extra, nullptr) == SS_OK);
      CHECK(next_head == d.hi && chunks >= 1 && chunks <= d.k && deltas == chunks && dqs == chunks);
      in_chunks += chunks > 1;
      CHECK(ss_packed_bwd(&d, a, a, a, cu, cu, kept ? a : nullptr, a, kept ? (const float*)a : nullptr, a, a, a, ws_begin, b - 1, nullptr) == SS_ERR_WORKSPACE);
    }
  }
  CHECK(ok > 1000 && bad > 1000 && in_chunks > 100);
  return 0;
}

static int cache() {
  long ok = 0, bad = 0, ok_attn = 0, bad_attn = 0;
  for (int it = 0; it < 40000; ++it) {
    ss_cache_desc d;
    const bool any = it % 3 == 0;
    d.n_pages = any ? wide() : pick(1, 5000); d.page = it % 5 ? 8 << pick(0, 7) : wide();
    d.HK = any ? wide() : pick(1, 12); d.D = it % 7 ? 64 * pick(1, 2) : pick(-1, 300);
    d.format = it % 11 ? pick(0, 2) : pick(-1, 4);
    d.n_seq = any ? wide() : pick(1, 70); d.max_pages = any ? wide() : pick(1, 400);
    size_t c = 0, s = 0;
    const int rc = ss_cache_bytes(&d, &c, &s);
    ss_cache_attn_desc a;
    a.T = any ? wide() : pick(1, 500); a.H = it % 2 ? (int)std::min<int64_t>((int64_t)std::max(d.HK, 0) * pick(1, 9), 2147483647) : wide();
    a.max_new = it % 4 ? pick(1, 64) : wide(); a.scale = 0.1f;
    a.q_stride_h = a.y_stride_h = d.D; a.q_stride_t = a.y_stride_t = (int64_t)a.H * d.D;
    if (it % 6 == 0) a.q_stride_t = (int64_t)(rnd() >> pick(1, 60)) & ~7ll;
    size_t w = 0;
    const int ra = ss_cache_attn_workspace_bytes(&d, &a, &w);
    void* p = (void*)256;
    const int32_t* i = (const int32_t*)256;
    float* f = (float*)256;
    const int rw = ss_cache_write(&d, a.T, p, p, a.q_stride_t, 128, i, i, i, p, f, p, f, nullptr);
    const int rr = ss_cache_read(&d, a.T, i, i, i, p, f, p, f, p, p, a.q_stride_t, 128, nullptr);
    CHECK(rw == rr);
    if (rc != SS_OK) {
      ++bad;
      CHECK(ra == rc && rw == rc);
      continue;
    }
    ++ok;
    CHECK(c == (size_t)d.n_pages * d.HK * d.page * d.D * (d.format ? 1 : 2) && s == (d.format ? (size_t)d.n_pages * d.HK * d.page * 4 : 0));
    const int rn = ss_cache_attn(&d, &a, p, i, i, nullptr, i, p, f, p, f, p, f, (void*)256, w, nullptr);
    CHECK(rn == ra);
    ra == SS_OK ? ++ok_attn : ++bad_attn;
    if (ra == SS_OK && w) CHECK(ss_cache_attn(&d, &a, p, i, i, nullptr, i, p, f, p, f, p, f, (void*)256, w - 1, nullptr) == SS_ERR_WORKSPACE);
  }
  CHECK(ok > 1000 && bad > 1000 && ok_attn > 1000 && bad_attn > 1000 && ssa::cache_launches > 1000);
  return 0;
}

int main() {
  if (packed() || cache()) return 1;
  std::puts("all checks passed");
  return 0;
}
