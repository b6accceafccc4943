// Attention over packed sequences, plainly: a wavefront per row and head, a lane per pair of columns, fp32 throughout.
#include "mfma_common.h"
#include "packed.h"

namespace ssa {
namespace {

__device__ inline float wave_sum(float x) {
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
// the sequence whose rows, by `cu`, hold row t; -1: none
__device__ inline int seq_of(const int32_t* cu, int n_seq, int t) {
  for (int b0 = 0; b0 < n_seq; b0 += 64) {
    const int b = b0 + (int)(threadIdx.x & 63);
    const uint64_t hit = __builtin_amdgcn_ballot_w64(b < n_seq && cu[min(b, n_seq - 1)] <= t && t < cu[min(b, n_seq - 1) + 1]);
    if (hit) return b0 + __builtin_ctzll(hit);
  }
  return -1;
}
__device__ inline float at(const void* x, int64_t i, int d, int D) { return d < D ? bf2f(((const uint16_t*)x)[i + d]) : 0.f; }

template <int WHAT>  // 0 forward, 1 statistics, 2 dQ
__global__ __launch_bounds__(64) void packed_row_kernel(PackedP p) {
  const int t = blockIdx.x, h = p.h0 * p.G + blockIdx.y, hk = h / p.G, lane = threadIdx.x, D = p.D;
  const int b = seq_of(p.cu_q, p.n_seq, t);
  if (b < 0) return;
  const PackedSeq s = packed_seq(p, b);
  const int keys = min(t - s.q0 + (s.m - s.n) + 1, s.m);  // visible
  const int64_t qi = t * p.q_st + h * p.q_sh, yi = t * p.y_st + h * p.y_sh;
  const float q0 = at(p.Q, qi, lane, D), q1 = at(p.Q, qi, lane + 64, D);
  const float g0 = WHAT ? at(p.dY, yi, lane, D) : 0.f, g1 = WHAT ? at(p.dY, yi, lane + 64, D) : 0.f;
  const int64_t si = (int64_t)(h - p.lse_h0) * p.Tq + t, di = (int64_t)(h - p.delta_h0) * p.Tq + t;
  const float lse = WHAT == 2 ? p.lse[si] : 0.f, delta = WHAT == 2 ? p.delta[di] : 0.f;
  float m = -INFINITY, l = 0.f, a0 = 0.f, a1 = 0.f;
  for (int j = 0; j < keys; ++j) {
    const int64_t ki = (int64_t)(s.k0 + j) * p.k_st + hk * p.k_sh;
    const float k0 = at(p.K, ki, lane, D), k1 = at(p.K, ki, lane + 64, D), v0 = at(p.V, ki, lane, D), v1 = at(p.V, ki, lane + 64, D);
    const float x = p.scale * wave_sum(q0 * k0 + q1 * k1);
    if (WHAT < 2) {
      const float mn = fmaxf(m, x), alpha = expf(m - mn), e = expf(x - mn);
      m = mn;
      l = l * alpha + e;
      a0 = a0 * alpha + e * v0;
      a1 = a1 * alpha + e * v1;
    } else {
      const float ds = expf(x - lse) * (wave_sum(g0 * v0 + g1 * v1) - delta);
      a0 += ds * k0;
      a1 += ds * k1;
    }
  }
  if (WHAT < 2) {
    const float r = l > 0.f ? 1.f / l : 0.f;
    a0 *= r;
    a1 *= r;
    if (lane == 0 && p.lse_out) p.lse_out[si] = l > 0.f ? m + logf(l) : -INFINITY;
    if (WHAT == 1) {
      const float d = wave_sum(a0 * g0 + a1 * g1);
      if (lane == 0) p.delta_out[di] = d;
      return;
    }
  } else {
    a0 *= p.scale;
    a1 *= p.scale;
  }
  uint16_t* out = WHAT == 0 ? (uint16_t*)p.Yo + yi : (uint16_t*)p.dQ + qi;
  if (lane < D) out[lane] = f2bf(a0);
  if (lane + 64 < D) out[lane + 64] = f2bf(a1);
}

__global__ __launch_bounds__(64) void packed_delta_kernel(PackedP p) {
  const int t = blockIdx.x, h = p.h0 * p.G + blockIdx.y, lane = threadIdx.x;
  if (seq_of(p.cu_q, p.n_seq, t) < 0) return;
  const int64_t yi = t * p.y_st + h * p.y_sh;
  const float d = wave_sum(at(p.Y, yi, lane, p.D) * at(p.dY, yi, lane, p.D) + at(p.Y, yi, lane + 64, p.D) * at(p.dY, yi, lane + 64, p.D));
  if (lane == 0) p.delta_out[(int64_t)(h - p.delta_h0) * p.Tq + t] = d;
}

__global__ __launch_bounds__(64) void packed_key_kernel(PackedP p) {
  const int t = blockIdx.x, hk = p.h0 + blockIdx.y, lane = threadIdx.x, D = p.D;
  const int b = seq_of(p.cu_k, p.n_seq, t);
  if (b < 0) return;
  const PackedSeq s = packed_seq(p, b);
  const int64_t ki = t * p.k_st + hk * p.k_sh;
  const float k0 = at(p.K, ki, lane, D), k1 = at(p.K, ki, lane + 64, D), v0 = at(p.V, ki, lane, D), v1 = at(p.V, ki, lane + 64, D);
  float dk0 = 0.f, dk1 = 0.f, dv0 = 0.f, dv1 = 0.f;
  for (int h = hk * p.G; h < (hk + 1) * p.G; ++h)
    for (int i = max(t - s.k0 - (s.m - s.n), 0); i < s.n; ++i) {
      const int64_t qi = (int64_t)(s.q0 + i) * p.q_st + h * p.q_sh, yi = (int64_t)(s.q0 + i) * p.y_st + h * p.y_sh;
      const float q0 = at(p.Q, qi, lane, D), q1 = at(p.Q, qi, lane + 64, D), g0 = at(p.dY, yi, lane, D), g1 = at(p.dY, yi, lane + 64, D);
      const float x = p.scale * wave_sum(q0 * k0 + q1 * k1);
      const float e = expf(x - p.lse[(int64_t)(h - p.lse_h0) * p.Tq + s.q0 + i]);
      const float ds = e * (wave_sum(g0 * v0 + g1 * v1) - p.delta[(int64_t)(h - p.delta_h0) * p.Tq + s.q0 + i]);
      dv0 += e * g0;
      dv1 += e * g1;
      dk0 += ds * q0;
      dk1 += ds * q1;
    }
  uint16_t *dK = (uint16_t*)p.dK + ki, *dV = (uint16_t*)p.dV + ki;
  if (lane < D) { dK[lane] = f2bf(p.scale * dk0); dV[lane] = f2bf(dv0); }
  if (lane + 64 < D) { dK[lane + 64] = f2bf(p.scale * dk1); dV[lane + 64] = f2bf(dv1); }
}

dim3 rows(const PackedP& p) { return dim3(p.Tq, (p.h1 - p.h0) * p.G); }

}  // namespace

hipError_t launch_packed_fwd(const PackedP& p, hipStream_t st) {
  packed_row_kernel<0><<<rows(p), 64, 0, st>>>(p);
  return hipGetLastError();
}
hipError_t launch_packed_stat(const PackedP& p, hipStream_t st) {
  packed_row_kernel<1><<<rows(p), 64, 0, st>>>(p);
  return hipGetLastError();
}
hipError_t launch_packed_delta(const PackedP& p, hipStream_t st) {
  packed_delta_kernel<<<rows(p), 64, 0, st>>>(p);
  return hipGetLastError();
}
hipError_t launch_packed_dq(const PackedP& p, hipStream_t st) {
  packed_row_kernel<2><<<rows(p), 64, 0, st>>>(p);
  return hipGetLastError();
}
hipError_t launch_packed_dkdv(const PackedP& p, hipStream_t st) {
  packed_key_kernel<<<dim3(p.Tk, p.h1 - p.h0), 64, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace ssa
