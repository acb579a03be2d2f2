// Routing of rows to experts: scores, a balance bias, expert groups, the k best
// experts and their weights.
//
//   s_e = softmax(l)_e or 1 / (1 + exp(-l_e)),  t_e = s_e + b_e
//   group value: the sum of the group's group_best (1 or 2) largest t; the
//   top_groups best groups stay, and of their experts the k largest t;
//   w_j = s of the j-th, divided by the sum of the k, times a factor.
//
// Which of two experts is taken hangs on the last digits of their scores, so
// scores are computed in 64 bits and ordered by 64-bit keys: the score's bits in
// an order that unsigned integers have, the lowest 10 of them replaced by
// 1023 - e.  Scores that agree in all but their last 10 bits count as equal, and
// the lower id goes first.
//
// One wavefront per row, E <= 64 * NPL.  The k best are found by rank: every
// lane counts for each of its experts the larger keys in a copy that the whole
// wavefront reads from LDS, so no step waits for the one before.
#include <math.h>

#include "common.h"
#include "kernels.h"

namespace darts {

constexpr int kRouteWaves = 4;       // rows per block
constexpr int kRouteMaxPerLane = 16;
constexpr uint64_t kRouteIdBits = 1023;

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// LDS written by this wavefront is read by its other lanes.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_s_waitcnt(0xc07f);    // lgkmcnt(0)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// Unsigned order of 64-bit floating numbers (no NaN).
__device__ __forceinline__ uint64_t order_bits(double v) {
  const uint64_t b = (uint64_t)__double_as_longlong(v);
  return b ^ ((b >> 63) ? ~(uint64_t)0 : (uint64_t)1 << 63);
}

template <int NPL>
__global__ void __launch_bounds__(64 * kRouteWaves) route_kernel(RouteArgs a) {
  __shared__ __attribute__((aligned(16))) uint64_t keys[kRouteWaves][64 * NPL];
  __shared__ double best_s[kRouteWaves][64];
  __shared__ int32_t best_id[kRouteWaves][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t r = (int64_t)blockIdx.x * kRouteWaves + w;
  if (r >= a.n_rows) return;
  const int E = a.n_experts, k = a.top_k;
  float l[NPL], b[NPL];
  float mx = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int j = 0; j < NPL; ++j) {
    const int e = lane + 64 * j;
    l[j] = -INFINITY;
    b[j] = 0.f;
    if (e < E) {
      l[j] = a.bf16 ? bf16_to_f32(((const bf16_t*)a.logits)[r * a.ld + e]) : ((const float*)a.logits)[r * a.ld + e];
      if (a.bias) b[j] = a.bias[e];
    }
    bad |= !(l[j] < INFINITY) || !(b[j] < INFINITY);     // NaN or +inf
    mx = fmaxf(mx, l[j]);
  }
  bad = __any(bad);
  mx = wave_max(mx);
  double s[NPL], total = 0.0;
#pragma unroll
  for (int j = 0; j < NPL; ++j) {
    if (l[j] == -INFINITY) s[j] = 0.0;
    else s[j] = a.sigmoid ? 1.0 / (1.0 + exp(-(double)l[j])) : exp((double)l[j] - (double)mx);
    total += s[j];
  }
  if (!a.sigmoid) {
    total = wave_sum_f64(total);
#pragma unroll
    for (int j = 0; j < NPL; ++j) s[j] = total > 0.0 ? s[j] / total : 0.0;
  }
  // key 0: not to be had
  uint64_t key[NPL];
#pragma unroll
  for (int j = 0; j < NPL; ++j) {
    const int e = lane + 64 * j;
    const bool have = !bad && l[j] > -INFINITY && b[j] > -INFINITY;
    key[j] = have ? (order_bits(s[j] + (double)b[j]) & ~kRouteIdBits) | (kRouteIdBits - (uint64_t)e) : 0;
    keys[w][e] = key[j];
  }
  if (a.n_groups > 1) {
    wave_lds_fence();
    const int per = E / a.n_groups;
    // lane g: the group's best keys, their scores to the keys' precision
    uint64_t k0 = 0, k1 = 0;
    if (lane < a.n_groups)
      for (int i = 0; i < per; ++i) {
        const uint64_t q = keys[w][lane * per + i];
        k1 = q > k0 ? k0 : q > k1 ? q : k1;
        k0 = q > k0 ? q : k0;
      }
    auto score = [](uint64_t q) {
      q &= ~kRouteIdBits;
      return __longlong_as_double((long long)((q >> 63) ? q ^ ((uint64_t)1 << 63) : ~q & ~kRouteIdBits));
    };
    double v = k0 ? score(k0) : -INFINITY;
    if (a.group_best == 2 && k1) v += score(k1);
    const uint64_t mine = lane < a.n_groups && k0 ? (order_bits(v) & ~kRouteIdBits) | (kRouteIdBits - (uint64_t)lane) : 0;
    int before = 0;
    for (int g = 0; g < a.n_groups; ++g) before += __shfl(mine, g, 64) > mine;
    const uint64_t chosen = __ballot(mine != 0 && before < a.top_groups);
    wave_lds_fence();
#pragma unroll
    for (int j = 0; j < NPL; ++j) {
      const int e = lane + 64 * j;
      if (e >= E || !((chosen >> (e / per)) & 1)) key[j] = 0;
      keys[w][e] = key[j];
    }
  }
  if (lane < k) best_id[w][lane] = -1;
  wave_lds_fence();
  int rank[NPL];
#pragma unroll
  for (int j = 0; j < NPL; ++j) rank[j] = 0;
  const int E2 = (E + 1) & ~1;
#pragma unroll 8
  for (int y = 0; y < E2; y += 2) {
    const uint4 q = *(const uint4*)&keys[w][y];             // the same address in every lane
    const uint64_t q0 = ((uint64_t)q.y << 32) | q.x, q1 = ((uint64_t)q.w << 32) | q.z;
#pragma unroll
    for (int j = 0; j < NPL; ++j) rank[j] += (q0 > key[j]) + (q1 > key[j]);
  }
#pragma unroll
  for (int j = 0; j < NPL; ++j)
    if (key[j] != 0 && rank[j] < k) {
      best_s[w][rank[j]] = s[j];
      best_id[w][rank[j]] = lane + 64 * j;
    }
  wave_lds_fence();
  const int id = lane < k ? best_id[w][lane] : -1;
  double v = id >= 0 ? best_s[w][lane] : 0.0;
  if (a.renorm) {
    const double sum = wave_sum_f64(v);
    v = sum > 0.0 ? v / sum : 0.0;
  }
  if (lane < k) {
    a.ids[r * k + lane] = id;
    a.weights[r * k + lane] = bad ? __uint_as_float(0x7fc00000u) : (float)(v * (double)a.factor);
  }
}

hipError_t launch_route(const RouteArgs& a, hipStream_t st) {
  if (a.n_rows <= 0) return hipSuccess;
  if (a.n_experts > 64 * kRouteMaxPerLane || a.top_k > 64 || a.n_groups > 64) return hipErrorInvalidValue;
  const dim3 grid((unsigned)((a.n_rows + kRouteWaves - 1) / kRouteWaves)), blk(64 * kRouteWaves);
  if (a.n_experts <= 64) hipLaunchKernelGGL(route_kernel<1>, grid, blk, 0, st, a);
  else if (a.n_experts <= 128) hipLaunchKernelGGL(route_kernel<2>, grid, blk, 0, st, a);
  else if (a.n_experts <= 256) hipLaunchKernelGGL(route_kernel<4>, grid, blk, 0, st, a);
  else hipLaunchKernelGGL(route_kernel<kRouteMaxPerLane>, grid, blk, 0, st, a);
  return hipGetLastError();
}

}  // namespace darts
