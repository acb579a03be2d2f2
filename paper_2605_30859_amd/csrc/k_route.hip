// Routing of rows to experts: scores, a balance bias, expert groups, the k best
// experts and their weights.
//
//   s_e = softmax(l)_e or 1 / (1 + exp(-l_e)),  t_e = s_e + b_e
//   group value: the sum of the group's group_best (1 or 2) largest t; the
//   top_groups best groups stay, and of their experts the k largest t;
//   w_j = s of the j-th, divided by the sum of the k, times a factor.
//
// Which of two experts is taken hangs on the last digits of their scores: by
// definition they have 64 bits, and equal ones go by the lower id.
//
// Few rows need the definition's arithmetic for all experts.  LPR lanes hold a row,
// NPL consecutive experts each, and the best are taken one after the other by a
// maximum over the row of
//  * the logits themselves where there is neither bias nor group: scores rise with
//    them, and equal logits have equal scores;
//  * t in float32 otherwise, off by less than 2^-20 (1 + |t|), with sigmoids 2^-22.
//    One more than k are taken, and these ordered by their 64-bit t.
// Where a value left out is so near to the last one taken (kNearSoftmax, kNearSigmoid;
// kNearLogit between any two logits) that the definition might see them otherwise, or
// scores saturate, the row is done again by the definition, by the whole wavefront.
//
// Bound by instructions.  32768 rows of 128 experts: 51 us by the definition alone
// (a wavefront per row, ranks by comparing every pair), 11 us so; reading the
// logits takes 3 us.  976 rows of 256 experts in 8 groups with a bias: 15 and 9 us.
#include <math.h>

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace darts {

constexpr int kRouteWaves = 4;       // wavefronts per block
// Logits: s_a / s_b >= 1 + (l_a - l_b) (1 - s_a), for l_a <= 15 and a distance of
// 2^-26 at least 1 + 4e-15, which 64 bits tell apart.
constexpr float kNearLogit = 1.490116119384765625e-08f;   // 2^-26
constexpr float kSigmoidTop = 15.f, kScoreLow = -700.f;
// Relative to 1 + |t|, for a pair of groups to 1 and the mean of either's experts' |t|:
// four errors of softmax scores (the exponentials', and their sum's); of sigmoids
// 1.25 2^-23 + 2^-24 |t| each and the sums' roundings.  A row done again costs a small
// call 6 to 9 us.
constexpr float kNearSoftmax = 3.814697265625e-06f, kNearSigmoid = 9.5367431640625e-07f;   // 2^-18, 2^-20

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
__device__ __forceinline__ float load_logit(const RouteArgs& a, int64_t r, int e) {
  return a.bf16 ? bf16_to_f32(((const bf16_t*)a.logits)[r * a.ld + e]) : ((const float*)a.logits)[r * a.ld + e];
}

// What a wavefront needs to do a row by the definition.
template <int NPL>
struct RouteLds {
  double t[64 * NPL];
};

// Row r by the definition, one wavefront, E <= 64 * NPL.
template <int NPL>
__device__ __forceinline__ void route_exact(const RouteArgs& a, int64_t r, RouteLds<NPL>& lds) {
  const int lane = threadIdx.x & 63;
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
      l[j] = load_logit(a, r, e);
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
  // t, -inf for an expert that is not to be had
  double t[NPL];
#pragma unroll
  for (int j = 0; j < NPL; ++j) {
    t[j] = !bad && l[j] > -INFINITY && b[j] > -INFINITY ? s[j] + (double)b[j] : -INFINITY;
    lds.t[lane + 64 * j] = t[j];
  }
  if (a.n_groups > 1) {
    wave_lds_fence();
    // lane g: the two best of group g, and its place among the groups
    const int per = E / a.n_groups;
    double v0 = -INFINITY, v1 = -INFINITY;
    if (lane < a.n_groups)
      for (int i = 0; i < per; ++i) {
        const double q = lds.t[lane * per + i];
        v1 = q > v0 ? v0 : q > v1 ? q : v1;
        v0 = q > v0 ? q : v0;
      }
    const double v = a.group_best == 2 && v1 > -INFINITY ? v0 + v1 : v0;
    int before = 0;
    for (int g = 0; g < a.n_groups; ++g) {
      const double u = __shfl(v, g, 64);
      before += u > v || (u == v && g < lane);
    }
    const uint64_t chosen = __ballot(lane < a.n_groups && before < a.top_groups);
    wave_lds_fence();
#pragma unroll
    for (int j = 0; j < NPL; ++j) {
      const int e = lane + 64 * j;
      if (e >= E || !((chosen >> (e / per)) & 1)) t[j] = -INFINITY;
      lds.t[e] = t[j];
    }
  }
  // the best that is left, k times
  int id = -1;
  double v = 0.0;
  for (int i = 0; i < k; ++i) {
    double m = t[0], ms = s[0];
    int me = lane;
#pragma unroll
    for (int j = 1; j < NPL; ++j)
      if (t[j] > m) {                                  // ids rise with j: the lower one of equals
        m = t[j];
        ms = s[j];
        me = lane + 64 * j;
      }
    double best = m;
    int e = me;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const double u = __shfl_xor(best, o, 64);
      const int f = __shfl_xor(e, o, 64);
      if (u > best || (u == best && f < e)) {
        best = u;
        e = f;
      }
    }
    if (best == -INFINITY) break;
    const double bs = __shfl(ms, e & 63, 64);
    if (lane == i) {
      id = e;
      v = bs;
    }
#pragma unroll
    for (int j = 0; j < NPL; ++j)
      if (e == lane + 64 * j) t[j] = -INFINITY;
  }
  if (a.renorm) {
    const double sum = wave_sum_f64(v);
    v = sum > 0.0 ? v / sum : 0.0;
  }
  if (lane < k) {
    a.ids[r * k + lane] = id;
    a.weights[r * k + lane] = bad ? __uint_as_float(0x7fc00000u) : (float)(v * (double)a.factor);
  }
}

// Over the LPR lanes of a row, the result in all of them.
template <int LPR, typename T, typename Op>
__device__ __forceinline__ T row_reduce(T v, Op op) {
  static_assert(sizeof(T) == 4, "32-bit values");
#define DARTS_ROR(N) \
  v = op(v, __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, true)));
  DARTS_ROR(8) DARTS_ROR(4) DARTS_ROR(2) DARTS_ROR(1)
#undef DARTS_ROR
  if (LPR >= 32) v = op(v, __shfl_xor(v, 16, 64));
  if (LPR >= 64) v = op(v, __shfl_xor(v, 32, 64));
  return v;
}
__device__ __forceinline__ float max_f(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float min_f(float a, float b) { return fminf(a, b); }
__device__ __forceinline__ float add_f(float a, float b) { return a + b; }

template <int NPL, bool VEC>
__device__ __forceinline__ void load_logits(const RouteArgs& a, int64_t r, int e0, float (&l)[NPL]) {
  if constexpr (VEC) {
    if (a.bf16) {
      const bf16_t* p = (const bf16_t*)a.logits + r * a.ld + e0;
#pragma unroll
      for (int j = 0; j < NPL; j += 4) {
        const u32x2_t v = *(const u32x2_t*)(p + j);
        l[j] = __uint_as_float(v[0] << 16);
        l[j + 1] = __uint_as_float(v[0] & 0xffff0000u);
        l[j + 2] = __uint_as_float(v[1] << 16);
        l[j + 3] = __uint_as_float(v[1] & 0xffff0000u);
      }
    } else {
      const float* p = (const float*)a.logits + r * a.ld + e0;
#pragma unroll
      for (int j = 0; j < NPL; j += 4) {
        const f32x4_t v = *(const f32x4_t*)(p + j);
        l[j] = v[0]; l[j + 1] = v[1]; l[j + 2] = v[2]; l[j + 3] = v[3];
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < NPL; ++j) l[j] = e0 + j < a.n_experts ? load_logit(a, r, e0 + j) : -INFINITY;
  }
}

// E <= LPR * NPL, k < LPR.  MODE: ordered by the logits (no bias, no groups), by t,
// or by t within groups of whole lanes whose number is a power of two.  VEC: E is
// a multiple of NPL and rows of logits are aligned for it.
enum RouteMode { ROUTE_LOGITS, ROUTE_SCORES, ROUTE_GROUPS };
template <int LPR, int NPL, int MODE, bool VEC>
__global__ void __launch_bounds__(64 * kRouteWaves) route_kernel(RouteArgs a) {
  constexpr int RPW = 64 / LPR;
  __shared__ RouteLds<LPR * NPL / 64> lds[kRouteWaves];
  __shared__ int32_t chosen[kRouteWaves][64];         // a row's ids in the order they are taken
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int sub = lane % LPR, first = lane - sub, e0 = sub * NPL;
  const int64_t r = ((int64_t)blockIdx.x * kRouteWaves + w) * RPW + lane / LPR;
  const bool live = r < a.n_rows;
  const int E = a.n_experts, k = a.top_k;
  const int64_t rr = live ? r : a.n_rows - 1;         // lanes past the end repeat the last row, unwritten
  float l[NPL], t[NPL];
#pragma unroll
  for (int j = 0; j < NPL; ++j) l[j] = -INFINITY;
  if (!VEC || e0 < E) load_logits<NPL, VEC>(a, rr, e0, l);
  float mx = -INFINITY, odd = -INFINITY;              // odd: +inf where a logit or bias is +inf or NaN
#pragma unroll
  for (int j = 0; j < NPL; ++j) {
    odd = l[j] < INFINITY ? odd : INFINITY;
    mx = fmaxf(mx, l[j]);
  }
  mx = row_reduce<LPR>(mx, max_f);
  if constexpr (MODE == ROUTE_LOGITS) {
#pragma unroll
    for (int j = 0; j < NPL; ++j) t[j] = l[j];
  } else {
    if (a.sigmoid) {
#pragma unroll
      for (int j = 0; j < NPL; ++j) t[j] = __fdiv_rn(1.0f, 1.0f + expf(-l[j]));
    } else {
      const float base = mx == -INFINITY ? 0.f : mx;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < NPL; ++j) {
        t[j] = __expf(l[j] - base);
        sum += t[j];
      }
      sum = row_reduce<LPR>(sum, add_f);
      const float inv = 1.0f / sum;
#pragma unroll
      for (int j = 0; j < NPL; ++j) t[j] *= inv;
    }
    if (a.bias) {
      float b[NPL];
#pragma unroll
      for (int j = 0; j < NPL; ++j) b[j] = a.bias[min(e0 + j, E - 1)];
#pragma unroll
      for (int j = 0; j < NPL; ++j) {
        odd = b[j] < INFINITY ? odd : INFINITY;
        t[j] += b[j];
      }
    }
#pragma unroll
    for (int j = 0; j < NPL; ++j) t[j] = l[j] == -INFINITY ? -INFINITY : t[j];
  }
  const bool bad = row_reduce<LPR>(odd, max_f) > 0.f;
  bool near = false;
  const float near_by = a.sigmoid ? kNearSigmoid : kNearSoftmax;
  auto too_near = [&](float hi, float lo) {           // hi >= lo, neighbours in the order; lo may be -inf
    const float gap = hi - lo;
    if (MODE == ROUTE_LOGITS) return gap > 0.f && gap < kNearLogit;
    return gap < near_by * (1.0f + fmaxf(fabsf(hi), fabsf(lo)));
  };
  if constexpr (MODE == ROUTE_GROUPS) {
    // the two best of each group's lanes, then the groups' values against each other
    const int lanes = E / a.n_groups / NPL;
    float v0 = -INFINITY, v1 = -INFINITY;
#pragma unroll
    for (int j = 0; j < NPL; ++j) {
      v1 = fmaxf(v1, fminf(v0, t[j]));
      v0 = fmaxf(v0, t[j]);
    }
    for (int o = 1; o < lanes; o <<= 1) {
      const float u0 = __shfl_xor(v0, o, 64), u1 = __shfl_xor(v1, o, 64);
      v1 = fmaxf(fminf(v0, u0), fmaxf(v1, u1));
      v0 = fmaxf(v0, u0);
    }
    // Half of a value, or of two experts' mean, which finite scores do not overflow.  Its
    // error goes by its own experts' sizes (of opposite signs they may have a small sum).
    const bool two = a.group_best == 2 && v1 > -INFINITY;
    const float f = a.group_best == 2 ? 0.25f : 0.5f;
    const float v = two ? f * v0 + f * v1 : f * v0;
    const float err = v0 > -INFINITY ? 0.5f * near_by * (f + f * fabsf(v0) + (two ? f * fabsf(v1) : 0.f)) : 0.f;
    const int g = sub / lanes;
    int before = 0;
#pragma unroll 4
    for (int i = 0; i < a.n_groups; ++i) {
      const float u = __shfl(v, first + i * lanes, 64);
      before += (u > v) | ((u == v) & (i < g));
    }
    const bool in = e0 < E, stays = in && before < a.top_groups;
    const float low = row_reduce<LPR>(stays ? v - err : INFINITY, min_f);
    const float high = row_reduce<LPR>(in && !stays ? v + err : -INFINITY, max_f);
    near = low > -INFINITY && low <= high;
#pragma unroll
    for (int j = 0; j < NPL; ++j) t[j] = stays ? t[j] : -INFINITY;
  }
  const uint64_t below = (((uint64_t)1 << sub) - 1) << first;      // lanes of this row with lower ids
  chosen[w][lane] = -1;
  // taken: k of the logits, whose neighbours are then k + 1; of scores k + 1, and the
  // one left out after them is a neighbour of the k-th
  constexpr int more = MODE == ROUTE_LOGITS ? 0 : 1;
  float last = INFINITY, mine = 0.f;
  for (int i = 0; i <= k + more; ++i) {
    float m = t[0];
#pragma unroll
    for (int j = 1; j < NPL; ++j) m = fmaxf(m, t[j]);
    const float best = row_reduce<LPR>(m, max_f);
    if (MODE == ROUTE_LOGITS || i == k + 1) near |= best > -INFINITY && too_near(last, best);
    if (MODE == ROUTE_LOGITS || i == k - 1) last = best;
    if (i == k + more) break;
    mine = sub == i ? best : mine;
    // of equals the lowest lane, and in it the lowest expert
    const uint64_t has = __ballot(m == best);
    bool own = m == best && (has & below) == 0 && best > -INFINITY;
    int id = -1;
#pragma unroll
    for (int j = 0; j < NPL; ++j) {
      const bool it = own && t[j] == best;
      t[j] = it ? -INFINITY : t[j];
      id = it ? e0 + j : id;
      own = own && !it;
    }
    if (id >= 0) chosen[w][first + i] = id;
  }
  wave_lds_fence();
  const int my_id = chosen[w][lane];
  float my_l = mine;
  if (MODE != ROUTE_LOGITS) my_l = my_id >= 0 ? load_logit(a, rr, my_id) : 0.f;
  // scores that saturate: sigmoids near 1, or exponentials near the end of their range
  if constexpr (MODE == ROUTE_LOGITS) {
    const float low = row_reduce<LPR>(my_id >= 0 ? my_l : INFINITY, min_f);
    near |= a.sigmoid ? mx > kSigmoidTop || low < kScoreLow : low - mx < kScoreLow;
  }
  double v = exp(a.sigmoid ? -(double)my_l : (double)my_l - (double)mx);
  if (a.sigmoid) {
    v = 1.0 / (1.0 + v);
  } else if (MODE != ROUTE_LOGITS || !a.renorm) {
    double total = 0.0;
#pragma unroll
    for (int j = 0; j < NPL; ++j) total += l[j] > -INFINITY ? exp((double)l[j] - (double)mx) : 0.0;
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) total += __shfl_xor(total, o, 64);
    v = v / total;
  }
  int place = sub;
  if constexpr (MODE != ROUTE_LOGITS) {
    const double t64 = my_id >= 0 ? v + (a.bias ? (double)a.bias[my_id] : 0.0) : -INFINITY;
    place = 0;
#pragma unroll 3
    for (int i = 0; i <= k; ++i) {
      const double u = __shfl(t64, first + i, 64);
      const int id = __shfl(my_id, first + i, 64);
      place += (u > t64) | ((u == t64) & (id < my_id));
    }
    if (my_id < 0 || bad) place = sub;                // behind those that were taken
    if (sub > k) place = k;
  }
  v = my_id >= 0 && place < k ? v : 0.0;
  if (a.renorm) {
    double sum = v;
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    v = sum > 0.0 ? v / sum : 0.0;
  }
  // near and bad are the same in the whole row; a row that is done again is written there
  // alone, as other lanes hold its places
  if (live && place < k && (bad || !near)) {
    a.ids[r * k + place] = bad ? -1 : my_id;
    a.weights[r * k + place] = bad ? __uint_as_float(0x7fc00000u) : (float)(v * (double)a.factor);
  }
  uint64_t again = __ballot(near && live && !bad && sub == 0);
  while (again) {
    const int f = __builtin_ctzll(again);
    again &= again - 1;
    route_exact<LPR * NPL / 64>(a, ((int64_t)blockIdx.x * kRouteWaves + w) * RPW + f / LPR, lds[w]);
  }
}

// Groups of any size, and 64 experts a row: by the definition alone.
template <int NPL>
__global__ void __launch_bounds__(64 * kRouteWaves) route_exact_kernel(RouteArgs a) {
  __shared__ RouteLds<NPL> lds[kRouteWaves];
  const int w = threadIdx.x >> 6;
  const int64_t r = (int64_t)blockIdx.x * kRouteWaves + w;
  if (r < a.n_rows) route_exact<NPL>(a, r, lds[w]);
}

template <int LPR, int NPL>
static void route_go(const RouteArgs& a, hipStream_t st) {
  constexpr int rows = kRouteWaves * (64 / LPR), npl = LPR * NPL / 64;
  const int per = a.n_experts / a.n_groups, lanes = per / NPL;
  const bool any = a.top_k >= LPR || (a.n_groups > 1 && (per % NPL || lanes & (lanes - 1)));
  const dim3 blk(64 * kRouteWaves);
  if (any) {
    hipLaunchKernelGGL(route_exact_kernel<npl>, dim3((unsigned)((a.n_rows + kRouteWaves - 1) / kRouteWaves)), blk, 0, st, a);
    return;
  }
  const dim3 grid((unsigned)((a.n_rows + rows - 1) / rows));
  const int align = a.bf16 ? 8 : 16;                   // four logits
  const bool vec = a.n_experts % NPL == 0 && ((uintptr_t)a.logits % align) == 0 && a.ld % 4 == 0;
#define DARTS_ROUTE(MODE)                                                                            \
  if (vec) hipLaunchKernelGGL((route_kernel<LPR, NPL, MODE, true>), grid, blk, 0, st, a);            \
  else hipLaunchKernelGGL((route_kernel<LPR, NPL, MODE, false>), grid, blk, 0, st, a);
  if (a.n_groups > 1) {
    DARTS_ROUTE(ROUTE_GROUPS)
  } else if (a.bias) {
    DARTS_ROUTE(ROUTE_SCORES)
  } else {
    DARTS_ROUTE(ROUTE_LOGITS)
  }
#undef DARTS_ROUTE
}

hipError_t launch_route(const RouteArgs& all, hipStream_t st) {
  if (all.n_experts > 1024 || all.top_k > 64 || all.n_groups > 64) return hipErrorInvalidValue;
  constexpr int most = 1 << 24;        // rows of a launch: up to 64 threads each, fewer than 2^32 in all
  for (int64_t r = 0; r < all.n_rows; r += most) {
    RouteArgs a = all;
    a.logits = (const char*)all.logits + r * all.ld * (all.bf16 ? 2 : 4);
    a.ids += r * all.top_k;
    a.weights += r * all.top_k;
    a.n_rows = (int)std::min<int64_t>(all.n_rows - r, most);
    if (a.n_experts <= 64 && a.top_k < 16) route_go<16, 4>(a, st);
    else if (a.n_experts <= 128 && a.top_k < 16) route_go<16, 8>(a, st);
    else if (a.n_experts <= 256 && a.top_k < 32) route_go<32, 8>(a, st);
    else if (a.n_experts <= 512) route_go<64, 8>(a, st);
    else route_go<64, 16>(a, st);
  }
  return hipGetLastError();
}

}  // namespace darts
