// Projections and routed experts in 8-bit integers.
//
//   rows to codes:  scale_r = max|x_r| / 127, code = rint(x * (127 / max|x_r|))
//   product:        C[m][n] = (sum_k a[m][k] w[n][k]) * a_scale[m] * w_scale[n]
//                   on v_mfma_i32_16x16x64_i8, the sum exact in 32 bits
//   experts:        rows to codes; gate/up over the routing lists with the SwiGLU
//                   epilogue; hidden rows to codes; down; the weighted sum of a
//                   row's experts in slot order
#include <math.h>

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace darts {

typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------ rows to codes
// The magnitude is found on the bits without the sign, whose order as integers
// puts infinities and NaN behind every finite number: a row that holds one gets
// the scale NaN and codes 0, so every product with it is NaN.  Rows whose
// magnitude is below 2^-119 (a scale would not be a normal number) get scale 0
// and codes 0.
constexpr uint32_t kTinyBits = 0x04000000u;      // 2^-119
__device__ __forceinline__ void row_scale(uint32_t top, float& up, float& scale) {
  const float m = __uint_as_float(top);
  up = top < kTinyBits || top >= 0x7f800000u ? 0.f : __fdiv_rn(127.0f, m);
  scale = top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : top < kTinyBits ? 0.f : __fdiv_rn(m, 127.0f);
}
// |x * up| <= 127 (1 + 2^-23), so a code stays within 127; up 0 gives code 0
// whatever x is.
__device__ __forceinline__ int code_of(float x, float up) {
  return up == 0.f ? 0 : (int)__builtin_rintf(x * up);
}

template <bool BF16>
__device__ __forceinline__ float load_x(const void* x, int64_t i) {
  return BF16 ? bf16_to_f32(((const bf16_t*)x)[i]) : ((const float*)x)[i];
}

// One block of 256 threads per row.
template <bool BF16>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const void* __restrict__ x, int cols, int64_t ldx,
                                                            int8_t* __restrict__ q, float* __restrict__ scale) {
  __shared__ uint32_t red[4];
  const int64_t r = blockIdx.x;
  uint32_t top = 0;
  for (int c = threadIdx.x; c < cols; c += 256)
    top = max(top, __float_as_uint(load_x<BF16>(x, r * ldx + c)) & 0x7fffffffu);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();
  top = max(max(red[0], red[1]), max(red[2], red[3]));
  float up, sc;
  row_scale(top, up, sc);
  if (threadIdx.x == 0) scale[r] = sc;
  for (int c = threadIdx.x; c < cols; c += 256) q[r * cols + c] = (int8_t)code_of(load_x<BF16>(x, r * ldx + c), up);
}

hipError_t launch_quantize_rows(const void* x, int64_t rows, int cols, int64_t ldx, bool bf16, int8_t* q, float* scale,
                                hipStream_t st) {
  for (int64_t r = 0; r < rows; r += INT32_MAX / 256) {
    const dim3 grid((unsigned)std::min<int64_t>(rows - r, INT32_MAX / 256));
    const char* xr = (const char*)x + r * ldx * (bf16 ? 2 : 4);
    if (bf16) hipLaunchKernelGGL(quantize_rows_kernel<true>, grid, dim3(256), 0, st, xr, cols, ldx, q + r * cols, scale + r);
    else hipLaunchKernelGGL(quantize_rows_kernel<false>, grid, dim3(256), 0, st, xr, cols, ldx, q + r * cols, scale + r);
  }
  return hipGetLastError();
}

// ------------------------------------------------------------------ products
__device__ __forceinline__ float silu_i8(float g) { return g / (1.0f + __expf(-g)); }

// What a tile of a product reads and writes.
struct I8Tile {
  const int8_t *a, *w;            // rows of K codes
  const float *a_scale, *w_scale;
  void* c;
  int rows, N, K, ldc;            // rows of the product; channels
  const int32_t* arow;            // NULL, or the row of a (and a_scale) of each of them
};

template <int EPI>
__device__ __forceinline__ void store_i8(void* c, int64_t at, float v) {
  if (EPI == EPI_F32) ((float*)c)[at] = v;
  else if (EPI == EPI_ADD_F32) ((float*)c)[at] += v;
  else ((bf16_t*)c)[at] = f32_to_bf16(v);
}

// A 64 x 64 tile by four wavefronts of 16 rows each; operands go straight from
// memory into the matrix instructions' registers.  Codes past K are zero, rows
// past the last repeat it and are not stored.
template <int EPI>
__device__ __forceinline__ void i8_tile(const I8Tile& t, int m0, int n0) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, fr = lane & 15, fq = lane >> 4;
  int row = min(m0 + 16 * w + fr, t.rows - 1);
  if (t.arow) row = t.arow[row];
  const int8_t* a = t.a + (int64_t)row * t.K;
  const int8_t* b[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) b[j] = t.w + (int64_t)min(n0 + 16 * j + fr, t.N - 1) * t.K;
  i32x4_t acc[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = (i32x4_t){0, 0, 0, 0};
  for (int k = 16 * fq; k < ((t.K + 63) & ~63); k += 64) {
    i32x4_t x = {0, 0, 0, 0}, y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = x;
    if (k < t.K) {
      x = *(const i32x4_t*)(a + k);
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = *(const i32x4_t*)(b[j] + k);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, y[j], acc[j], 0, 0, 0);
  }
  // lane: rows 4 * (lane / 16) + i, column lane % 16
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + 16 * w + 4 * fq + i;
    if (m >= t.rows) continue;
    const float sa = t.a_scale[t.arow ? t.arow[m] : m];
#pragma unroll
    for (int j = 0; j < 4; j += EPI == EPI_SWIGLU ? 2 : 1) {
      const int n = n0 + 16 * j + fr;
      if (n >= t.N) continue;
      const float v = (float)acc[j][i] * sa * t.w_scale[n];
      if constexpr (EPI == EPI_SWIGLU) {
        const float u = (float)acc[j + 1][i] * sa * t.w_scale[n + 16];
        store_i8<EPI_BF16>(t.c, (int64_t)m * t.ldc + (n >> 5) * 16 + fr, silu_i8(v) * u);
      } else {
        store_i8<EPI>(t.c, (int64_t)m * t.ldc + n, v);
      }
    }
  }
}

template <int EPI>
__global__ void __launch_bounds__(256) gemm_i8_kernel(I8Tile t, int mt) {
  i8_tile<EPI>(t, (int)(blockIdx.x % mt) * 64, (int)(blockIdx.x / mt) * 64);
}

// Expert e owns rows [off[e], off[e] + cnt[e]) of C, and of A or of the row list
// into A; mtiles lists the non-empty row tiles.
struct I8Groups {
  const int32_t *off, *cnt, *mtiles, *n_mtiles;
};
template <int EPI>
__global__ void __launch_bounds__(256) gemm_i8_grouped_kernel(I8Tile t, I8Groups g, int nt) {
  const int total = g.n_mtiles[0] * nt;
  for (int it = blockIdx.x; it < total; it += gridDim.x) {
    const int mt = g.mtiles[it / nt], e = mt >> 16;
    const int64_t off = g.off[e];
    I8Tile u = t;
    if (t.arow) {
      u.arow = t.arow + off;
    } else {
      u.a = t.a + off * t.K;
      u.a_scale = t.a_scale + off;
    }
    u.w = t.w + (int64_t)e * t.N * t.K;
    u.w_scale = t.w_scale + (int64_t)e * t.N;
    u.c = (char*)t.c + off * t.ldc * (EPI == EPI_F32 || EPI == EPI_ADD_F32 ? 4 : 2);
    u.rows = g.cnt[e];
    i8_tile<EPI>(u, (mt & 0xffff) * 64, it % nt * 64);
  }
}

size_t gemm_i8_workspace_bytes(int, int, int) { return 0; }

hipError_t launch_gemm_i8(const int8_t* a, const float* a_scale, const int8_t* w, const float* w_scale, void* c, int M,
                          int N, int K, int epi, void*, size_t, hipStream_t st) {
  if (M <= 0) return hipSuccess;
  const int mt = (M + 63) / 64;
  const int64_t blocks = (int64_t)mt * ((N + 63) / 64);
  if (blocks > INT32_MAX / 256) return hipErrorInvalidValue;
  const I8Tile t{a, w, a_scale, w_scale, c, M, N, K, epi == EPI_SWIGLU ? N / 2 : N, nullptr};
  const dim3 grid((unsigned)blocks), blk(256);
  switch (epi) {
    case EPI_F32: hipLaunchKernelGGL(gemm_i8_kernel<EPI_F32>, grid, blk, 0, st, t, mt); break;
    case EPI_BF16: hipLaunchKernelGGL(gemm_i8_kernel<EPI_BF16>, grid, blk, 0, st, t, mt); break;
    case EPI_ADD_F32: hipLaunchKernelGGL(gemm_i8_kernel<EPI_ADD_F32>, grid, blk, 0, st, t, mt); break;
    case EPI_SWIGLU: hipLaunchKernelGGL(gemm_i8_kernel<EPI_SWIGLU>, grid, blk, 0, st, t, mt); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

// ------------------------------------------------------------ routed experts
// out[r] = sum_j w[r][j] * y[pos(r, j)] in slot order, fp32 sums, 8 columns per
// thread.  A place without an expert adds w * 0: nothing, or NaN for the weight
// NaN of a row that the router could not read.
template <int EPI>
__global__ void __launch_bounds__(256) combine_i8_kernel(const bf16_t* __restrict__ y, int d, int k,
                                                         const int32_t* __restrict__ pos_of,
                                                         const float* __restrict__ weights, void* __restrict__ out) {
  const int64_t r = blockIdx.x;
  for (int c = threadIdx.x * 8; c < d; c += 256 * 8) {
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < k; ++j) {
      const int p = pos_of[r * k + j];
      const float wj = weights[r * k + j];
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (p >= 0) v = *(const uint4*)(y + (int64_t)p * d + c);
      const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[2 * i] = fmaf(wj, bf16_to_f32((bf16_t)(u[i] & 0xffffu)), s[2 * i]);
        s[2 * i + 1] = fmaf(wj, bf16_to_f32((bf16_t)(u[i] >> 16)), s[2 * i + 1]);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) store_i8<EPI>(out, r * d + c + i, s[i]);
  }
}

// Workspace of the expert layer, in this order, each part 256-byte aligned.
struct FfnWork {
  int8_t *q, *hq;
  float *q_scale, *h_scale;
  int32_t *counts, *offsets, *mtiles, *n_mtiles, *mtiles_dn, *n_mtiles_dn, *blk, *pos_of, *row_of;
  bf16_t *h, *y;
};
static size_t ffn_layout(int64_t rows, int d, int E, int k, int Fe, char* base, FfnWork* f) {
  size_t at = 0;
  auto part = [&](size_t bytes) {
    char* p = base ? base + at : nullptr;
    at += (bytes + 255) / 256 * 256;
    return p;
  };
  const size_t pairs = (size_t)rows * k;
  FfnWork t;
  t.q = (int8_t*)part((size_t)rows * d);
  t.q_scale = (float*)part((size_t)rows * 4);
  t.counts = (int32_t*)part((size_t)E * 4);
  t.offsets = (int32_t*)part((size_t)E * 4);
  t.mtiles = (int32_t*)part((pairs / kGroupedTileRowsMin + E) * 4);
  t.n_mtiles = (int32_t*)part(4);
  t.mtiles_dn = (int32_t*)part((pairs / kGroupedTileRowsMin + E) * 4);
  t.n_mtiles_dn = (int32_t*)part(4);
  t.blk = (int32_t*)part((size_t)kMoeBlocks * E * 4);
  t.pos_of = (int32_t*)part(pairs * 4);
  t.row_of = (int32_t*)part(pairs * 4);
  t.h = (bf16_t*)part(pairs * Fe * 2);
  t.hq = (int8_t*)part(pairs * Fe);
  t.h_scale = (float*)part(pairs * 4);
  t.y = (bf16_t*)part(pairs * d * 2);
  if (f) *f = t;
  return at;
}
size_t moe_ffn_i8_workspace_bytes(int64_t rows, int d, int E, int k, int Fe) {
  return ffn_layout(rows, d, E, k, Fe, nullptr, nullptr);
}

hipError_t launch_moe_ffn_i8(const FfnI8Args& a, hipStream_t st) {
  if (a.n_rows <= 0) return hipSuccess;
  FfnWork f;
  if (ffn_layout(a.n_rows, a.d, a.E, a.k, a.Fe, (char*)a.ws, &f) > a.ws_bytes) return hipErrorInvalidValue;
  hipError_t e = launch_quantize_rows(a.x, a.n_rows, a.d, a.d, true, f.q, f.q_scale, st);
  if (e != hipSuccess) return e;
  const int n_pairs = a.n_rows * a.k;
  MoeListArgs l{};
  l.topk_id = a.ids; l.n_pairs = n_pairs; l.E = a.E; l.k = a.k;
  l.counts = f.counts; l.offsets = f.offsets;
  l.mtiles = f.mtiles; l.n_mtiles = f.n_mtiles; l.mtiles_dn = f.mtiles_dn; l.n_mtiles_dn = f.n_mtiles_dn;
  l.tile_rows = l.tile_rows_dn = kGroupedTileRowsMin;
  l.blk = f.blk; l.pos_of = f.pos_of; l.row_of = f.row_of;
  if ((e = launch_moe_lists(l, st)) != hipSuccess) return e;
  const I8Groups gu{f.offsets, f.counts, f.mtiles, f.n_mtiles}, dn{f.offsets, f.counts, f.mtiles_dn, f.n_mtiles_dn};
  const I8Tile t1{f.q, a.w_gu, f.q_scale, a.s_gu, f.h, 0, 2 * a.Fe, a.d, a.Fe, f.row_of};
  hipLaunchKernelGGL(gemm_i8_grouped_kernel<EPI_SWIGLU>, dim3(1024), dim3(256), 0, st, t1, gu, (2 * a.Fe + 63) / 64);
  if ((e = launch_quantize_rows(f.h, n_pairs, a.Fe, a.Fe, true, f.hq, f.h_scale, st)) != hipSuccess) return e;
  const I8Tile t2{f.hq, a.w_down, f.h_scale, a.s_down, f.y, 0, a.d, a.Fe, a.d, nullptr};
  hipLaunchKernelGGL(gemm_i8_grouped_kernel<EPI_BF16>, dim3(1024), dim3(256), 0, st, t2, dn, (a.d + 63) / 64);
  if (a.epi == EPI_ADD_F32)
    hipLaunchKernelGGL(combine_i8_kernel<EPI_ADD_F32>, dim3(a.n_rows), dim3(256), 0, st, f.y, a.d, a.k, f.pos_of,
                       a.weights, a.out);
  else
    hipLaunchKernelGGL(combine_i8_kernel<EPI_BF16>, dim3(a.n_rows), dim3(256), 0, st, f.y, a.d, a.k, f.pos_of, a.weights,
                       a.out);
  return hipGetLastError();
}

}  // namespace darts
