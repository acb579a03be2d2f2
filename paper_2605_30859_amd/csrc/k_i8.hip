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
#include <atomic>

#include "common.h"
#include "gemm_tiles.h"
#include "kernels.h"
#include "moe_lists.h"

namespace darts {

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

// Eight elements of a row as float32, and eight codes.
template <bool BF16>
struct X8;
template <>
struct X8<true> {
  u32x4_t v;
  __device__ __forceinline__ void load(const void* x, int64_t i) { v = *(const u32x4_t*)((const bf16_t*)x + i); }
  __device__ __forceinline__ float at(int e) const {
    return __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16);
  }
};
template <>
struct X8<false> {
  f32x4_t v[2];
  __device__ __forceinline__ void load(const void* x, int64_t i) {
    v[0] = *(const f32x4_t*)((const float*)x + i);
    v[1] = *(const f32x4_t*)((const float*)x + i + 4);
  }
  __device__ __forceinline__ float at(int e) const { return v[e >> 2][e & 3]; }
};
template <bool BF16>
__device__ __forceinline__ float load_x(const void* x, int64_t i) {
  return BF16 ? bf16_to_f32(((const bf16_t*)x)[i]) : ((const float*)x)[i];
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

// WPR wavefronts per row, in blocks of four or sixteen.  VEC: rows of whole 16-byte pieces, codes
// ldq apart with zeros between them (else ldq is cols); the first kQuantKeep pieces
// of a lane stay in registers between the two passes, so rows of up to
// 64 * WPR * 32 elements are read once.
constexpr int kQuantKeep = 4;
template <bool BF16, bool VEC, int WPR>
__device__ __forceinline__ void quantize_row(const void* __restrict__ x, int64_t r, int t, uint32_t* red, int cols, int64_t ldx,
                                             int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale) {
  constexpr int T = 64 * WPR;                          // threads of the row
  X8<BF16> keep[kQuantKeep];
  uint32_t top = 0;
  const int n8 = cols / 8;
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < kQuantKeep; ++i)
      if (t + T * i < n8) keep[i].load(x, r * ldx + (t + T * i) * 8);
#pragma unroll
    for (int i = 0; i < kQuantKeep; ++i)
      if (t + T * i < n8)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(keep[i].at(e)) & 0x7fffffffu);
    for (int c = t + T * kQuantKeep; c < n8; c += T) {
      X8<BF16> v;
      v.load(x, r * ldx + c * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v.at(e)) & 0x7fffffffu);
    }
  } else {
    for (int c = t; c < cols; c += T) top = max(top, __float_as_uint(load_x<BF16>(x, r * ldx + c)) & 0x7fffffffu);
  }
  top = wave_max_u32(top);
  if constexpr (WPR > 1) {                             // in a block, every row at once
    if ((t & 63) == 0) red[t >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WPR; ++i) top = max(top, red[i]);
  }
  float up, sc;
  row_scale(top, up, sc);
  if (t == 0) scale[r] = sc;
  auto store = [&](const X8<BF16>& v, int c) {
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      w[h] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[h] |= ((uint32_t)code_of(v.at(4 * h + e), up) & 0xffu) << (8 * e);
    }
    *(uint2*)(q + r * ldq + c * 8) = make_uint2(w[0], w[1]);
  };
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < kQuantKeep; ++i)
      if (t + T * i < n8) store(keep[i], t + T * i);
    for (int c = t + T * kQuantKeep; c < n8; c += T) {
      X8<BF16> v;
      v.load(x, r * ldx + c * 8);
      store(v, c);
    }
    for (int c = n8 + t; c < ldq / 8; c += T) *(uint2*)(q + r * ldq + c * 8) = make_uint2(0u, 0u);
  } else {
    for (int c = t; c < cols; c += T) q[r * ldq + c] = (int8_t)code_of(load_x<BF16>(x, r * ldx + c), up);
  }
}

template <bool BF16, bool VEC, int WPR>
__global__ void __launch_bounds__(std::max(256, 64 * WPR))
    quantize_rows_kernel(const void* __restrict__ x, int64_t rows, int cols, int64_t ldx, int8_t* __restrict__ q, int64_t ldq,
                         float* __restrict__ scale) {
  __shared__ uint32_t red[WPR];
  const int64_t r = WPR == 1 ? (int64_t)blockIdx.x * 4 + threadIdx.x / 64 : blockIdx.x;
  if (WPR == 1 && r >= rows) return;
  quantize_row<BF16, VEC, WPR>(x, r, threadIdx.x % (64 * WPR), red, cols, ldx, q, ldq, scale);
}

template <bool BF16, bool VEC>
static hipError_t quantize_go(const void* x, int64_t rows, int cols, int64_t ldx, int8_t* q, int64_t ldq, float* scale,
                              hipStream_t st) {
  // A wavefront per row where it holds the row, and there are rows for every CU; four
  // up to what they hold, and 16 beyond.  Four and 16, bf16, us: 45 rows of 8192 2.8 /
  // 2.8, of 12288 3.5 / 3.0, of 24576 5.9 / 3.7; 7808 rows 30 / 38, 49 / 46, 132 / 99.
  constexpr int hold = 64 * 8 * kQuantKeep;
  const int wpr = cols <= hold && rows >= 2048 ? 1 : cols <= 4 * hold ? 4 : 16;
  const int64_t most = (int64_t)1 << 21;               // rows per launch
  for (int64_t r = 0; r < rows; r += most) {
    const int64_t n = std::min(rows - r, most);
    const char* xr = (const char*)x + r * ldx * (BF16 ? 2 : 4);
    auto go = [&](auto kern, unsigned blocks, int threads) {
      hipLaunchKernelGGL(kern, dim3(blocks), dim3(threads), 0, st, xr, n, cols, ldx, q + r * ldq, ldq, scale + r);
    };
    if (wpr == 1) go(quantize_rows_kernel<BF16, VEC, 1>, (unsigned)((n + 3) / 4), 256);
    else if (wpr == 4) go(quantize_rows_kernel<BF16, VEC, 4>, (unsigned)n, 256);
    else go(quantize_rows_kernel<BF16, VEC, 16>, (unsigned)n, 1024);
  }
  return hipGetLastError();
}

hipError_t launch_quantize_rows(const void* x, int64_t rows, int cols, int64_t ldx, bool bf16, int8_t* q, int64_t ldq,
                                float* scale, hipStream_t st) {
  const bool vec = cols % 8 == 0 && ldq % 8 == 0 && ((uintptr_t)x & 15) == 0 && ((uintptr_t)q & 7) == 0 &&
                   ldx * (bf16 ? 2 : 4) % 16 == 0;
  if (!vec && ldq != cols) return hipErrorInvalidValue;
  if (bf16) return vec ? quantize_go<true, true>(x, rows, cols, ldx, q, ldq, scale, st)
                       : quantize_go<true, false>(x, rows, cols, ldx, q, ldq, scale, st);
  return vec ? quantize_go<false, true>(x, rows, cols, ldx, q, ldq, scale, st)
             : quantize_go<false, false>(x, rows, cols, ldx, q, ldq, scale, st);
}

// ------------------------------------------------------------------ products
// The kernels of the bf16 products on codes (gemm_tiles.h): a 16-byte chunk holds
// 16 codes where it held 8 bf16, so the same tiles, LDS layouts and loads feed
// v_mfma_i32_16x16x64_i8, which takes as long as v_mfma_f32_16x16x32_bf16 and does
// twice the products.  K2 = K / 2 is K in the 16-bit units of those kernels.
//  * skinny (few rows): operands go straight from memory into registers, 8
//    wavefronts of a block split K and are added through LDS;
//  * ring: tiles through a ring of LDS stages;
//  * alternating groups (many rows): 256-row tiles on persistent blocks.
// The last two may split K over blocks: the partial sums are integers in a
// workspace, so neither the plan nor the order changes any result.

// Up to 16 * MT rows.  WK wavefronts share a strip of 16 channels, each a range of
// kw codes of K (a multiple of 64), and a block has 8 / WK strips.  Lane (r, q)
// loads 16 codes of row r; the loads of U steps of 64 are issued before the
// products of the U steps before.  (One row, 6144 x 4096 from memory: 7.7 us with U
// 2, 7.9 with 4, 7.6 with 8, 24576 x 4096 19.9, 22.7, 20.9; non-temporal loads 8.6
// and 25 us with U 4, and 20-40% behind where a cache holds the weights.)
template <int MT, int WK, int EPI>
__global__ void __launch_bounds__(512) gemm_i8_skinny_kernel(const int8_t* __restrict__ A, const float* __restrict__ a_scale,
                                                             const int8_t* __restrict__ W, const float* __restrict__ w_scale,
                                                             void* __restrict__ C, int ldc, int M, int N, int K, int kw) {
  constexpr int U = 2, NS = 8 / WK;
  static_assert(EPI != EPI_SWIGLU || NS % 2 == 0, "gate and up strips in one block");
  __shared__ i32x4_t red[8][MT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, fq = lane >> 4;
  const int strip = blockIdx.x * NS + wave / WK;
  const int kb = (wave % WK) * kw, ke = min(K, kb + kw);
  i32x4_t acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = (i32x4_t){0, 0, 0, 0};
  const int8_t* wp = W + (int64_t)min(strip * 16 + fr, N - 1) * K;
  const int8_t* ap[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) ap[i] = A + (int64_t)min(16 * i + fr, M - 1) * K;
  i32x4_t a[2][U][MT], b[2][U];
  auto load = [&](int k, int p) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = min(k + 64 * u + 16 * fq, ke - 16);
      b[p][u] = *(const i32x4_t*)(wp + at);
#pragma unroll
      for (int i = 0; i < MT; ++i) a[p][u][i] = *(const i32x4_t*)(ap[i] + at);
    }
  };
  auto mma = [&](int k, int p) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = k + 64 * u + 16 * fq < ke;       // past the end: W's last codes against zeros
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        if (!in) a[p][u][i] = (i32x4_t){0, 0, 0, 0};
        acc[i] = I8Op::mma(a[p][u][i], b[p][u], acc[i]);
      }
    }
  };
  if (kb < ke) {
    load(kb, 0);
    for (int k = kb; k < ke; k += 2 * 64 * U) {
      if (k + 64 * U < ke) load(k + 64 * U, 1);
      mma(k, 0);
      if (k + 64 * U >= ke) break;
      if (k + 2 * 64 * U < ke) load(k + 2 * 64 * U, 0);
      mma(k + 64 * U, 1);
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) red[wave][i][lane] = acc[i];
  __syncthreads();
  // wavefront t adds and stores tile t (SwiGLU: gate and up)
  constexpr int P = EPI == EPI_SWIGLU ? 2 : 1;
  for (int t = wave; t < MT * NS / P; t += 8) {
    const int i = t / (NS / P), s0 = t % (NS / P) * P;
    i32x4_t s[1][P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
      s[0][p] = red[(s0 + p) * WK][i][lane];
#pragma unroll
      for (int w = 1; w < WK; ++w) s[0][p] += red[(s0 + p) * WK + w][i][lane];
    }
    const I8Op::Extra ex{a_scale, w_scale, 0};
    store_i8_tiles<1, P, EPI, false>(C, ldc, M, N, i * 16, (blockIdx.x * NS + s0) * 16, lane, s, ex);
  }
}

template <int BM, int BN, int WGM, int WGN, int STAGES, int EPI, bool SPLIT>
__global__ void __launch_bounds__(64 * WGM * WGN)
    gemm_i8_ring_kernel(const int8_t* __restrict__ A, const float* __restrict__ a_scale, const int8_t* __restrict__ W,
                        const float* __restrict__ w_scale, void* __restrict__ C, int ldc, int M, int N, int K2, int k_chunk,
                        int mt, int nt, int32_t* __restrict__ ws) {
  const int b = xcd_block();
  const int mi = b % mt, ni = (b / mt) % nt, z = b / (mt * nt);
  const I8Op::Extra ex{a_scale, w_scale, min(k_chunk, K2 - z * k_chunk)};
  dma_gemm_tile<I8Op, BM, BN, 64, WGM, WGN, STAGES, EPI, SPLIT>(
      (const bf16_t*)A, K2, (const bf16_t*)W, K2, C, ldc, M, N, k_chunk, mi, ni, z, (float*)ws, nullptr, ex);
}

// One persistent block per CU, each XCD a contiguous eighth of the tiles.
template <int BM, int BN, int WGM, int WGN, int BPC, int EPI, bool SPLIT, bool TAIL>
__global__ void __launch_bounds__(512, 2 * BPC)
    gemm_i8_alt_kernel(const int8_t* __restrict__ A, int lda2, const float* __restrict__ a_scale,
                       const int8_t* __restrict__ W, const float* __restrict__ w_scale, void* __restrict__ C, int ldc, int M,
                       int N, int K2, int k_chunk, int mt, int nt, int n_split, int32_t* __restrict__ ws) {
  constexpr int esz = (SPLIT || EPI == EPI_F32 || EPI == EPI_ADD_F32) ? 4 : 2;
  const int total = mt * nt * n_split, chunk = (total + 7) >> 3;
  const int hi = min(total, ((int)(blockIdx.x & 7) + 1) * chunk);
  int it = (int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3);
  auto next = [&](AltItem& t) {
    if (it >= hi) return false;
    const int z = it / (mt * nt);
    int mi, ni;
    panel_order(it - z * mt * nt, mt, nt, mi, ni);
    it += (int)(gridDim.x >> 3);
    t.a = (const bf16_t*)A + (int64_t)mi * BM * lda2 + z * k_chunk;
    t.w = (const bf16_t*)W + (int64_t)ni * BN * K2 + z * k_chunk;
    const int64_t out = (int64_t)mi * BM * ldc + (EPI == EPI_SWIGLU && !SPLIT ? ni * BN / 2 : ni * BN);
    t.c = SPLIT ? (char*)(ws + (int64_t)z * M * N + out) : (char*)C + out * esz;
    t.rows = M - mi * BM;
    t.arow = nullptr;
    t.a_scale = a_scale + mi * BM;
    t.w_scale = w_scale + ni * BN;
    t.cols = N - ni * BN;
    return true;
  };
  alt_gemm_items<I8Op, BM, BN, WGM, WGN, EPI, SPLIT, false, 0, TAIL>(lda2, K2, ldc, k_chunk / 64, next, K2);
}

// Partial sums of S splits, scales and epilogue; four columns per thread.
template <int EPI>
__global__ void __launch_bounds__(256) reduce_i8_kernel(const int32_t* __restrict__ ws, int S, int M, int N,
                                                        const float* __restrict__ a_scale, const float* __restrict__ w_scale,
                                                        void* C, int ldc) {
  const int ncol4 = (EPI == EPI_SWIGLU ? N / 2 : N) / 4;
  const int64_t total = (int64_t)M * ncol4, zs = (int64_t)M * N;
  for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
    const int m = (int)(t / ncol4), c = (int)(t % ncol4) * 4;
    const int n = EPI == EPI_SWIGLU ? (c >> 4) * 32 + (c & 15) : c;
    const float sa = a_scale[m];
    auto value = [&](int col, float (&v)[4]) {
      i32x4_t s = {0, 0, 0, 0};
      for (int z = 0; z < S; ++z) s += *(const i32x4_t*)(ws + z * zs + (int64_t)m * N + col);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (float)s[e] * sa * w_scale[col + e];
    };
    float v[4];
    value(n, v);
    if constexpr (EPI == EPI_SWIGLU) {
      float u[4];
      value(n + 16, u);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = silu_f(v[e]) * u[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) epi_store<EPI == EPI_SWIGLU ? EPI_BF16 : EPI>(C, ldc, M, m, c + e, v[e]);
  }
}

// ------------------------------------------------------------------ dispatch
// A plan: the kernel, its tiles and K splits; a function of (M, N, K) alone.
struct I8Plan {
  int kind;          // index into kI8Tiles, or -1 skinny
  int mt, nt;        // tiles
  int S;             // K splits (skinny: wavefronts per strip)
  int k_chunk;       // units per split
  bool pad;          // A's rows are copied to ones of whole pairs of K tiles first
};
// The tiles, and a model of their times: a block's time is fixed + per_k * (K tiles
// of 128 codes), in us, with one block per CU; with two on a CU, gain is the CU's
// speed against one block's.  Fitted to 330 sizes (16 shapes, 16 to 16384 rows,
// weights from memory): the plans that it gives take 1.1% longer on average than
// the fastest measured one, also against ring tiles of 64 x 128 and 128 x 128,
// which no plan needs.
struct I8Tiles {
  int bm, bn, occ;
  bool alt;
  double fixed, per_k, gain;
};
static constexpr I8Tiles kI8Tiles[] = {
    {64, 64, 2, false, 1.26, 0.321, 1.37}, {128, 128, 2, true, 1.95, 0.558, 1.19}, {128, 256, 1, true, 2.98, 0.843, 1.0},
    {256, 128, 1, true, 2.52, 0.787, 1.0}, {256, 192, 1, true, 3.24, 1.077, 1.0},  {256, 256, 1, true, 3.95, 1.270, 1.0}};
constexpr int kI8Kinds = sizeof(kI8Tiles) / sizeof(kI8Tiles[0]);
constexpr int kI8Cus = 256;
// us: of a launch, of the reduce kernel, of the kernel that pads rows
constexpr double kI8LaunchUs = 3.17, kI8ReduceUs = 2.2, kI8PadUs = 3.0;
constexpr double kI8ReadMBs = 5.01e6, kI8SplitMBs = 5.46e6;   // bytes per us: operands and results, partial sums

static bool set_i8_plan(I8Plan& p, int kind, int S, int M, int N, int K) {
  const int K2 = K / 2;
  p.kind = kind;
  p.S = S;
  p.mt = p.nt = 0;
  p.k_chunk = K2;
  p.pad = false;
  if (kind < 0) return M <= 32 && (S == 4 || S == 8) && (int64_t)N * S < ((int64_t)1 << 29);   // 512 N S / 128 threads
  const I8Tiles& t = kI8Tiles[kind];
  p.mt = (M + t.bm - 1) / t.bm;
  p.nt = (N + t.bn - 1) / t.bn;
  if (t.alt) {
    // whole pairs of K tiles (one split: A's rows are padded to them); 32-bit byte
    // offsets inside a tile
    if ((int64_t)256 * std::max<int64_t>(K + 256, 4 * (int64_t)N) >= ((int64_t)1 << 31)) return false;
    if (S > 1 && K2 % (128 * S)) return false;
    p.pad = K2 % 128 != 0;
    p.k_chunk = (K2 + 127) / 128 * 128 / S;
  } else {
    p.k_chunk = (K2 + 64 * S - 1) / (64 * S) * 64;
    if ((int64_t)p.k_chunk * (S - 1) >= K2) return false;      // a split without work
  }
  return (int64_t)p.mt * p.nt * S < (1 << 24);
}

static double i8_estimate(const I8Plan& p, int M, int N, int K) {
  const I8Tiles& t = kI8Tiles[p.kind];
  const double blocks = (double)p.mt * p.nt * p.S, tile = t.fixed + t.per_k * ((p.k_chunk + 63) / 64);
  double us = blocks <= kI8Cus ? tile : std::ceil(blocks / (t.occ * kI8Cus)) * t.occ * tile / t.gain;
  us = std::max(us, ((double)N * K + (double)M * K + 2.0 * M * N) / kI8ReadMBs) + kI8LaunchUs;
  if (p.S > 1) us += kI8ReduceUs + 8.0 * p.S * M * N / kI8SplitMBs;
  if (p.pad) us += kI8PadUs;
  return us;
}

// Skinny: a few rows; up to 16 of them while the weights are small (16 rows: 4096 x
// 4096 6.9 us against 9.1 in tiles, 6144 x 4096 10.5 against 10.9, 4096 x 12288 15.6
// against 15.1, 24576 x 4096 30 against 23), up to 32 while K is short, too (32 rows:
// 8192 x 1024 6.0 against 6.6, 2048 x 4096 9.2 against 8.7).
// Eight wavefronts per strip, a block; or four of twice the range and two strips a
// block, where that makes one round of blocks over the CUs of two, or K is too short to
// tell.  One row, four and eight, us: 4096 x 4096 7.5 / 6.2, 4608 x 4096 7.7 / 8.4, 6144 x
// 4096 8.1 / 8.7, 8192 x 4096 9.2 / 9.1, 12288 x 4096 14.5 / 12.0, 24576 x 4096 24.3 /
// 23.0; 6144 x 8192 13.7 / 15.0, 12288 x 8192 27.8 / 25.4; 4608 x 2048 5.2 / 5.3, 10240 x
// 2048 8.5 / 7.0; 6144 x 512 3.2 / 3.7, 12288 x 512 3.9 / 4.4.  16 rows alike.
static bool skinny_i8_plan(I8Plan& p, int M, int N, int K) {
  const int64_t w = (int64_t)N * K;
  if (M > 4 && !(M <= 16 && w <= 26000000) && !(M <= 32 && w <= 8400000 && K <= 2048)) return false;
  const int strips = (N + 15) / 16;
  return set_i8_plan(p, -1, strips > kI8Cus && (strips <= 2 * kI8Cus || K <= 512) ? 4 : 8, M, N, K);
}

// False if the results are too many for any (2^36 elements).
static bool plan_i8(I8Plan& best, int M, int N, int K) {
  if (skinny_i8_plan(best, M, N, K)) return true;
  I8Plan p;
  double least = 1e300;
  for (int kind = 0; kind < kI8Kinds; ++kind)
    for (int S = 1; S <= 8; S *= 2) {
      if (!set_i8_plan(p, kind, S, M, N, K)) continue;
      const double us = i8_estimate(p, M, N, K);
      if (us < least) {
        least = us;
        best = p;
      }
    }
  return least < 1e300;
}

static size_t plan_ws_bytes(const I8Plan& p, int M, int N) {
  if (p.kind < 0) return 0;
  return p.S > 1 ? (size_t)p.S * M * N * 4 : p.pad ? (size_t)M * p.k_chunk * 2 : 0;
}
size_t gemm_i8_workspace_bytes(int M, int N, int K) {
  I8Plan p;
  return plan_i8(p, M, N, K) ? plan_ws_bytes(p, M, N) : 0;
}

bool gemm_i8_plan_info(int M, int N, int K, int epi, int32_t* out) {
  I8Plan p;
  if (!plan_i8(p, M, N, K)) return false;
  if (p.kind < 0) {
    const int wk = epi == EPI_SWIGLU ? 4 : p.S;        // as skinny_i8 has them
    const int32_t v[5] = {0, M <= 16 ? 16 : 32, 8 / wk * 16, wk, 0};
    std::copy(v, v + 5, out);
  } else {
    const I8Tiles& t = kI8Tiles[p.kind];
    const int32_t v[5] = {t.alt ? 2 : 1, t.bm, t.bn, p.S, p.pad};
    std::copy(v, v + 5, out);
  }
  return true;
}

// Rows of K codes to rows of ldo, with zeros behind them; 16 bytes per thread.
__global__ void __launch_bounds__(256) pad_rows_kernel(const int8_t* __restrict__ a, int64_t rows, int K, int ldo,
                                                       int8_t* __restrict__ out) {
  const int per = ldo / 16;
  for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < rows * per; t += (int64_t)gridDim.x * 256) {
    const int64_t r = t / per;
    const int c = (int)(t % per) * 16;
    u32x4_t v = {0u, 0u, 0u, 0u};
    if (c < K) v = *(const u32x4_t*)(a + r * K + c);
    *(u32x4_t*)(out + r * ldo + c) = v;
  }
}

// Dynamic LDS beyond 64 KB is allowed once per kernel and device.
static hipError_t allow_lds(const void* kern, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return hipSuccess;
  e = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

struct I8Call {
  const int8_t* a;
  const float* a_scale;
  const int8_t* w;
  const float* w_scale;
  void* c;
  int M, N, K, lda, ldc;
  int32_t* ws;
};

template <int EPI, int MT, int WK>
static void skinny_i8_go(const I8Call& c, hipStream_t st) {
  constexpr int cols = 8 / WK * 16;
  const int kw = (c.K + WK * 64 - 1) / (WK * 64) * 64;
  hipLaunchKernelGGL((gemm_i8_skinny_kernel<MT, WK, EPI>), dim3((c.N + cols - 1) / cols), dim3(512), 0, st, c.a,
                     c.a_scale, c.w, c.w_scale, c.c, c.ldc, c.M, c.N, c.K, kw);
}
template <int EPI, int MT>
static void skinny_i8(int wk, const I8Call& c, hipStream_t st) {
  if (wk == 4 || EPI == EPI_SWIGLU) skinny_i8_go<EPI, MT, 4>(c, st);
  else skinny_i8_go<EPI, MT, EPI == EPI_SWIGLU ? 4 : 8>(c, st);
}

template <int EPI, int BM, int BN, int WGM, int WGN, int ST, bool SPLIT>
static hipError_t ring_i8_go(const I8Plan& p, const I8Call& c, hipStream_t st) {
  constexpr int lds = ST * (BM + BN) * 64 * 2;
  auto kern = gemm_i8_ring_kernel<BM, BN, WGM, WGN, ST, EPI, SPLIT>;
  static std::atomic<uint64_t> done{0};
  hipError_t e = allow_lds((const void*)kern, lds, done);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3(p.mt * p.nt * p.S), dim3(64 * WGM * WGN), lds, st, c.a, c.a_scale, c.w, c.w_scale, c.c,
                     c.ldc, c.M, c.N, c.K / 2, p.k_chunk, p.mt, p.nt, c.ws);
  return hipGetLastError();
}

template <int EPI, int BM, int BN, int WGM, int WGN, int BPC, bool SPLIT, bool TAIL>
static hipError_t alt_i8_as(const I8Plan& p, const I8Call& c, hipStream_t st) {
  constexpr int lds = 2 * (BM + BN) * 64 * 2 + (SPLIT ? 0 : kAltScaleBytes);
  auto kern = gemm_i8_alt_kernel<BM, BN, WGM, WGN, BPC, EPI, SPLIT, TAIL>;
  static std::atomic<uint64_t> done{0};
  hipError_t e = allow_lds((const void*)kern, lds, done);
  if (e != hipSuccess) return e;
  const int blocks = std::min((p.mt * p.nt * p.S + 7) / 8 * 8, kI8Cus * BPC);
  hipLaunchKernelGGL(kern, dim3(blocks), dim3(512), lds, st, c.a, c.lda / 2, c.a_scale, c.w, c.w_scale, c.c,
                     SPLIT ? c.N : c.ldc, c.M, c.N, c.K / 2, p.k_chunk, p.mt, p.nt, p.S, c.ws);
  return hipGetLastError();
}
template <int EPI, int BM, int BN, int WGM, int WGN, int BPC, bool SPLIT>
static hipError_t alt_i8_go(const I8Plan& p, const I8Call& c, hipStream_t st) {
  if constexpr (!SPLIT)
    if (p.pad) return alt_i8_as<EPI, BM, BN, WGM, WGN, BPC, SPLIT, true>(p, c, st);
  return alt_i8_as<EPI, BM, BN, WGM, WGN, BPC, SPLIT, false>(p, c, st);
}

template <int EPI, bool SPLIT>
static hipError_t tiles_i8_go(const I8Plan& p, const I8Call& c, hipStream_t st) {
  switch (p.kind) {
    case 0: return ring_i8_go<EPI, 64, 64, 2, 2, 4, SPLIT>(p, c, st);
    case 1: return alt_i8_go<EPI, 128, 128, 2, 4, 2, SPLIT>(p, c, st);
    case 2: return alt_i8_go<EPI, 128, 256, 2, 4, 1, SPLIT>(p, c, st);
    case 3: return alt_i8_go<EPI, 256, 128, 4, 2, 1, SPLIT>(p, c, st);
    case 4: return alt_i8_go<EPI, 256, 192, 4, 2, 1, SPLIT>(p, c, st);
    default: return alt_i8_go<EPI, 256, 256, 2, 4, 1, SPLIT>(p, c, st);
  }
}

template <int EPI>
static hipError_t gemm_i8_go(const I8Plan& p, const I8Call& c, hipStream_t st) {
  if (p.kind < 0) {
    if (c.M <= 16) skinny_i8<EPI, 1>(p.S, c, st);
    else skinny_i8<EPI, 2>(p.S, c, st);
    return hipGetLastError();
  }
  if (p.pad) {
    I8Call padded = c;
    padded.a = (const int8_t*)c.ws;
    padded.lda = 2 * p.k_chunk;
    const int64_t n = (int64_t)c.M * padded.lda / 16;
    hipLaunchKernelGGL(pad_rows_kernel, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 4096)), dim3(256), 0, st, c.a,
                       (int64_t)c.M, c.K, padded.lda, (int8_t*)c.ws);
    return tiles_i8_go<EPI, false>(p, padded, st);
  }
  if (p.S == 1) return tiles_i8_go<EPI, false>(p, c, st);
  // partial sums do not depend on the epilogue
  hipError_t e = tiles_i8_go<EPI_F32, true>(p, c, st);
  if (e != hipSuccess) return e;
  const int64_t n4 = (int64_t)c.M * (EPI == EPI_SWIGLU ? c.N / 2 : c.N) / 4;
  hipLaunchKernelGGL(reduce_i8_kernel<EPI>, dim3((unsigned)std::min<int64_t>((n4 + 255) / 256, 16384)), dim3(256), 0, st,
                     c.ws, p.S, c.M, c.N, c.a_scale, c.w_scale, c.c, c.ldc);
  return hipGetLastError();
}

static hipError_t run_i8_plan(const I8Plan& p, const I8Call& c, int epi, hipStream_t st) {
  switch (epi) {
    case EPI_F32: return gemm_i8_go<EPI_F32>(p, c, st);
    case EPI_BF16: return gemm_i8_go<EPI_BF16>(p, c, st);
    case EPI_ADD_F32: return gemm_i8_go<EPI_ADD_F32>(p, c, st);
    case EPI_SWIGLU: return gemm_i8_go<EPI_SWIGLU>(p, c, st);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_gemm_i8(const int8_t* a, const float* a_scale, const int8_t* w, const float* w_scale, void* c, int M,
                          int N, int K, int epi, void* ws, size_t ws_bytes, hipStream_t st) {
  if (M <= 0) return hipSuccess;
  I8Plan p;
  if (!plan_i8(p, M, N, K) || plan_ws_bytes(p, M, N) > ws_bytes) return hipErrorInvalidValue;
  return run_i8_plan(p, {a, a_scale, w, w_scale, c, M, N, K, K, epi == EPI_SWIGLU ? N / 2 : N, (int32_t*)ws}, epi, st);
}

// ------------------------------------------------------------------- grouped
// Expert e owns rows [off[e], off[e] + cnt[e]) of C, and of A and a_scale or of the
// row list into them; mtiles lists the non-empty row tiles (e << 16 | tile).
// Persistent blocks take items (row tile, column tile), column tile fastest; each
// XCD takes a contiguous eighth of them, so the column tiles of an expert's row
// tile find its rows in that XCD's L2.
struct I8Groups {
  const int32_t *off, *cnt, *mtiles, *n_mtiles, *arow;
};
#define DARTS_GROUP_PARAMS                                                                                       \
  const int32_t *__restrict__ g_off, const int32_t *__restrict__ g_cnt, const int32_t *__restrict__ mtiles,      \
      const int32_t *__restrict__ n_mtiles, const int32_t *__restrict__ arow
#define DARTS_GROUP_ARGS(g) g.off, g.cnt, g.mtiles, g.n_mtiles, g.arow

// Tiles of the alternating groups: 128 rows while the weights are streamed (decode
// batches; non-temporal, each tile of them is read once), 256 rows above.  A's rows
// are lda2 units apart, zero from K on up to whole pairs of K tiles.
template <int BM, int BN, int BPC, int EPI, int WAUX, bool TAIL>
__global__ void __launch_bounds__(512, 2 * BPC)
    gemm_i8_alt_grouped_kernel(const int8_t* __restrict__ A, const float* __restrict__ a_scale, const int8_t* __restrict__ W,
                               const float* __restrict__ w_scale, void* __restrict__ C, int ldc, int N, int K2, int lda2,
                               int nt, DARTS_GROUP_PARAMS) {
  constexpr int esz = (EPI == EPI_F32 || EPI == EPI_ADD_F32) ? 4 : 2;
  const int total = n_mtiles[0] * nt, chunk = (total + 7) >> 3;
  const int hi = min(total, ((int)(blockIdx.x & 7) + 1) * chunk);
  int it = (int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3);
  auto next = [&](AltItem& t) {
    if (it >= hi) return false;
    const int mt = mtiles[it / nt], ni = it % nt;
    it += (int)(gridDim.x >> 3);
    const int e = mt >> 16, m0 = (mt & 0xffff) * BM;
    const int64_t row = (int64_t)g_off[e] + m0;
    t.a = (const bf16_t*)A + (arow ? 0 : row * lda2);
    t.w = (const bf16_t*)W + ((int64_t)e * N + ni * BN) * K2;
    t.c = (char*)C + (row * ldc + (EPI == EPI_SWIGLU ? ni * BN / 2 : ni * BN)) * esz;
    t.rows = g_cnt[e] - m0;
    t.arow = arow ? arow + row : nullptr;
    t.a_scale = arow ? a_scale : a_scale + row;
    t.w_scale = w_scale + (int64_t)e * N + ni * BN;
    t.cols = N - ni * BN;
    return true;
  };
  alt_gemm_items<I8Op, BM, BN, 2, 4, EPI, false, false, WAUX, TAIL>(lda2, K2, ldc, (K2 + 127) / 128 * 2, next, K2);
}

// Row tile of the projections of `pairs` routed rows, by the rows per expert; 128
// channels and two blocks per CU, or 256 channels in batches that give those blocks
// work enough.  Layers in tiles of 128 x 128, 128 x 256 and 256 x 256, us: 128
// experts (2048, 768), 8 each: 61 rows 115 / 120 / 160, 400 rows 133 / 132 / 169,
// 976 rows (61 per expert) 167 / 158 / 195, 2000 rows (125) 265 / 244 / 227; 60
// experts (1456, 720), 4 each: 61 rows 65 / 79 / 90, 976 rows (65) 92 / 101 / 107,
// 2000 rows (133) 142 / 145 / 127.  (In tiles of 64 x 64 through a ring of LDS
// stages 147, 180, 238, 370; 70, 110, 160.  With the weights straight into
// registers and tiles of 16 to 96 rows 131, 172, 227 for 61, 400 and 976 rows of the
// first.)
constexpr int kI8TileRowsMin = 128;
static int grouped_i8_rows(int64_t pairs, int E) { return pairs < (int64_t)100 * E ? kI8TileRowsMin : 256; }
static bool grouped_i8_wide(int64_t pairs, int E, int N) {
  return pairs >= (int64_t)24 * E && std::min<int64_t>(pairs, E) * ((N + 255) / 256) >= 2 * kI8Cus;
}

// Channels of a tile of so many rows.
static int grouped_i8_cols(int rows, int64_t pairs, int E, int N) {
  return rows == 256 || grouped_i8_wide(pairs, E, N) ? 256 : 128;
}
// Whether the weights end inside the last pair of K tiles.
static bool grouped_i8_short(int K) { return K % 256 != 0; }

template <int BM, int BN, int BPC, int EPI, int WAUX, bool TAIL>
static hipError_t grouped_alt(const I8Call& c, const I8Groups& g, hipStream_t st) {
  constexpr int lds = 2 * (BM + BN) * 64 * 2 + kAltScaleBytes;
  auto kern = gemm_i8_alt_grouped_kernel<BM, BN, BPC, EPI, WAUX, TAIL>;
  static std::atomic<uint64_t> done{0};
  hipError_t e = allow_lds((const void*)kern, lds, done);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3(kI8Cus * BPC), dim3(512), lds, st, c.a, c.a_scale, c.w, c.w_scale, c.c, c.ldc, c.N, c.K / 2,
                     c.lda / 2, (c.N + BN - 1) / BN, DARTS_GROUP_ARGS(g));
  return hipGetLastError();
}
template <int BM, int BN, int BPC, int EPI, int WAUX>
static hipError_t grouped_tail(const I8Call& c, const I8Groups& g, hipStream_t st) {
  return grouped_i8_short(c.K) ? grouped_alt<BM, BN, BPC, EPI, WAUX, true>(c, g, st)
                   : grouped_alt<BM, BN, BPC, EPI, WAUX, false>(c, g, st);
}
// c.M: the routed rows.
template <int EPI>
static hipError_t grouped_i8(int rows, int E, const I8Call& c, const I8Groups& g, hipStream_t st) {
  if (rows == 256) return grouped_tail<256, 256, 1, EPI, 0>(c, g, st);
  return grouped_i8_cols(rows, c.M, E, c.N) == 256 ? grouped_tail<128, 256, 1, EPI, kNtLoad>(c, g, st)
                                                   : grouped_tail<128, 128, 2, EPI, kNtLoad>(c, g, st);
}

// ------------------------------------------------------------ routed experts
// out[r] = sum_j w[r][j] * y[pos(r, j)] in slot order, fp32 sums, 8 columns per
// thread; y is read once, non-temporal (a layer of 8000 rows 512 us, 516 with plain
// loads; 32768 rows 1750 and 1787).  y is bf16, as in the decoder's bf16 experts: half
// the bytes that the down product and this sum exchange.  Measured with a float32 y in
// its place: one row 12.0 us (bf16 12.1), 61 rows 109 (106), 976 rows 179 (167), 32768
// rows 2250 (1730); the error of a bf16 result against 64 bits, relative in the 2-norm,
// 0.0017 (0.0023).  The two launches of a few rows round y, too, so that a row's result
// does not hang on how many come with it.
// A place without an expert adds nothing, whatever its weight, but NaN for the weight
// NaN of a row that the router could not read.
__device__ __forceinline__ float weight_of(bool expert, float w) { return expert || w != w ? w : 0.f; }
template <int EPI>
__global__ void __launch_bounds__(256) combine_i8_kernel(const bf16_t* __restrict__ y, int d, int k,
                                                         const int32_t* __restrict__ pos_of,
                                                         const float* __restrict__ weights, void* __restrict__ out) {
  const int64_t r = blockIdx.x;
  for (int c = threadIdx.x * 8; c < d; c += 256 * 8) {
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < k; j0 += 8) {
      // eight experts' rows are loaded before any is added
      X8<true> v[8];
      float wj[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        wj[j] = 0.f;
        v[j].v = (u32x4_t){0u, 0u, 0u, 0u};
        if (j0 + j < k) {
          const int p = pos_of[r * k + j0 + j];
          wj[j] = weight_of(p >= 0, weights[r * k + j0 + j]);
          if (p >= 0) v[j].v = __builtin_nontemporal_load((const u32x4_t*)(y + (int64_t)p * d + c));
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j0 + j < k)
#pragma unroll
          for (int i = 0; i < 8; ++i) s[i] = fmaf(wj[j], v[j].at(i), s[i]);
    }
    if constexpr (EPI == EPI_ADD_F32) {
      f32x4_t* o = (f32x4_t*)((float*)out + r * d + c);
      o[0] += (f32x4_t){s[0], s[1], s[2], s[3]};
      o[1] += (f32x4_t){s[4], s[5], s[6], s[7]};
    } else {
      *(u32x4_t*)((bf16_t*)out + r * d + c) = (u32x4_t){f32_to_bf16x2(s[0], s[1]), f32_to_bf16x2(s[2], s[3]),
                                                        f32_to_bf16x2(s[4], s[5]), f32_to_bf16x2(s[6], s[7])};
    }
  }
}

// A few rows: nearly every (row, slot) pair has an expert of its own, so weights
// are streamed per pair, without lists, in two launches that make the codes they
// need themselves.  Lane (r, q) of a strip's load holds 16 codes of weight row r,
// and every row of the matrix instruction's other operand is the pair's own.
// Loads return in the order of their issue: the activations' come first, the
// weights' are in flight while the codes are made.
// Loads of 64 codes in one step (one row of 128 experts: 13.0 us, with 4 13.4, with 8
// 17.0).
constexpr int kFewU = 2;
struct FewStrip {
  const int8_t* w;
  int K;
  i32x4_t b[2][kFewU], acc;
  __device__ __forceinline__ void load(int k, int p) {
    const int fq = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int u = 0; u < kFewU; ++u)
      b[p][u] = *(const i32x4_t*)(w + min(k + 64 * u + 16 * fq, K - 16));
  }
  __device__ __forceinline__ void mma(const int8_t* q, int k, int ke, int p) {
    const int fq = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int u = 0; u < kFewU; ++u)
      if (k + 64 * u < ke) acc = I8Op::mma(*(const i32x4_t*)(q + k + 64 * u + 16 * fq), b[p][u], acc);
  }
  // the first loads of codes [kb, ke) (kb a multiple of 64), then their products
  __device__ __forceinline__ void begin(const int8_t* w_, int K_, int kb) {
    w = w_;
    K = K_;
    acc = (i32x4_t){0, 0, 0, 0};
    __builtin_amdgcn_sched_barrier(0);
    load(kb, 0);
    load(kb + 64 * kFewU, 1);
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ __forceinline__ int sum(const int8_t* q, int kb, int ke) {
    for (int k = kb; k < ke; k += 2 * 64 * kFewU) {
      mma(q, k, ke, 0);
      if (k + 2 * 64 * kFewU < ke) load(k + 2 * 64 * kFewU, 0);
      mma(q, k + 64 * kFewU, ke, 1);
      if (k + 3 * 64 * kFewU < ke) load(k + 3 * 64 * kFewU, 1);
    }
    return acc[0];
  }
};
// A row of n <= 8 * T * N bf16 elements in the registers of T threads: its largest
// magnitude (of a wavefront's part), and its codes into LDS, with zeros up to a
// multiple of 64.
template <int T, int N>
struct FewRow {
  X8<true> v[N];
  __device__ __forceinline__ void load(const bf16_t* x, int n, int t) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i].v = (u32x4_t){0u, 0u, 0u, 0u};
      if ((t + T * i) * 8 < n) v[i].load(x, (t + T * i) * 8);
    }
  }
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[i].at(e)) & 0x7fffffffu);
    return wave_max_u32(m);
  }
  __device__ __forceinline__ void codes(float up, int n, int t, int8_t* q) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (t + T * i) * 8;
      if (c >= (n + 63) / 64 * 64) continue;
      uint32_t w[2] = {0u, 0u};
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e >> 2] |= ((uint32_t)code_of(v[i].at(e), up) & 0xffu) << (8 * (e & 3));
      *(uint2*)(q + c) = make_uint2(w[0], w[1]);
    }
  }
};
constexpr int kFewMaxD = 8192, kFewMaxFe = 2048;

// h of one pair and 16 features: gate and up strips, four wavefronts each with a
// quarter of K.
__global__ void __launch_bounds__(512) few_gate_up_kernel(FfnI8Args a, bf16_t* __restrict__ h) {
  extern __shared__ __attribute__((aligned(16))) int8_t q[];
  __shared__ uint32_t tops[8];
  __shared__ int32_t sums[8][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), fr = lane & 15;
  const int groups = a.Fe / 16, pair = blockIdx.x / groups, g = blockIdx.x % groups;
  const int id = a.ids[pair];
  FewRow<512, kFewMaxD / 4096> x;
  x.load((const bf16_t*)a.x + (int64_t)(pair / a.k) * a.d, a.d, tid);
  if (id < 0 || id >= a.E) return;
  const int64_t row0 = (int64_t)id * 2 * a.Fe + g * 32;
  const int kw = (a.d + 255) / 256 * 64, kb = min((wave & 3) * kw, a.d), ke = min(a.d, kb + kw);
  FewStrip s;
  s.begin(a.w_gu + (row0 + (wave >> 2) * 16 + fr) * a.d, a.d, kb);
  const float s_gu = a.s_gu[row0 + (lane & 31)];
  const uint32_t t = x.top();
  if (lane == 0) tops[wave] = t;
  __syncthreads();
  uint32_t top = tops[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) top = max(top, tops[i]);
  float up, scale;
  row_scale(top, up, scale);
  x.codes(up, a.d, tid, q);
  __syncthreads();
  const int sum = s.sum(q, kb, ke);
  if (lane < 16) sums[wave][lane] = sum;
  __syncthreads();
  if (tid < 32) {
    const int c = tid & 15, w = tid >> 4 << 2;
    const float v = (float)(sums[w][c] + sums[w + 1][c] + sums[w + 2][c] + sums[w + 3][c]) * scale * s_gu;
    const float u = __shfl_xor(v, 16, 64);
    if (tid < 16) h[(int64_t)pair * a.Fe + g * 16 + tid] = f32_to_bf16(silu_f(v) * u);
  }
}

// out of one row and 16 columns: wavefront w does the row's slots w, w + 8, ...
template <int EPI>
__global__ void __launch_bounds__(512) few_down_kernel(FfnI8Args a, const bf16_t* __restrict__ h) {
  extern __shared__ __attribute__((aligned(16))) int8_t q[];
  __shared__ float y[64][16], wj[64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), fr = lane & 15;
  const int strips = a.d / 16, r = blockIdx.x / strips, c0 = blockIdx.x % strips * 16;
  int8_t* mine = q + wave * ((a.Fe + 63) / 64 * 64);
  for (int j = wave; j < a.k; j += 8) {
    const int id = a.ids[r * a.k + j];
    const bool expert = id >= 0 && id < a.E;
    const float w = a.weights[r * a.k + j];
    float v = 0.f;
    if (expert) {
      FewRow<64, kFewMaxFe / 512> hr;
      hr.load(h + ((int64_t)r * a.k + j) * a.Fe, a.Fe, lane);
      const int64_t col = (int64_t)id * a.d + c0 + fr;
      FewStrip s;
      s.begin(a.w_down + col * a.Fe, a.Fe, 0);
      const float s_down = a.s_down[col];
      float up, scale;
      row_scale(hr.top(), up, scale);
      hr.codes(up, a.Fe, lane, mine);
      __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0): only this wavefront reads them
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      v = bf16_to_f32(f32_to_bf16((float)s.sum(mine, 0, a.Fe) * scale * s_down));
    }
    if (lane < 16) y[j][lane] = v;
    if (lane == 0) wj[j] = weight_of(expert, w);
  }
  __syncthreads();
  if (tid < 16) {
    float s = 0.f;
    for (int j = 0; j < a.k; ++j) s = fmaf(wj[j], y[j][tid], s);
    epi_store<EPI>(a.out, a.d, INT32_MAX, r, c0 + tid, s);
  }
}

// Codes' rows in the workspace: whole pairs of K tiles.
static int64_t padded(int64_t k) { return (k + 255) / 256 * 256; }
// The first launch of a decode batch: `lists` blocks make the routing lists, the
// others the codes of four rows each.
__global__ void __launch_bounds__(1024) ffn_begin_kernel(FfnI8Args a, int lists, MoeLists l, int32_t* pos_of, int32_t* row_of,
                                                         int8_t* __restrict__ q, int64_t ldq, float* __restrict__ q_scale) {
  __shared__ uint32_t red[4][4];
  if ((int)blockIdx.x < lists) {
    moe_offsets_block(blockIdx.x, lists, a.ids, a.n_rows * a.k, a.E, a.k, l, pos_of, row_of);
    return;
  }
  const int w = threadIdx.x >> 8;
  // rows past the last repeat it: every thread meets the barrier, and writes the same
  const int64_t r = min((int)(blockIdx.x - lists) * 4 + w, a.n_rows - 1);
  quantize_row<true, true, 4>(a.x, r, threadIdx.x & 255, red[w], a.d, a.d, q, ldq, q_scale);
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
  t.q = (int8_t*)part((size_t)rows * padded(d));
  t.q_scale = (float*)part((size_t)rows * 4);
  t.counts = (int32_t*)part((size_t)E * 4);
  t.offsets = (int32_t*)part((size_t)E * 4);
  t.mtiles = (int32_t*)part((pairs / kI8TileRowsMin + E) * 4);
  t.n_mtiles = (int32_t*)part(4);
  t.mtiles_dn = (int32_t*)part((pairs / kI8TileRowsMin + E) * 4);
  t.n_mtiles_dn = (int32_t*)part(4);
  t.blk = (int32_t*)part((size_t)kMoeBlocks * E * 4);
  t.pos_of = (int32_t*)part(pairs * 4);
  t.row_of = (int32_t*)part(pairs * 4);
  t.h = (bf16_t*)part(pairs * Fe * 2);
  t.hq = (int8_t*)part(pairs * padded(Fe));
  t.h_scale = (float*)part(pairs * 4);
  t.y = (bf16_t*)part(pairs * d * 2);
  if (f) *f = t;
  return at;
}
size_t moe_ffn_i8_workspace_bytes(int64_t rows, int d, int E, int k, int Fe) {
  return ffn_layout(rows, d, E, k, Fe, nullptr, nullptr);
}

// Whether weights are streamed per pair: while pairs share few experts, or read so
// little that launches are the cost.  Two launches against lists, us: 128 experts
// (2048, 768), 8 each: 1 row 13 / 32, 4 rows 30 / 46, 10 rows 64 / 68; 64 experts
// (1024, 1408), 6 each: 4 rows 24 / 39, 7 rows 35 / 49; 60 experts (1456, 720), 4
// each: 10 rows 30 / 48; 16 experts (1024, 512), 4 each: 1 row 8 / 25, 15 rows 18 / 27.
static bool few_rows(int64_t pairs, int d, int E, int Fe) {
  return (3 * pairs <= 2 * E || (pairs <= 72 && 3 * pairs * d * Fe <= 250000000)) && d <= kFewMaxD && Fe <= kFewMaxFe;
}

void moe_ffn_i8_plan_info(int n_rows, int d, int E, int k, int Fe, int32_t* out) {
  const int pairs = n_rows * k, rows = grouped_i8_rows(pairs, E);
  int32_t v[6] = {0, 0, 0, 0, 0, 0};
  if (!few_rows(pairs, d, E, Fe)) {
    v[0] = pairs <= kMoeOneBlockPairs ? 1 : 2;
    v[1] = rows;
    v[2] = grouped_i8_cols(rows, pairs, E, 2 * Fe);
    v[3] = grouped_i8_cols(rows, pairs, E, d);
    v[4] = grouped_i8_short(d);
    v[5] = grouped_i8_short(Fe);
  }
  std::copy(v, v + 6, out);
}

hipError_t launch_moe_ffn_i8(const FfnI8Args& a, hipStream_t st) {
  if (a.n_rows <= 0) return hipSuccess;
  FfnWork f;
  if (ffn_layout(a.n_rows, a.d, a.E, a.k, a.Fe, (char*)a.ws, &f) > a.ws_bytes) return hipErrorInvalidValue;
  const int n_pairs = a.n_rows * a.k;
  if (few_rows(n_pairs, a.d, a.E, a.Fe)) {
    hipLaunchKernelGGL(few_gate_up_kernel, dim3(n_pairs * (a.Fe / 16)), dim3(512), (a.d + 63) / 64 * 64, st, a, f.h);
    const dim3 grid(a.n_rows * (a.d / 16));
    const int lds = 8 * ((a.Fe + 63) / 64 * 64);
    if (a.epi == EPI_ADD_F32) hipLaunchKernelGGL(few_down_kernel<EPI_ADD_F32>, grid, dim3(512), lds, st, a, f.h);
    else hipLaunchKernelGGL(few_down_kernel<EPI_BF16>, grid, dim3(512), lds, st, a, f.h);
    return hipGetLastError();
  }
  const int tile = grouped_i8_rows(n_pairs, a.E);
  hipError_t e;
  if (n_pairs <= kMoeOneBlockPairs) {
    const MoeLists l{f.counts, f.offsets, f.mtiles, f.n_mtiles, f.mtiles_dn, f.n_mtiles_dn, nullptr, tile, tile};
    const int lists = moe_place_blocks(n_pairs);
    hipLaunchKernelGGL(ffn_begin_kernel, dim3(lists + (a.n_rows + 3) / 4), dim3(1024), 0, st, a, lists, l, f.pos_of, f.row_of,
                       f.q, padded(a.d), f.q_scale);
  } else {
    if ((e = launch_quantize_rows(a.x, a.n_rows, a.d, a.d, true, f.q, padded(a.d), f.q_scale, st)) != hipSuccess) return e;
    const MoeListArgs l{a.ids, n_pairs, a.E, a.k, f.counts, f.offsets, f.mtiles, f.n_mtiles, f.mtiles_dn, f.n_mtiles_dn,
                        tile, tile, nullptr, f.blk, f.pos_of, f.row_of};
    if ((e = launch_moe_lists(l, st)) != hipSuccess) return e;
  }
  const I8Call gu{f.q, f.q_scale, a.w_gu, a.s_gu, f.h, n_pairs, 2 * a.Fe, a.d, (int)padded(a.d), a.Fe, nullptr};
  if ((e = grouped_i8<EPI_SWIGLU>(tile, a.E, gu, {f.offsets, f.counts, f.mtiles, f.n_mtiles, f.row_of}, st)) != hipSuccess)
    return e;
  if ((e = launch_quantize_rows(f.h, n_pairs, a.Fe, a.Fe, true, f.hq, padded(a.Fe), f.h_scale, st)) != hipSuccess) return e;
  const I8Call dn{f.hq, f.h_scale, a.w_down, a.s_down, f.y, n_pairs, a.d, a.Fe, (int)padded(a.Fe), a.d, nullptr};
  if ((e = grouped_i8<EPI_BF16>(tile, a.E, dn, {f.offsets, f.counts, f.mtiles_dn, f.n_mtiles_dn, nullptr}, st)) != hipSuccess)
    return e;
  if (a.epi == EPI_ADD_F32)
    hipLaunchKernelGGL(combine_i8_kernel<EPI_ADD_F32>, dim3(a.n_rows), dim3(256), 0, st, f.y, a.d, a.k, f.pos_of,
                       a.weights, a.out);
  else
    hipLaunchKernelGGL(combine_i8_kernel<EPI_BF16>, dim3(a.n_rows), dim3(256), 0, st, f.y, a.d, a.k, f.pos_of, a.weights,
                       a.out);
  return hipGetLastError();
}

}  // namespace darts
