// Device code of the matrix products C[M,N] = A[M,K] * W[N,K]^T, shared by the bf16
// (k_gemm.hip) and the 8-bit integer kernels (k_i8.hip): the ring of LDS tiles and
// the alternating wavefront groups.  Operands are addressed in units of 16 bits:
// one bf16 element, or two 8-bit codes, so a chunk of 16 bytes is a matrix
// instruction's operand in both and K counts units.
#pragma once
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace darts {

typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));

// The two kinds of operands.  Extra is what a tile's epilogue and K loop need
// beside the addresses.
struct Bf16Op {
  typedef bf16x8_t frag;
  typedef f32x4_t acc;
  struct Extra {};
  static constexpr bool kI8 = false;
  static __device__ __forceinline__ acc mma(const frag& a, const frag& b, const acc& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};
// Codes: sums in 32-bit integers, exact.  a_scale[m] belongs to row m of the
// output, w_scale[n] to its column n.  N is any
// multiple of 16, K (in codes) of 16: the ring fills the last K tile with zeros
// past klen units, and columns past N repeat W's last row and are not stored.
struct I8Op {
  typedef i32x4_t frag;
  typedef i32x4_t acc;
  struct Extra {
    const float *a_scale, *w_scale;
    int klen;               // units of this tile's K range
  };
  static constexpr bool kI8 = true;
  static __device__ __forceinline__ acc mma(const frag& a, const frag& b, const acc& c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
  }
};
// Zeros that lanes past the end of K load.
static __device__ __attribute__((aligned(16))) uint32_t kZeroChunk[4];

__device__ __forceinline__ float silu_f(float g) { return g / (1.0f + __expf(-g)); }

template <int EPI>
__device__ __forceinline__ void epi_store(void* C, int ldc, int M, int m, int n, float v) {
  if (m >= M) return;
  if (EPI == EPI_F32) ((float*)C)[(int64_t)m * ldc + n] = v;
  else if (EPI == EPI_BF16) ((bf16_t*)C)[(int64_t)m * ldc + n] = f32_to_bf16(v);
  else if (EPI == EPI_ADD_F32) ((float*)C)[(int64_t)m * ldc + n] += v;
}

// Write a 16x16 MFMA output tile pair / single tile.  acc layout: lane holds
// rows r0 + 4*(lane/16) + i, column c0 + lane%16.
template <int EPI>
__device__ __forceinline__ void store_tile(void* C, int ldc, int M, int r0, int c0, int lane,
                                           const f32x4_t& v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) epi_store<EPI>(C, ldc, M, r0 + 4 * (lane >> 4) + i, c0 + (lane & 15), v[i]);
}
// gate tile (physical cols 32g..32g+15) and up tile (32g+16..32g+31) -> H cols 16g..16g+15
__device__ __forceinline__ void store_swiglu(bf16_t* H, int ldc, int M, int r0, int pc0, int lane,
                                             const f32x4_t& g, const f32x4_t& u) {
  const int col = (pc0 >> 5) * 16 + (lane & 15);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = r0 + 4 * (lane >> 4) + i;
    if (m < M) H[(int64_t)m * ldc + col] = f32_to_bf16(silu_f(g[i]) * u[i]);
  }
}
__device__ __forceinline__ void store_partial(float* P, int M, int N, int r0, int c0, int lane,
                                              const f32x4_t& v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = r0 + 4 * (lane >> 4) + i;
    if (m < M) P[(int64_t)m * N + c0 + (lane & 15)] = v[i];
  }
}

// ------------------------------------------------------------ strip layout
// Strip-packed weights: a [N][K] matrix (N % 16 == 0, K % 32 == 0) is stored
// as N/16 strips of 16 consecutive rows; strip g holds K/32 blocks of 64 x 8
// bf16, and lane l of block s holds W[16g + l%16][32s + 8(l/16), +8), the B
// operand of v_mfma_f32_16x16x32_bf16 for that strip and K step.  A strip
// occupies the same 16*K elements as in the row-major layout, only reordered.
// Element offset of the 8-element chunk W[n][k, k+8), k % 8 == 0:
__device__ __forceinline__ int64_t strip_off(int n, int k, int K) {
  return (((int64_t)(n >> 4) * (K >> 5) + (k >> 5)) * 64 + (n & 15) + 16 * ((k >> 3) & 3)) * 8;
}

// A wavefront's accumulators of codes: lane (r, q) holds rows 4q + i of column r of
// each 16 x 16 tile.  SPLIT: partial sums, still integers.
template <int TM, int TN, int EPI, bool SPLIT>
__device__ __forceinline__ void store_i8_tiles(void* C, int ldc, int M, int N, int rb, int cb, int lane,
                                               const i32x4_t (&acc)[TM][TN], const I8Op::Extra& ex) {
  const int fr = lane & 15, fq = lane >> 4;
  float sw[TN];
  if constexpr (!SPLIT) {
#pragma unroll
    for (int j = 0; j < TN; ++j) sw[j] = ex.w_scale[min(cb + 16 * j + fr, N - 1)];
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    float sa[4];
    if constexpr (!SPLIT) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sa[e] = ex.a_scale[min(rb + 16 * i + 4 * fq + e, M - 1)];
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int n = cb + 16 * j;                       // 16 columns are inside N or outside it together
      if (n >= N) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = rb + 16 * i + 4 * fq + e;
        if (m >= M) continue;
        if constexpr (SPLIT) {
          ((int32_t*)C)[(int64_t)m * ldc + n + fr] = acc[i][j][e];
        } else if constexpr (EPI == EPI_SWIGLU) {
          if (j % 2 == 0)
            ((bf16_t*)C)[(int64_t)m * ldc + (n >> 5) * 16 + fr] =
                f32_to_bf16(silu_f((float)acc[i][j][e] * sa[e] * sw[j]) *
                            ((float)acc[i][j + 1 < TN ? j + 1 : j][e] * sa[e] * sw[j + 1 < TN ? j + 1 : j]));
        } else {
          epi_store<EPI>(C, ldc, M, m, n + fr, (float)acc[i][j][e] * sa[e] * sw[j]);
        }
      }
    }
  }
}

// ------------------------------------------------------------------ tiled
// Operand tiles travel global -> LDS with direct 16-byte LDS loads (no
// staging registers) through a STAGES-deep ring of LDS buffers.  A KB-wide K
// slice of a row is KB/8 chunks of 16 bytes, stored in a swizzled chunk order
// (dma_swz) so that the 16-byte fragment reads of consecutive rows hit
// distinct banks.  Rows of A past M load row M-1 (their results are never
// stored).  Each wavefront owns a (BM/WGM) x (BN/WGN) register tile of
// 16x16 MFMA accumulators.
// s_waitcnt vmcnt(N) (gfx9 encoding: vmcnt bits 3:0 and 15:14; expcnt and
// lgkmcnt left at their "don't wait" maxima)
template <int N>
__device__ __forceinline__ void vm_wait() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

typedef __attribute__((address_space(3))) void lds_void_t;

// Cache-policy operand of the direct LDS loads that marks them non-temporal
// (the nt bit of gfx950's global loads).  A streaming read of 8 GiB measured
// 7.0 TB/s with non-temporal 16-byte loads against 6.3 TB/s with plain ones;
// the weight streams of the MoE expert GEMMs gain 4-13% from it wherever each
// weight tile is read once per launch.
constexpr int kNtLoad = 2;

// LDS chunk swizzle for a tile row of KB bf16 (KB/8 chunks of 16 bytes): the
// chunk order of row r is permuted so that the 8 rows a 16-byte fragment read
// touches in one LDS pass land in distinct banks.
template <int KB>
__device__ __forceinline__ int dma_swz(int r) {
  if constexpr (KB == 64) return r & 7;
  else return (r >> 1) & 3;
}

// One BM x BN output tile (rows m0.., cols n0.., K range [z*k_chunk, +k_chunk)).
// arow != NULL: row r of the tile's A operand is row arow[r] of A (a gather).
// PW: W is strip-packed (pack_strips_kernel; ldw = K): the same LDS tile is
// filled from the packed addresses, so results are bitwise those of the
// row-major layout.  WAUX: cache policy of the W loads (kNtLoad: non-temporal,
// for weights a launch reads once).
template <typename Op, int BM, int BN, int KB, int WGM, int WGN, int STAGES, int EPI, bool SPLIT, bool PW = false,
          int WAUX = 0>
__device__ __forceinline__ void dma_gemm_tile(const bf16_t* __restrict__ A, int lda,
                                              const bf16_t* __restrict__ W, int ldw,
                                              void* __restrict__ C, int ldc, int M, int N,
                                              int k_chunk, int mi, int ni, int z,
                                              float* __restrict__ ws,
                                              const int32_t* __restrict__ arow = nullptr,
                                              typename Op::Extra ex = {}) {
  static_assert(KB == 32 || KB == 64, "K tile");
  constexpr int NW = WGM * WGN;                    // wavefronts per block
  constexpr int WM = BM / WGM, WN = BN / WGN, TM = WM / 16, TN = WN / 16;
  constexpr int CH = KB / 8, RPI = 64 / CH;        // chunks per row, rows per 1 KB load instruction
  constexpr int AI = BM / (RPI * NW), WI = BN / (RPI * NW);   // load instructions per wave per stage
  static_assert(AI * RPI * NW == BM && WI * RPI * NW == BN, "tile rows must split over the waves");
  constexpr int KH = KB / 32;                      // 32-wide MFMA K steps per tile
  constexpr int STAGE_ELEMS = (BM + BN) * KB;      // bf16 elements per stage
  extern __shared__ __attribute__((aligned(16))) bf16_t smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave / WGN, wn = wave % WGN;
  const int m0 = mi * BM, n0 = ni * BN;
  const int kbeg = z * k_chunk;
  int nk = k_chunk / KB;
  if constexpr (Op::kI8) nk = (ex.klen + KB - 1) / KB;

  // per-lane global source rows for this wave's load instructions: lane i fills
  // LDS bytes [16i, 16i+16) of the instruction's RPI rows, which hold source
  // chunk (i % CH) ^ swizzle(row)
  const int lrow = lane / CH;
  const int gchunk = (lane % CH) ^ dma_swz<KB>(lrow);
  const bf16_t* asrc[AI];
  const bf16_t* wsrc[WI];
#pragma unroll
  for (int j = 0; j < AI; ++j) {
    int r = m0 + wave * (BM / NW) + RPI * j + lrow;
    r = r < M ? r : M - 1;
    if (arow) r = arow[r];
    asrc[j] = A + (int64_t)r * lda + kbeg + gchunk * 8;
  }
#pragma unroll
  for (int j = 0; j < WI; ++j) {
    int n = n0 + wave * (BN / NW) + RPI * j + lrow;
    if constexpr (Op::kI8) n = n < N ? n : N - 1;
    if constexpr (PW) wsrc[j] = W + strip_off(n, kbeg + gchunk * 8, ldw);
    else wsrc[j] = W + (int64_t)n * ldw + kbeg + gchunk * 8;
  }
  // one KB-wide K step moves a row-major source KB elements on, a packed one
  // KB/32 blocks of 512 elements
  constexpr int WSTEP = PW ? KB * 16 : KB;

  auto issue = [&](int kt, int buf) {
    bf16_t* sa = smem + buf * STAGE_ELEMS;
    bf16_t* sw = sa + BM * KB;
    if constexpr (Op::kI8) {
      if (kt * KB + KB > ex.klen) {                    // the last K tile, not full: zeros past the end
        const bool in = kt * KB + gchunk * 8 < ex.klen;
#pragma unroll
        for (int j = 0; j < AI; ++j)
          __builtin_amdgcn_global_load_lds(in ? (const void*)(asrc[j] + kt * KB) : (const void*)kZeroChunk,
                                           (lds_void_t*)(sa + (wave * (BM / NW) + RPI * j) * KB), 16, 0, 0);
#pragma unroll
        for (int j = 0; j < WI; ++j)
          __builtin_amdgcn_global_load_lds(in ? (const void*)(wsrc[j] + kt * WSTEP) : (const void*)kZeroChunk,
                                           (lds_void_t*)(sw + (wave * (BN / NW) + RPI * j) * KB), 16, 0, WAUX);
        return;
      }
    }
#pragma unroll
    for (int j = 0; j < AI; ++j)
      __builtin_amdgcn_global_load_lds((const void*)(asrc[j] + kt * KB),
                                       (lds_void_t*)(sa + (wave * (BM / NW) + RPI * j) * KB), 16, 0, 0);
#pragma unroll
    for (int j = 0; j < WI; ++j)
      __builtin_amdgcn_global_load_lds((const void*)(wsrc[j] + kt * WSTEP),
                                       (lds_void_t*)(sw + (wave * (BN / NW) + RPI * j) * KB), 16, 0, WAUX);
  };

  typedef typename Op::frag frag_t;
  typename Op::acc acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = (typename Op::acc){0, 0, 0, 0};

#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s)
    if (s < nk) issue(s, s);

  const int fr = lane & 15, fq = lane >> 4;
  for (int kt = 0; kt < nk; ++kt) {
    // this wave's loads of stage kt are done once at most the (STAGES-2) later
    // stages' loads are outstanding (all outstanding in the last stages); the
    // raw barrier then publishes every wave's stage kt (no memory fence: it
    // would drain the prefetches still in flight)
    if (kt + STAGES - 2 < nk) vm_wait<(STAGES - 2) * (AI + WI)>();
    else vm_wait<0>();
    __builtin_amdgcn_s_barrier();
    if (kt + STAGES - 1 < nk) issue(kt + STAGES - 1, (kt + STAGES - 1) % STAGES);
    const bf16_t* sa = smem + (kt % STAGES) * STAGE_ELEMS;
    const bf16_t* sw = sa + BM * KB;
    // fragments of every 32-wide K step are read before the first MFMA, so
    // LDS latency overlaps matrix work
    frag_t a[KH][TM], bb[KH][TN];
#pragma unroll
    for (int ks = 0; ks < KH; ++ks) {
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int r = wm * WM + 16 * i + fr;
        a[ks][i] = *(const frag_t*)(sa + r * KB + (((ks * 4 + fq) ^ dma_swz<KB>(r)) * 8));
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int r = wn * WN + 16 * j + fr;
        bb[ks][j] = *(const frag_t*)(sw + r * KB + (((ks * 4 + fq) ^ dma_swz<KB>(r)) * 8));
      }
    }
#pragma unroll
    for (int ks = 0; ks < KH; ++ks)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = Op::mma(a[ks][i], bb[ks][j], acc[i][j]);
  }

  const int rb = m0 + wm * WM, cb = n0 + wn * WN;
  if constexpr (Op::kI8) {
    store_i8_tiles<TM, TN, EPI, SPLIT>(SPLIT ? (void*)(ws + (int64_t)z * M * N) : C, SPLIT ? N : ldc, M, N, rb, cb, lane,
                                       acc, ex);
  } else if constexpr (SPLIT) {
    float* P = ws + (int64_t)z * M * N;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) store_partial(P, M, N, rb + 16 * i, cb + 16 * j, lane, acc[i][j]);
  } else if constexpr (EPI == EPI_SWIGLU) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; j += 2)
        store_swiglu((bf16_t*)C, ldc, M, rb + 16 * i, cb + 16 * j, lane, acc[i][j], acc[i][j + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) store_tile<EPI>(C, ldc, M, rb + 16 * i, cb + 16 * j, lane, acc[i][j]);
  }
}

// 16 bytes to buffer r at voff + soff. A vector instruction that writes one of
// the last three data registers right after such a store can still change what
// is stored (seen here: accumulators, converted for the next store, in memory
// in place of results). The compiler puts the two wait states between them only
// where soff is a constant, so they stand here, and the data, an input of the
// same statement, keeps its registers until then.
__device__ __forceinline__ void store_b128(u32x4_t v, __amdgpu_buffer_rsrc_t r, int voff, int soff) {
  __builtin_amdgcn_raw_buffer_store_b128(v, r, voff, soff, 0);
  asm volatile("s_nop 1" ::"v"(v) : "memory");
}

// ------------------------------------------------------- alternating groups
// BM x BN output tile for compute-bound launches: 8 wavefronts in two groups
// of four (one wavefront of each group per SIMD) that alternate between
// fetching operands from LDS and issuing MFMAs, so the matrix cores of a SIMD
// run one wavefront's products while the other wavefront reads its next
// fragments.  The second group runs one barrier behind the first.
//
// A 64-wide K tile is four half tiles in LDS (A0, A1 of BM/2 rows, B0, B1 of
// BN/2 rows of W), double-buffered.  A wavefront owns TM x TN 16x16
// accumulators of each of the four A half x B half quadrants and takes two
// quadrants per phase: (A0,B0) (A0,B1), then (A1,B0) (A1,B1).  The first phase
// reads A0 and B1 (B0's fragments are there already), the second A1 and the
// next K tile's B0, so both read equally much and the reads of one group last
// about as long as the MFMAs of the other.  Each phase also issues the direct
// LDS loads of two half tiles one or two K tiles ahead, into the half tiles
// read one phase earlier, and waits until at most the four youngest half tiles
// are in flight; the barrier that ends the fetch section then publishes the
// half tiles the next phase reads.
//
// MFMAs take W as the first operand, so a lane's four accumulators are four
// consecutive columns of one output row and the epilogue stores them together.
// For SwiGLU B0 holds the gate rows and B1 the up rows of the tile's columns,
// so a lane has both of a feature.  The sums run over K in the same order as
// in dma_gemm_tile, so results are bitwise those of the tiled kernel.
//
// Bound by the matrix cores, at the clock that the card's power allows: a
// library GEMM of the same sizes reaches 1530 TFLOP/s.  Measured on the
// Qwen3-8B gate/up projection against the tiled kernel, where every wavefront
// reads its fragments and then issues its MFMAs behind one barrier per K tile:
// 16384 rows 2080 us (1590 TFLOP/s) against 2880 us, 4096 rows 535 against 747
// us, 389 rows (256x192 tiles, weights cold) 76 against 96 us; QKV at 4096 rows
// 154 against 187 us.  Four phases of one quadrant each (8 barriers per K tile)
// took 561 us at 4096 rows.
template <int N>
__device__ __forceinline__ void vm_lgkm_wait() {   // vmcnt(N) and lgkmcnt(0)
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (0x7 << 4));
}
// Neither memory accesses nor MFMAs are moved across.
__device__ __forceinline__ void order_fence() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
// The same with a raw barrier.
__device__ __forceinline__ void fenced_barrier() {
  order_fence();
  __builtin_amdgcn_s_barrier();
  order_fence();
}

// One output tile of alt_gemm_items.
struct AltItem {
  const bf16_t* a;       // its first row of A (arow set: A itself), at the first column of its K range
  const bf16_t* w;       // its first row of W, at the first column of its K range
  char* c;               // its first output element
  int rows;              // rows of the output from the tile's first one on (> 0)
  const int32_t* arow;   // NULL, or the A row of each of them
  // codes: the scales of A's rows (as arow counts them, else from the tile's first
  // row) and of the tile's first column of W, and W's rows from the tile's first one
  // on (a multiple of 16, > 0)
  const float *a_scale, *w_scale;
  int cols;
};

// A block's items, one after the other; next(item) yields the first, then each
// following one, or false.  nk: 64-wide K tiles of every item, even.  PW: W is
// strip-packed (ldw = K).  An item's row list is read during the last K tiles of
// the item before it, and its first loads are issued before that item's results
// are stored, so neither latency is waited for (EPI_ADD_F32 reads the results'
// old values behind those loads, and waits for them).  TAIL: W's rows hold w_units of
// K, less than nk tiles; A's are zero from there on, and W's loads past the end read
// codes before it instead.
constexpr int kAltScaleBytes = 2 * 512 * 4;   // codes: dynamic LDS beyond the tiles
template <typename Op, int BM, int BN, int WGM, int WGN, int EPI, bool SPLIT, bool PW, int WAUX = 0, bool TAIL = false, typename Next>
__device__ __forceinline__ void alt_gemm_items(int lda, int ldw, int ldc, int nk, Next next, [[maybe_unused]] int w_units = 0) {
#ifdef __HIP_DEVICE_COMPILE__   // the host pass knows no buffer resources
  constexpr int KB = 64, NW = 8;
  static_assert(WGM * WGN == NW, "8 wavefronts");
  constexpr int HM = BM / 2, HN = BN / 2;             // half tile rows
  constexpr int TM = HM / WGM / 16, TN = HN / WGN / 16;
  static_assert(TM * WGM * 16 == HM && TN * WGN * 16 == HN, "half tiles split evenly over the wavefronts");
  // 1 KB (8-row) loads per half tile, load i by wavefront i % 8; per wavefront
  // of the first and of the second group
  constexpr int IA = HM / 8, IB = HN / 8;
  constexpr int LA = IA / NW, LB = (IB + NW - 1) / NW;
  static_assert(IA % NW == 0 && IB % 4 == 0 && IB >= NW, "a group's wavefronts issue equally many loads");
  constexpr int LB1 = IB / NW;                        // second group
  // LDS: the two stages of A0, of A1, of B0, of B1, so that either operand's
  // fragment reads differ by constants that fit the instruction's offset
  constexpr int HA = HM * KB, HB = HN * KB;
  constexpr bool kSwiglu = !SPLIT && EPI == EPI_SWIGLU;
  constexpr int kEsz = !SPLIT && (EPI == EPI_BF16 || EPI == EPI_SWIGLU) ? 2 : 4;   // output element
  // stores of a whole tile per lane (16 bytes, or 8 at addresses that are not
  // adjacent, so that none are merged)
  constexpr int kStores = 2 * TM * TN * (kSwiglu ? 1 : 2) / (kEsz == 2 && TN % 2 == 0 ? 2 : 1);
  extern __shared__ __attribute__((aligned(16))) bf16_t smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool first = wave < 4;                        // group
  const int wm = wave / WGN, wn = wave % WGN;

  // Source addresses are a buffer resource, a 32-bit lane offset in bytes that
  // stays the same over K, and a uniform offset that moves on (no vector
  // registers or instructions per load).  Gathered A rows are offsets from A
  // itself (the launcher checks that they fit), others from the tile's first row.
  const int lrow = lane >> 3;
  const int gchunk = (lane & 7) ^ lrow;               // source chunk of this lane's LDS slot
  // Order of W's rows in a half tile.  With 16-bit results and an even number
  // of column tiles per wavefront, two tiles t = 0, 1 share 32 columns, column
  // c of tile t being column 8*(c/4) + 4*t + c%4 of them: a lane's four
  // accumulators of either tile are then 8 consecutive columns, one 16-byte
  // store, and a row's four lanes write 64 bytes in one piece.  (8-byte stores
  // in 32-byte pieces cost the MoE down projection of 32768 rows, 1.07 GB of
  // results, 0.43 ms of its 1.03 ms.)  Otherwise rows are in order.
  constexpr bool kPair = kEsz == 2 && TN % 2 == 0;
  const int wlane = kPair ? 8 * (lrow >> 2) + (lrow & 3) : lrow;   // row in a strip of 16, but for a uniform part
  int woff = PW ? ((gchunk & 3) * 16 + wlane) * 16 + (gchunk >> 2) * 1024 : (wlane * ldw + gchunk * 8) * 2;
  constexpr bool kScales = Op::kI8 && !SPLIT;
  [[maybe_unused]] int srow = 0;                      // codes: the row whose scale this lane fetches
  auto row_ids = [&](const AltItem& t, int (&row)[2][LA]) {
    if constexpr (kScales) {
      int s = lane + 64 * (wave & 3);
      asm volatile("" : "+v"(s));
      s = min(s, t.rows - 1);
      srow = t.arow && first ? t.arow[s] : s;
    }
    int row0 = lrow;
    asm volatile("" : "+v"(row0));                    // recomputed here, not kept over the K loop
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < LA; ++j) {
        int r = min(h * HM + (wave + NW * j) * 8 + row0, t.rows - 1);
        row[h][j] = t.arow ? t.arow[r] : r;
      }
  };
  AltItem cur;
  int arow[2][LA], aoff[2][LA];
  if (!next(cur)) return;
  row_ids(cur, arow);
  auto ares = __builtin_amdgcn_make_buffer_rsrc((void*)cur.a, 0, -1, 0x00020000);
  auto wres = __builtin_amdgcn_make_buffer_rsrc((void*)cur.w, 0, -1, 0x00020000);
  // K tile kt belongs in stage kt & 1, which the callers know as a constant
  auto issue_a = [&](int kt, int stage, int h) {
    bf16_t* s = smem + (2 * h + stage) * HA + wave * 8 * KB;
#pragma unroll
    for (int j = 0; j < LA; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ares, (lds_void_t*)(s + NW * j * 8 * KB), 16, aoff[h][j],
                                               kt * (KB * 2), 0, 0);
  };
  [[maybe_unused]] int w_rows = 0;
  [[maybe_unused]] const int w_full = w_units / KB, w_rest = w_units % KB;   // whole K tiles of W, units of the next
  // woff for whole K tiles, and for the one that W ends in
  [[maybe_unused]] auto w_offset = [&](bool end) {
    int l = lane;
    asm volatile("" : "+v"(l));                       // computed where it changes, not kept
    const int r = l >> 3, c = (l & 7) ^ r;
    return ((kPair ? 8 * (r >> 2) + (r & 3) : r) * ldw + (end && c * 8 >= w_rest ? 0 : c * 8)) * 2;
  };
  if constexpr (Op::kI8) w_rows = cur.cols;
  auto issue_b = [&](int kt, int stage, int h) {
    bf16_t* s = smem + 4 * HA + (2 * h + stage) * HB + wave * 8 * KB;
    if constexpr (TAIL)
      if (kt >= w_full) {
        kt = w_rest ? w_full : w_full - 1;
        if (w_rest) woff = w_offset(true);
      }
#pragma unroll
    for (int j = 0; j < LB; ++j) {
      if (j == LB1 && !first) break;
      const int q = wave + NW * j;                    // 8 rows of the half tile: of which strip, from which row
      const int strip = kPair ? (q >> 2) * 2 + (q & 1) : q >> 1, sub = kPair ? ((q >> 1) & 1) * 4 : (q & 1) * 8;
      // a wavefront's TN column tiles of B0 and then its TN of B1 are neighbours
      int row = (kSwiglu ? strip * 2 + h : strip / TN * 2 * TN + h * TN + strip % TN) * 16;
      if constexpr (Op::kI8) row = min(row, w_rows - 16);   // a strip past W's last one repeats it
      const int off = PW ? row * 2 * ldw + sub * 16 + kt * (KB * 32) : (row + sub) * 2 * ldw + kt * (KB * 2);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(wres, (lds_void_t*)(s + NW * j * 8 * KB), 16, woff, off, 0, WAUX);
    }
  };

  const int fr = lane & 15, fq = lane >> 4;
  const int cvoff = (fr * ldc + fq * (kPair ? 8 : 4)) * kEsz;
  // fragments [K step][tile]: of an A half, of B1, and of B0 for this K tile
  // and the next (by parity of the K tile)
  typedef typename Op::frag frag_t;
  frag_t a[2][TM], b1[2][TN], b0[2][2][TN];
  typename Op::acc acc[2][2][TM][TN];
  // rows are multiples of 16 apart, so the swizzle of a lane's row is fr & 7
  const bf16_t* pa = smem + (wm * TM * 16 + fr) * KB;
  const bf16_t* pb = smem + 4 * HA + (wn * TN * 16 + fr) * KB;
  const int c0 = (fq ^ (fr & 7)) * 8, c1 = ((4 + fq) ^ (fr & 7)) * 8;
  auto read_a = [&](int stage, int h) {
    const bf16_t* s = pa + (2 * h + stage) * HA;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      a[0][i] = *(const frag_t*)(s + i * 16 * KB + c0);
      a[1][i] = *(const frag_t*)(s + i * 16 * KB + c1);
    }
  };
  auto read_b = [&](int stage, int h, frag_t (&f)[2][TN]) {
    const bf16_t* s = pb + (2 * h + stage) * HB;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      f[0][j] = *(const frag_t*)(s + j * 16 * KB + c0);
      f[1][j] = *(const frag_t*)(s + j * 16 * KB + c1);
    }
  };
  auto mma = [&](int h, const frag_t (&f0)[2][TN]) {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[h][0][i][j] = Op::mma(f0[ks][j], a[ks][i], acc[h][0][i][j]);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[h][1][i][j] = Op::mma(b1[ks][j], a[ks][i], acc[h][1][i][j]);
    __builtin_amdgcn_s_setprio(0);
  };
  // row of W (from the tile's first) of an accumulator's first column
  [[maybe_unused]] auto col_of = [&](int g, int j) {
    const int f = kPair ? 8 * fq + 4 * (j & 1) : 4 * fq, t = kPair ? j & ~1 : j;
    if constexpr (kSwiglu) return (wn * TN + t + (f >> 4)) * 32 + g * 16 + (f & 15);
    else return ((2 * wn + g) * TN + t) * 16 + f;
  };
  // The fetch section ends: this wavefront's fragments are in registers, and
  // all but the NA youngest A and NB youngest B half tiles have landed (vector
  // memory operations retire in order).  MAYBE, stored: the kStores stores of
  // the item before may be younger than those half tiles, too.
  auto landed = [&](auto NA, auto NB, auto MAYBE, bool stored) {
    constexpr int na = decltype(NA)::value, nb = decltype(NB)::value, st = decltype(MAYBE)::value ? kStores : 0;
    static_assert(na * LA + nb * LB + st < 64, "vmcnt range");
    if (st && stored) {
      if (LB1 == LB || first) vm_lgkm_wait<na * LA + nb * LB + st>();
      else vm_lgkm_wait<na * LA + nb * LB1 + st>();
    } else {
      if (LB1 == LB || first) vm_lgkm_wait<na * LA + nb * LB>();
      else vm_lgkm_wait<na * LA + nb * LB1>();
    }
    fenced_barrier();
  };
  constexpr std::integral_constant<int, 0> n0{};
  constexpr std::integral_constant<int, 1> n1{};
  constexpr std::integral_constant<int, 2> n2{};
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  // LEFT: 0 in the steady loop, 1 for the last tile but one, 2 for the last
  auto tile = [&](int kt, auto P, auto LEFT, auto MAYBE, bool stored) {
    constexpr int p = decltype(P)::value, left = decltype(LEFT)::value;
    if constexpr (left < 2) issue_a(kt + 1, 1 - p, 1);
    if constexpr (left < 1) issue_b(kt + 2, p, 0);
    read_a(p, 0);
    read_b(p, 1, b1);
    if constexpr (left == 0) landed(n2, n2, MAYBE, stored);
    else if constexpr (left == 1) landed(n2, n1, MAYBE, stored);
    else landed(n0, n0, MAYBE, false);
    mma(0, b0[p]);
    fenced_barrier();
    if constexpr (left < 1) { issue_a(kt + 2, p, 0); issue_b(kt + 2, p, 1); }
    read_a(p, 1);
    if constexpr (left < 2) read_b(1 - p, 0, b0[1 - p]);
    if constexpr (left == 0) landed(n2, n2, MAYBE, stored);
    else if constexpr (left == 1) landed(n1, n0, MAYBE, stored);
    else landed(n0, n0, MAYBE, false);
    mma(1, b0[p]);
    fenced_barrier();
  };
  // Codes: an item's scales (of its 256 rows, then of its channels) go to LDS
  // with its first loads, into one of two places by turns, since that is before
  // the results of the item before are scaled.
  [[maybe_unused]] float* scales = (float*)(smem + 4 * (HA + HB));
  [[maybe_unused]] int turn = 0;
  // the first loads of cur, whose rows are in arow
  auto start = [&]() {
    if constexpr (TAIL)
      if (w_rest) woff = w_offset(false);
    if constexpr (kScales) {
      int t = lane + 64 * (wave & 3);
      asm volatile("" : "+v"(t));                     // recomputed here, not kept over the K loop
      const float* src = first ? cur.a_scale + srow : cur.w_scale + min(t, min(cur.cols, BN) - 1);
      __builtin_amdgcn_global_load_lds((const void*)src, (lds_void_t*)(scales + turn * 512 + wave * 64), 4, 0, 0);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < LA; ++j)
        aoff[h][j] = (int)(((uint32_t)arow[h][j] * (uint32_t)lda + gchunk * 8) * 2u);
    ares = __builtin_amdgcn_make_buffer_rsrc((void*)cur.a, 0, -1, 0x00020000);
    wres = __builtin_amdgcn_make_buffer_rsrc((void*)cur.w, 0, -1, 0x00020000);
    issue_b(0, 0, 0); issue_a(0, 0, 0); issue_b(0, 0, 1);
    issue_a(0, 0, 1); issue_b(1, 1, 0); issue_a(1, 1, 0); issue_b(1, 1, 1);
  };

  start();
  bool stored = false;
  while (true) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) acc[h][g][i][j] = (typename Op::acc){0, 0, 0, 0};
    landed(n2, n2, yes, stored);
    read_b(0, 0, b0[0]);
    landed(n2, n2, yes, stored);
    if (!first) fenced_barrier();                     // the second group runs one barrier behind
    if (nk > 2) {
      tile(0, n0, n0, yes, stored);
      tile(1, n1, n0, no, false);
      for (int kt = 2; kt < nk - 2; kt += 2) {
        tile(kt, n0, n0, no, false);
        tile(kt + 1, n1, n0, no, false);
      }
    }
    AltItem nxt;
    const bool more = next(nxt);
    if (more) row_ids(nxt, arow);                     // read while the last two K tiles are computed
    tile(nk - 2, n0, n1, no, false);
    tile(nk - 1, n1, n2, no, false);
    if (first) fenced_barrier();

    const auto cres = __builtin_amdgcn_make_buffer_rsrc((void*)cur.c, 0, -1, 0x00020000);
    const int rows = cur.rows;
    [[maybe_unused]] int out_cols = 0;                // codes: output columns from the tile's first one on
    if constexpr (Op::kI8) out_cols = kSwiglu ? cur.cols / 2 : cur.cols;
    [[maybe_unused]] const float* sc = scales + turn * 512;
    if (more) {
      cur = nxt;
      if constexpr (Op::kI8) w_rows = cur.cols;
      turn ^= 1;
      start();
    }
    // the value of an accumulator
    auto value = [&](int h, int g, int i, int j) {
      if constexpr (kScales) {
        const float sa = sc[h * HM + (wm * TM + i) * 16 + fr];
        const f32x4_t sw = *(const f32x4_t*)(sc + 256 + col_of(g, j));
        f32x4_t v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)acc[h][g][i][j][e] * sa * sw[e];
        return v;
      } else {
        return __builtin_bit_cast(f32x4_t, acc[h][g][i][j]);
      }
    };
    order_fence();   // landed() counts the stores below as younger than start()'s loads
    // accumulators: row 16*i + lane%16, columns 16*j + 4*(lane/16) .. +3, or with
    // kPair those of tiles j, j + 1 columns 16*j + 8*(lane/16) .. +7
    auto store = [&](int h, int i, auto EDGE) {
      // EDGE: some columns may lie past N (16 of them are inside or outside together)
      [[maybe_unused]] auto inside = [&](int g, int j) {
        if constexpr (Op::kI8 && decltype(EDGE)::value)
          return ((kSwiglu ? wn : 2 * wn + g) * TN + j) * 16 + fq * (kPair ? 8 : 4) < out_cols;
        else return true;
      };
      const int m = h * HM + (wm * TM + i) * 16;      // this wavefront's 16 rows
      if constexpr (kEsz == 2) {
#pragma unroll
        for (int g = 0; g < (kSwiglu ? 1 : 2); ++g) {
          uint2 v[TN];
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            f32x4_t u = value(h, g, i, j);
            if constexpr (kSwiglu) {
              const f32x4_t up = value(h, 1, i, j);
#pragma unroll
              for (int e = 0; e < 4; ++e) u[e] = silu_f(u[e]) * up[e];
            }
            v[j] = make_uint2(f32_to_bf16x2(u[0], u[1]), f32_to_bf16x2(u[2], u[3]));
          }
#pragma unroll
          for (int j = 0; j < TN; j += kPair ? 2 : 1) {
            const int o = (m * ldc + ((kSwiglu ? wn : 2 * wn + g) * TN + j) * 16) * kEsz;
            if (!inside(g, j)) continue;
            if constexpr (kPair)
              store_b128((u32x4_t){v[j].x, v[j].y, v[j + 1].x, v[j + 1].y}, cres, cvoff, o);
            else
              __builtin_amdgcn_raw_buffer_store_b64((u32x2_t){v[j].x, v[j].y}, cres, cvoff, o, 0);
          }
        }
      } else {
        f32x4_t r[2][TN];
        if constexpr (!SPLIT && EPI == EPI_ADD_F32) {
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int j = 0; j < TN; ++j)
              if (inside(g, j))
                r[g][j] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                                                          cres, cvoff, (m * ldc + ((kSwiglu ? wn : 2 * wn + g) * TN + j) * 16) * kEsz, 0));
        }
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            if (!inside(g, j)) continue;
            f32x4_t v = value(h, g, i, j);
            if constexpr (!SPLIT && EPI == EPI_ADD_F32) v += r[g][j];
            store_b128(__builtin_bit_cast(u32x4_t, v), cres, cvoff,
                       (m * ldc + ((kSwiglu ? wn : 2 * wn + g) * TN + j) * 16) * kEsz);
          }
      }
    };
    stored = rows >= BM;
    if constexpr (Op::kI8) stored = stored && out_cols >= (kSwiglu ? BN / 2 : BN);
    if (stored) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < TM; ++i) store(h, i, no);
    } else {
      int row0 = fr;
      asm volatile("" : "+v"(row0));
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < TM; ++i)
          if (row0 < rows - (h * HM + (wm * TM + i) * 16)) store(h, i, yes);
    }
    if (!more) break;
  }
#endif
}

// Blocks are renumbered so that the blocks one XCD runs (dispatch is round
// robin over the 8 XCDs) are consecutive tiles and share operands in its L2.
__device__ __forceinline__ int xcd_block() {
  const int nb = gridDim.x;
  int b = blockIdx.x;
  const int full = (nb / 8) * 8;
  if (b < full) b = (b % 8) * (full / 8) + b / 8;
  return b;
}

// Tile order of one XCD's run of consecutive tiles: panels of kPanel row tiles,
// column tiles fastest after the panel's rows, so that the 32 tiles the XCD has
// in flight are about 8 x 4 and read 12 operand tiles, not 33.
constexpr int kPanel = 8;
__device__ __forceinline__ void panel_order(int b, int mt, int nt, int& mi, int& ni) {
  const int p = b / (kPanel * nt), rows = min(kPanel, mt - p * kPanel);
  const int r = b - p * kPanel * nt;
  mi = p * kPanel + r % rows;
  ni = r / rows;
}

}  // namespace darts
