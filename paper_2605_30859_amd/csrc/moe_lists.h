// Routing lists of decode batches (k_moe.hip, and the 8-bit experts' first launch).
#pragma once
#include "common.h"
#include "kernels.h"

namespace darts {

// Lists of a routing: per-expert counts and their exclusive scan, and the
// non-empty expert row tiles (e << 16 | tile) of either projection.
struct MoeLists {
  int32_t *counts, *offsets, *mtiles, *n_mtiles, *mtiles2, *n_mtiles2, *touched_out;
  int tile_rows, tile_rows2;
};
// The lists from thread e's count v of expert e (0 for e >= E), by one block of
// 1024 threads; returns the expert's offset.  write: the same in the whole block.
__device__ __forceinline__ int moe_lists(const MoeLists& l, int v, int E, int32_t* sh, bool write = true) {
  const int tid = threadIdx.x;
  int total;
  const int ex = block_excl_scan1024(v, sh, &total);
  if (!write) return ex;
  const int nt = (v + l.tile_rows - 1) / l.tile_rows;
  int ntiles;
  const int tex = block_excl_scan1024(nt, sh, &ntiles);
  if (tid < E) {
    l.counts[tid] = v;
    l.offsets[tid] = ex;
    for (int j = 0; j < nt; ++j) l.mtiles[tex + j] = (tid << 16) | j;
  }
  if (tid == 0) *l.n_mtiles = ntiles;
  // the second list (another row tile for the other projection)
  const int nt2 = (v + l.tile_rows2 - 1) / l.tile_rows2;
  int ntiles2;
  const int tex2 = block_excl_scan1024(nt2, sh, &ntiles2);
  if (tid < E)
    for (int j = 0; j < nt2; ++j) l.mtiles2[tex2 + j] = (tid << 16) | j;
  if (tid == 0) *l.n_mtiles2 = ntiles2;
  if (l.touched_out) {
    const int nz = __syncthreads_count(v > 0);
    if (tid == 0) *l.touched_out = nz;
  }
  return ex;
}
// Decode batches: one launch, counts by an LDS histogram of the n_pairs routed
// (row, slot) pairs.  A thread keeps its pairs' experts and their places among the
// expert's pairs (what the histogram's adds return) in registers.  Every block
// counts all pairs, the first writes the lists, and each places the pairs of its
// own share of the experts: the stores to 64 different lines per instruction are
// what placing costs (7808 pairs 18 us in one block that counted twice, 15 in one
// that counted once, 9.8 so).
constexpr int kMoePlaceBlocks = 16, kMoePlaceAlone = 512;   // blocks, from so many pairs on
constexpr int kMoeOneBlockPairs = 16384;
// Block `blk` of `blks` blocks of 1024 threads.
__device__ __forceinline__ void moe_offsets_block(int blk, int blks, const int32_t* __restrict__ topk_id, int n_pairs, int E,
                                                  int k, const MoeLists& lists, int32_t* __restrict__ pos_of,
                                                  int32_t* __restrict__ row_of) {
  constexpr int N = kMoeOneBlockPairs / 1024;
  __shared__ int32_t hist[1024];
  __shared__ int32_t sh[32];
  const int tid = threadIdx.x;
  int e[N], at[N];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    e[u] = -1;
    if (1024 * u < n_pairs && tid + 1024 * u < n_pairs) e[u] = topk_id[tid + 1024 * u];
  }
  hist[tid] = 0;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < N; ++u) {
    at[u] = -1;
    if (1024 * u < n_pairs && e[u] >= 0 && e[u] < E) at[u] = atomicAdd(&hist[e[u]], 1);
  }
  __syncthreads();
  const int ex = moe_lists(lists, tid < E ? hist[tid] : 0, E, sh, blk == 0);
  hist[tid] = tid < E ? ex : 0;          // the experts' first positions
  __syncthreads();
  const int lo = blk * E / blks, hi = (blk + 1) * E / blks;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int i = tid + 1024 * u;
    if (1024 * u >= n_pairs || i >= n_pairs) continue;
    if (at[u] < 0) {
      if (blk == 0) pos_of[i] = -1;
    } else if (e[u] >= lo && e[u] < hi) {
      const int p = hist[e[u]] + at[u];
      row_of[p] = i / k;
      pos_of[i] = p;
    }
  }
}
inline int moe_place_blocks(int n_pairs) { return n_pairs < kMoePlaceAlone ? 1 : kMoePlaceBlocks; }

}  // namespace darts
