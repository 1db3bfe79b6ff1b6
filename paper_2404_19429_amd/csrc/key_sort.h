// Stable placement by a small key: items 0 .. N - 1, each with a key in [0, D),
// D <= 512, or none, get the positions that a stable sort by key gives them.
//
// An item's position is the first position of its key (a prefix sum over the
// keys' totals), plus the items of that key in earlier tiles, in earlier waves
// of its tile, and earlier in its wave.  A block of NT threads takes a tile of
// 4 NT items, its waves 256 each, in order; a wave takes 64 at a time and finds
// the lanes of the same key with one ballot per key bit.  One tile is one launch;
// past that the tiles' counts come from a launch before it, and every block sums
// those of the tiles before its own: D numbers a tile, tiles^2 D reads in all, out of
// the L2s while they are few megabytes.  Past kSortSumTiles tiles a launch between
// the two turns the counts into those sums (sort_scan), so that the work grows with
// the items.  Integers only, no atomics on device memory: the same positions every time.
//
// A block is a chain of latencies (keys, the tiles' counts, barriers, scattered
// stores of a line a lane), so small tiles on many CUs are the faster ones until
// the sums over the tiles are the longer part: 1024 items up to 64 tiles of them,
// 4096 beyond.  Counting and placing 12000 items of 160 keys in tiles of 4096: 2.6 +
// 9.5 us, of 1024: 3.1 + 6.3.
#pragma once

#include "internal.h"

namespace lmoe {

constexpr int kSortMaxD = 512, kSortRounds = 4;
constexpr int kSortSmall = 256, kSortLarge = 1024;   // threads of a block
inline int sort_threads(int64_t n) { return n <= 64 * kSortRounds * kSortSmall ? kSortSmall : kSortLarge; }
inline int64_t sort_tiles(int64_t n) {
  const int64_t tile = kSortRounds * sort_threads(n);
  return (n + tile - 1) / tile;
}
// Tiles up to which every block sums the others' counts.  Lookup gradient of 2^21 + 1 tokens (513 tiles), 500 ids of
// width 8: 280 us summed, 213 scanned; of 2^26 43 ms and 7.3; the smaller batches are as they were.
constexpr int64_t kSortSumTiles = 512;
// Numbers of `counts`: D a tile, and where they are scanned the keys' totals behind them.
inline int64_t sort_counts(int64_t tiles, int D) { return (tiles + (tiles > kSortSumTiles ? 1 : 0)) * D; }

// Lanes whose item has the same key (of `bits` bits) as this lane's.
__device__ __forceinline__ uint64_t same_key(int key, int bits) {
  uint64_t m = __ballot(key >= 0);
#pragma unroll
  for (int b = 0; b < 9; ++b) {
    if (b >= bits) break;
    const bool one = (key >> b) & 1;
    const uint64_t ones = __ballot(one);
    m &= one ? ones : ~ones;
  }
  return m;
}

// counts[tile][key] of the tiles.  key(i): the key of item i, -1 if it has none.
template <int NT, typename Key>
__device__ __forceinline__ void sort_count(const Key& key, int64_t N, int D, int32_t* __restrict__ counts, int64_t tile,
                                           int32_t (&hist)[kSortMaxD]) {
  for (int e = threadIdx.x; e < D; e += NT) hist[e] = 0;
  int k[kSortRounds];
#pragma unroll
  for (int q = 0; q < kSortRounds; ++q) {
    const int64_t i = tile * (kSortRounds * NT) + q * NT + threadIdx.x;
    k[q] = i < N ? key(i) : -1;
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kSortRounds; ++q)
    if (k[q] >= 0) atomicAdd(&hist[k[q]], 1);
  __syncthreads();
  for (int e = threadIdx.x; e < D; e += NT) counts[tile * D + e] = hist[e];
}

// counts[tile][key] -> the sums over the tiles before it, and the keys' totals behind
// the last tile's.  A block takes kScanKeys keys by kScanParts shares of the tiles,
// whose sums meet in LDS.
constexpr int kScanKeys = 16, kScanParts = 64;
static __global__ __launch_bounds__(kScanKeys * kScanParts) void sort_scan_kernel(int32_t* __restrict__ counts, int64_t tiles, int D) {
  __shared__ int32_t sum[kScanParts][kScanKeys];
  const int q = threadIdx.x % kScanKeys, part = threadIdx.x / kScanKeys;
  const int e = blockIdx.x * kScanKeys + q;
  const int64_t share = (tiles + kScanParts - 1) / kScanParts;
  const int64_t a = min(tiles, part * share), b = e < D ? min(tiles, a + share) : a;
  constexpr int U = 8;   // tiles in flight
  int32_t n[U];
  int32_t mine = 0;
  for (int64_t t = a; t < b; t += U) {
#pragma unroll
    for (int u = 0; u < U; ++u) n[u] = t + u < b ? counts[(t + u) * D + e] : 0;
#pragma unroll
    for (int u = 0; u < U; ++u) mine += n[u];
  }
  sum[part][q] = mine;
  __syncthreads();
  int32_t run = 0;
  for (int p = 0; p < part; ++p) run += sum[p][q];
  for (int64_t t = a; t < b; t += U) {
#pragma unroll
    for (int u = 0; u < U; ++u) n[u] = t + u < b ? counts[(t + u) * D + e] : 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t + u < b) counts[(t + u) * D + e] = run;
      run += n[u];
    }
  }
  if (part == kScanParts - 1 && e < D) counts[tiles * D + e] = run;
}
// The launch between counting and placing, if there is one.
inline void launch_sort_scan(int32_t* counts, int64_t tiles, int D, hipStream_t s) {
  if (tiles > kSortSumTiles)
    launch_kernel(sort_scan_kernel, dim3((unsigned)((D + kScanKeys - 1) / kScanKeys)), dim3(kScanKeys * kScanParts), 0, s,
                  counts, tiles, D);
}

template <int NT>
struct SortLds {
  static constexpr int W = NT / kWave;
  int32_t cnt[W][kSortMaxD];   // a wave's items of a key, then the position of the first of them from the key's first
  int32_t first[kSortMaxD], total[kSortMaxD];   // a key's first position (a multiple of `align`), its items
  int32_t wsum[W];
  int32_t used;                // positions up to the last key's end, rounded up to `align`
};

// Places the tile's items: emit(i, position) for each, position -1 for an item
// without a key.  Leaves first, total and used in L for the caller.
template <int NT, typename Key, typename Emit>
__device__ __forceinline__ void sort_place(const Key& key, const Emit& emit, int64_t N, int D, int align,
                                           const int32_t* __restrict__ counts, int64_t tile, int64_t tiles,
                                           SortLds<NT>& L) {
  constexpr int W = SortLds<NT>::W, KT = (kSortMaxD + NT - 1) / NT;   // waves; keys a thread
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int bits = D > 1 ? 32 - __builtin_clz(D - 1) : 0;
  const int64_t i0 = tile * (kSortRounds * NT) + wave * (kSortRounds * kWave) + lane;
  int k[kSortRounds], rank[kSortRounds];
#pragma unroll
  for (int q = 0; q < kSortRounds; ++q) k[q] = i0 + q * kWave < N ? key(i0 + q * kWave) : -1;
  // The other tiles' counts, on their way while this one's are made (thread: keys KT x .. KT x + KT - 1).
  int run[KT], total[KT];
#pragma unroll
  for (int h = 0; h < KT; ++h) run[h] = total[h] = 0;
  const int e0 = threadIdx.x * KT;
  if (tiles > kSortSumTiles) {   // (sums already)
#pragma unroll
    for (int h = 0; h < KT; ++h)
      if (e0 + h < D) {
        run[h] = counts[tile * D + e0 + h];
        total[h] = counts[tiles * D + e0 + h];
      }
  } else if (tiles > 1 && e0 < D) {
    constexpr int U = 8;   // tiles whose counts are read together
    for (int64_t t = 0; t < tiles; t += U) {
      int n[U][KT];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < KT; ++h) n[u][h] = t + u < tiles && e0 + h < D ? counts[(t + u) * D + e0 + h] : 0;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < KT; ++h) {
          run[h] += t + u < tile ? n[u][h] : 0;
          total[h] += n[u][h];
        }
    }
  }
#pragma unroll
  for (int w = 0; w < W; ++w)
    for (int e = threadIdx.x; e < D; e += NT) L.cnt[w][e] = 0;
  __syncthreads();
  const uint64_t below = lane == 0 ? 0ull : ~0ull >> (64 - lane);
#pragma unroll
  for (int q = 0; q < kSortRounds; ++q) {
    const uint64_t m = same_key(k[q], bits);
    int before = 0;
    const int lead = m ? __builtin_ctzll(m) : lane;
    if (k[q] >= 0 && lane == lead) before = atomicAdd(&L.cnt[wave][k[q]], __popcll(m));   // (the wave's own counter)
    rank[q] = __shfl(before, lead, kWave) + __popcll(m & below);
  }
  __syncthreads();
  int room[KT], all = 0;
#pragma unroll
  for (int h = 0; h < KT; ++h) {
    room[h] = 0;
    const int e = e0 + h;
    if (e < D) {
      int n[W], sum = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) n[w] = L.cnt[w][e];
#pragma unroll
      for (int w = 0; w < W; ++w) {
        L.cnt[w][e] = run[h] + sum;
        sum += n[w];
      }
      if (tiles <= 1) total[h] = sum;
      room[h] = (total[h] + align - 1) / align * align;
      all += room[h];
    }
  }
  // Sums of the keys' rooms before each thread's.
  int end = all;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int u = __shfl_up(end, o, kWave);
    if (lane >= o) end += u;
  }
  if (lane == kWave - 1) L.wsum[wave] = end;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w) end += w < wave ? L.wsum[w] : 0;
  int at = end - all;
#pragma unroll
  for (int h = 0; h < KT; ++h)
    if (e0 + h < D) {
      L.first[e0 + h] = at;
      L.total[e0 + h] = total[h];
      at += room[h];
      if (e0 + h == D - 1) L.used = at;
    }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kSortRounds; ++q) {
    const int64_t i = i0 + q * kWave;
    if (i < N) emit(i, k[q] >= 0 ? L.first[k[q]] + L.cnt[wave][k[q]] + rank[q] : -1);
  }
}

}  // namespace lmoe
