// Stable placement by a small key: items 0 .. N - 1, each with a key in [0, D),
// D <= 512, or none, get the positions that a stable sort by key gives them.
//
// An item's position is the first position of its key (a prefix sum over the
// keys' totals), plus the items of that key in earlier tiles, in earlier waves
// of its tile, and earlier in its wave.  A tile is 4096 items, sixteen waves of
// 256 in order; a wave takes 64 at a time and finds the lanes of the same key
// with one ballot per key bit.  Up to one tile it is one launch; past that the
// tiles' counts come from a launch before it, and every block sums those of the
// tiles before its own (D numbers a tile, L2-resident).  Integers only, no
// atomics on device memory: the same positions every time.  A block is a chain of
// latencies (keys, the tiles' counts, three barriers), so what can be in flight
// together is.
#pragma once

#include "internal.h"

namespace lmoe {

constexpr int kSortTile = 4096, kSortThreads = 1024, kSortWaves = kSortThreads / kWave, kSortMaxD = 512;
constexpr int kSortRounds = kSortTile / kSortThreads;
inline int64_t sort_tiles(int64_t n) { return (n + kSortTile - 1) / kSortTile; }

// Lanes whose item has the same key (of `bits` bits) as this lane's.
__device__ __forceinline__ uint64_t same_key(int key, int bits) {
  uint64_t m = __ballot(key >= 0);
  for (int b = 0; b < bits; ++b) {
    const bool one = (key >> b) & 1;
    const uint64_t ones = __ballot(one);
    m &= one ? ones : ~ones;
  }
  return m;
}

// Inclusive sums of v over the block's threads (whole waves, at most 16 of them).
__device__ __forceinline__ int block_scan(int v, int (&wsum)[kSortWaves]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int u = __shfl_up(v, o, kWave);
    if (lane >= o) v += u;
  }
  if (lane == kWave - 1) wsum[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v += wsum[w];
  __syncthreads();
  return v;
}

// counts[tile][key] of the tiles.  key(i): the key of item i, -1 if it has none.
template <typename Key>
__device__ __forceinline__ void sort_count(const Key& key, int64_t N, int D, int32_t* __restrict__ counts, int64_t tile,
                                           int32_t (&hist)[kSortMaxD]) {
  for (int e = threadIdx.x; e < D; e += kSortThreads) hist[e] = 0;
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kSortRounds; ++q) {
    const int64_t i = tile * kSortTile + q * kSortThreads + threadIdx.x;
    const int k = i < N ? key(i) : -1;
    if (k >= 0) atomicAdd(&hist[k], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < D; e += kSortThreads) counts[tile * D + e] = hist[e];
}

struct SortLds {
  int32_t cnt[kSortWaves][kSortMaxD];   // a wave's items of a key, then the position of the first of them
  int32_t first[kSortMaxD], total[kSortMaxD];   // a key's first position (a multiple of `align`), its items
  int32_t wsum[kSortWaves];
  int32_t used;                         // positions up to the last key's end, rounded up to `align`
};

// Places the tile's items: emit(i, position) for each, position -1 for an item
// without a key.  Leaves first, total and used in L for the caller.
template <typename Key, typename Emit>
__device__ __forceinline__ void sort_place(const Key& key, const Emit& emit, int64_t N, int D, int align,
                                           const int32_t* __restrict__ counts, int64_t tile, int64_t tiles, SortLds& L) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int bits = D > 1 ? 32 - __builtin_clz(D - 1) : 0;
  for (int i = threadIdx.x; i < kSortWaves * D; i += kSortThreads) L.cnt[i / D][i % D] = 0;
  __syncthreads();
  const uint64_t below = lane == 0 ? 0ull : ~0ull >> (64 - lane);
  const int64_t i0 = tile * kSortTile + wave * (kSortTile / kSortWaves) + lane;
  int k[kSortRounds], rank[kSortRounds];
#pragma unroll
  for (int q = 0; q < kSortRounds; ++q) {
    const int64_t i = i0 + q * kWave;
    k[q] = i < N ? key(i) : -1;
  }
#pragma unroll
  for (int q = 0; q < kSortRounds; ++q) {
    const uint64_t m = same_key(k[q], bits);
    int before = 0;
    const int lead = m ? __builtin_ctzll(m) : lane;
    if (k[q] >= 0 && lane == lead) before = atomicAdd(&L.cnt[wave][k[q]], __popcll(m));   // (the wave's own counter)
    rank[q] = __shfl(before, lead, kWave) + __popcll(m & below);
  }
  __syncthreads();
  int total = 0, run = 0;
  const int e = threadIdx.x;
  if (e < D) {
    if (tiles > 1) {
      constexpr int U = 8;   // tiles whose counts are read together
      const int32_t* c = counts + e;
      for (int64_t t = 0; t < tiles; t += U) {
        int n[U];
#pragma unroll
        for (int u = 0; u < U; ++u) n[u] = t + u < tiles ? c[(t + u) * D] : 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          run += t + u < tile ? n[u] : 0;
          total += n[u];
        }
      }
    }
    int n[kSortWaves], sum = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) n[w] = L.cnt[w][e];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      L.cnt[w][e] = run + sum;
      sum += n[w];
    }
    if (tiles <= 1) total = sum;
  }
  const int room = (total + align - 1) / align * align;
  const int end = block_scan(room, L.wsum);
  if (e < D) {
    L.first[e] = end - room;
    L.total[e] = total;
    if (e == D - 1) L.used = end;
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kSortRounds; ++q) {
    const int64_t i = i0 + q * kWave;
    if (i < N) emit(i, k[q] >= 0 ? L.first[k[q]] + L.cnt[wave][k[q]] + rank[q] : -1);
  }
}

}  // namespace lmoe
