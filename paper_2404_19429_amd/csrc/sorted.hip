// Tokens sorted by expert and back, without a capacity: every choice gets a row,
// the rows of an expert lie together, in (token, choice) order.
//
// rows and dO are what the products read (bfloat16: 16 x 32 blocks), expert_out
// and dXe row-major.  An expert's rows start at a multiple of sixteen in
// bfloat16, so a block of sixteen rows belongs to one expert.
#include "internal.h"
#include "key_sort.h"

namespace lmoe {

int64_t sorted_rows(const moe_sorted_cfg& c) {
  const int64_t n = c.T * c.k;
  return c.dtype == MOE_BF16 ? pad16(n + 15 * std::min<int64_t>(c.E, n)) : n;
}

// ------------------------------------------------------------------------ sort
struct ExpertOf {   // the expert of choice i, -1: none
  const int32_t* idx;
  int E;
  __device__ __forceinline__ int operator()(int64_t i) const {
    const int e = idx[i];
    return e >= 0 && e < E ? e : -1;
  }
};

template <int NT>
__global__ __launch_bounds__(NT) void sorted_count_kernel(const int32_t* __restrict__ idx, int64_t N, int E,
                                                          int32_t* __restrict__ counts) {
  __shared__ int32_t hist[kSortMaxD];
  sort_count<NT>(ExpertOf{idx, E}, N, E, counts, blockIdx.x, hist);
}

// The row ranges, and which rows hold no choice: those between an expert's last
// and the next one's first, and those past the last (none(r) for each, shared by
// the grid's threads).
template <int NT, typename None>
__device__ __forceinline__ void sorted_ranges(const SortLds<NT>& L, int E, int align, int64_t R, int32_t* row_begin,
                                              int32_t* row_end, int64_t block, int64_t blocks, const None& none) {
  for (int e = threadIdx.x; e < E; e += NT) {
    const int b = L.first[e], n = L.total[e];
    if (block == 0) {
      row_begin[e] = b;
      row_end[e] = b + n;
    }
    if (block == 0)
      for (int r = b + n; r < b + (n + align - 1) / align * align; ++r) none(r);
  }
  for (int64_t r = L.used + block * NT + threadIdx.x; r < R; r += blocks * NT) none(r);
}

// slot and src of a tile's choices; block 0 also writes the row ranges.
template <int NT>
__global__ __launch_bounds__(NT) void sorted_place_kernel(const int32_t* __restrict__ idx, int64_t N, int E, int align,
                                                          int64_t R, const int32_t* __restrict__ counts,
                                                          int32_t* __restrict__ row_begin, int32_t* __restrict__ row_end,
                                                          int32_t* __restrict__ slot, int32_t* __restrict__ src) {
  __shared__ SortLds<NT> L;
  sort_place<NT>(ExpertOf{idx, E}, [&](int64_t i, int at) {
    slot[i] = at;
    if (at >= 0) src[at] = (int32_t)i;
  }, N, E, align, counts, blockIdx.x, gridDim.x, L);
  sorted_ranges<NT>(L, E, align, R, row_begin, row_end, blockIdx.x, gridDim.x, [&](int64_t r) { src[r] = -1; });
}

size_t sorted_dispatch_ws_bytes(const moe_sorted_cfg& c) {
  const int64_t tiles = sort_tiles(c.T * c.k);
  return tiles > 1 ? (size_t)sort_counts(tiles, c.E) * sizeof(int32_t) : 0;
}

// ---------------------------------------------------------------------- gather
// rows[r] = x[src[r] / k].  A wave moves sixteen rows by U * 8 vectors of columns:
// eight lanes a row, so that a load and a store are whole cache lines (a bfloat16
// block's half is 512 bytes in one run).  Bound: bytes; 16384 x 2 rows of 2048 in
// bfloat16: 201 MB moved in 41 us (traced); four lanes a row, whose accesses were half
// lines, 48.
template <typename T, int U, bool S>
__device__ __forceinline__ void gather_rows(const T* __restrict__ x, T* __restrict__ rows, int64_t r0, const int (&i)[2], int d,
                                            int k, int c0) {
  constexpr int V = Vec<T>::N;
  u32x4 v[2][U];
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (i[h] >= 0) {
      const T* from = x + (int64_t)((uint32_t)i[h] / (uint32_t)k) * d;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c0 + u * 8 * V < d) v[h][u] = *reinterpret_cast<const u32x4*>(from + c0 + u * 8 * V);
    }
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (i[h] >= 0)
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c0 + u * 8 * V < d) store16<S>((void*)(rows + ebuf_off<T>(r0 + 8 * h, c0 + u * 8 * V, d)), v[h][u]);
}
template <typename T, int U, bool S>
__global__ __launch_bounds__(256) void sorted_gather_kernel(const T* __restrict__ x, const int32_t* __restrict__ src,
                                                            T* __restrict__ rows, int64_t R, int64_t N, int d, int k,
                                                            int cols) {
  const int64_t w = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 6;
  const int lane = threadIdx.x & 63;
  const int64_t r = w / cols * 16 + (lane >> 3);
  int i[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    i[h] = r + 8 * h < R ? src[r + 8 * h] : -1;
    if (i[h] >= N) i[h] = -1;
  }
  gather_rows<T, U, S>(x, rows, r, i, d, k, ((int)(w % cols) * U * 8 + (lane & 7)) * Vec<T>::N);
}

// One tile of choices (a decode batch): every block places it for itself, a couple
// of microseconds beside a launch and its wait, and moves its share of the rows;
// block 0 writes what the caller keeps.
template <typename T, int U>
__global__ __launch_bounds__(kSortSmall) void sorted_small_kernel(const T* __restrict__ x, const int32_t* __restrict__ idx,
                                                                  int N, int E, int align, int R, int32_t* row_begin,
                                                                  int32_t* row_end, int32_t* slot, int32_t* src,
                                                                  T* __restrict__ rows, int d, int k, int cols) {
  constexpr int NT = kSortSmall;
  __shared__ SortLds<NT> L;
  __shared__ int16_t held[kSortRounds * NT + 15 * kSortMaxD + 16];   // the choice that a row holds
  const bool first = blockIdx.x == 0;
  sort_place<NT>(ExpertOf{idx, E}, [&](int64_t i, int at) {
    if (first) slot[i] = at;
    if (at >= 0) held[at] = (int16_t)i;
  }, N, E, align, nullptr, 0, 1, L);
  for (int e = threadIdx.x; e < E; e += NT) {
    const int b = L.first[e], n = L.total[e];
    if (first) {
      row_begin[e] = b;
      row_end[e] = b + n;
    }
    for (int r = b + n; r < b + (n + align - 1) / align * align; ++r) held[r] = -1;
  }
  __syncthreads();
  const int used = L.used;
  if (first)
    for (int r = threadIdx.x; r < R; r += NT) src[r] = r < used ? held[r] : -1;
  const int lane = threadIdx.x & 63;
  for (int w = blockIdx.x * (NT / kWave) + (threadIdx.x >> 6); w / cols * 16 < used; w += gridDim.x * (NT / kWave)) {
    const int r = w / cols * 16 + (lane >> 3);
    const int i[2] = {r < used ? held[r] : -1, r + 8 < used ? held[r + 8] : -1};
    gather_rows<T, U, false>(x, rows, r, i, d, k, (w % cols * U * 8 + (lane & 7)) * Vec<T>::N);
  }
}

void launch_sorted_dispatch(const moe_sorted_cfg& c, const void* x, const int32_t* idx, int32_t* row_begin,
                            int32_t* row_end, int32_t* slot, int32_t* src, void* rows, void* ws, hipStream_t s) {
  const int64_t N = c.T * c.k, R = sorted_rows(c), tiles = std::max<int64_t>(1, sort_tiles(N));
  const int align = c.dtype == MOE_BF16 ? 16 : 1;
  int32_t* counts = (int32_t*)ws;
  auto place = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    if (tiles > 1)
      launch_kernel(sorted_count_kernel<NT>, dim3((unsigned)tiles), dim3(NT), 0, s, idx, N, c.E, counts);
    launch_sort_scan(counts, tiles, c.E, s);
    launch_kernel(sorted_place_kernel<NT>, dim3((unsigned)tiles), dim3(NT), 0, s, idx, N, c.E, align, R, counts, row_begin,
                  row_end, slot, src);
  };
  auto go = [&](auto tag) {
    using T = decltype(tag);
    constexpr int U = 1;
    const int cols = (c.d_model + U * 8 * Vec<T>::N - 1) / (U * 8 * Vec<T>::N);
    const int64_t strips = (R + 15) / 16, waves = strips * cols;   // of sixteen rows
    if (tiles == 1 && N > 0) {
      const unsigned blocks = (unsigned)std::min<int64_t>(256, (waves + 3) / 4);
      launch_kernel((sorted_small_kernel<T, U>), dim3(blocks), dim3(kSortSmall), 0, s, (const T*)x, idx, (int)N, c.E, align,
                    (int)R, row_begin, row_end, slot, src, (T*)rows, c.d_model, c.k, cols);
      return;
    }
    if (sort_threads(N) == kSortSmall) place(std::integral_constant<int, kSortSmall>{});
    else place(std::integral_constant<int, kSortLarge>{});
    auto gather = [&](auto stream) {
      each_launch(strips, (int64_t)cols * kWave, [&](int64_t b, int64_t n) {   // (rows of whole strips lie together)
        launch_kernel((sorted_gather_kernel<T, U, decltype(stream)::value>), dim3((unsigned)((n * cols + 3) / 4)),
                      dim3(256), 0, s, (const T*)x, src + 16 * b, (T*)rows + 16 * b * c.d_model,
                      std::min(16 * n, R - 16 * b), N, c.d_model, c.k, cols);
      });
    };
    if (R == 0) return;
    if (stream_bytes(R * c.d_model * (int64_t)sizeof(T))) gather(std::true_type{});
    else gather(std::false_type{});
  };
  if (c.dtype == MOE_BF16) go(uint16_t{});
  else go(float{});
}

// -------------------------------------------------- rows back to their tokens
// W: y[t] = sum over r of w[t][r] rows[slot[t][r]] (combine).  Otherwise the sum
// alone (the dispatch's gradient), G: plus sum over j of dlogits[t][j] Wg[j] (the
// gate's).  Float sums in choice order; a thread owns 16 bytes of a token.  Bound:
// bytes, 201 MB in 34 and 36 us (traced; 16384 tokens, two choices, 2048 in bfloat16).
template <typename T, bool W, bool G, bool S>
__global__ __launch_bounds__(256) void sorted_back_kernel(const T* __restrict__ rows, const int32_t* __restrict__ slot,
                                                          const float* __restrict__ w, const T* __restrict__ Wg,
                                                          const float* __restrict__ dl, T* __restrict__ y,
                                                          int64_t T_tokens, int64_t R, int d, int k, int E) {
  constexpr int V = Vec<T>::N, U = 4;
  const int nc = d / V;
  const int64_t gid = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t t = gid / nc;
  if (t >= T_tokens) return;
  const int c = (int)(gid - t * nc) * V;
  float acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.f;
  for (int r0 = 0; r0 < k; r0 += U) {
    u32x4 v[U];
    float wr[U];
    bool on[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      on[u] = false;
      if (r0 + u < k) {
        const int at = slot[t * k + r0 + u];
        on[u] = at >= 0 && at < R;
        if (on[u]) {
          v[u] = *reinterpret_cast<const u32x4*>(rows + (int64_t)at * d + c);
          wr[u] = W ? w[t * k + r0 + u] : 1.f;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (on[u]) {
        float f[V];
        Vec<T>::load(&v[u], f);
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = W ? fmaf(wr[u], f[i], acc[i]) : acc[i] + f[i];
      }
  }
  if constexpr (G) {
    for (int j = 0; j < E; ++j) {
      const float a = dl[t * E + j];
      if (a == 0.f) continue;   // (an expert that the token did not choose, under renormalised weights)
      float f[V];
      Vec<T>::load(Wg + (int64_t)j * d + c, f);
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] = fmaf(a, f[i], acc[i]);
    }
  }
  store16<S>(y + t * d + c, acc);
}

template <bool W>
static void launch_back(const moe_sorted_cfg& c, const void* rows, const int32_t* slot, const float* w, const void* Wg,
                        const float* dl, void* y, hipStream_t s) {
  if (c.T == 0) return;
  auto go = [&](auto tag, auto gate, auto stream) {
    using T = decltype(tag);
    const int64_t nc = c.d_model / Vec<T>::N;
    each_launch(c.T, nc, [&](int64_t t0, int64_t n) {
      launch_kernel((sorted_back_kernel<T, W, decltype(gate)::value, decltype(stream)::value>),
                    dim3((unsigned)((n * nc + 255) / 256)), dim3(256), 0, s, (const T*)rows, slot + t0 * c.k,
                    W ? w + t0 * c.k : nullptr, (const T*)Wg, dl ? dl + t0 * c.E : nullptr, (T*)y + t0 * c.d_model, n,
                    sorted_rows(c), c.d_model, c.k, c.E);
    });
  };
  auto type = [&](auto gate, auto stream) {
    if (c.dtype == MOE_BF16) go(uint16_t{}, gate, stream);
    else go(float{}, gate, stream);
  };
  auto gated = [&](auto stream) {
    if (Wg) type(std::true_type{}, stream);
    else type(std::false_type{}, stream);
  };
  if (stream_bytes(c.T * c.d_model * (c.dtype == MOE_BF16 ? 2 : 4))) gated(std::true_type{});
  else gated(std::false_type{});
}

void launch_sorted_combine(const moe_sorted_cfg& c, const void* O, const int32_t* slot, const float* w, void* y,
                           hipStream_t s) {
  launch_back<true>(c, O, slot, w, nullptr, nullptr, y, s);
}
void launch_sorted_dispatch_bwd(const moe_sorted_cfg& c, const int32_t* slot, const void* dXe, const void* Wg,
                                const float* dl, void* dx, hipStream_t s) {
  launch_back<false>(c, dXe, slot, nullptr, Wg, dl, dx, s);
}

// ------------------------------------------------------------ combine backward
// dO[row] = w dy[t], dw = <dy[t], O[row]> for the choice that the row holds.  A
// block takes sixteen rows, each wave a run of columns of all of them (eight lanes
// a row, as in the gather); the waves' dot products meet in LDS, in wave order.
// The blocks past the rows (of the first launch) write the zeros of the choices that have none.  Bound:
// bytes, 336 MB in 67 us (traced; as above).
template <typename T, int U, bool S>
__global__ __launch_bounds__(256) void sorted_combine_bwd_kernel(const T* __restrict__ O, const int32_t* __restrict__ slot,
                                                                 const int32_t* __restrict__ src,
                                                                 const float* __restrict__ w, const T* __restrict__ dy,
                                                                 T* __restrict__ dO, float* __restrict__ dw, int64_t R,
                                                                 int64_t all_rows, int64_t N, int d, int k) {
  constexpr int V = Vec<T>::N;
  __shared__ float part[4][16];
  const int64_t rb = (R + 15) / 16;   // R: the launch's rows, of all_rows
  if (blockIdx.x >= rb) {
    const int64_t i = ((int64_t)blockIdx.x - rb) * blockDim.x + threadIdx.x;
    if (i < N && (slot[i] < 0 || slot[i] >= all_rows)) dw[i] = 0.f;
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t r0 = (int64_t)blockIdx.x * 16 + (lane >> 3);
  int i[2];
  float wr[2], dot[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    i[h] = r0 + 8 * h < R ? src[r0 + 8 * h] : -1;
    if (i[h] >= N) i[h] = -1;
    wr[h] = i[h] >= 0 ? w[i[h]] : 0.f;
    dot[h] = 0.f;
  }
  for (int c0 = (wave * U * 8 + (lane & 7)) * V; c0 < d; c0 += 4 * U * 8 * V) {
    u32x4 a[2][U], b[2][U];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (i[h] >= 0) {
        const T *g = dy + (int64_t)((uint32_t)i[h] / (uint32_t)k) * d, *o = O + (r0 + 8 * h) * d;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (c0 + u * 8 * V < d) {
            a[h][u] = *reinterpret_cast<const u32x4*>(g + c0 + u * 8 * V);
            b[h][u] = *reinterpret_cast<const u32x4*>(o + c0 + u * 8 * V);
          }
      }
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (i[h] >= 0)
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (c0 + u * 8 * V < d) {
            float p[V], q[V];
            Vec<T>::load(&a[h][u], p);
            Vec<T>::load(&b[h][u], q);
#pragma unroll
            for (int j = 0; j < V; ++j) {
              dot[h] = fmaf(p[j], q[j], dot[h]);
              p[j] *= wr[h];
            }
            store16<S>(dO + ebuf_off<T>(r0 + 8 * h, c0 + u * 8 * V, d), p);
          }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) dot[h] += __shfl_xor(dot[h], o, kWave);
    if ((lane & 7) == 0) part[wave][8 * h + (lane >> 3)] = dot[h];
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int q = 8 * h + (lane >> 3);
    if (wave == 0 && (lane & 7) == 0 && i[h] >= 0) dw[i[h]] = ((part[0][q] + part[1][q]) + part[2][q]) + part[3][q];
  }
}

void launch_sorted_combine_bwd(const moe_sorted_cfg& c, const void* O, const int32_t* slot, const int32_t* src,
                               const float* w, const void* dy, void* dO, float* dw, hipStream_t s) {
  const int64_t N = c.T * c.k, R = sorted_rows(c);
  if (N == 0) return;
  auto go = [&](auto tag, auto stream) {
    using T = decltype(tag);
    each_launch((R + 15) / 16, 256, [&](int64_t b, int64_t n) {   // (beside N threads at most: together under 2^32)
      const int64_t r0 = 16 * b, zeros = b == 0 ? (N + 255) / 256 : 0;
      launch_kernel((sorted_combine_bwd_kernel<T, 2, decltype(stream)::value>), dim3((unsigned)(n + zeros)), dim3(256), 0, s,
                    (const T*)O + r0 * c.d_model, slot, src + r0, w, (const T*)dy, (T*)dO + r0 * c.d_model, dw,
                    std::min(16 * n, R - r0), R, N, c.d_model, c.k);
    });
  };
  auto type = [&](auto stream) {
    if (c.dtype == MOE_BF16) go(uint16_t{}, stream);
    else go(float{}, stream);
  };
  if (stream_bytes(R * c.d_model * (c.dtype == MOE_BF16 ? 2 : 4))) type(std::true_type{});
  else type(std::false_type{});
}

}  // namespace lmoe
