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

__global__ __launch_bounds__(kSortThreads) void sorted_count_kernel(const int32_t* __restrict__ idx, int64_t N, int E,
                                                                    int32_t* __restrict__ counts) {
  __shared__ int32_t hist[kSortMaxD];
  sort_count(ExpertOf{idx, E}, N, E, counts, blockIdx.x, hist);
}

// slot and src of a tile's choices; block 0 also writes the row ranges.  Rows
// between an expert's last and the next one's first, and past the last, hold none.
__global__ __launch_bounds__(kSortThreads) void sorted_place_kernel(const int32_t* __restrict__ idx, int64_t N, int E,
                                                                    int align, int64_t R,
                                                                    const int32_t* __restrict__ counts,
                                                                    int32_t* __restrict__ row_begin,
                                                                    int32_t* __restrict__ row_end,
                                                                    int32_t* __restrict__ slot,
                                                                    int32_t* __restrict__ src) {
  __shared__ SortLds L;
  sort_place(ExpertOf{idx, E}, [&](int64_t i, int at) {
    slot[i] = at;
    if (at >= 0) src[at] = (int32_t)i;
  }, N, E, align, counts, blockIdx.x, gridDim.x, L);
  const int e = threadIdx.x;
  if (blockIdx.x == 0 && e < E) {
    const int b = L.first[e], n = L.total[e];
    row_begin[e] = b;
    row_end[e] = b + n;
    for (int r = b + n; r < b + (n + align - 1) / align * align; ++r) src[r] = -1;
  }
  const int64_t step = (int64_t)gridDim.x * kSortThreads;
  for (int64_t r = L.used + (int64_t)blockIdx.x * kSortThreads + threadIdx.x; r < R; r += step) src[r] = -1;
}

size_t sorted_dispatch_ws_bytes(const moe_sorted_cfg& c) {
  const int64_t tiles = sort_tiles(c.T * c.k);
  return tiles > 1 ? (size_t)tiles * c.E * sizeof(int32_t) : 0;
}

// ---------------------------------------------------------------------- gather
// rows[r] = x[src[r] / k].  A wave moves sixteen rows by U * 4 vectors of columns:
// four lanes a row, so that a bfloat16 block is written as one KiB.
template <typename T, int U>
__global__ __launch_bounds__(256) void sorted_gather_kernel(const T* __restrict__ x, const int32_t* __restrict__ src,
                                                            T* __restrict__ rows, int64_t R, int64_t N, int d, int k,
                                                            int cols) {
  constexpr int V = Vec<T>::N;
  const int64_t w = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 6;
  const int lane = threadIdx.x & 63;
  const int64_t r = w / cols * 16 + (lane >> 2);
  if (r >= R) return;
  const int i = src[r];
  if (i < 0 || i >= N) return;
  const T* from = x + (int64_t)((uint32_t)i / (uint32_t)k) * d;
  const int c0 = ((int)(w % cols) * U * 4 + (lane & 3)) * V;
  u32x4 v[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (c0 + u * 4 * V < d) v[u] = *reinterpret_cast<const u32x4*>(from + c0 + u * 4 * V);
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (c0 + u * 4 * V < d) *reinterpret_cast<u32x4*>(rows + ebuf_off<T>(r, c0 + u * 4 * V, d)) = v[u];
}

void launch_sorted_dispatch(const moe_sorted_cfg& c, const void* x, const int32_t* idx, int32_t* row_begin,
                            int32_t* row_end, int32_t* slot, int32_t* src, void* rows, void* ws, hipStream_t s) {
  const int64_t N = c.T * c.k, R = sorted_rows(c), tiles = std::max<int64_t>(1, sort_tiles(N));
  int32_t* counts = (int32_t*)ws;
  if (tiles > 1)
    hipLaunchKernelGGL(sorted_count_kernel, dim3((unsigned)tiles), dim3(kSortThreads), 0, s, idx, N, c.E, counts);
  hipLaunchKernelGGL(sorted_place_kernel, dim3((unsigned)tiles), dim3(kSortThreads), 0, s, idx, N, c.E,
                     c.dtype == MOE_BF16 ? 16 : 1, R, counts, row_begin, row_end, slot, src);
  if (R == 0) return;
  auto go = [&](auto tag) {
    using T = decltype(tag);
    constexpr int U = 4;
    const int cols = (c.d_model + U * 4 * Vec<T>::N - 1) / (U * 4 * Vec<T>::N);
    const int64_t waves = (R + 15) / 16 * cols;
    hipLaunchKernelGGL((sorted_gather_kernel<T, U>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, (const T*)x, src,
                       (T*)rows, R, N, c.d_model, c.k, cols);
  };
  if (c.dtype == MOE_BF16) go(uint16_t{});
  else go(float{});
}

// -------------------------------------------------- rows back to their tokens
// W: y[t] = sum over r of w[t][r] rows[slot[t][r]] (combine).  Otherwise the sum
// alone (the dispatch's gradient), G: plus sum over j of dlogits[t][j] Wg[j] (the
// gate's).  Float sums in choice order; a thread owns 16 bytes of a token.
template <typename T, bool W, bool G>
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
  Vec<T>::store(y + t * d + c, acc);
}

template <bool W>
static void launch_back(const moe_sorted_cfg& c, const void* rows, const int32_t* slot, const float* w, const void* Wg,
                        const float* dl, void* y, hipStream_t s) {
  if (c.T == 0) return;
  auto go = [&](auto tag, auto gate) {
    using T = decltype(tag);
    const int64_t n = c.T * (c.d_model / Vec<T>::N);
    hipLaunchKernelGGL((sorted_back_kernel<T, W, decltype(gate)::value>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0,
                       s, (const T*)rows, slot, w, (const T*)Wg, dl, (T*)y, c.T, sorted_rows(c), c.d_model, c.k, c.E);
  };
  auto type = [&](auto gate) {
    if (c.dtype == MOE_BF16) go(uint16_t{}, gate);
    else go(float{}, gate);
  };
  if (Wg) type(std::true_type{});
  else type(std::false_type{});
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
// block takes sixteen rows, each wave a run of columns of all of them (four lanes
// a row, as in the gather); the waves' dot products meet in LDS, in wave order.
// The blocks past the rows write the zeros of the choices that have none.
template <typename T, int U>
__global__ __launch_bounds__(256) void sorted_combine_bwd_kernel(const T* __restrict__ O, const int32_t* __restrict__ slot,
                                                                 const int32_t* __restrict__ src,
                                                                 const float* __restrict__ w, const T* __restrict__ dy,
                                                                 T* __restrict__ dO, float* __restrict__ dw, int64_t R,
                                                                 int64_t N, int d, int k) {
  constexpr int V = Vec<T>::N;
  __shared__ float part[4][16];
  const int64_t rb = (R + 15) / 16;
  if (blockIdx.x >= rb) {
    const int64_t i = ((int64_t)blockIdx.x - rb) * blockDim.x + threadIdx.x;
    if (i < N && (slot[i] < 0 || slot[i] >= R)) dw[i] = 0.f;
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t r = (int64_t)blockIdx.x * 16 + (lane >> 2);
  int i = r < R ? src[r] : -1;
  if (i >= N) i = -1;
  float dot = 0.f;
  if (i >= 0) {
    const float wr = w[i];
    const T* g = dy + (int64_t)((uint32_t)i / (uint32_t)k) * d;
    const T* o = O + r * d;
    for (int c0 = (wave * U * 4 + (lane & 3)) * V; c0 < d; c0 += 4 * U * 4 * V) {
      u32x4 a[U], b[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c0 + u * 4 * V < d) {
          a[u] = *reinterpret_cast<const u32x4*>(g + c0 + u * 4 * V);
          b[u] = *reinterpret_cast<const u32x4*>(o + c0 + u * 4 * V);
        }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c0 + u * 4 * V < d) {
          float p[V], q[V];
          Vec<T>::load(&a[u], p);
          Vec<T>::load(&b[u], q);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            dot = fmaf(p[j], q[j], dot);
            p[j] *= wr;
          }
          Vec<T>::store(dO + ebuf_off<T>(r, c0 + u * 4 * V, d), p);
        }
    }
  }
  dot += __shfl_xor(dot, 1, kWave);
  dot += __shfl_xor(dot, 2, kWave);
  if ((lane & 3) == 0) part[wave][lane >> 2] = dot;
  __syncthreads();
  if (wave == 0 && (lane & 3) == 0 && i >= 0) {
    const int q = lane >> 2;
    dw[i] = ((part[0][q] + part[1][q]) + part[2][q]) + part[3][q];
  }
}

void launch_sorted_combine_bwd(const moe_sorted_cfg& c, const void* O, const int32_t* slot, const int32_t* src,
                               const float* w, const void* dy, void* dO, float* dw, hipStream_t s) {
  const int64_t N = c.T * c.k, R = sorted_rows(c);
  if (N == 0) return;
  auto go = [&](auto tag) {
    using T = decltype(tag);
    hipLaunchKernelGGL((sorted_combine_bwd_kernel<T, 4>), dim3((unsigned)((R + 15) / 16 + (N + 255) / 256)), dim3(256), 0,
                       s, (const T*)O, slot, src, w, (const T*)dy, (T*)dO, dw, R, N, c.d_model, c.k);
  };
  if (c.dtype == MOE_BF16) go(uint16_t{});
  else go(float{});
}

}  // namespace lmoe
