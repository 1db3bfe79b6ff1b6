// Lookup of token ids in a scaled table, and its gradient at the table.
#include "internal.h"
#include "key_sort.h"

namespace lmoe {

// ---------------------------------------------------------------------- lookup
// y[t] = scale W[ids[t]], 0 for an id outside the table.  A thread owns 16 bytes.
template <typename T>
__global__ __launch_bounds__(256) void embed_kernel(const int32_t* __restrict__ ids, const T* __restrict__ W,
                                                    T* __restrict__ y, int64_t T_tokens, int V_rows, int d, float scale) {
  constexpr int V = Vec<T>::N;
  const int nc = d / V;
  const int64_t gid = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t t = gid / nc;
  if (t >= T_tokens) return;
  const int c = (int)(gid - t * nc) * V;
  const int id = ids[t];
  float f[V];
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = 0.f;
  if (id >= 0 && id < V_rows) {
    Vec<T>::load(W + (int64_t)id * d + c, f);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] *= scale;
  }
  Vec<T>::store(y + t * d + c, f);
}

void launch_embed(const moe_embed_cfg& c, const int32_t* ids, const void* W, void* y, hipStream_t s) {
  if (c.T == 0) return;
  auto go = [&](auto tag) {
    using T = decltype(tag);
    const int64_t n = c.T * (c.d_model / Vec<T>::N);
    hipLaunchKernelGGL(embed_kernel<T>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, ids, (const T*)W, (T*)y, c.T,
                       c.V, c.d_model, c.scale);
  };
  if (c.dtype == MOE_BF16) go(uint16_t{});
  else go(float{});
}

// -------------------------------------------------------------------- gradient
// dW[v] = scale * sum of dy[t] over the tokens with ids[t] = v, in token order: the
// tokens are sorted by id (digits of at most nine bits, lowest first, each pass a
// stable placement), then a thread owns 16 bytes of a run of kRun sorted tokens,
// adds in float and stores where the id changes.  An id whose tokens cross a run's
// border leaves partial sums (one at the run's head, one at its tail), which a last
// launch adds in run order: the same bits every time, whatever the ids.
constexpr int kRun = 32;

struct EmbedPlan {
  int passes, bits;
  int64_t tiles, runs;
  size_t key[2], tok[2], counts, part, bytes;   // offsets into the workspace
};
static EmbedPlan embed_plan(const moe_embed_cfg& c) {
  EmbedPlan p{};
  const int all = 32 - __builtin_clz((unsigned)c.V);   // ids 0 .. V - 1, and V for none
  p.passes = (all + 8) / 9;
  p.bits = (all + p.passes - 1) / p.passes;
  p.tiles = std::max<int64_t>(1, sort_tiles(c.T));
  p.runs = (c.T + kRun - 1) / kRun;
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t o = at;
    at += (n + 255) / 256 * 256;
    return o;
  };
  for (int i = 0; i < 2; ++i) {
    p.key[i] = take((size_t)c.T * 4);
    p.tok[i] = take((size_t)c.T * 4);
  }
  p.counts = take((size_t)p.tiles * (1 << p.bits) * 4);
  p.part = take((size_t)p.runs * 2 * c.d_model * 4);
  p.bytes = at;
  return p;
}
size_t embed_bwd_ws_bytes(const moe_embed_cfg& c) { return c.T == 0 ? 0 : embed_plan(c).bytes; }

struct Digit {   // the digit of sorted item i (pass 0: of token i)
  const int32_t* ids;   // pass 0
  const int32_t* keys;  // later passes
  int V, shift, mask;
  __device__ __forceinline__ int key(int64_t i) const {
    if (keys) return keys[i];
    const int id = ids[i];
    return id >= 0 && id < V ? id : V;
  }
  __device__ __forceinline__ int operator()(int64_t i) const { return (key(i) >> shift) & mask; }
};

// Zeros for the table's gradient, 16-byte vectors [a, b), from the blocks that a
// launch has beside its sorting ones: the table is written while the few blocks
// of the sort wait for one another.
__device__ __forceinline__ void fill_zero(u32x4* z, int64_t a, int64_t b, int64_t block, int64_t blocks) {
  for (int64_t i = a + block * blockDim.x + threadIdx.x; i < b; i += blocks * blockDim.x) z[i] = u32x4{0u, 0u, 0u, 0u};
}

__global__ __launch_bounds__(kSortThreads) void embed_count_kernel(Digit dg, int64_t N, int D, int32_t* __restrict__ counts,
                                                                   int64_t tiles, u32x4* z, int64_t za, int64_t zb) {
  __shared__ int32_t hist[kSortMaxD];
  if (blockIdx.x >= tiles) return fill_zero(z, za, zb, blockIdx.x - tiles, gridDim.x - tiles);
  sort_count(dg, N, D, counts, blockIdx.x, hist);
}

__global__ __launch_bounds__(kSortThreads) void embed_place_kernel(Digit dg, const int32_t* __restrict__ toks, int64_t N,
                                                                   int D, const int32_t* __restrict__ counts, int64_t tiles,
                                                                   int32_t* __restrict__ key_out,
                                                                   int32_t* __restrict__ tok_out, u32x4* z, int64_t za,
                                                                   int64_t zb) {
  __shared__ SortLds L;
  if (blockIdx.x >= tiles) return fill_zero(z, za, zb, blockIdx.x - tiles, gridDim.x - tiles);
  sort_place(dg, [&](int64_t i, int at) {
    key_out[at] = dg.key(i);
    tok_out[at] = toks ? toks[i] : (int32_t)i;
  }, N, D, 1, counts, blockIdx.x, tiles, L);
}

template <typename T>
__device__ __forceinline__ void embed_row(T* dW, int64_t at, const float (&acc)[Vec<T>::N], float scale, bool accum) {
  constexpr int V = Vec<T>::N;
  float o[V];
#pragma unroll
  for (int i = 0; i < V; ++i) o[i] = 0.f;
  if (accum) Vec<T>::load(dW + at, o);
#pragma unroll
  for (int i = 0; i < V; ++i) o[i] = accum ? fmaf(scale, acc[i], o[i]) : scale * acc[i];
  Vec<T>::store(dW + at, o);
}

template <typename T>
__global__ __launch_bounds__(256) void embed_runs_kernel(const int32_t* __restrict__ key, const int32_t* __restrict__ tok,
                                                         const T* __restrict__ dy, T* __restrict__ dW,
                                                         float* __restrict__ part, int64_t N, int64_t runs, int V_rows, int d,
                                                         float scale, int accum) {
  constexpr int V = Vec<T>::N, U = 8;
  const int nc = d / V;
  const int64_t gid = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t run = gid / nc;
  if (run >= runs) return;
  const int c = (int)(gid - run * nc) * V;
  const int64_t j0 = run * kRun, j1 = min(N, j0 + kRun);
  int cur = key[j0];
  bool head = j0 > 0 && key[j0 - 1] == cur;
  float acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.f;
  auto partial = [&](int which) {
    float* o = part + (run * 2 + which) * d + c;
#pragma unroll
    for (int i = 0; i < V; i += 4) *reinterpret_cast<f32x4*>(o + i) = f32x4{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
  };
  for (int64_t j = j0; j < j1; j += U) {
    u32x4 v[U];
    int k[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      k[u] = j + u < j1 ? key[j + u] : V_rows;
      if (k[u] < V_rows) v[u] = *reinterpret_cast<const u32x4*>(dy + (int64_t)tok[j + u] * d + c);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (j + u >= j1) break;
      if (k[u] != cur) {   // (ids go up: past the last id of the table come the tokens without one)
        if (head) partial(0);
        else embed_row(dW, (int64_t)cur * d + c, acc, scale, accum);
        head = false;
        cur = k[u];
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = 0.f;
      }
      if (cur < V_rows) {
        float f[V];
        Vec<T>::load(&v[u], f);
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] += f[i];
      }
    }
  }
  if (cur >= V_rows) return;
  if (head) partial(0);
  else if (j1 < N && key[j1] == cur) partial(1);
  else embed_row(dW, (int64_t)cur * d + c, acc, scale, accum);
}

// The ids that began in a run and went on past it: its tail, and the heads of the runs up to the last one that they reach.
template <typename T>
__global__ __launch_bounds__(256) void embed_join_kernel(const int32_t* __restrict__ key, T* __restrict__ dW,
                                                         const float* __restrict__ part, int64_t N, int64_t runs, int V_rows,
                                                         int d, float scale, int accum) {
  constexpr int V = Vec<T>::N;
  const int nc = d / V;
  const int64_t gid = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t run = gid / nc;
  if (run >= runs) return;
  const int c = (int)(gid - run * nc) * V;
  const int64_t j0 = run * kRun, j1 = j0 + kRun;
  if (j1 >= N) return;
  const int cur = key[j1 - 1];
  if (cur >= V_rows || key[j1] != cur || (j0 > 0 && key[j0 - 1] == cur)) return;
  float acc[V];
  auto add = [&](int64_t at, bool first) {
    const float* o = part + at * d + c;
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(o + i);
#pragma unroll
      for (int u = 0; u < 4; ++u) acc[i + u] = first ? v[u] : acc[i + u] + v[u];
    }
  };
  add(run * 2 + 1, true);
  for (int64_t m = run + 1; m < runs; ++m) {
    add(m * 2, false);
    const int64_t end = (m + 1) * kRun;
    if (end >= N || key[end] != cur) break;
  }
  embed_row(dW, (int64_t)cur * d + c, acc, scale, accum);
}

void launch_embed_bwd(const moe_embed_cfg& c, const int32_t* ids, const void* dy, void* dW, void* ws, hipStream_t s) {
  const int esz = c.dtype == MOE_BF16 ? 2 : 4;
  const int64_t zeros = c.accum ? 0 : (int64_t)c.V * c.d_model * esz / 16;
  const unsigned zblocks = zeros ? (unsigned)std::min<int64_t>(1024, (zeros + 4 * kSortThreads - 1) / (4 * kSortThreads)) : 0;
  u32x4* z = (u32x4*)dW;
  if (c.T == 0) {
    if (zeros)
      hipLaunchKernelGGL(embed_count_kernel, dim3(zblocks), dim3(kSortThreads), 0, s, Digit{}, (int64_t)0, 0, nullptr,
                         (int64_t)0, z, (int64_t)0, zeros);
    return;
  }
  const EmbedPlan p = embed_plan(c);
  char* w = (char*)ws;
  int32_t* counts = (int32_t*)(w + p.counts);
  const bool count = p.tiles > 1;
  const int launches = p.passes * (count ? 2 : 1);
  int done = 0;
  auto za = [&](int i) { return zeros * i / launches; };
  const unsigned grid = (unsigned)p.tiles + zblocks;
  const int D = 1 << p.bits;
  for (int q = 0; q < p.passes; ++q) {
    const int32_t *kin = q ? (const int32_t*)(w + p.key[(q - 1) & 1]) : nullptr,
                  *tin = q ? (const int32_t*)(w + p.tok[(q - 1) & 1]) : nullptr;
    const Digit dg{ids, kin, c.V, q * p.bits, D - 1};
    if (count) {
      hipLaunchKernelGGL(embed_count_kernel, dim3(grid), dim3(kSortThreads), 0, s, dg, c.T, D, counts, p.tiles, z,
                         za(done), za(done + 1));
      ++done;
    }
    hipLaunchKernelGGL(embed_place_kernel, dim3(grid), dim3(kSortThreads), 0, s, dg, tin, c.T, D, counts, p.tiles,
                       (int32_t*)(w + p.key[q & 1]), (int32_t*)(w + p.tok[q & 1]), z, za(done), za(done + 1));
    ++done;
  }
  const int last = (p.passes - 1) & 1;
  const int32_t *key = (const int32_t*)(w + p.key[last]), *tok = (const int32_t*)(w + p.tok[last]);
  auto go = [&](auto tag) {
    using T = decltype(tag);
    const int64_t n = p.runs * (c.d_model / Vec<T>::N);
    const unsigned blocks = (unsigned)((n + 255) / 256);
    hipLaunchKernelGGL(embed_runs_kernel<T>, dim3(blocks), dim3(256), 0, s, key, tok, (const T*)dy, (T*)dW,
                       (float*)(w + p.part), c.T, p.runs, c.V, c.d_model, c.scale, c.accum);
    if (p.runs > 1)
      hipLaunchKernelGGL(embed_join_kernel<T>, dim3(blocks), dim3(256), 0, s, key, (T*)dW, (const float*)(w + p.part), c.T,
                         p.runs, c.V, c.d_model, c.scale, c.accum);
  };
  if (c.dtype == MOE_BF16) go(uint16_t{});
  else go(float{});
}

}  // namespace lmoe
