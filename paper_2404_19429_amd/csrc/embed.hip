// Lookup of token ids in a scaled table, and its gradient at the table.
#include "internal.h"
#include "key_sort.h"

namespace lmoe {

// ---------------------------------------------------------------------- lookup
// y[t] = scale W[ids[t]], 0 for an id outside the table.  A thread owns 16 bytes.
template <typename T, bool S>
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
  store16<S>(y + t * d + c, f);
}

void launch_embed(const moe_embed_cfg& c, const int32_t* ids, const void* W, void* y, hipStream_t s) {
  if (c.T == 0) return;
  auto go = [&](auto tag, auto stream) {
    using T = decltype(tag);
    const int64_t nc = c.d_model / Vec<T>::N;
    each_launch(c.T, nc, [&](int64_t t0, int64_t n) {
      launch_kernel((embed_kernel<T, decltype(stream)::value>), dim3((unsigned)((n * nc + 255) / 256)), dim3(256), 0, s,
                    ids + t0, (const T*)W, (T*)y + t0 * c.d_model, n, c.V, c.d_model, c.scale);
    });
  };
  auto type = [&](auto stream) {
    if (c.dtype == MOE_BF16) go(uint16_t{}, stream);
    else go(float{}, stream);
  };
  if (stream_bytes(c.T * c.d_model * (c.dtype == MOE_BF16 ? 2 : 4))) type(std::true_type{});
  else type(std::false_type{});
}

// -------------------------------------------------------------------- gradient
// dW[v] = scale * sum of dy[t] over the tokens with ids[t] = v, in token order: the
// tokens are sorted by id (digits of at most nine bits, lowest first, each pass a
// stable placement; few tokens by comparing all pairs, in one launch), then a
// thread owns 16 bytes of a run of kRun sorted tokens, has their rows in flight
// together, adds in float and stores where the id changes.  An id whose tokens cross
// a run's border leaves partial sums (one at the run's head, one at its tail), which
// a last launch adds in run order: the same bits every time, whatever the ids.
// Bound: bytes, the table's gradient written once and dy read once: 16384 tokens of
// 50257 rows of 2048 in bfloat16, lookup and gradient 366 MB in 93 us, of which the
// sort's chain of latencies is 43 with 206 MB of zeros beside it.
constexpr int kRun = 16;

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
  auto take = [&](size_t n) {   // (whole runs of keys and tokens can be read)
    const size_t o = at;
    at += (n + 255) / 256 * 256;
    return o;
  };
  for (int i = 0; i < 2; ++i) {
    p.key[i] = take((size_t)c.T * 4);
    p.tok[i] = take((size_t)c.T * 4);
  }
  p.counts = take((size_t)sort_counts(p.tiles, 1 << p.bits) * 4);
  p.part = take((size_t)p.runs * 2 * c.d_model * 4);
  p.bytes = at;
  return p;
}
size_t embed_bwd_ws_bytes(const moe_embed_cfg& c) { return c.T == 0 ? 0 : embed_plan(c).bytes; }

// A token's id as a key; V for a token without one.
__device__ __forceinline__ int id_key(const int32_t* ids, int64_t t, int V) {
  const int id = ids[t];
  return id >= 0 && id < V ? id : V;
}
struct Digit {   // the digit of sorted item i (pass 0: of token i)
  const int32_t* ids;   // pass 0
  const int32_t* keys;  // later passes
  int V, shift, mask;
  __device__ __forceinline__ int key(int64_t i) const { return keys ? keys[i] : id_key(ids, i, V); }
  __device__ __forceinline__ int operator()(int64_t i) const { return (key(i) >> shift) & mask; }
};

// Zeros for the table's gradient, 16-byte vectors [a, b), from the blocks that a
// launch has beside its sorting ones: the table is written while the few blocks
// of the sort wait for one another.  The table's gradient is the optimiser's next, far
// behind: stored past the caches (16384 tokens, 50257 rows of 2048: 113 -> 103 us).
__device__ __forceinline__ void fill_zero(u32x4* z, int64_t a, int64_t b, int64_t block, int64_t blocks) {
  for (int64_t i = a + block * blockDim.x + threadIdx.x; i < b; i += blocks * blockDim.x) store16<true>((void*)(z + i), u32x4{0u, 0u, 0u, 0u});
}

template <int NT>
__global__ __launch_bounds__(NT) void embed_count_kernel(Digit dg, int64_t N, int D, int32_t* __restrict__ counts,
                                                         int64_t tiles, u32x4* z, int64_t za, int64_t zb) {
  __shared__ int32_t hist[kSortMaxD];
  if (blockIdx.x >= tiles) return fill_zero(z, za, zb, blockIdx.x - tiles, gridDim.x - tiles);
  sort_count<NT>(dg, N, D, counts, blockIdx.x, hist);
}

template <int NT>
__global__ __launch_bounds__(NT) void embed_place_kernel(Digit dg, const int32_t* __restrict__ toks, int64_t N, int D,
                                                         const int32_t* __restrict__ counts, int64_t tiles,
                                                         int32_t* __restrict__ key_out, int32_t* __restrict__ tok_out, u32x4* z,
                                                         int64_t za, int64_t zb) {
  __shared__ SortLds<NT> L;
  if (blockIdx.x >= tiles) return fill_zero(z, za, zb, blockIdx.x - tiles, gridDim.x - tiles);
  sort_place<NT>(dg, [&](int64_t i, int at) {
    key_out[at] = dg.key(i);
    tok_out[at] = toks ? toks[i] : (int32_t)i;
  }, N, D, 1, counts, blockIdx.x, tiles, L);
}

// Few tokens: a token's place is the number of tokens whose id is smaller, or the
// same and earlier.  A block takes 64 tokens, each of its waves compares them with a
// quarter of all ids (in LDS, four to a read): N^2 / 64 comparisons of a wave, over
// many CUs, against the radix passes' chain of launches (1111 tokens: 9.5 us against
// 12.3 for two passes in one block; at 16384 tokens 74 against 43 for the passes).
constexpr int kPairs = 8192;
__global__ __launch_bounds__(256) void embed_pairs_kernel(const int32_t* __restrict__ ids, int N, int V, int blocks,
                                                          int32_t* __restrict__ key_out, int32_t* __restrict__ tok_out,
                                                          u32x4* z, int64_t zb) {
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  extern __shared__ __attribute__((aligned(16))) int flat[];   // the ids, padded to whole chunks for four waves
  __shared__ int part[4][64];
  const i32x4* keys = (const i32x4*)flat;
  if (blockIdx.x >= blocks) return fill_zero(z, 0, zb, blockIdx.x - blocks, gridDim.x - blocks);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int padded = (N + 255) / 256 * 256;
  for (int i = threadIdx.x; i < padded; i += 256) flat[i] = i < N ? id_key(ids, i, V) : 0x7fffffff;
  __syncthreads();
  const int t0 = blockIdx.x * 64, t = t0 + lane;
  const int mine = flat[min(t, padded - 1)];
  int n = 0;
  const int quarter = padded / 4;   // a multiple of 64
  for (int b = wave * quarter; b < (wave + 1) * quarter; b += 64) {
    if (b != t0) {
      const int limit = mine + (b < t0 ? 1 : 0);   // (ids are at most 2^30)
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const i32x4 k = keys[b / 4 + q];
#pragma unroll
        for (int u = 0; u < 4; ++u) n += k[u] < limit ? 1 : 0;
      }
    } else {
      for (int j = 0; j < 64; ++j) n += flat[b + j] < mine + (j < lane ? 1 : 0) ? 1 : 0;
    }
  }
  part[wave][lane] = n;
  __syncthreads();
  if (wave == 0 && t < N) {
    const int at = part[0][lane] + part[1][lane] + part[2][lane] + part[3][lane];
    key_out[at] = mine;
    tok_out[at] = t;
  }
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
  store16<true>(dW + at, o);
}

template <typename T>
__global__ __launch_bounds__(256) void embed_runs_kernel(const int32_t* __restrict__ key, const int32_t* __restrict__ tok,
                                                         const T* __restrict__ dy, T* __restrict__ dW,
                                                         float* __restrict__ part, int64_t N, int64_t run0, int64_t runs,
                                                         int V_rows, int d, float scale, int accum) {
  constexpr int V = Vec<T>::N;
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  const int nc = d / V;
  const int64_t gid = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t local = gid / nc, run = run0 + local;   // of the launch's runs, run0 .. runs - 1
  if (run >= runs) return;
  const int c = (int)(gid - local * nc) * V;
  const int64_t j0 = run * kRun;
  const int n = (int)min((int64_t)kRun, N - j0);   // the run's tokens
  int k[kRun + 1], t[kRun];
#pragma unroll
  for (int q = 0; q < kRun; q += 4) {
    const i32x4 a = *reinterpret_cast<const i32x4*>(key + j0 + q), b = *reinterpret_cast<const i32x4*>(tok + j0 + q);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      k[q + u] = q + u < n ? a[u] : V_rows;
      t[q + u] = q + u < n ? b[u] : 0;
    }
  }
  const int prev = j0 > 0 ? key[j0 - 1] : -1;
  k[kRun] = j0 + kRun < N ? key[j0 + kRun] : V_rows;
  u32x4 v[kRun];
#pragma unroll
  for (int u = 0; u < kRun; ++u)   // (a token without an id has a row too; it is not added)
    v[u] = *reinterpret_cast<const u32x4*>(dy + (int64_t)t[u] * d + c);
  float acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.f;
  bool head = prev == k[0];
#pragma unroll
  for (int u = 0; u < kRun; ++u) {   // (ids go up: past the last id of the table come the tokens without one)
    if (k[u] >= V_rows) break;
    float f[V];
    Vec<T>::load(&v[u], f);
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] += f[i];
    if (k[u + 1] == k[u] && u + 1 < kRun) continue;
    const bool tail = k[u + 1] == k[u];
    if (head || tail) {
      float* o = part + (run * 2 + (head ? 0 : 1)) * d + c;
#pragma unroll
      for (int i = 0; i < V; i += 4) *reinterpret_cast<f32x4*>(o + i) = f32x4{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
    } else {
      embed_row(dW, (int64_t)k[u] * d + c, acc, scale, accum);
    }
    head = false;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
  }
}

// The ids that began in a run and went on past it: its tail, and the heads of the
// runs up to the last one that they reach.  A block is kJoinCols vectors of columns
// by four equal shares of those runs, which meet in LDS in order (an id that most
// tokens have is a long chain).
constexpr int kJoinCols = 64;
template <typename T>
__global__ __launch_bounds__(4 * kJoinCols) void embed_join_kernel(const int32_t* __restrict__ key, T* __restrict__ dW,
                                                                   const float* __restrict__ part, int64_t N, int64_t run0,
                                                                   int64_t runs, int V_rows, int d, int slabs, float scale, int accum) {
  constexpr int V = Vec<T>::N;
  __shared__ f32x4 red[3][kJoinCols][V / 4];
  const int64_t run = run0 + (int64_t)blockIdx.x / slabs;
  const int64_t j0 = run * kRun, j1 = j0 + kRun;
  if (j1 >= N) return;
  const int cur = key[j1 - 1];
  if (cur >= V_rows || key[j1] != cur || (j0 > 0 && key[j0 - 1] == cur)) return;
  // The last run that begins with this id: steps that double, then halve.
  int64_t lo = run + 1, step = 1;
  while (lo + step < runs && key[(lo + step) * kRun] == cur) {
    lo += step;
    step *= 2;
  }
  for (; step > 0; step /= 2)
    if (lo + step < runs && key[(lo + step) * kRun] == cur) lo += step;
  const int64_t heads = lo - run;   // runs run + 1 .. lo
  const int share = threadIdx.x / kJoinCols, lc = threadIdx.x % kJoinCols;
  const int c = ((int)(blockIdx.x % slabs) * kJoinCols + lc) * V;
  const bool on = c < d;
  const int64_t a = run + 1 + heads * share / 4, b = run + 1 + heads * (share + 1) / 4;
  float acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.f;
  if (on) {
    if (share == 0)
#pragma unroll
      for (int q = 0; q < V / 4; ++q) Vec<float>::load(part + (run * 2 + 1) * d + c + 4 * q, acc + 4 * q);
    constexpr int U = 8;
    for (int64_t m = a; m < b; m += U) {
      f32x4 p[U][V / 4];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < V / 4; ++q)
          p[u][q] = *reinterpret_cast<const f32x4*>(part + min(m + u, b - 1) * 2 * d + c + 4 * q);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (m + u < b)
#pragma unroll
          for (int i = 0; i < V; ++i) acc[i] += p[u][i / 4][i % 4];
    }
    if (share > 0)
#pragma unroll
      for (int q = 0; q < V / 4; ++q) red[share - 1][lc][q] = f32x4{acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]};
  }
  __syncthreads();
  if (share > 0 || !on) return;
#pragma unroll
  for (int s = 0; s < 3; ++s)
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] += red[s][lc][i / 4][i % 4];
  embed_row(dW, (int64_t)cur * d + c, acc, scale, accum);
}

void launch_embed_bwd(const moe_embed_cfg& c, const int32_t* ids, const void* dy, void* dW, void* ws, hipStream_t s) {
  const int esz = c.dtype == MOE_BF16 ? 2 : 4;
  const int64_t zeros = c.accum ? 0 : (int64_t)c.V * c.d_model * esz / 16;
  const unsigned zblocks = zeros ? (unsigned)std::min<int64_t>(512, (zeros + 1023) / 1024) : 0;   // of 256 threads
  u32x4* z = (u32x4*)dW;
  if (c.T == 0) {
    if (zeros)
      launch_kernel(embed_pairs_kernel, dim3(zblocks), dim3(256), 0, s, ids, 0, c.V, 0, nullptr, nullptr, z, zeros);
    return;
  }
  const EmbedPlan p = embed_plan(c);
  char* w = (char*)ws;
  int32_t* counts = (int32_t*)(w + p.counts);
  int32_t *key = (int32_t*)(w + p.key[0]), *tok = (int32_t*)(w + p.tok[0]);
  auto radix = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    const int launches = 2 * p.passes, D = 1 << p.bits;
    const unsigned grid = (unsigned)p.tiles + (zblocks * 256 + NT - 1) / NT;
    auto za = [&](int i) { return zeros * i / launches; };
    for (int q = 0; q < p.passes; ++q) {
      const Digit dg{ids, q ? key : nullptr, c.V, q * p.bits, D - 1};
      const int32_t* from = q ? tok : nullptr;
      key = (int32_t*)(w + p.key[q & 1]);
      tok = (int32_t*)(w + p.tok[q & 1]);
      launch_kernel(embed_count_kernel<NT>, dim3(grid), dim3(NT), 0, s, dg, c.T, D, counts, p.tiles, z, za(2 * q),
                    za(2 * q + 1));
      launch_sort_scan(counts, p.tiles, D, s);
      launch_kernel(embed_place_kernel<NT>, dim3(grid), dim3(NT), 0, s, dg, from, c.T, D, counts, p.tiles, key, tok, z,
                    za(2 * q + 1), za(2 * q + 2));
    }
  };
  if (c.T <= kPairs) {
    const int blocks = (int)((c.T + 63) / 64), lds = (int)((c.T + 255) / 256 * 256 * 4);
    static std::atomic<uint64_t> lds_ok{0};
    allow_dyn_lds((const void*)embed_pairs_kernel, kPairs * 4, lds_ok);
    launch_kernel(embed_pairs_kernel, dim3(blocks + zblocks), dim3(256), lds, s, ids, (int)c.T, c.V, blocks, key, tok, z,
                  zeros);
  } else if (sort_threads(c.T) == kSortSmall) {
    radix(std::integral_constant<int, kSortSmall>{});
  } else {
    radix(std::integral_constant<int, kSortLarge>{});
  }
  auto go = [&](auto tag) {
    using T = decltype(tag);
    const int nc = c.d_model / Vec<T>::N, slabs = (nc + kJoinCols - 1) / kJoinCols;
    each_launch(p.runs, nc, [&](int64_t r0, int64_t n) {
      launch_kernel(embed_runs_kernel<T>, dim3((unsigned)((n * nc + 255) / 256)), dim3(256), 0, s, key, tok, (const T*)dy,
                    (T*)dW, (float*)(w + p.part), c.T, r0, r0 + n, c.V, c.d_model, c.scale, c.accum);
    });
    each_launch(p.runs - 1, (int64_t)slabs * 4 * kJoinCols, [&](int64_t r0, int64_t n) {
      launch_kernel(embed_join_kernel<T>, dim3((unsigned)(n * slabs)), dim3(4 * kJoinCols), 0, s, key, (T*)dW,
                    (const float*)(w + p.part), c.T, r0, p.runs, c.V, c.d_model, slabs, c.scale, c.accum);
    });
  };
  if (c.dtype == MOE_BF16) go(uint16_t{});
  else go(float{});
}

}  // namespace lmoe
