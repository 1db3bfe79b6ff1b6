// The experts' FFNs on 4-bit weights, from one token on, and the weights' quantiser.
//
// y_t = sum_r w_tr W2_e act(W1_e x_t).  With n = T k choices, two products over the
// chosen experts (act(W1 x) of every choice goes through the workspace) and a sum over
// a token's choices.  The weights are read once and bound the time; 16 output rows x
// 128 inputs of them are one 16-byte load a lane, which v_cvt_scalef32_pk_bf16_fp4
// turns into bfloat16 exactly, scale included (eight codes in four instructions), for
// v_mfma_f32_16x16x32_bf16 against up to 16 tokens.
//
// A matrix instruction wants lane (i = lane & 15, q = lane >> 4) to hold row i, and 16
// rows are 16 cache lines: loads straight into that order are bound by the L1's line
// look-ups (64 per load; measured, 48 tokens against 16 experts of 1024 x 4096: 19 + 26
// us where 36 + 36 MB take 14, and the two products take 12.5 + 13.7 now).  So a wave loads
// 8 rows x 256 inputs at a time, whole 128-byte lines, and turns them in LDS.  Of a row's
// 256 inputs lane q gets 32 q .. 32 q + 31 of each half, one scale group; MFMA j of a half takes inputs 8 j .. 8 j + 7
// of these from weights and tokens alike, so the product's k-index stands for the same
// input in both operands, which is all a dot product needs.
#include <type_traits>

#include "internal.h"

namespace lmoe {

// Up to so many choices a block finds its expert's tokens by itself, past that a launch sorts
// them (whole calls, us, by itself and sorted: 64 experts of 1024 x 2048, 400 choices 48.5 and
// 52.8, 640 62.7 and 66.9, 1000 78.6 and 76.0; 16 of 736 x 512, 720 29.3 and 28.6, 1000 37.6
// and 29.5: the tiles of an expert with many tokens are then blocks of their own).
constexpr int kW4Scan = 640;
constexpr int kW4Tile = 16;        // tokens of one pass over the weights: a matrix instruction's columns
constexpr int kW4ListThreads = 1024;
constexpr int kW4Splits = 4;       // of the second product's K, at most
constexpr int kMaxGridY = 65535;
// Waves of a block that splits K over waves, at most; and of a SIMD, by registers: 168, which
// the three parts of float inputs with 32 rows spill out of (20-100 bytes a lane), the rest not.
constexpr int kW4Waves = 8, kW4PerSimd = 3;

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

// -------------------------------------------------------------------- choices
// More than kW4Scan choices: their numbers sorted by expert (the order inside an
// expert is left to the atomics: rows do not mix, so it changes no value) and the
// table of token tiles {expert, first, count}.
struct W4Tile {
  int32_t e, first, count, pad;
};
__global__ __launch_bounds__(kW4ListThreads) void w4_list_kernel(const int32_t* __restrict__ idx, int n, int E,
                                                                 int32_t* __restrict__ list,
                                                                 W4Tile* __restrict__ tiles,
                                                                 int32_t* __restrict__ ntiles) {
  __shared__ int32_t cnt[kRouterMaxE], at[kRouterMaxE], sum[2][kRouterMaxE];
  const int tid = threadIdx.x;
  for (int e = tid; e < kRouterMaxE; e += kW4ListThreads) cnt[e] = 0;
  __syncthreads();
  for (int i = tid; i < n; i += kW4ListThreads) {
    const int e = idx[i];
    if (e >= 0 && e < E) atomicAdd(&cnt[e], 1);
  }
  __syncthreads();
  // exclusive sums of the counts and of the tiles
  if (tid < kRouterMaxE) {
    sum[0][tid] = cnt[tid];
    sum[1][tid] = (cnt[tid] + kW4Tile - 1) / kW4Tile;
  }
  __syncthreads();
  for (int o = 1; o < kRouterMaxE; o <<= 1) {
    int a = 0, b = 0;
    if (tid < kRouterMaxE && tid >= o) {
      a = sum[0][tid - o];
      b = sum[1][tid - o];
    }
    __syncthreads();
    if (tid < kRouterMaxE) {
      sum[0][tid] += a;
      sum[1][tid] += b;
    }
    __syncthreads();
  }
  if (tid < kRouterMaxE) {
    const int c = cnt[tid], nt = (c + kW4Tile - 1) / kW4Tile;
    const int first = sum[0][tid] - c, t0 = sum[1][tid] - nt;
    at[tid] = first;
    for (int j = 0; j < nt; ++j) tiles[t0 + j] = W4Tile{tid, first + j * kW4Tile, min(kW4Tile, c - j * kW4Tile), 0};
    if (tid == kRouterMaxE - 1) *ntiles = sum[1][tid];
  }
  __syncthreads();
  for (int i = tid; i < n; i += kW4ListThreads) {
    const int e = idx[i];
    if (e >= 0 && e < E) list[atomicAdd(&at[e], 1)] = i;
  }
}

// ------------------------------------------------------------------- products
struct W4Args {
  const uint8_t *codes, *scales;   // [E][N][K/2], [E][N][K/32]
  const void* in;                  // rows of K: x by token, or the parts of act(W1 x) by choice
  void* out;                       // FIRST: the parts [parts][n][N] bf16; else float [splits][n][N]
  const int32_t *idx, *list;
  const W4Tile* tiles;             // null: the blocks find their tokens
  const int32_t* ntiles;
  int32_t N, K, n, k, E, act;
  int32_t by_choice;               // blockIdx.y is a choice, not an expert (fewer choices than experts)
  int32_t steps;                   // steps of 256 inputs of one split (blocks of 128 rows)
  int32_t tile0;                   // the tile of blockIdx.y 0
};

// Eight codes to bfloat16.
__device__ __forceinline__ bf16x8 w4_frag(uint32_t c, float s) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
  return __builtin_bit_cast(bf16x8, r);
}

// A float's leading eight significand bits (truncated: never past the largest
// bfloat16), and what is left of it; of an infinity nothing is left (what is left of a
// finite value or NaN is none).
template <bool FINITE = false>
__device__ __forceinline__ float part_of(float& v) {
  const float h = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
  v = !FINITE && h == v ? 0.f : v - h;
  return h;
}

// The 16-byte pieces that eight inputs of a token come from, and their NS bfloat16 parts.
template <typename T, int NS, bool FIRST> struct W4In {
  static constexpr int NP = FIRST && sizeof(T) == 4 ? 2 : NS;
  u32x4 raw[NP];
  __device__ __forceinline__ void load(const W4Args& a, int64_t off) {
    if constexpr (FIRST && sizeof(T) == 4) {
      const u32x4* p = reinterpret_cast<const u32x4*>((const float*)a.in + off);
      raw[0] = p[0];
      raw[1] = p[1];
    } else {
#pragma unroll
      for (int s = 0; s < NS; ++s)
        raw[s] = *reinterpret_cast<const u32x4*>((const uint16_t*)a.in + (int64_t)s * a.n * a.K + off);
    }
  }
  __device__ __forceinline__ void parts(bf16x8 (&b)[NS]) const {
    if constexpr (FIRST && sizeof(T) == 4) {
      u32x4 r[NS];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float lo = __uint_as_float(raw[i >> 1][(2 * i) & 3]), hi = __uint_as_float(raw[i >> 1][(2 * i + 1) & 3]);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          const float l = s == 0 ? part_of(lo) : part_of<true>(lo), h = s == 0 ? part_of(hi) : part_of<true>(hi);
          r[s][i] = (__float_as_uint(l) >> 16) | __float_as_uint(h);
        }
      }
#pragma unroll
      for (int s = 0; s < NS; ++s) b[s] = __builtin_bit_cast(bf16x8, r[s]);
    } else {
#pragma unroll
      for (int s = 0; s < NS; ++s) b[s] = __builtin_bit_cast(bf16x8, raw[s]);
    }
  }
};

// The weights of 16 RT rows x 256 inputs (a step), on their way: lane l has 16-byte piece
// l % 8 of row l / 8 of every eight rows, and the scales of row l (l < 16 RT).
// Where K is no multiple of a step the scales' rows have any alignment: lane l then has
// byte l % 8 of row l / 8 of every eight rows (past K the row's last).
constexpr int kStep = 256;
template <int RT, bool FULL> struct W4Scales {
  u32x2 v;
  __device__ __forceinline__ void load(const uint8_t* scales, int K, int col) {
    const int lane = threadIdx.x & 63;
    v = *reinterpret_cast<const u32x2*>(scales + (int64_t)(lane & (16 * RT - 1)) * (K / 32) + col / 32);
  }
  __device__ __forceinline__ void store(u32x2* rows) const {
    const int lane = threadIdx.x & 63;
    if (lane < 16 * RT) rows[lane] = v;
  }
};
template <int RT> struct W4Scales<RT, false> {
  uint8_t v[2 * RT];
  __device__ __forceinline__ void load(const uint8_t* scales, int K, int col) {
    const int lane = threadIdx.x & 63;
    const uint8_t* p = scales + (int64_t)(lane >> 3) * (K / 32) + min(col / 32 + (lane & 7), K / 32 - 1);
#pragma unroll
    for (int i = 0; i < 2 * RT; ++i) v[i] = p[(int64_t)8 * i * (K / 32)];
  }
  __device__ __forceinline__ void store(u32x2* rows) const {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < 2 * RT; ++i) ((uint8_t*)rows)[64 * i + lane] = v[i];
  }
};
template <int RT, bool FULL> struct W4Step {
  u32x4 code[2 * RT];
  W4Scales<RT, FULL> sc;
  // codes, scales: at the first of the rows; col: the step's first input.
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, int K, int col) {
    const int lane = threadIdx.x & 63;
    const int at = col + (lane & 7) * 32;
    const bool ok = FULL || at < K;   // (K is a multiple of 32)
#pragma unroll
    for (int g = 0; g < 2 * RT; ++g) {
      const u32x4 v = __builtin_nontemporal_load(
          reinterpret_cast<const u32x4*>(codes + (int64_t)(8 * g + (lane >> 3)) * (K / 2) + (ok ? at : col) / 2));
      code[g] = ok ? v : u32x4{0u, 0u, 0u, 0u};
    }
    sc.load(scales, K, col);
  }
};
template <int RT> struct W4Lds {   // a wave's step, turned
  u32x4 code[RT][16][8];           // [row][piece ^ row % 8]: neither side meets a bank conflict
  u32x2 sc[RT][16];
};

// (one activation's code for four values, not four switches: it is most of the kernel's)
__device__ __forceinline__ void w4_act(float (&h)[4], int act) {
  auto all = [&](auto kind) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = act_fwd_nan(h[i], decltype(kind)::value);
  };
  if (act == MOE_ACT_RELU) all(std::integral_constant<int, MOE_ACT_RELU>{});
  else if (act == MOE_ACT_GELU_TANH) all(std::integral_constant<int, MOE_ACT_GELU_TANH>{});
  else if (act == MOE_ACT_GELU_ERF) all(std::integral_constant<int, MOE_ACT_GELU_ERF>{});
}

__device__ __forceinline__ void w4_wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Rows row .. row + 3 of a choice's product: act of it in parts, or itself.
template <bool FIRST, int NO>
__device__ __forceinline__ void w4_out(const W4Args& a, int choice, int row, f32x4 s) {
  const int64_t off = (int64_t)choice * a.N + row;
  if constexpr (FIRST) {
    float h[4] = {s[0], s[1], s[2], s[3]};
    w4_act(h, a.act);
#pragma unroll
    for (int p = 0; p < NO; ++p) {
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = p + 1 < NO || NO == 3 ? part_of(h[i]) : h[i];   // two parts: the second rounds
      *reinterpret_cast<u32x2*>((uint16_t*)a.out + (int64_t)p * a.n * a.N + off) =
          u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
  } else {
    *reinterpret_cast<f32x4*>((float*)a.out + (int64_t)blockIdx.z * a.n * a.N + off) = s;
  }
}

// Tokens list[0 .. cnt) of one expert, 16 at most, against the block's 16 RT rows; the
// block's waves split K into interleaved steps (w: the wave's first, on its way).
template <typename T, bool FIRST, int NS, int NO, int RT, bool FULL>
__device__ __forceinline__ void w4_tile(const W4Args& a, int waves, int cnt, const int32_t* list, const uint8_t* codes,
                                        const uint8_t* scales, W4Step<RT, FULL>& w, W4Lds<RT>* lds) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int i16 = lane & 15, q = lane >> 4;
  const int row0 = blockIdx.x * 16 * RT;
  W4Lds<RT>& mine = lds[wv];
  f32x4 acc[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int choice = list[min(i16, cnt - 1)];   // columns past the count repeat the last
  const int64_t in_off = (int64_t)(FIRST ? choice / a.k : choice) * a.K;
  for (int col = wv * kStep; col < a.K; col += waves * kStep) {
    w4_wave_fence();
#pragma unroll
    for (int g = 0; g < 2 * RT; ++g) mine.code[g >> 1][8 * (g & 1) + (lane >> 3)][(lane & 7) ^ (lane >> 3)] = w.code[g];
    w.sc.store(&mine.sc[0][0]);
    w4_wave_fence();
    // The inputs are asked for ahead of the next weights: loads return in order, and a
    // wait for inputs behind them would be a wait for memory.
    W4In<T, NS, FIRST> in[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = col + 128 * h + 32 * q;
#pragma unroll
      for (int j = 0; j < 4; ++j) in[h][j].load(a, in_off + (FULL || at < a.K ? at : col) + 8 * j);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (col + waves * kStep < a.K) w.load(codes, scales, a.K, col + waves * kStep);
    __builtin_amdgcn_sched_barrier(0);
    u32x2 sc[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) sc[r] = mine.sc[r][i16];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool ok = FULL || col + 128 * h + 32 * q < a.K;
      u32x4 code[RT];
      float s[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        code[r] = mine.code[r][i16][(4 * h + q) ^ (i16 & 7)];
        s[r] = __uint_as_float(((sc[r][h] >> (8 * q)) & 0xffu) << 23);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8 b[NS];
        in[h][j].parts(b);
        if (!FULL)   // (weights past K are zeros, but the inputs read in their place may be infinite)
#pragma unroll
          for (int x = 0; x < NS; ++x)
            b[x] = __builtin_bit_cast(bf16x8, ok ? __builtin_bit_cast(u32x4, b[x]) : u32x4{0u, 0u, 0u, 0u});
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const bf16x8 f = w4_frag(code[r][j], s[r]);
#pragma unroll
          for (int x = NS - 1; x >= 0; --x) acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, b[x], acc[r], 0, 0, 0);
        }
      }
    }
  }
  // The waves' sums meet in LDS and are added in wave order, every wave its rows.
  f32x4 (*red)[64] = reinterpret_cast<f32x4(*)[64]>(lds);
  static_assert(sizeof(f32x4) * 64 * RT <= sizeof(W4Lds<RT>), "");
  __syncthreads();
#pragma unroll
  for (int r = 0; r < RT; ++r) red[wv * RT + r][lane] = acc[r];
  __syncthreads();
  if (wv < RT && i16 < cnt) {
    f32x4 v[kW4Waves];
#pragma unroll
    for (int x = 0; x < kW4Waves; ++x) v[x] = red[min(x, waves - 1) * RT + wv][lane];
    f32x4 s = v[0];
#pragma unroll
    for (int x = 1; x < kW4Waves; ++x) s = x < waves ? s + v[x] : s;
    w4_out<FIRST, NO>(a, choice, row0 + wv * 16 + 4 * q, s);
  }
}

// How a block finds its expert and tokens (blockIdx.y): by the list's tiles; every wave by
// itself in up to 64 choices (a choice, if it is the first of its expert, or an expert); or the
// block in up to kW4Scan: by expert, or by choice.  (Whole calls, us.  By wave and by block:
// one token, top-2 of 16 experts of 1024 x 4096 13.0 and 13.9, 32 tokens 29.4 and 29.1.  By
// choice and by expert: the one token 13.0 and 19.8; top-6 of 160 experts of 1536 x 768, 11
// tokens 32.2 and 36.9, 20 tokens 46.2 both.)
enum { kFindTiles, kFindWave, kFindExpert, kFindChoice };
// list and their number (0: none, or another block has them).  first() runs as soon as the
// expert is known.  Four or eight waves; every one ends with the same answer.
struct W4Found {
  int e, cnt;
  const int32_t* list;
};
template <int HOW, typename F>
__device__ __forceinline__ W4Found w4_find(const W4Args& a, int waves, int32_t (&lists)[kW4Scan], int32_t& found, F first) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  W4Found r{-1, 0, lists};
  if constexpr (HOW == kFindTiles) {
    const int tile = a.tile0 + blockIdx.y;
    if (tile >= *a.ntiles) return r;
    const W4Tile t = a.tiles[tile];
    r.e = t.e;
    first(r.e);
    if ((int)threadIdx.x < t.count) lists[threadIdx.x] = a.list[t.first + threadIdx.x];
    __syncthreads();
    r.cnt = t.count;
  } else if constexpr (HOW == kFindWave) {
    const int my = lane < a.n ? a.idx[lane] : -1;
    r.e = a.by_choice ? __builtin_amdgcn_readlane(my, (int)blockIdx.y) : (int)blockIdx.y;
    if (r.e < 0 || r.e >= a.E) return r;
    const uint64_t same = __ballot(my == r.e);
    if (same == 0 || (a.by_choice && __builtin_ctzll(same) != (int)blockIdx.y)) return r;
    first(r.e);
    int32_t* mine = lists + wv * kWave;
    if (my == r.e) mine[__popcll(same & ((1ull << lane) - 1))] = lane;
    r.list = mine;
    w4_wave_fence();
    r.cnt = __popcll(same);
  } else {
    // The expert's choices, in any order (rows do not mix).  By expert most have some, and
    // the weights are asked for right behind the choices, not behind the answer.
    constexpr int NI = (kW4Scan + 255) / 256;
    int at[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) at[i] = a.idx[min((int)threadIdx.x + 64 * waves * i, a.n - 1)];
    r.e = HOW == kFindChoice ? a.idx[blockIdx.y] : (int)blockIdx.y;
    if (HOW == kFindChoice && (r.e < 0 || r.e >= a.E)) return r;
    if constexpr (HOW == kFindExpert) {
      __builtin_amdgcn_sched_barrier(0);
      first(r.e);
    }
    if (threadIdx.x == 0) found = 0;
    __syncthreads();
    bool earlier = false;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int c = threadIdx.x + 64 * waves * i;
      if (c < a.n && at[i] == r.e) {
        lists[atomicAdd(&found, 1)] = c;
        earlier |= c < (int)blockIdx.y;
      }
    }
    if constexpr (HOW == kFindChoice) {   // the first choice of an expert stands for all of them
      if (__syncthreads_or(earlier)) return r;
      first(r.e);
    } else {
      __syncthreads();
    }
    r.cnt = found;
  }
  return r;
}

template <typename T, bool FIRST, int NS, int NO, int RT, bool FULL, int HOW>
__global__ __launch_bounds__(64 * kW4Waves, kW4PerSimd) void w4_product_kernel(W4Args a) {
  extern __shared__ __attribute__((aligned(16))) char w4_lds[];
  W4Lds<RT>* lds = reinterpret_cast<W4Lds<RT>*>(w4_lds);   // one a wave
  __shared__ int32_t found, lists[kW4Scan];
  const int wv = threadIdx.x >> 6, waves = blockDim.x >> 6;
  W4Step<RT, FULL> w;
  const uint8_t *codes = nullptr, *scales = nullptr;
  auto weights = [&](int e) __attribute__((always_inline)) {   // the wave's first step
    const int64_t row = (int64_t)e * a.N + blockIdx.x * 16 * RT;
    codes = a.codes + row * (a.K / 2);
    scales = a.scales + row * (a.K / 32);
    if (wv * kStep < a.K) w.load(codes, scales, a.K, wv * kStep);
  };
  const W4Found f = w4_find<HOW>(a, waves, lists, found, weights);
  for (int c0 = 0; c0 < f.cnt; c0 += kW4Tile) {
    if (c0) {
      weights(f.e);
      __syncthreads();   // the sums of the tile before have been read
    }
    w4_tile<T, FIRST, NS, NO, RT, FULL>(a, waves, min(kW4Tile, f.cnt - c0), f.list + c0, codes, scales, w, lds);
  }
}

// ------------------------------------------------------------- blocks of 128 rows
// Where there are blocks enough, four waves take 32 rows each over the whole K (of
// blockIdx.z's split), and the tokens' inputs go through LDS once for all of them: with K
// split over the waves every 16 or 32 rows fetched them anew, four times the weights' bytes.
// Bound by the latency of a block's steps: 48 tokens, 16 experts of 1024 x 4096, 12.5 and
// 13.7 us for 36 MB each, and still 10-11 with everything in cache.  (Blocks of 64 rows,
// twice as many: 12.0 for the first product, 17.0 for the second, whose inputs are two parts.
// Three steps on their way instead of one: 14.2 and 18.3; the registers, and the loads after
// the last step, cost more than they hide.)
template <typename T, bool FIRST, int NS, int NO, bool FULL, int HOW>
__global__ __launch_bounds__(256, NS == 3 ? 1 : 2) void w4_rows_kernel(W4Args a) {
  constexpr int RT = 2, WR = 16 * RT, BR = 4 * WR;   // rows of a wave, of the block
  __shared__ u32x4 wcode[2][BR][8];        // [row][piece ^ row % 8]
  __shared__ u32x2 wsc[2][BR];
  __shared__ u32x4 tok[2][NS][16][32];             // [part][token][piece ^ token % 8]
  __shared__ int32_t found, lists[kW4Scan];
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, q = lane >> 4;
  const int row0 = blockIdx.x * BR;
  const bool on = row0 + WR * wv < a.N;            // (N is a multiple of 32)
  const int k0 = blockIdx.z * a.steps * kStep;
  const int k1 = min(a.K, k0 + a.steps * kStep);
  const uint8_t *codes = nullptr, *scales = nullptr;
  u32x4 wreg[2 * RT];
  W4Scales<RT, FULL> sreg;
  auto load_w = [&](int col) __attribute__((always_inline)) {
    const int at = col + (lane & 7) * 32;
    const bool ok = FULL || at < k1;
#pragma unroll
    for (int i = 0; i < 2 * RT; ++i) {
      const u32x4 v = __builtin_nontemporal_load(
          reinterpret_cast<const u32x4*>(codes + (int64_t)(8 * i + (lane >> 3)) * (a.K / 2) + (ok ? at : col) / 2));
      wreg[i] = ok ? v : u32x4{0u, 0u, 0u, 0u};
    }
    sreg.load(scales, a.K, col);
  };
  auto first = [&](int e) __attribute__((always_inline)) {   // the wave's rows
    const int64_t row = (int64_t)e * a.N + (on ? row0 + WR * wv : 0);
    codes = a.codes + row * (a.K / 2);
    scales = a.scales + row * (a.K / 32);
    load_w(k0);
  };
  const W4Found fnd = w4_find<HOW>(a, 4, lists, found, first);
  for (int c0 = 0; c0 < fnd.cnt; c0 += kW4Tile) {
    const int cnt = min(kW4Tile, fnd.cnt - c0);
    const int32_t* list = fnd.list + c0;
    if (c0) load_w(k0);
    // Thread: inputs 8 (tid % 32) .. of tokens tid / 32 and 8 + tid / 32.
    int64_t src[2];
    bool has[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = 8 * i + (tid >> 5);
      has[i] = t < cnt;
      const int choice = list[has[i] ? t : 0];
      src[i] = (int64_t)(FIRST ? choice / a.k : choice) * a.K;
    }
    W4In<T, NS, FIRST> in[2];
    auto load_t = [&](int col) __attribute__((always_inline)) {
      const int at = col + 8 * (tid & 31);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (has[i]) in[i].load(a, src[i] + (FULL || at < k1 ? at : col));
    };
    auto store = [&](int b, int col) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 2 * RT; ++i) wcode[b][WR * wv + 8 * i + (lane >> 3)][(lane & 7) ^ (lane >> 3)] = wreg[i];
      sreg.store(&wsc[b][WR * wv]);
      const bool ok = FULL || col + 8 * (tid & 31) < k1;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (has[i]) {
          bf16x8 p[NS];
          in[i].parts(p);
          const int t = 8 * i + (tid >> 5);
#pragma unroll
          for (int x = 0; x < NS; ++x)   // (weights past K are zeros, but the inputs read in their place may be infinite)
            tok[b][x][t][(tid & 31) ^ (t & 7)] = ok ? __builtin_bit_cast(u32x4, p[x]) : u32x4{0u, 0u, 0u, 0u};
        }
    };
    f32x4 acc[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[r] = f32x4{0.f, 0.f, 0.f, 0.f};
    load_t(k0);
    if (c0) __syncthreads();   // the tile before has been read
    store(0, k0);
    __syncthreads();
    int b = 0;
    for (int col = k0; col < k1; col += kStep, b ^= 1) {
      // (After the last step the loads ask for what is there already: a branch around a load
      // has its results copied, and so waited for, right behind it.)
      const int after = col + kStep < k1 ? col + kStep : col;
      load_t(after);
      load_w(after);
      __builtin_amdgcn_sched_barrier(0);
      u32x2 sc[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) sc[r] = wsc[b][WR * wv + 16 * r + i16];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (!FULL && col + 128 * h >= k1) break;
        u32x4 code[RT];
        float s[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          code[r] = wcode[b][WR * wv + 16 * r + i16][(4 * h + q) ^ (i16 & 7)];
          s[r] = __uint_as_float(((sc[r][h] >> (8 * q)) & 0xffu) << 23);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          bf16x8 t[NS];
#pragma unroll
          for (int x = 0; x < NS; ++x) t[x] = __builtin_bit_cast(bf16x8, tok[b][x][i16][(16 * h + 4 * q + j) ^ (i16 & 7)]);
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            const bf16x8 f = w4_frag(code[r][j], s[r]);
#pragma unroll
            for (int x = NS - 1; x >= 0; --x) acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, t[x], acc[r], 0, 0, 0);
          }
        }
      }
      store(b ^ 1, after);
      __syncthreads();
    }
    if (on && i16 < cnt) {
      const int choice = list[i16];
#pragma unroll
      for (int r = 0; r < RT; ++r) w4_out<FIRST, NO>(a, choice, row0 + WR * wv + 16 * r + 4 * q, acc[r]);
    }
  }
}

// Thread: four columns of a token (blockIdx.y; further ones past the grid's limit).  NR
// choices at a time, every load of them and of their SP splits ahead of the sums: with few
// tokens the kernel is the latency of its loads (512 tokens, top-2, four splits: 6.8 us;
// four choices at a time and the splits one by one 7.9).
template <typename T, int SP, int NR>
__global__ __launch_bounds__(256) void w4_combine_kernel(const float* __restrict__ O, const int32_t* __restrict__ idx,
                                                         const float* __restrict__ w, T* __restrict__ y, int64_t T_tokens,
                                                         int d, int E, int k) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= d) return;
  for (int64_t t = blockIdx.y; t < T_tokens; t += gridDim.y) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    for (int r0 = 0; r0 < k; r0 += NR) {
      int e[NR];
      float wr[NR];
      f32x4 o[NR][SP];
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const int64_t i = t * k + min(r0 + r, k - 1);
        e[r] = idx[i];
        wr[r] = w[i];
#pragma unroll
        for (int z = 0; z < SP; ++z) o[r][z] = *reinterpret_cast<const f32x4*>(O + (z * T_tokens * k + i) * d + c);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int r = 0; r < NR; ++r) {
#pragma unroll
        for (int z = 1; z < SP; ++z) o[r][0] += o[r][z];
        if (r0 + r < k && e[r] >= 0 && e[r] < E)   // (of another choice O and w may hold anything)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[i] = fmaf(wr[r], o[r][0][i], s[i]);
      }
    }
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<u32x2*>(y + t * d + c) = u32x2{pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3])};
    else
      *reinterpret_cast<f32x4*>(y + t * d + c) = s;
  }
}
template <typename T>
static void launch_w4_combine(const moe_w4_cfg& c, const float* O, const int32_t* idx, const float* w, void* y, int splits,
                              hipStream_t s) {
  const dim3 grid((c.d_model + 1023) / 1024, (unsigned)std::min<int64_t>(c.T, 32768));
  auto go = [&](auto kern) { launch_kernel(kern, grid, dim3(256), 0, s, O, idx, w, (T*)y, c.T, c.d_model, c.E, c.k); };
  auto choices = [&](auto sp) {
    constexpr int SP = decltype(sp)::value;
    if (c.k <= 2) go(w4_combine_kernel<T, SP, 2>);
    else if (c.k <= 4) go(w4_combine_kernel<T, SP, 4>);
    else go(w4_combine_kernel<T, SP, 8>);
  };
  static_assert(kW4Splits == 4, "a case for each");
  if (splits == 1) choices(std::integral_constant<int, 1>{});
  else if (splits == 2) choices(std::integral_constant<int, 2>{});
  else if (splits == 3) choices(std::integral_constant<int, 3>{});
  else choices(std::integral_constant<int, 4>{});
}

// ------------------------------------------------------------------ many tokens
// bfloat16, two dozen tokens an expert and more: the products are matrix products
// again.  The tokens' rows are laid out by expert, padded to 16, in the order in which the
// matrix instructions take them (x by w4_pack_kernel, act(W1 x) by the first product), so
// both sides of a 128-row x 160-token block go through LDS in whole lines: the codes of 256
// inputs, the tokens' values of 64, each with the next on its way.  Four waves, 64 rows by
// half the tokens each.  512 tokens, top-2 of 8 experts of 2048 x 8192: 51 and 52 us for 34
// GFLOP each, bound by what stands beside the matrix instructions (a code conversion for
// every four of them, both sides' LDS reads) with one round of two blocks a CU.
// The tokens' rows are padded to whole 128s with zeros; rows and inputs past the matrix are
// read inside it (WHOLE: there are none), such codes taken as zeros and such rows written as
// zeros, which the second product meets as its inputs' padding.
// act(W1 x) is rounded once to bfloat16 here, as moe_expert_ffn_fwd does: a second part
// would double the second product, which is no longer hidden behind the weights.
constexpr int kGemmRows = 128, kGemmToks = 160, kGemmT = kGemmToks / 32;   // kGemmT: 16-token tiles of a wave
struct W4Group {   // where an expert's rows are
  int32_t e, row, rows, pad;   // first padded row of a token tile, its rows (a multiple of 16)
};

// choice_of[row] (-1: padding), the token tiles and their number; an expert's tiles are
// alike in size.
__global__ __launch_bounds__(kW4ListThreads) void w4_group_kernel(const int32_t* __restrict__ idx, int n, int E,
                                                                  int32_t* __restrict__ choice_of,
                                                                  W4Group* __restrict__ tiles,
                                                                  int32_t* __restrict__ ntiles, int max_rows) {
  __shared__ int32_t cnt[kRouterMaxE], at[kRouterMaxE], sum[2][kRouterMaxE];
  const int tid = threadIdx.x;
  for (int e = tid; e < kRouterMaxE; e += kW4ListThreads) cnt[e] = 0;
  for (int i = tid; i < max_rows; i += kW4ListThreads) choice_of[i] = -1;
  __syncthreads();
  for (int i = tid; i < n; i += kW4ListThreads) {
    const int e = idx[i];
    if (e >= 0 && e < E) atomicAdd(&cnt[e], 1);
  }
  __syncthreads();
  if (tid < kRouterMaxE) {
    sum[0][tid] = (cnt[tid] + 15) / 16;
    sum[1][tid] = (cnt[tid] + kGemmToks - 1) / kGemmToks;
  }
  __syncthreads();
  for (int o = 1; o < kRouterMaxE; o <<= 1) {
    int a = 0, b = 0;
    if (tid < kRouterMaxE && tid >= o) {
      a = sum[0][tid - o];
      b = sum[1][tid - o];
    }
    __syncthreads();
    if (tid < kRouterMaxE) {
      sum[0][tid] += a;
      sum[1][tid] += b;
    }
    __syncthreads();
  }
  if (tid < kRouterMaxE) {
    const int t16 = (cnt[tid] + 15) / 16, nt = (cnt[tid] + kGemmToks - 1) / kGemmToks;
    const int first = 16 * (sum[0][tid] - t16), t0 = sum[1][tid] - nt;
    at[tid] = first;
    const int each = nt ? (t16 + nt - 1) / nt : 0;   // 16-row tiles of a token tile
    for (int j = 0; j < nt; ++j) tiles[t0 + j] = W4Group{tid, first + 16 * j * each, 16 * max(0, min(each, t16 - j * each)), 0};
    if (tid == kRouterMaxE - 1) *ntiles = sum[1][tid];
  }
  __syncthreads();
  for (int i = tid; i < n; i += kW4ListThreads) {
    const int e = idx[i];
    if (e >= 0 && e < E) choice_of[atomicAdd(&at[e], 1)] = i;
  }
}

static int w4_pad(int x) { return (x + 127) / 128 * 128; }

// Element (row, input) of the laid-out tokens [row / 16][input / 128][j][lane][8]; K: padded.
__host__ __device__ __forceinline__ int64_t w4_tok_off(int64_t row, int in, int K) {
  return (((row >> 4) * (K >> 7) + (in >> 7)) * 4 + ((in & 31) >> 3)) * 512 + (((in >> 5) & 3) * 16 + (row & 15)) * 8 + (in & 7);
}

// One thread per 8 values, in the output's order.
__global__ __launch_bounds__(256) void w4_pack_kernel(const uint16_t* __restrict__ x, const int32_t* __restrict__ choice_of,
                                                      uint16_t* __restrict__ out, int K, int k, int64_t pieces) {
  for (int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x; p < pieces; p += (int64_t)gridDim.x * 256) {
    const int lane = (int)(p & 63), j = (int)(p >> 6) & 3;
    const int64_t chunk = p >> 8;
    const int nc = (K + 127) >> 7;
    const int64_t t16 = chunk / nc;
    const int c = (int)(chunk - t16 * nc);
    const int choice = choice_of[t16 * 16 + (lane & 15)];
    const int in = c * 128 + (lane >> 4) * 32 + 8 * j;
    u32x4 v = {0u, 0u, 0u, 0u};
    if (choice >= 0 && in < K) v = *reinterpret_cast<const u32x4*>(x + (int64_t)(choice / k) * K + in);
    *reinterpret_cast<u32x4*>(out + p * 8) = v;
  }
}

struct W4GemmArgs {
  const uint8_t *codes, *scales;
  const uint16_t* in;    // laid-out tokens of K values (padded to 128)
  void* out;             // FIRST: laid-out tokens of N values (padded to 128); else float [splits][n][N]
  const int32_t* choice_of;
  const W4Group* tiles;
  const int32_t* ntiles;
  int32_t N, K, n, act, steps;   // steps of 256 inputs of one split
};

// The activation of values that are then rounded to bfloat16.  (erf's code once, not at
// each of a lane's twenty places: unrolled it is most of the kernel.)
__device__ __noinline__ f32x4 w4_act_erf(f32x4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = act_fwd_t<MOE_ACT_GELU_ERF>(v[i]);
  return v;
}
__device__ __forceinline__ f32x4 w4_act_rounded(f32x4 v, int act) {
  if (act == MOE_ACT_GELU_ERF) return w4_act_erf(v);
  f32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float t = act_fwd_t<MOE_ACT_GELU_TANH>(v[i]);
    r[i] = act == MOE_ACT_GELU_TANH ? t : act == MOE_ACT_RELU && v[i] < 0.f ? 0.f : v[i];
  }
  return r;
}

template <bool FIRST, bool WHOLE>
__global__ __launch_bounds__(256, 2) void w4_gemm_kernel(W4GemmArgs a) {
  __shared__ u32x4 wcode[2][kGemmRows][8];     // [row][piece ^ row % 8]
  __shared__ uint32_t wsc[2][2][kGemmRows];    // [half][row]: four groups' bytes
  __shared__ u32x4 tok[2][2 * kGemmT][2][64];  // [16-token tile][j][lane]
  if ((int)blockIdx.y >= *a.ntiles) return;
  const W4Group g = a.tiles[blockIdx.y];
  if (g.rows == 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, q = lane >> 4;
  const int rg = wv & 1, tg = wv >> 1;
  const int row0 = blockIdx.x * kGemmRows;
  const int nt16 = g.rows >> 4;                                  // 16-token tiles of the block
  const int t0 = tg * ((nt16 + 1) / 2), mine = tg ? nt16 - t0 : (nt16 + 1) / 2;   // of the wave
  const int k0 = blockIdx.z * a.steps * kStep;
  const int Kp = WHOLE ? a.K : (a.K + 127) & ~127, Np = WHOLE ? a.N : (a.N + 127) & ~127;
  const int k1 = min(Kp, k0 + a.steps * kStep);
  if (k0 >= k1) return;   // (the launch leaves no split empty)
  const uint8_t* codes = a.codes + ((int64_t)g.e * a.N + row0) * (a.K / 2);
  const uint8_t* scales = a.scales + ((int64_t)g.e * a.N + row0) * (a.K / 32);
  const uint16_t* toks = a.in + (int64_t)(g.row >> 4) * Kp * 16;

  // (k1 is a multiple of 128.  A half step past k1 is not looked at, nor are tiles past
  // nt16: their loads are of something inside the arrays, and wait for no branch.)
  u32x4 wreg[4];
  uint32_t sreg[2];
  const int last_row = a.N - 1 - row0, groups = a.K / 32;
  auto load_w = [&](int col) __attribute__((always_inline)) {
    const int at = col + (lane & 7) * 32, in = at < k1 ? at : col;
    const bool ok = WHOLE || in < a.K;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 32 * wv + 8 * i + (lane >> 3);
      const u32x4 v = *reinterpret_cast<const u32x4*>(codes + (int64_t)(WHOLE ? row : min(row, last_row)) * (a.K / 2) +
                                                      (ok ? in : 0) / 2);
      wreg[i] = ok ? v : u32x4{0u, 0u, 0u, 0u};
    }
    if constexpr (WHOLE) {
      const uint8_t* p = scales + (int64_t)(tid & (kGemmRows - 1)) * groups;
      sreg[0] = *reinterpret_cast<const uint32_t*>(p + col / 32);
      sreg[1] = *reinterpret_cast<const uint32_t*>(p + (col + 128 < k1 ? col + 128 : col) / 32);
    } else {   // rows of any alignment: a half step of one row a thread (past K the row's last)
      const uint8_t* p = scales + (int64_t)min(tid & (kGemmRows - 1), last_row) * groups;
      const int g0 = (col + 128 * (tid / kGemmRows)) / 32;
      sreg[0] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) sreg[0] |= (uint32_t)p[min(g0 + i, groups - 1)] << (8 * i);
    }
  };
  auto store_w = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) wcode[b][32 * wv + 8 * i + (lane >> 3)][(lane & 7) ^ (lane >> 3)] = wreg[i];
    if constexpr (!WHOLE) {
      wsc[b][tid / kGemmRows][tid & (kGemmRows - 1)] = sreg[0];
    } else if (tid < kGemmRows) {
      wsc[b][0][tid] = sreg[0];
      wsc[b][1][tid] = sreg[1];
    }
  };
  // Values of 64 inputs: those of pair jp (j = 2 jp, 2 jp + 1) of the 128 from `col` on.
  u32x4 treg[kGemmT];
  auto load_t = [&](int col, int jp) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kGemmT; ++i) {
      const int f = wv + 4 * i, t = min(f >> 1, nt16 - 1), j = 2 * jp + (f & 1);   // every fourth fragment
      treg[i] = *reinterpret_cast<const u32x4*>(toks + (((int64_t)t * (Kp >> 7) + (col >> 7)) * 4 + j) * 512 + lane * 8);
    }
  };
  auto store_t = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kGemmT; ++i) tok[b][(wv + 4 * i) >> 1][wv & 1][lane] = treg[i];
  };

  f32x4 acc[4][kGemmT];
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int t = 0; t < kGemmT; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};

  load_w(k0);
  load_t(k0, 0);
  store_w(0);
  store_t(0);
  __syncthreads();
  int wb = 0;
  for (int col = k0; col < k1; col += kStep, wb ^= 1) {
    // (After the last step the loads ask for what is there already: a branch around a load
    // has its results copied, and so waited for, right behind it.)
    const bool two = col + 128 < k1;
    const int after = col + kStep < k1 ? col + kStep : col;
    u32x4 code[4];
    float sc[4];
    // 64 inputs: half h, pair jp.  (Straight code, no loop over the four: ahead of a loop
    // the compiler waits for the weights that are still on their way.)
    auto sub = [&](auto hc, auto jc) __attribute__((always_inline)) {
      constexpr int h = decltype(hc)::value, jp = decltype(jc)::value;
      if constexpr (jp == 0) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 64 * rg + 16 * r + i16;
          code[r] = wcode[wb][row][(4 * h + q) ^ (i16 & 7)];
          sc[r] = __uint_as_float(((wsc[wb][h][row] >> (8 * q)) & 0xffu) << 23);
        }
      }
      const bool last = jp == 1 && (h == 1 || !two);
      load_t(jp == 0 ? col + 128 * h : last ? after : col + 128, jp ^ 1);
      // loads return in order: the next weights behind these, not ahead of them
      if constexpr (h == 0 && jp == 0) load_w(after);
      __builtin_amdgcn_sched_barrier(0);
      // Both j's reads ahead of the products, which wait for the first j's only.  (An empty
      // asm uses the values where they are waited for: left alone the compiler moves each
      // read into the branch of its products, and every product waits for LDS.)
      u32x4 b[2][kGemmT];
#pragma unroll
      for (int jj = 0; jj < 2; ++jj)
#pragma unroll
        for (int t = 0; t < kGemmT; ++t) b[jj][t] = tok[jp][t0 + t][jj][lane];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
        bf16x8 f[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) f[r] = w4_frag(code[r][2 * jp + jj], sc[r]);
#pragma unroll
        for (int t = 0; t < kGemmT; ++t) asm volatile("" : "+v"(b[jj][t]));
#pragma unroll
        for (int t = 0; t < kGemmT; ++t)
          if (t < mine)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              acc[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[r], __builtin_bit_cast(bf16x8, b[jj][t]), acc[r][t], 0, 0, 0);
      }
      store_t(jp ^ 1);
      if (last) store_w(wb ^ 1);
      __syncthreads();
    };
    constexpr std::integral_constant<int, 0> c0;
    constexpr std::integral_constant<int, 1> c1;
    sub(c0, c0);
    sub(c0, c1);
    if (two) {
      sub(c1, c0);
      sub(c1, c1);
    }
  }
#pragma unroll
  for (int t = 0; t < kGemmT; ++t) {
    if (t >= mine) break;
    const int64_t row = g.row + 16 * (t0 + t) + i16;
    const int choice = FIRST ? 0 : a.choice_of[row];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int f = row0 + 64 * rg + 16 * r + 4 * q;
      if constexpr (FIRST) {   // (padding rows: act(0) = 0)
        const f32x4 h = w4_act_rounded(acc[r][t], a.act);
        const bool in = WHOLE || f < a.N;
        *reinterpret_cast<u32x2*>((uint16_t*)a.out + w4_tok_off(row, f, Np)) =
            u32x2{in ? pack_bf16x2(h[0], h[1]) : 0u, in ? pack_bf16x2(h[2], h[3]) : 0u};
      } else {
        if (choice >= 0 && (WHOLE || f < a.N))
          *reinterpret_cast<f32x4*>((float*)a.out + ((int64_t)blockIdx.z * a.n + choice) * a.N + f) = acc[r][t];
      }
    }
  }
}

// The laid-out form serves: bfloat16, tokens and work enough.  Its time hardly grows with the
// tokens, the other form's does with every 16 of an expert; but it has two launches more,
// and of few blocks' long chains if there are few rows.  Whole call, us, other form against
// this one.  By choices an expert: 16 experts of 1024 x 4096, 16: 48.5 and 54.0, 24: 54.9 and
// 55.0, 32: 70.2 and 56.6; 64 experts of 2048 x 1408, 18: 109.7 and 114.5, 24: 118.8 and 117.5,
// 36: 158.4 and 124.4.  By choices x d x f in 10^9: f 1056, 0.27: 29 and 34, 0.45: 49 and 40,
// 0.57: 43 and 42, 0.67: 68 and 45; f 1024, 0.54: 44 and 40; f 512, 0.54: 34 and 41,
// 0.63: 43 and 53, 0.77: 40 and 46; f 256, 0.54: 33 and 59.
constexpr int kGemmFrom = 24;   // choices an expert, on average
static bool w4_gemm(const moe_w4_cfg& c) {
  const int64_t n = c.T * c.k;
  return c.dtype == MOE_BF16 && n >= (int64_t)kGemmFrom * c.E &&
         n * c.d_model * c.d_ff >= (c.d_ff >= 1024 ? (int64_t)3 << 27 : (int64_t)1 << 30);
}

// Workspace: list (or choices by row), tiles, tile count | parts (or laid-out act(W1 x)) |
// O | laid-out x.
struct W4Ws {
  size_t list, tiles, ntiles, parts, O, x, total;
  int max_tiles;
  int64_t rows;   // laid-out rows at most
};
static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
static W4Ws w4_ws(const moe_w4_cfg& c) {
  W4Ws w;
  const int64_t n = c.T * c.k;
  const bool bf = c.dtype == MOE_BF16;
  w.rows = n + 15 * std::min<int64_t>(n, c.E);
  w.rows = (w.rows + 15) / 16 * 16;
  static_assert(kGemmToks >= kW4Tile, "the laid-out products have no more tiles than the others");
  w.max_tiles = (int)(std::min<int64_t>(n, c.E) + n / kW4Tile);
  w.list = 0;
  w.tiles = up256(4 * (size_t)w.rows);
  w.ntiles = w.tiles + sizeof(W4Tile) * (size_t)w.max_tiles;
  w.parts = up256(w.ntiles + 4);
  w.O = up256(w.parts + std::max((size_t)(bf ? 2 : 3) * n * c.d_ff, bf ? (size_t)w.rows * w4_pad(c.d_ff) : 0) * 2);
  w.x = up256(w.O + (size_t)kW4Splits * n * c.d_model * 4);
  w.total = up256(w.x + (bf ? (size_t)w.rows * w4_pad(c.d_model) * 2 : 0));
  return w;
}
size_t experts_w4_ws_bytes(const moe_w4_cfg& c) { return w4_ws(c).total; }

// A product over gy experts or tiles; the splits it was done in.  Blocks of 128 rows where
// there are three for two CUs (the second product's K split to get there): 48 tokens, 16
// experts of 1024 x 4096, 512 blocks, 12.3 and 13.6 us; one token, top-2 of them, 64 blocks,
// 8.3 and 7.0 us where 16 rows take 4.9 and 6.0.  Else 16 or 32 rows, 32 where there are two
// blocks a CU of them: 5 float tokens, 15 choices, d 736, f 1888, first product (885 blocks of
// 32) 10.1 us, with 16 rows 14.4, with 128 11.7; second (690 blocks of 16) 9.4, with 32 rows
// 11.9, with 128 11.4.
template <typename T, bool FIRST, int NS, int NO, bool FULL>
static int launch_w4_rows(W4Args a, int gy, hipStream_t s) {
  const int cus = num_cus();
  const int64_t blocks = (int64_t)((a.N + 127) / 128) * gy;
  const int steps = (a.K + kStep - 1) / kStep;
  int splits = FIRST ? 1 : (int)std::min<int64_t>(std::min(kW4Splits, steps), std::max<int64_t>(1, 2 * cus / blocks));
  a.steps = (steps + splits - 1) / splits;
  splits = (steps + a.steps - 1) / a.steps;   // whole steps, no split empty
  auto how = [&](auto go) {
    if (a.tiles) go(std::integral_constant<int, kFindTiles>{});
    else if (a.n <= kWave) go(std::integral_constant<int, kFindWave>{});
    else if (a.by_choice) go(std::integral_constant<int, kFindChoice>{});
    else go(std::integral_constant<int, kFindExpert>{});
  };
  if (2 * blocks * splits >= 3 * cus) {
    for (; a.tile0 < gy; a.tile0 += kMaxGridY)   // (only a list's tiles pass the grid's limit)
      how([&](auto h) {
        launch_kernel((w4_rows_kernel<T, FIRST, NS, NO, FULL, decltype(h)::value>),
                      dim3((a.N + 127) / 128, std::min(kMaxGridY, gy - a.tile0), splits), dim3(256), 0, s, a);
      });
    return splits;
  }
  const int rt = (int64_t)(a.N / 16) * gy >= 4 * cus ? 2 : 1;
  // Eight waves split K finer than four, but more of such blocks wait for a place: rounds of
  // blocks times a wave's steps and the latencies ahead of the first, as long as three.
  // (Second product of the one token: 6.0 us with eight, 6.7 with four; of the 5 float
  // tokens 11.9 and 9.4, their first 14.3 and 10.1.)
  auto cost = [&](int wv) {
    const int64_t places = (int64_t)cus * (4 * kW4PerSimd / wv);
    return ((int64_t)(a.N / (16 * rt)) * gy + places - 1) / places * (3 + (steps + wv - 1) / wv);
  };
  const int waves = cost(kW4Waves) < cost(4) ? kW4Waves : 4;
  how([&](auto h) {   // (gy is within a grid's limit: more tiles are blocks of 128 rows)
    constexpr int H = decltype(h)::value;
    auto go = [&](auto kern, size_t lds) {
      launch_kernel(kern, dim3(a.N / (16 * rt), gy), dim3(64 * waves), waves * lds, s, a);
    };
    if (rt == 2) go(w4_product_kernel<T, FIRST, NS, NO, 2, FULL, H>, sizeof(W4Lds<2>));
    else go(w4_product_kernel<T, FIRST, NS, NO, 1, FULL, H>, sizeof(W4Lds<1>));
  });
  return 1;
}
template <typename T, bool FIRST, int NS, int NO>
static int launch_w4_product(const W4Args& a, int gy, hipStream_t s) {
  return a.K % kStep == 0 ? launch_w4_rows<T, FIRST, NS, NO, true>(a, gy, s)
                          : launch_w4_rows<T, FIRST, NS, NO, false>(a, gy, s);
}

static void launch_w4_gemm(const moe_w4_cfg& c, const void* x, const int32_t* idx, const float* w, const uint8_t* W1c,
                           const uint8_t* W1s, const uint8_t* W2c, const uint8_t* W2s, void* y, void* ws, hipStream_t s) {
  const W4Ws L = w4_ws(c);
  const int n = (int)(c.T * c.k), d = c.d_model, f = c.d_ff;
  char* base = (char*)ws;
  int32_t* choice_of = (int32_t*)(base + L.list);
  W4Group* tiles = (W4Group*)(base + L.tiles);
  int32_t* ntiles = (int32_t*)(base + L.ntiles);
  static_assert(sizeof(W4Group) == sizeof(W4Tile), "one table's room");
  launch_kernel(w4_group_kernel, dim3(1), dim3(kW4ListThreads), 0, s, idx, n, c.E, choice_of, tiles, ntiles,
                (int)L.rows);
  const int64_t pieces = L.rows * (w4_pad(d) / 8);
  launch_kernel(w4_pack_kernel, dim3((unsigned)std::min<int64_t>((pieces + 255) / 256, 1 << 20)), dim3(256), 0, s,
                (const uint16_t*)x, (const int32_t*)choice_of, (uint16_t*)(base + L.x), d, c.k, pieces);
  const int gy = std::min<int64_t>(n, c.E) + n / kGemmToks;
  const W4GemmArgs a{W1c, W1s, (const uint16_t*)(base + L.x), base + L.parts, choice_of, tiles, ntiles, f, d, n, c.act,
                     (d + kStep - 1) / kStep};
  const bool whole = d % kGemmRows == 0 && f % kGemmRows == 0;
  static_assert(kGemmRows == 128, "the padding of a layout's rows");
  auto go = [&](auto kern, int N, int splits, const W4GemmArgs& g) {
    launch_kernel(kern, dim3(w4_pad(N) / kGemmRows, gy, splits), dim3(256), 0, s, g);
  };
  whole ? go(w4_gemm_kernel<true, true>, f, 1, a) : go(w4_gemm_kernel<true, false>, f, 1, a);
  // K is split where the blocks would not fill the CUs twice; whole steps, no split empty.
  const int steps = (f + kStep - 1) / kStep;
  const int64_t blocks = (int64_t)(w4_pad(d) / kGemmRows) * c.E * ((n / c.E + kGemmToks - 1) / kGemmToks);   // for an even load
  int splits = (int)std::min<int64_t>(std::min(kW4Splits, steps), std::max<int64_t>(1, 2 * num_cus() / std::max<int64_t>(1, blocks)));
  const int per = (steps + splits - 1) / splits;
  splits = (steps + per - 1) / per;
  const W4GemmArgs b{W2c, W2s, (const uint16_t*)(base + L.parts), base + L.O, choice_of, tiles, ntiles, d, f, n, c.act, per};
  whole ? go(w4_gemm_kernel<false, true>, d, splits, b) : go(w4_gemm_kernel<false, false>, d, splits, b);
  launch_w4_combine<uint16_t>(c, (const float*)(base + L.O), idx, w, y, splits, s);
}

template <typename T, int NX, int NA>
static void launch_w4_t(const moe_w4_cfg& c, const void* x, const int32_t* idx, const float* w, const uint8_t* W1c,
                        const uint8_t* W1s, const uint8_t* W2c, const uint8_t* W2s, void* y, void* ws, hipStream_t s) {
  const W4Ws L = w4_ws(c);
  const int n = (int)(c.T * c.k);
  char* base = (char*)ws;
  int32_t* list = (int32_t*)(base + L.list);
  W4Tile* tiles = (W4Tile*)(base + L.tiles);
  int32_t* ntiles = (int32_t*)(base + L.ntiles);
  const bool scan = n <= kW4Scan;
  const int by_choice = scan && n < c.E;
  if (!scan)
    launch_kernel(w4_list_kernel, dim3(1), dim3(kW4ListThreads), 0, s, idx, n, c.E, list, tiles, ntiles);
  else
    tiles = nullptr;
  const int gy = !scan ? L.max_tiles : by_choice ? n : c.E;
  const W4Args a{W1c, W1s, x, base + L.parts, idx, list, tiles, ntiles, c.d_ff, c.d_model, n, c.k, c.E, c.act,
                 by_choice, 0, 0};
  launch_w4_product<T, true, NX, NA>(a, gy, s);
  const W4Args b{W2c, W2s, base + L.parts, base + L.O, idx, list, tiles, ntiles, c.d_model, c.d_ff, n, c.k, c.E, c.act,
                 by_choice, 0, 0};
  const int splits = launch_w4_product<T, false, NA, NA>(b, gy, s);
  launch_w4_combine<T>(c, (const float*)(base + L.O), idx, w, y, splits, s);
}

void launch_experts_w4(const moe_w4_cfg& c, const void* x, const int32_t* idx, const float* w, const uint8_t* W1c,
                       const uint8_t* W1s, const uint8_t* W2c, const uint8_t* W2s, void* y, void* ws, hipStream_t s) {
  if (c.T == 0) return;
  if (w4_gemm(c)) launch_w4_gemm(c, x, idx, w, W1c, W1s, W2c, W2s, y, ws, s);
  else if (c.dtype == MOE_BF16) launch_w4_t<uint16_t, 1, 2>(c, x, idx, w, W1c, W1s, W2c, W2s, y, ws, s);
  else launch_w4_t<float, 3, 3>(c, x, idx, w, W1c, W1s, W2c, W2s, y, ws, s);
}

// ------------------------------------------------------------------ quantiser
// One thread per group of 32 weights (run once per weight load).
template <typename T>
__global__ __launch_bounds__(256) void w4_quantize_kernel(const T* __restrict__ W, uint8_t* __restrict__ codes,
                                                          uint8_t* __restrict__ scales, int64_t groups) {
  for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < groups; g += (int64_t)gridDim.x * 256) {
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; i += Vec<T>::N) Vec<T>::load(W + g * 32 + i, v + i);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    const bool bad = m >= 0x7f800000u;
    // amax = f 2^e with f in [1/2, 1): 7 * 2^s = 7/8 * 2^(s + 3)
    int e = 0;
    const float f = bad || m == 0 ? 0.f : frexpf(__uint_as_float(m), &e);
    int s = m == 0 || bad ? -100 : f <= 0.875f ? e - 3 : e - 2;
    s = min(max(s, -100), 125);
    const float inv = ldexpf(1.f, -s);
    u32x4 out = {0u, 0u, 0u, 0u};
    if (!bad) {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const float a = fabsf(v[i]) * inv;
        // nearest of 0 0.5 1 1.5 2 3 4 6; half way the code with the even mantissa
        const uint32_t c = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.f);
        out[i >> 3] |= (c | (__float_as_uint(v[i]) >> 31 << 3)) << (4 * (i & 7));
      }
    }
    *reinterpret_cast<u32x4*>(codes + g * 16) = out;
    scales[g] = bad ? 255 : (uint8_t)(s + 127);
  }
}

void launch_w4_quantize(int64_t rows, int K, int dtype, const void* W, uint8_t* codes, uint8_t* scales,
                        hipStream_t s) {
  const int64_t groups = rows * (K / 32);
  if (groups == 0) return;
  const dim3 grid((unsigned)std::min<int64_t>((groups + 255) / 256, 1 << 16));
  if (dtype == MOE_BF16)
    launch_kernel(w4_quantize_kernel<uint16_t>, grid, dim3(256), 0, s, (const uint16_t*)W, codes, scales, groups);
  else
    launch_kernel(w4_quantize_kernel<float>, grid, dim3(256), 0, s, (const float*)W, codes, scales, groups);
}

}  // namespace lmoe
