// Softmax cross entropy of rows x over the vocabulary W, a piece of it at a time,
// without keeping the logits, and its gradients.
//
//   forward: l = x W^T, lse = log sum exp l, loss = lse - l[target].  The product's
//     epilogue leaves of each row and run of columns the largest logit and the sum of
//     exp(l - largest) (EPI_LSE), 8 bytes; one launch joins them.  A run is what the
//     narrowest tile allowed has in a wave: 64 columns in bfloat16, 32 in float, half of
//     that up to 1024 tokens.  Where the logits were 4 T V bytes the runs are T V / 8
//     (bfloat16), T V / 4 (float), twice that up to 1024 tokens.
//   backward: dl = g (exp(l - lse) - [v = target]) in the type of x, computed again
//     piece by piece (EPI_DL); dx += dl W in float over the pieces, dW = dl^T x.  dl's
//     rounding to bfloat16 (relative to the largest g) is half a step of each, as of
//     every operand of the products.
//
// A piece's dl takes kDlBytes, or 2048 columns where those are more (past 131072 tokens
// of bfloat16, 65536 of float), but no more than the products address, 2 GiB (float: 4),
// with 64 columns at the least.  Every piece reads and writes dx's float sums, so fewer are
// faster (16384 tokens, 50257 classes, width 2048, bfloat16, one step: 128 MiB 13.41 ms, 256
// 12.08, 512 11.77, 1024 11.53), and 512 MiB are a third of that dl.
#include "gemm_wide.h"

namespace lmoe {

// gemm.hip
int xent_run_columns(int dtype, int64_t T);
int launch_xent_lse(int dtype, int form, int64_t T, int d, const void* x, const void* W, const XentParams& xp,
                    hipStream_t s);
void launch_xent_dl(int dtype, int form, int64_t T, int d, const void* x, const void* W, const XentParams& xp, void* dl,
                    int ld, hipStream_t s);
void launch_xent_dx(int dtype, int64_t T, int d, int cols, const void* dl, int ld, const void* W, const float* acc_in,
                    float* acc_out, void* dx, const float* scale, void* part, hipStream_t s);
size_t xent_slices_bytes(int64_t T, int d, int cols);
void launch_xent_dx_whole(int64_t T, int d, int cols, const void* dl, int ld, const void* W, void* dx, const float* scale,
                          void* part, hipStream_t s);
void launch_xent_dw(int dtype, int64_t T, int d, int cols, const void* dl, int ld, const void* x, void* dW,
                    const float* scale, void* part, hipStream_t s);
size_t xent_part_bytes();

namespace {

constexpr int64_t kDlBytes = (int64_t)512 << 20;
constexpr int64_t kWBytes = (int64_t)128 << 20;  // of W in blocks, in the forward
// From how many tokens on the forward copies x, and x and W, to blocks, and the backward W (x it always does).  Blocks
// feed the products' loads whole cache lines, for a pass over the operand.  Forward, no copy / x / both, us (50257
// classes): 64 tokens, width 1024 33.1 / 32.0 / 58.1; 2048 232.8 / 201.8 / 222.4; 4096, width 2048 834 / 715 / 721; 8192,
// width 1024 863 / 761 / 739.  Backward, W as it is / copied: 4096 tokens 2497 / 2510, 8192 (32000 classes) 2697 / 2632.
constexpr int64_t kFwdX = 64, kFwdBlocked = 8192, kBwdBlocked = 8192;
constexpr int64_t kCus = 256;   // compute units (the sizes below are asked for on hosts without a device too)
constexpr int64_t kOperand = (int64_t)1 << 31;   // the bf16 products' operands: 32-bit byte offsets

int64_t esize(const moe_xent_cfg& c) { return c.dtype == MOE_BF16 ? 2 : 4; }

int fwd_form(const moe_xent_cfg& c) {
  if (c.dtype != MOE_BF16 || c.T < kFwdX) return kXentRows;
  return c.T < kFwdBlocked ? kXentX : kXentBlocked;
}
struct FwdPlan {
  int form, cols;         // kXent*; columns of a piece
  int64_t blocks;         // runs of columns, at most
  size_t part, tl, x, W, bytes;
};
FwdPlan fwd_plan(const moe_xent_cfg& c) {
  FwdPlan p{};
  p.form = fwd_form(c);
  const int64_t room = p.form == kXentBlocked ? kWBytes : kOperand - 1;
  p.cols = (int)std::min<int64_t>(c.V, std::max<int64_t>(256, room / (c.d_model * 2) / 256 * 256));
  if (c.dtype == MOE_F32) {   // (the float product has a block of 256 threads for every 64 x 64 tile)
    const int64_t tiles = kMostThreads / 256 / ((c.T + 15 + 63) / 64);
    p.cols = (int)std::min<int64_t>(p.cols, std::max<int64_t>(1, tiles) * 64);
  }
  const int run = xent_run_columns(c.dtype, c.T);
  const int64_t pieces = (c.V + p.cols - 1) / p.cols;
  p.blocks = (c.V + run - 1) / run + (int64_t)(512 / run) * pieces;   // (a piece is two products at most)
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t o = at;
    at += (n + 255) / 256 * 256;
    return o;
  };
  p.part = take((size_t)p.blocks * c.T * sizeof(float2));
  p.tl = take((size_t)c.T * sizeof(float));
  if (p.form >= kXentX) p.x = take(pad16(c.T) * c.d_model * 2);
  if (p.form == kXentBlocked) p.W = take(pad16(p.cols) * c.d_model * 2);
  p.bytes = at;
  return p;
}
struct BwdPlan {
  int cols, pieces, ld;   // columns of a piece, pieces, columns of dl's rows
  size_t scale, x, W, dl, acc, part, bytes;
  int form;               // kXentX or kXentBlocked
};
BwdPlan bwd_plan(const moe_xent_cfg& c) {
  BwdPlan p{};
  const int64_t e = esize(c), rows = pad16(c.T);
  int64_t most = std::max<int64_t>(2048, kDlBytes / (rows * e) / 256 * 256);
  // Pieces that are whole rounds of the tiles of dW (and, with as many tokens, of the others).
  const int64_t unit = kCus / std::min<int64_t>(kCus, (c.d_model + 255) / 256) * 256;
  if (c.dtype == MOE_BF16 && most < c.V && most >= unit) most = most / unit * unit;
  most = std::min(most, (kOperand - 1) / (c.d_model * 2) / 256 * 256);
  most = std::min(most, std::max<int64_t>(64, (kOperand - 1) / (rows * 2) / 64 * 64));
  p.cols = (int)std::min<int64_t>(c.V, most);
  p.pieces = (c.V + p.cols - 1) / p.cols;
  const int pad = c.dtype == MOE_BF16 ? 64 : 8;
  p.ld = (p.cols + pad - 1) / pad * pad;
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t o = at;
    at += (n + 255) / 256 * 256;
    return o;
  };
  p.form = c.dtype == MOE_BF16 && c.T >= kBwdBlocked ? kXentBlocked : kXentX;
  p.scale = take(sizeof(float));
  p.x = take(rows * c.d_model * e);
  if (p.form == kXentBlocked) p.W = take(pad16(p.cols) * c.d_model * 2);
  p.dl = take(rows * p.ld * e);
  if (c.dtype == MOE_BF16 && p.pieces > 1) p.acc = take((size_t)c.T * c.d_model * 4);
  if (c.dtype == MOE_BF16) p.part = take(xent_part_bytes());
  if (c.dtype == MOE_F32) p.part = take(xent_slices_bytes(c.T, c.d_model, p.cols));
  p.bytes = at;
  return p;
}

// lse and loss of a row from its runs.  A block takes TX rows, TY slices of the runs each.
__global__ __launch_bounds__(256) void xent_join_kernel(const float2* __restrict__ part, const float* __restrict__ tl,
                                                        const int32_t* __restrict__ target, int blocks, int64_t T, int V,
                                                        int tx, float* __restrict__ loss, float* __restrict__ lse) {
  __shared__ float2 red[256];
  const int lx = threadIdx.x % tx, ly = threadIdx.x / tx, ny = 256 / tx;
  const int64_t t = (int64_t)blockIdx.x * tx + lx;
  // Sums under the largest so far, in base 2; a NaN logit is in its run's sum.
  auto join = [](float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x), at = m > -INFINITY ? m : 0.f;
    return make_float2(m, a.y * __builtin_amdgcn_exp2f(a.x - at) + b.y * __builtin_amdgcn_exp2f(b.x - at));
  };
  float2 v = make_float2(-INFINITY, 0.f);
  if (t < T)
    for (int b = ly; b < blocks; b += 4 * ny) {
      float2 q[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) q[u] = b + u * ny < blocks ? part[(int64_t)(b + u * ny) * T + t] : make_float2(-INFINITY, 0.f);
      v = join(v, join(join(q[0], q[1]), join(q[2], q[3])));
    }
  red[threadIdx.x] = v;
  __syncthreads();
  for (int h = ny / 2; h > 0; h >>= 1) {
    if (ly < h) red[threadIdx.x] = join(red[threadIdx.x], red[threadIdx.x + h * tx]);
    __syncthreads();
  }
  if (ly == 0 && t < T) {
    const float z = (red[threadIdx.x].x + log2f(red[threadIdx.x].y)) * kLn2;
    const int id = target[t];
    lse[t] = z;
    loss[t] = id >= 0 && id < V ? z - tl[t] : 0.f;
  }
}

// The largest |g| of the tokens that count (1 if there is none, or none that is finite): what bf16's dl is relative to.
// One block's work.
__device__ __forceinline__ void largest_g(const float* __restrict__ g, const int32_t* __restrict__ target, int64_t T, int V,
                                          float* __restrict__ out) {
  __shared__ float red[4];
  float m = 0.f;
  constexpr int U = 16;
  for (int64_t t0 = threadIdx.x; t0 < T; t0 += U * 256) {
    float v[U];
    int id[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t t = t0 + u * 256;
      v[u] = t < T ? fabsf(g[t]) : 0.f;
      id[u] = t < T ? target[t] : -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) m = id[u] >= 0 && id[u] < V ? fmaxf(m, v[u]) : m;   // (NaN: left out)
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    *out = m > 0.f && m < INFINITY ? m : 1.f;
  }
}

// x for the backward's products: the rows whose target is no class as zeros, so that
// whatever padding holds stays out of dW.  bf16: 16 x 32 blocks, a wave each.
// target NULL: every row as it is.  scale (nullable): the first block finds largest_g.
__global__ __launch_bounds__(256) void xent_pack_kernel(const uint16_t* __restrict__ x, const int32_t* __restrict__ target,
                                                        uint16_t* __restrict__ out, int64_t T, int V, int d,
                                                        const float* __restrict__ g, float* __restrict__ scale) {
  if (scale && blockIdx.x == 0) return largest_g(g, target, T, V, scale);
  const int64_t b = ((int64_t)(blockIdx.x - (scale ? 1 : 0)) * blockDim.x + threadIdx.x) >> 6;
  const int lane = threadIdx.x & 63, kb = d >> 5;
  const int64_t rb = b / kb;
  if (rb * 16 >= pad16(T)) return;
  const int64_t row = rb * 16 + (lane >> 2);
  const int col = (int)(b - rb * kb) * 32 + (lane & 3) * 8;
  u32x4 v = u32x4{0u, 0u, 0u, 0u};
  if (row < T && (target == nullptr || (target[row] >= 0 && target[row] < V))) v = *reinterpret_cast<const u32x4*>(x + row * d + col);
  *reinterpret_cast<u32x4*>(out + b * 512 + lane * 8) = v;
}
__global__ __launch_bounds__(256) void xent_copy_kernel(const float* __restrict__ x, const int32_t* __restrict__ target,
                                                        float* __restrict__ out, int64_t T, int V, int d) {
  const int64_t i = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * 4;
  const int64_t row = i / d;
  if (row >= T) return;
  const bool on = target[row] >= 0 && target[row] < V;
  *reinterpret_cast<f32x4*>(out + i) = on ? *reinterpret_cast<const f32x4*>(x + i) : f32x4{0.f, 0.f, 0.f, 0.f};
}
__global__ __launch_bounds__(256) void xent_zero_kernel(u32x4* z, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) z[i] = u32x4{0u, 0u, 0u, 0u};
}

void launch_pack(const void* src, const int32_t* target, void* dst, int64_t rows, int V, int d, hipStream_t s,
                 const float* g = nullptr, float* scale = nullptr) {
  const int64_t blocks = (pad16(rows) / 16 * (d / 32) * 64 + 255) / 256 + (scale ? 1 : 0);
  launch_kernel(xent_pack_kernel, dim3((unsigned)blocks), dim3(256), 0, s, (const uint16_t*)src, target,
                (uint16_t*)dst, rows, V, d, g, scale);
}

}  // namespace

size_t xent_ws_bytes(const moe_xent_cfg& c, bool backward) {
  if (c.T == 0) return 0;
  if (backward) return bwd_plan(c).bytes;
  return fwd_plan(c).bytes;
}

void launch_xent(const moe_xent_cfg& c, const void* x, const void* W, const int32_t* target, float* loss, float* lse,
                 void* ws, hipStream_t s) {
  if (c.T == 0) return;
  const FwdPlan p = fwd_plan(c);
  char* w = (char*)ws;
  XentParams xp{};
  xp.target = target;
  xp.part = (float2*)(w + p.part);
  xp.tl = (float*)(w + p.tl);
  xp.stride = c.T;
  xp.V = c.V;
  if (p.form >= kXentX) {
    launch_pack(x, nullptr, w + p.x, c.T, c.V, c.d_model, s);
    x = w + p.x;
  }
  for (int64_t v = 0; v < c.V; v += p.cols) {
    xp.col0 = (int)v;
    xp.cols = (int)std::min<int64_t>(p.cols, c.V - v);
    const void* Wv = (const char*)W + v * c.d_model * esize(c);
    if (p.form == kXentBlocked) {
      launch_pack(Wv, nullptr, w + p.W, xp.cols, c.V, c.d_model, s);
      Wv = w + p.W;
    }
    xp.block0 += launch_xent_lse(c.dtype, p.form, c.T, c.d_model, x, Wv, xp, s);
  }
  // Rows a block: enough blocks for every CU, 64 bytes of a run's rows at least where there are as many.
  int tx = 1;
  while (tx < 64 && tx < c.T && (tx < 8 || c.T >= (int64_t)1024 * tx)) tx *= 2;
  launch_kernel(xent_join_kernel, dim3((unsigned)((c.T + tx - 1) / tx)), dim3(256), 0, s, xp.part, xp.tl, target,
                xp.block0, c.T, c.V, tx, loss, lse);
}

void launch_xent_bwd(const moe_xent_cfg& c, const void* x, const void* W, const int32_t* target, const float* lse,
                     const float* dloss, void* dx, void* dW, void* ws, hipStream_t s) {
  const int64_t d = c.d_model, e = esize(c);
  if (c.T == 0) {
    const int64_t n = c.V * d * e / 16;
    if (dW)
      launch_kernel(xent_zero_kernel, dim3((unsigned)std::min<int64_t>(4096, (n + 255) / 256)), dim3(256), 0, s,
                    (u32x4*)dW, n);
    return;
  }
  const BwdPlan p = bwd_plan(c);
  char* w = (char*)ws;
  void *xp_ = w + p.x, *dl = w + p.dl;
  const bool bf = c.dtype == MOE_BF16;
  if (bf)
    launch_pack(x, target, xp_, c.T, c.V, (int)d, s, dloss, (float*)(w + p.scale));
  else
    launch_kernel(xent_copy_kernel, dim3((unsigned)((c.T * d / 4 + 255) / 256)), dim3(256), 0, s, (const float*)x,
                  target, (float*)xp_, c.T, c.V, (int)d);
  XentParams xp{};
  xp.target = target;
  xp.lse = lse;
  xp.g = dloss;
  const float* scale = bf ? (const float*)(w + p.scale) : nullptr;
  xp.scale = scale;
  xp.stride = c.T;
  xp.V = c.V;
  float* acc = bf ? (float*)(w + p.acc) : (float*)dx;
  for (int64_t v = 0; v < c.V; v += p.cols) {
    xp.col0 = (int)v;
    xp.cols = (int)std::min<int64_t>(p.cols, c.V - v);
    const int unit = bf ? 64 : 8, ld = (xp.cols + unit - 1) / unit * unit;
    const void* Wv = (const char*)W + v * d * e;
    if (p.form == kXentBlocked) launch_pack(Wv, nullptr, w + p.W, xp.cols, c.V, (int)d, s);
    launch_xent_dl(c.dtype, p.form, c.T, (int)d, xp_, p.form == kXentBlocked ? w + p.W : Wv, xp, dl, ld, s);
    if (dx && bf && p.pieces == 1) {
      launch_xent_dx_whole(c.T, (int)d, xp.cols, dl, ld, Wv, dx, scale, w + p.part, s);
    } else if (dx) {
      const bool last = v + p.cols >= c.V;
      launch_xent_dx(c.dtype, c.T, (int)d, xp.cols, dl, ld, Wv, v > 0 ? acc : nullptr, acc, bf && last ? dx : nullptr,
                     scale, w + p.part, s);
    }
    if (dW) launch_xent_dw(c.dtype, c.T, (int)d, xp.cols, dl, ld, xp_, (char*)dW + v * d * e, scale, w + p.part, s);
  }
}

}  // namespace lmoe
