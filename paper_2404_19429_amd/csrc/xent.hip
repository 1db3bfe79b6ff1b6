// Softmax cross entropy of rows x over the vocabulary W, a piece of it at a time,
// without keeping the logits, and its gradients.
//
//   forward: l = x W^T, lse = log sum exp l, loss = lse - l[target].  The product's
//     epilogue leaves of each row and run of 32 or 64 columns the largest logit and
//     the sum of exp(l - largest) (EPI_LSE), T V / 8 bytes at most where the logits
//     were 4 T V; one launch joins them.
//   backward: dl = g (exp(l - lse) - [v = target]) in the type of x, computed again
//     piece by piece (EPI_DL); dx += dl W in float over the pieces, dW = dl^T x.  dl's
//     rounding to bfloat16 is half a step of each, as every operand of the products.
//
// A piece's dl takes kDlBytes at most, which the last-level cache holds between the
// product that writes it and the two that read it.
#include "gemm_wide.h"

namespace lmoe {

// gemm.hip
int xent_run_columns(int dtype, int64_t T);
int launch_xent_lse(int dtype, int64_t T, int d, const void* x, const void* W, const XentParams& xp, hipStream_t s);
void launch_xent_dl(int dtype, int64_t T, int d, const void* x, const void* W, const XentParams& xp, void* dl, int ld,
                    hipStream_t s);
void launch_xent_dx(int dtype, int64_t T, int d, int cols, const void* dl, int ld, const void* W, const float* acc_in,
                    float* acc_out, void* dx, hipStream_t s);
void launch_xent_dx_whole(int64_t T, int d, int cols, const void* dl, int ld, const void* W, void* dx, void* part,
                          hipStream_t s);
void launch_xent_dw(int dtype, int64_t T, int d, int cols, const void* dl, int ld, const void* x, void* dW, hipStream_t s);
size_t xent_part_bytes();

namespace {

constexpr int64_t kDlBytes = (int64_t)256 << 20;
constexpr int64_t kOperand = (int64_t)1 << 31;   // the bf16 products' operands: 32-bit byte offsets

int64_t esize(const moe_xent_cfg& c) { return c.dtype == MOE_BF16 ? 2 : 4; }

// Columns of a piece: as many as `most`, in equal pieces of whole tiles.
int piece_columns(const moe_xent_cfg& c, int64_t most) {
  if (c.V <= most) return c.V;
  const int64_t n = (c.V + most - 1) / most, even = (c.V + n - 1) / n;
  return (int)std::min<int64_t>(most, (even + 255) / 256 * 256);
}
int fwd_columns(const moe_xent_cfg& c) {
  return piece_columns(c, (kOperand - 1) / (c.d_model * 2) / 256 * 256);
}
struct BwdPlan {
  int cols, pieces, ld;   // columns of a piece, pieces, columns of dl's rows
  size_t x, dl, acc, part, bytes;
};
BwdPlan bwd_plan(const moe_xent_cfg& c) {
  BwdPlan p{};
  const int64_t e = esize(c), rows = pad16(c.T);
  int64_t most = std::max<int64_t>(2048, kDlBytes / (rows * e) / 256 * 256);
  most = std::min(most, (kOperand - 1) / (c.d_model * 2) / 256 * 256);
  most = std::min(most, std::max<int64_t>(64, (kOperand - 1) / (rows * 2) / 64 * 64));
  p.cols = piece_columns(c, most);
  p.pieces = (c.V + p.cols - 1) / p.cols;
  const int unit = c.dtype == MOE_BF16 ? 64 : 8;
  p.ld = (p.cols + unit - 1) / unit * unit;
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t o = at;
    at += (n + 255) / 256 * 256;
    return o;
  };
  p.x = take(rows * c.d_model * e);
  p.dl = take(rows * p.ld * e);
  if (c.dtype == MOE_BF16 && p.pieces > 1) p.acc = take((size_t)c.T * c.d_model * 4);
  if (c.dtype == MOE_BF16 && p.pieces == 1) p.part = take(xent_part_bytes());
  p.bytes = at;
  return p;
}
// Forward: the runs' (largest, sum) of every row, then the targets' logits.
int64_t fwd_blocks(const moe_xent_cfg& c) {
  const int run = xent_run_columns(c.dtype, c.T), cols = fwd_columns(c);
  return (c.V + run - 1) / run + (int64_t)(256 / run) * ((c.V + cols - 1) / cols);
}

// lse and loss of a row from its runs.  A block takes TX rows, TY slices of the runs each.
__global__ __launch_bounds__(256) void xent_join_kernel(const float2* __restrict__ part, const float* __restrict__ tl,
                                                        const int32_t* __restrict__ target, int blocks, int64_t T, int V,
                                                        int tx, float* __restrict__ loss, float* __restrict__ lse) {
  __shared__ float2 red[256];
  const int lx = threadIdx.x % tx, ly = threadIdx.x / tx, ny = 256 / tx;
  const int64_t t = (int64_t)blockIdx.x * tx + lx;
  // Sums of exp(l - m) under the largest so far; a NaN logit is in its run's sum.
  auto join = [](float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x), at = m > -INFINITY ? m : 0.f;
    return make_float2(m, a.y * __builtin_amdgcn_exp2f((a.x - at) * kLog2e) + b.y * __builtin_amdgcn_exp2f((b.x - at) * kLog2e));
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
    const float z = red[threadIdx.x].x + logf(red[threadIdx.x].y);
    const int id = target[t];
    lse[t] = z;
    loss[t] = id >= 0 && id < V ? z - tl[t] : 0.f;
  }
}

// x for the backward's products: the rows whose target is no class as zeros, so that
// whatever padding holds stays out of dW.  bf16: 16 x 32 blocks, a wave each.
__global__ __launch_bounds__(256) void xent_pack_kernel(const uint16_t* __restrict__ x, const int32_t* __restrict__ target,
                                                        uint16_t* __restrict__ out, int64_t T, int V, int d) {
  const int64_t b = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 6;
  const int lane = threadIdx.x & 63, kb = d >> 5;
  const int64_t rb = b / kb;
  if (rb * 16 >= pad16(T)) return;
  const int64_t row = rb * 16 + (lane >> 2);
  const int col = (int)(b - rb * kb) * 32 + (lane & 3) * 8;
  u32x4 v = u32x4{0u, 0u, 0u, 0u};
  if (row < T && target[row] >= 0 && target[row] < V) v = *reinterpret_cast<const u32x4*>(x + row * d + col);
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

}  // namespace

size_t xent_ws_bytes(const moe_xent_cfg& c, bool backward) {
  if (c.T == 0) return 0;
  if (backward) return bwd_plan(c).bytes;
  return (size_t)fwd_blocks(c) * c.T * sizeof(float2) + (size_t)c.T * sizeof(float);
}

void launch_xent(const moe_xent_cfg& c, const void* x, const void* W, const int32_t* target, float* loss, float* lse,
                 void* ws, hipStream_t s) {
  if (c.T == 0) return;
  const int cols = fwd_columns(c);
  XentParams xp{};
  xp.target = target;
  xp.part = (float2*)ws;
  xp.tl = (float*)(xp.part + fwd_blocks(c) * c.T);
  xp.stride = c.T;
  xp.V = c.V;
  for (int v = 0; v < c.V; v += cols) {
    xp.col0 = v;
    xp.cols = std::min(cols, c.V - v);
    xp.block0 += launch_xent_lse(c.dtype, c.T, c.d_model, x, (const char*)W + (int64_t)v * c.d_model * esize(c), xp, s);
  }
  int tx = 1;
  while (tx < 64 && tx < c.T) tx *= 2;
  hipLaunchKernelGGL(xent_join_kernel, dim3((unsigned)((c.T + tx - 1) / tx)), dim3(256), 0, s, xp.part, xp.tl, target,
                     xp.block0, c.T, c.V, tx, loss, lse);
}

void launch_xent_bwd(const moe_xent_cfg& c, const void* x, const void* W, const int32_t* target, const float* lse,
                     const float* dloss, void* dx, void* dW, void* ws, hipStream_t s) {
  const int64_t d = c.d_model, e = esize(c);
  if (c.T == 0) {
    const int64_t n = c.V * d * e / 16;
    if (dW)
      hipLaunchKernelGGL(xent_zero_kernel, dim3((unsigned)std::min<int64_t>(4096, (n + 255) / 256)), dim3(256), 0, s,
                         (u32x4*)dW, n);
    return;
  }
  const BwdPlan p = bwd_plan(c);
  char* w = (char*)ws;
  void *xp_ = w + p.x, *dl = w + p.dl;
  const bool bf = c.dtype == MOE_BF16;
  if (bf)
    hipLaunchKernelGGL(xent_pack_kernel, dim3((unsigned)((pad16(c.T) / 16 * (d / 32) * 64 + 255) / 256)), dim3(256), 0, s,
                       (const uint16_t*)x, target, (uint16_t*)xp_, c.T, c.V, (int)d);
  else
    hipLaunchKernelGGL(xent_copy_kernel, dim3((unsigned)((c.T * d / 4 + 255) / 256)), dim3(256), 0, s, (const float*)x,
                       target, (float*)xp_, c.T, c.V, (int)d);
  XentParams xp{};
  xp.target = target;
  xp.lse = lse;
  xp.g = dloss;
  xp.stride = c.T;
  xp.V = c.V;
  float* acc = bf ? (float*)(w + p.acc) : (float*)dx;
  for (int v = 0; v < c.V; v += p.cols) {
    xp.col0 = v;
    xp.cols = std::min(p.cols, c.V - v);
    const int unit = bf ? 64 : 8, ld = (xp.cols + unit - 1) / unit * unit;
    const void* Wv = (const char*)W + (int64_t)v * d * e;
    launch_xent_dl(c.dtype, c.T, (int)d, xp_, Wv, xp, dl, ld, s);
    if (dx && bf && p.pieces == 1) {
      launch_xent_dx_whole(c.T, (int)d, xp.cols, dl, ld, Wv, dx, w + p.part, s);
    } else if (dx) {
      const bool last = v + p.cols >= c.V;
      launch_xent_dx(c.dtype, c.T, (int)d, xp.cols, dl, ld, Wv, v > 0 ? acc : nullptr, acc, bf && last ? dx : nullptr, s);
    }
    if (dW) launch_xent_dw(c.dtype, c.T, (int)d, xp.cols, dl, ld, xp_, (char*)dW + (int64_t)v * d * e, s);
  }
}

}  // namespace lmoe
