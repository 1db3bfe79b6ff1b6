// The router: scores, choice with balance bias and groups, weights, loads; and its
// gradient at the logits.
//
// Forward, one wavefront per token: lane l holds experts l, l + 64, ...  The choice
// value c = s + b is compared in double, so that the choice is the one of any other
// evaluation in 64 bits (two values of a token closer than 1e-15 aside).
#include "internal.h"

namespace lmoe {

constexpr int kRouteWavesPerBlock = 4;

__device__ __forceinline__ double wave_max_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmax(v, __shfl_xor(v, o, kWave));
  return v;
}
__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// 1 / (1 + e^-l); l = -inf gives 0.
__device__ __forceinline__ double sigmoid_f64(double l) { return 1.0 / (1.0 + exp(-l)); }

template <int NE>
__global__ __launch_bounds__(64 * kRouteWavesPerBlock) void route_kernel(
    const float* __restrict__ logits, const float* __restrict__ bias, int32_t* __restrict__ idx,
    float* __restrict__ w, int32_t* __restrict__ load, int64_t T, int E, int k, int score, int renorm, int groups,
    int top_groups, float scale) {
  __shared__ double keys[kRouteWavesPerBlock][64 * NE];
  __shared__ double gval[kRouteWavesPerBlock][64 * NE];
  __shared__ uint8_t gkeep[kRouteWavesPerBlock][64 * NE];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int64_t t = (int64_t)blockIdx.x * kRouteWavesPerBlock + wv;
  const bool on = t < T;
  double l[NE], s[NE], key[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const int e = i * 64 + lane;
    const float f = on && e < E ? logits[t * E + e] : -INFINITY;
    l[i] = f > -INFINITY ? (double)f : -INFINITY;
  }
  if (score == MOE_SCORE_SOFTMAX) {
    double m = l[0], z = 0.0;
#pragma unroll
    for (int i = 1; i < NE; ++i) m = fmax(m, l[i]);
    m = wave_max_f64(m);
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      s[i] = l[i] == -INFINITY ? 0.0 : l[i] == m ? 1.0 : exp(l[i] - m);
      z += s[i];
    }
    z = wave_sum_f64(z);
#pragma unroll
    for (int i = 0; i < NE; ++i) s[i] = z > 0.0 ? s[i] / z : 0.0;
  } else {
#pragma unroll
    for (int i = 0; i < NE; ++i) s[i] = sigmoid_f64(l[i]);
  }
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const int e = i * 64 + lane;
    double c = l[i];
    if (bias || groups > 1) {
      c = s[i] + (bias && e < E ? (double)bias[e] : 0.0);
      if (!(c > -INFINITY) || l[i] == -INFINITY) c = -INFINITY;
    }
    key[i] = c;
    keys[wv][e] = c;
  }
  if (groups > 1) {
    __syncthreads();
    const int n = E / groups;
    for (int g = lane; g < groups; g += 64) {
      double a = -INFINITY, b = -INFINITY;
      for (int j = 0; j < n; ++j) {
        const double c = keys[wv][g * n + j];
        b = fmax(b, fmin(a, c));
        a = fmax(a, c);
      }
      gval[wv][g] = a == -INFINITY ? a : b == -INFINITY ? a : a + b;
    }
    __syncthreads();
    for (int g = lane; g < groups; g += 64) {
      int rank = 0;
      for (int h = 0; h < groups; ++h)
        rank += gval[wv][h] > gval[wv][g] || (gval[wv][h] == gval[wv][g] && h < g);
      gkeep[wv][g] = rank < top_groups;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const int e = i * 64 + lane;
      if (e < E && !gkeep[wv][e / n]) key[i] = -INFINITY;
    }
  }
  if (!on) return;
  double mine = 0.0, sum = 0.0;
  int mine_e = -1;
  for (int r = 0; r < k; ++r) {
    double best = -INFINITY;
    int be = 1 << 30;
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (key[i] > best) {
        best = key[i];
        be = i * 64 + lane;
      }
    const double m = wave_max_f64(best);
    if (m == -INFINITY) break;
    int e = best == m ? be : 1 << 30;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) e = min(e, __shfl_xor(e, o, kWave));
    double se = 0.0;
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (i * 64 + lane == e) {
        key[i] = -INFINITY;
        se = s[i];
      }
    se = __shfl(se, e & 63, kWave);
    sum += se;
    if (lane == r) {
      mine = se;
      mine_e = e;
    }
  }
  if (lane < k) {
    idx[t * k + lane] = mine_e;
    double v = scale * mine;
    if (renorm) v = sum > 0.0 ? v / sum : 0.0;
    w[t * k + lane] = (float)v;
    if (load && mine_e >= 0) atomicAdd(load + mine_e, 1);
  }
}

void launch_route(const moe_route_cfg& c, const float* logits, const float* bias, int32_t* idx, float* w,
                  int32_t* load, hipStream_t s) {
  if (c.T == 0) return;
  const unsigned blocks = (unsigned)((c.T + kRouteWavesPerBlock - 1) / kRouteWavesPerBlock);
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(64 * kRouteWavesPerBlock), 0, s, logits, bias, idx, w, load, c.T, c.E,
                       c.k, c.score, c.renorm, c.groups, c.top_groups, c.scale);
  };
  if (c.E <= 64) go(route_kernel<1>);
  else if (c.E <= 128) go(route_kernel<2>);
  else if (c.E <= 256) go(route_kernel<4>);
  else go(route_kernel<8>);
}

// ------------------------------------------------------------------- gradient
template <int NE>
__global__ __launch_bounds__(64 * kRouteWavesPerBlock) void route_bwd_kernel(
    const float* __restrict__ logits, const int32_t* __restrict__ idx, const float* __restrict__ w,
    const float* __restrict__ dw, float* __restrict__ dlogits, int64_t T, int E, int k, int score, int renorm,
    float scale) {
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * kRouteWavesPerBlock + (threadIdx.x >> 6);
  if (t >= T) return;
  int er = lane < k ? idx[t * k + lane] : -1;
  if (er < 0 || er >= E) er = -1;
  const float wr = er >= 0 ? w[t * k + lane] : 0.f, gr = er >= 0 ? dw[t * k + lane] : 0.f;
  const float G = wave_sum(wr * gr);
  float v = wr * (renorm ? gr - G / scale : gr);
  if (score == MOE_SCORE_SIGMOID && er >= 0) v *= 1.f / (1.f + expf(logits[t * E + er]));   // 1 - s
  float p[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) p[i] = 0.f;
  if (score == MOE_SCORE_SOFTMAX && !renorm) {
    float l[NE], m = -INFINITY, z = 0.f;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const int e = i * 64 + lane;
      l[i] = e < E ? logits[t * E + e] : -INFINITY;
      if (!(l[i] > -INFINITY)) l[i] = -INFINITY;
      m = fmaxf(m, l[i]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      p[i] = l[i] == -INFINITY ? 0.f : l[i] == m ? 1.f : expf(l[i] - m);
      z += p[i];
    }
    z = wave_sum(z);
#pragma unroll
    for (int i = 0; i < NE; ++i) p[i] = z > 0.f ? -G * (p[i] / z) : 0.f;
  }
  for (int r = 0; r < k; ++r) {
    const int e = __shfl(er, r, kWave);
    const float a = __shfl(v, r, kWave);
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (i * 64 + lane == e) p[i] += a;
  }
#pragma unroll
  for (int i = 0; i < NE; ++i)
    if (i * 64 + lane < E) dlogits[t * E + i * 64 + lane] = p[i];
}

void launch_route_bwd(const moe_route_cfg& c, const float* logits, const int32_t* idx, const float* w,
                      const float* dw, float* dlogits, hipStream_t s) {
  if (c.T == 0) return;
  const unsigned blocks = (unsigned)((c.T + kRouteWavesPerBlock - 1) / kRouteWavesPerBlock);
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, dim3(blocks), dim3(64 * kRouteWavesPerBlock), 0, s, logits, idx, w, dw, dlogits, c.T, c.E,
                       c.k, c.score, c.renorm, c.scale);
  };
  if (c.E <= 64) go(route_bwd_kernel<1>);
  else if (c.E <= 128) go(route_bwd_kernel<2>);
  else if (c.E <= 256) go(route_bwd_kernel<4>);
  else go(route_bwd_kernel<8>);
}

}  // namespace lmoe
