// The router: scores, choice with balance bias and groups, weights, loads; and its
// gradient at the logits.
//
// The choice is defined on the values c = s + b compared as doubles (so that it is the
// one of any other evaluation in 64 bits, two values of a token closer than 1e-15 aside).
// Doubles for every expert would bound the kernel, so tokens are routed in float first:
// a team of 4 or 16 lanes holds a token's row, and every step that compares two values
// also sees whether they are too close for float to tell (route_eps, above the sum of
// the errors).  Such a token (a few in a thousand of ordinary logits; all of them where
// logits tie) goes the exact way, one wavefront for the token in double, in the same launch.
// Bound by the comparisons, not by the 4 E bytes a token: 32768 tokens, 256 experts in 8
// groups, k 8, 23.2-24.3 us (8.7 for the bytes; 16 without the exact way, whose registers leave
// five waves a SIMD); all in double 270.  8192 tokens, 64 experts, k 2: 3.3 us.
#include <utility>

#include "internal.h"

namespace lmoe {

struct RouteArgs {
  const float *logits, *bias;
  int32_t* idx;
  float* w;
  int64_t T;
  int32_t E, k, score, renorm, groups, top_groups;
  float scale;
  int64_t first;   // the launch's first token
};

template <int CTRL>
__device__ __forceinline__ float dpp_f(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ double dpp_f64(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xf, 0xf, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double readlane_f64(double v, int l) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, l), hi = __builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), l);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// ------------------------------------------------------------------- exact way
// Within rows of 16 lanes by rotations, then the four rows' results: a fifth of the
// latency of six exchanges through LDS, and a rare token's latency is the kernel's tail.
template <typename F>
__device__ __forceinline__ double wave_reduce_f64(double v, F f) {
  v = f(v, dpp_f64<0x128>(v));
  v = f(v, dpp_f64<0x124>(v));
  v = f(v, dpp_f64<0x122>(v));
  v = f(v, dpp_f64<0x121>(v));
  return f(f(readlane_f64(v, 0), readlane_f64(v, 16)), f(readlane_f64(v, 32), readlane_f64(v, 48)));
}
__device__ __forceinline__ double wave_max_f64(double v) {
  return wave_reduce_f64(v, [](double a, double b) __attribute__((always_inline)) { return fmax(a, b); });
}
__device__ __forceinline__ double wave_sum_f64(double v) {
  return wave_reduce_f64(v, [](double a, double b) __attribute__((always_inline)) { return a + b; });
}

// LDS written by a lane of the wave, read by another.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A wave's: MG groups at most (0: there are none).
template <int NE, int MG>
struct RouteLds {
  double key[64 * NE], gval[MG];
  uint8_t keep[MG];
};
template <int NE>
struct RouteLds<NE, 0> {};

// Token t by the whole wave: lane l holds experts l, l + 64, ...
template <int NE, int MG>
__device__ __forceinline__ void route_exact(const RouteArgs& a, int64_t t, RouteLds<NE, MG>& lds) {
  const int lane = threadIdx.x & 63;
  const int E = a.E;
  double l[NE], s[NE], key[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const int e = i * 64 + lane;
    const float f = e < E ? a.logits[t * E + e] : -INFINITY;
    l[i] = f > -INFINITY ? (double)f : -INFINITY;
  }
  if (a.score == MOE_SCORE_SOFTMAX) {
    double m = l[0], z = 0.0;
#pragma unroll
    for (int i = 1; i < NE; ++i) m = fmax(m, l[i]);
    m = wave_max_f64(m);
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      s[i] = l[i] == -INFINITY ? 0.0 : l[i] == m ? 1.0 : exp(l[i] - m);   // (+inf logits: an even share)
      z += s[i];
    }
    z = wave_sum_f64(z);
#pragma unroll
    for (int i = 0; i < NE; ++i) s[i] = z > 0.0 ? s[i] / z : 0.0;
  } else {
#pragma unroll
    for (int i = 0; i < NE; ++i) s[i] = 1.0 / (1.0 + exp(-l[i]));
  }
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const int e = i * 64 + lane;
    key[i] = l[i];
    if (a.bias || a.groups > 1) {
      const double c = s[i] + (a.bias && e < E ? (double)a.bias[e] : 0.0);
      key[i] = c > -INFINITY && l[i] > -INFINITY ? c : -INFINITY;
    }
  }
  if constexpr (MG > 0) if (a.groups > 1) {
    const int n = E / a.groups;
    wave_lds_fence();
#pragma unroll
    for (int i = 0; i < NE; ++i) lds.key[i * 64 + lane] = key[i];
    wave_lds_fence();
    for (int g = lane; g < a.groups; g += 64) {
      double x = -INFINITY, y = -INFINITY;
#pragma unroll 8
      for (int j = 0; j < n; ++j) {
        const double c = lds.key[g * n + j];
        y = fmax(y, fmin(x, c));
        x = fmax(x, c);
      }
      lds.gval[g] = y == -INFINITY ? x : x + y;
    }
    wave_lds_fence();
    for (int g = lane; g < a.groups; g += 64) {
      const double v = lds.gval[g];
      int rank = 0;
#pragma unroll 8
      for (int h = 0; h < a.groups; ++h) rank += lds.gval[h] > v || (lds.gval[h] == v && h < g);
      lds.keep[g] = rank < a.top_groups;
    }
    wave_lds_fence();
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const int e = i * 64 + lane;
      if (e < E && !lds.keep[e / n]) key[i] = -INFINITY;
    }
  }
  double mine = 0.0, sum = 0.0;
  int mine_e = -1;
  for (int r = 0; r < a.k; ++r) {
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
    int e = 1 << 30;
    for (uint64_t at = __ballot(best == m); at; at &= at - 1)   // (several lanes: a tie)
      e = min(e, __builtin_amdgcn_readlane(be, __builtin_ctzll(at)));
    double se = 0.0;
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (i * 64 + lane == e) {
        key[i] = -INFINITY;
        se = s[i];
      }
    se = readlane_f64(se, e & 63);
    sum += se;
    if (lane == r) {
      mine = se;
      mine_e = e;
    }
  }
  if (lane < a.k) {
    double v = a.scale * mine;
    if (a.renorm) v = sum > 0.0 ? v / sum : 0.0;
    a.idx[t * a.k + lane] = mine_e;
    a.w[t * a.k + lane] = (float)v;
  }
}

// -------------------------------------------------------------------- float way
constexpr float kRouteMasked = -3e38f;    // a masked expert's value; every other is clamped to +-1e30
constexpr float kRouteNone = -2e38f;      // below: masked
constexpr float kRouteFar = 1e30f;
// Two values of a row held NV a lane are told apart if they differ by more than
// route_eps(NV) max(1, |value|): the element numbers in their low bits move each by at most
// (NV - 1) 2^-23 of its size; the sum of a softmax (NV - 1 additions of a lane, 4 of the
// team) moves their difference, 1 at most, by (NV + 3) 2^-24; and 1e-6 is for the scores by
// themselves (2 * 4.1e-7: v_exp_f32 and v_rcp_f32 of 1 ulp each, the rounded argument of the
// exponential, the product, + b).
constexpr float route_eps(int nv) { return (float)(5 * nv - 1) * 0x1p-24f + 1e-6f; }
// Two groups, sums of two values: 15 2^-22 each for the lane's number in the low bits,
// 2^-23 for the sum, and as above for four scores in 32 a lane: 1.12e-5.
constexpr float kRouteGroupEps = 1.25e-5f;
constexpr int kRouteGroupsFast = 16;      // one lane of a team for each group
constexpr int kRouteWaves = 4;            // per block (eight: 32768 tokens, 256 experts 23.6 us, four 22.8)

template <int CTRL>
__device__ __forceinline__ int dpp_i(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true);
}
// Exchanges within 4 lanes (quad_perm) or 16 (row_ror): every lane ends with the result.
template <int LPT>
__device__ __forceinline__ int team_max(int v) {
  if constexpr (LPT == 4) {
    v = max(v, dpp_i<0xB1>(v));
    v = max(v, dpp_i<0x4E>(v));
  } else {
    v = max(v, dpp_i<0x128>(v));
    v = max(v, dpp_i<0x124>(v));
    v = max(v, dpp_i<0x122>(v));
    v = max(v, dpp_i<0x121>(v));
  }
  return v;
}
template <int LPT>
__device__ __forceinline__ float team_sum(float v) {
  if constexpr (LPT == 4) {
    v += dpp_f<0xB1>(v);
    v += dpp_f<0x4E>(v);
  } else {
    v += dpp_f<0x128>(v);
    v += dpp_f<0x124>(v);
    v += dpp_f<0x122>(v);
    v += dpp_f<0x121>(v);
  }
  return v;
}
// The value of the team's lane before this one (of its last lane for the first).
template <int LPT>
__device__ __forceinline__ int team_before(int v) {
  if constexpr (LPT == 4) return dpp_i<0x93>(v);   // quad_perm 3 0 1 2
  else return dpp_i<0x121>(v);
}

// A float's place in the order, as a signed integer, and back.  Integers sort without the
// canonicalising copies that a float maximum of unknown bits takes.
__device__ __forceinline__ int order_key(float f) {
  const int i = __float_as_int(f);
  return i ^ (int)((uint32_t)(i >> 31) >> 1);
}
__device__ __forceinline__ float from_order_key(int i) { return __int_as_float(i ^ (int)((uint32_t)(i >> 31) >> 1)); }

// Batcher's odd-even merge sort: the comparisons of N values.
template <int N>
struct SortNet {
  int n = 0;
  uint8_t a[N * 6] = {}, b[N * 6] = {};
  constexpr SortNet() {
    for (int p = 1; p < N; p *= 2)
      for (int q = p; q >= 1; q /= 2)
        for (int j = q % p; j <= N - 1 - q; j += 2 * q)
          for (int i = 0; i < q; ++i)
            if (i + j + q < N && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
              a[n] = (uint8_t)(i + j);
              b[n++] = (uint8_t)(i + j + q);
            }
  }
};
// f(0), f(1), .. f(N - 1), the number a constant of each.
template <typename F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each_of(F f) {
  each_of(f, std::make_integer_sequence<int, N>{});
}
template <int N>
__device__ __forceinline__ void sort_desc(int (&v)[N]) {
  each_of<SortNet<N>().n>([&](auto i) __attribute__((always_inline)) {
    constexpr SortNet<N> net;
    constexpr int a = net.a[decltype(i)::value], b = net.b[decltype(i)::value];
    const int hi = max(v[a], v[b]);
    v[b] = min(v[a], v[b]);
    v[a] = hi;
  });
}

// Lane j's chunks of a row of E >= 4: experts 4 (j + LPT c) .., those past its end `none`.
// One load a chunk from inside the row (of any alignment); where E is no multiple of four
// the last is shifted.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
template <int LPT, int NCH>
__device__ __forceinline__ void load_row(const float* row, int j, int E, float none, float (&v)[4 * NCH]) {
  int past[NCH];
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int e = 4 * (j + LPT * c), at = min(e, E - 4);
    past[c] = e - at;
    const f32x4 x = *reinterpret_cast<const f32x4_any*>(row + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[4 * c + i] = x[i];
  }
  if (E & 3) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const float x1 = v[4 * c + 1], x2 = v[4 * c + 2], x3 = v[4 * c + 3];
      v[4 * c + 3] = past[c] > 0 ? none : x3;
      v[4 * c + 2] = past[c] > 1 ? none : past[c] > 0 ? x3 : x2;
      v[4 * c + 1] = past[c] > 2 ? none : past[c] > 1 ? x3 : past[c] > 0 ? x2 : x1;
      v[4 * c] = past[c] > 3 ? none : past[c] > 2 ? x3 : past[c] > 1 ? x2 : past[c] > 0 ? x1 : v[4 * c];
    }
  } else if (E < 4 * LPT * NCH) {
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * c + i] = past[c] > 0 ? none : v[4 * c + i];
  }
}

// exp(l - m): e^d (1 + what the rounding of d = l - m has lost), which is up to half of 2^-17
// for the scores of e^-64 and below, 64 half steps of the result.
__device__ __forceinline__ float exp_diff(float l, float m) {
  const float d = l - m, b = l - d;
  const float lost = (l - (d + b)) - (m - b);
  const float s = expf(d);
  return fmaf(s, lost, s);
}

// LPT lanes per token, NCH chunks of four experts per lane (chunk c of lane j: experts
// 4 (j + LPT c) ..), up to KT choices.
template <int LPT, int NCH, int KT, bool GROUPS>
__global__ __launch_bounds__(64 * kRouteWaves) void route_kernel(RouteArgs a) {
  constexpr int NV = 4 * NCH, TPW = kWave / LPT, NE = (LPT * NV + 63) / 64;
  constexpr int NL = NV < KT + 1 ? NV : KT + 1;     // entries of a lane's sorted list that can matter
  constexpr int NM = KT / LPT + 1;                  // rounds (the choices and the next best) a lane keeps
  const int masked = order_key(kRouteMasked), none = order_key(kRouteNone);
  __shared__ RouteLds<NE, GROUPS ? kRouteGroupsFast : 0> lds[kRouteWaves];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int j = lane % LPT, team = lane / LPT;
  const int E = a.E, k = a.k;
  const bool use_c = a.bias || GROUPS;                                   // the choice is by c, else by the logits
  const bool soft = a.score == MOE_SCORE_SOFTMAX;
  const bool use_z = soft && (use_c || !a.renorm);

  const int64_t tb = a.first + ((int64_t)blockIdx.x * kRouteWaves + wv) * TPW;   // the wave's tokens
  uint64_t redo = 0;
  if (tb < a.T) {
    const int64_t t = tb + team;
    const bool on = t < a.T;
    const float* row = a.logits + (on ? t : a.T - 1) * E;
    float v[NV];
    load_row<LPT, NCH>(row, j, E, -INFINITY, v);
    float m = kRouteMasked;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      v[i] = v[i] > -INFINITY ? fmaxf(v[i], -kRouteFar) : kRouteMasked;   // (a NaN compares false)
      m = fmaxf(m, v[i]);
    }
    bool amb = m > kRouteFar;   // (among them +inf)
    float z = 1.f;
    if (soft) {
      m = from_order_key(team_max<LPT>(order_key(m)));
      amb |= m <= -kRouteFar && m > kRouteNone;   // no live logit above the clamp: the shares are those of the logits themselves
    }
    if (use_c || use_z) {
      // scores; 0 for a masked expert but in rows without any other
      float x[NV];
      if (soft) {
        z = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          x[i] = __builtin_amdgcn_exp2f((v[i] - m) * 1.44269504f);
          z += x[i];
        }
        z = team_sum<LPT>(z);
        const float rz = __builtin_amdgcn_rcpf(z);
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] *= rz;
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v[i] * -1.44269504f));
      }
      if (use_c) {
        if (a.bias) {
          float b[NV];
          load_row<LPT, NCH>(a.bias, j, E, 0.f, b);
#pragma unroll
          for (int i = 0; i < NV; ++i) {   // (a NaN compares false, and the clamp of one is not looked at)
            x[i] += b[i];
            x[i] = x[i] > -INFINITY ? __builtin_amdgcn_fmed3f(x[i], -kRouteFar, kRouteFar) : kRouteMasked;
          }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = v[i] > kRouteNone ? x[i] : kRouteMasked;
      }
    }
    if constexpr (GROUPS) {
      static_assert(sizeof(float2) * TPW * LPT * NCH <= sizeof(lds[0].key), "the chunks' two largest share the exact way's memory");
      float2* mine = (float2*)lds[wv].key + team * (LPT * NCH);
      wave_lds_fence();
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const float h0 = fmaxf(v[4 * c], v[4 * c + 1]), l0 = fminf(v[4 * c], v[4 * c + 1]);
        const float h1 = fmaxf(v[4 * c + 2], v[4 * c + 3]), l1 = fminf(v[4 * c + 2], v[4 * c + 3]);
        mine[j + LPT * c] = make_float2(fmaxf(h0, h1), fmaxf(fminf(h0, h1), fmaxf(l0, l1)));
      }
      wave_lds_fence();
      const int n4 = E / a.groups / 4;      // chunks of a group
      const float rn4 = 1.f / (float)n4;
      float x = kRouteMasked, y = kRouteMasked;
      if (j < a.groups) {
#pragma unroll 4
        for (int q = 0; q < n4; ++q) {
          const float2 f = mine[j * n4 + q];
          y = fmaxf(fmaxf(y, f.y), fminf(x, f.x));
          x = fmaxf(x, f.x);
        }
      }
      const float gv = x > kRouteNone ? (y > kRouteNone ? x + y : x) : kRouteMasked;
      const float big = x > kRouteNone ? fmaxf(fabsf(x), y > kRouteNone ? fabsf(y) : 0.f) : 0.f;
      const float most = from_order_key(team_max<LPT>(order_key(big)));
      amb |= most >= kRouteFar;   // a clamped value keeps its place in the order, but not in a sum
      const float eps = kRouteGroupEps * fmaxf(1.f, most);
      // The best groups one after the other (the lane in the low bits keeps them apart).
      const int gk = j < a.groups ? (order_key(gv) & ~15) | (15 - j) : (int)0x80000000;
      int rest = gk, last = 0;
      for (int i = 0; i < a.top_groups; ++i) {
        last = team_max<LPT>(rest);
        rest = rest == last ? (int)0x80000000 : rest;
      }
      const int next = team_max<LPT>(rest);
      amb |= next > none && from_order_key(last) - from_order_key(next) <= eps;
      const uint32_t kept = (uint32_t)(__ballot(gk >= last) >> (lane & 48));
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        // (whole numbers below 128 and a reciprocal within 2^-24: the half keeps the quotient exact)
        const int g = (int)(((float)(j + LPT * c) + 0.5f) * rn4);
        const bool out = !((kept >> (g & 15)) & 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * c + i] = out ? kRouteMasked : v[4 * c + i];
      }
    }
    // The element's number in the low bits: the values of a lane are distinct, and sort with it.
    int key[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) key[i] = (order_key(v[i]) & ~(NV - 1)) | i;
    sort_desc(key);
    // Round r finds the team's r-th largest among the heads of the lanes' lists (KT + 1
    // rounds whatever k is: leaving early costs more in branches than the rounds).  Lane
    // r keeps it, and the lanes that hold it.
    int kept_key[NM];
    uint32_t kept_at[NM];
#pragma unroll
    for (int q = 0; q < NM; ++q) {
      kept_key[q] = masked;
      kept_at[q] = 1;
    }
    each_of<KT + 1>([&](auto rc) __attribute__((always_inline)) {
      constexpr int r = decltype(rc)::value;
      const int M = team_max<LPT>(key[0]);
      const bool win = key[0] == M;
      const uint32_t at = (uint32_t)(__ballot(win) >> (lane & ~(LPT - 1)));
      kept_key[r / LPT] = j == r % LPT ? M : kept_key[r / LPT];
      kept_at[r / LPT] = j == r % LPT ? at : kept_at[r / LPT];
      if constexpr (r < KT) {
#pragma unroll
        for (int q = 0; q + 1 < NL; ++q) key[q] = win ? key[q + 1] : key[q];
        key[NL - 1] = win ? masked : key[NL - 1];
      }
    });
    // Neighbours in the order too close to tell, the next best after the last choice too.
#pragma unroll
    for (int q = 0; q < NM; ++q) {
      const int r = q * LPT + j;
      // (both exchanges by every lane: in the arms of a condition their sources would be idle)
      const int here = team_before<LPT>(kept_key[q]), there = team_before<LPT>(kept_key[q > 0 ? q - 1 : 0]);
      const int before = j == 0 ? there : here;
      const float x = from_order_key(kept_key[q]), p = from_order_key(before);
      amb |= r >= 1 && r <= k && x > kRouteNone && p - x <= route_eps(NV) * fmaxf(1.f, fabsf(p));
      amb |= r <= k && x > kRouteNone && __popc(kept_at[q] & (LPT == 16 ? 0xffffu : 0xfu)) > 1;   // two alike
    }
    float s[NM], sum = 0.f;
    int e[NM];
#pragma unroll
    for (int q = 0; q < NM; ++q) {
      const int r = q * LPT + j;
      s[q] = 0.f;
      e[q] = -1;
      if (r < k && kept_key[q] > none) {
        const int i = kept_key[q] & (NV - 1);
        e[q] = 4 * (__builtin_ctz(kept_at[q]) + LPT * (i >> 2)) + (i & 3);
        const float l = row[e[q]];
        s[q] = soft ? exp_diff(l, m) : 1.f / (1.f + expf(-l));
        // Next to float's smallest numbers.  (A plain softmax's weight is its share times the scale:
        // below e^-210 that is none whatever the scale is.)
        const float x = soft ? l - m : l;
        amb |= x < -80.f && (a.renorm || !soft || x > -210.f);
      }
      sum += s[q];
    }
    float f = a.scale;
    if (a.renorm) {
      sum = team_sum<LPT>(sum);
      f = sum > 0.f ? a.scale / sum : 0.f;
      amb |= f == INFINITY;   // a weight is at most the scale, whatever its factors are
    } else if (soft) {
      f = a.scale / z;
    }
    redo = __ballot(amb && on);
    const uint64_t lanes = (LPT == 16 ? 0xffffull : 0xfull) << (lane & ~(LPT - 1));
    if (on && !(redo & lanes)) {
#pragma unroll
      for (int q = 0; q < NM; ++q) {
        const int r = q * LPT + j;
        if (r < k) {
          a.idx[t * k + r] = e[q];
          a.w[t * k + r] = s[q] * f;
        }
      }
    }
  }
  while (redo) {
    const int l = __builtin_ctzll(redo) / LPT;
    redo &= ~((LPT == 16 ? 0xffffull : 0xfull) << (l * LPT));
    route_exact(a, tb + l, lds[wv]);
  }
}

// Every token the exact way.
template <int NE>
__global__ __launch_bounds__(256) void route_exact_kernel(RouteArgs a) {
  __shared__ RouteLds<NE, 64 * NE> lds[4];
  const int wv = threadIdx.x >> 6;
  for (int64_t t = (int64_t)blockIdx.x * 4 + wv; t < a.T; t += (int64_t)gridDim.x * 4) route_exact(a, t, lds[wv]);
}

// load[e] += the choices of e.  A launch of its own, with few blocks: a count is one
// address, and atomics on it are served one after the other (from every routing block
// they took 12 us of 28 for 32768 tokens; integers, so their order changes nothing).
constexpr int kLoadThreads = 1024;
__global__ __launch_bounds__(kLoadThreads) void route_load_kernel(const int32_t* __restrict__ idx, int64_t n, int E,
                                                                  int32_t* __restrict__ load) {
  __shared__ int32_t hist[kRouterMaxE];
  for (int e = threadIdx.x; e < E; e += kLoadThreads) hist[e] = 0;
  __syncthreads();
  const int64_t step = (int64_t)gridDim.x * kLoadThreads;
#pragma unroll 4
  for (int64_t i = (int64_t)blockIdx.x * kLoadThreads + threadIdx.x; i < n; i += step) {
    const int e = idx[i];
    if (e >= 0) atomicAdd(&hist[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kLoadThreads)
    if (hist[e]) atomicAdd(load + e, hist[e]);
}

template <int LPT, int NCH, bool GROUPS>
static void launch_route_n(const RouteArgs& a, hipStream_t s) {
  const int64_t tokens = (int64_t)kRouteWaves * (kWave / LPT);   // of a block
  const int64_t most = tokens << 22;                             // of a launch (its thread count is 32 bits)
  auto go = [&](auto kern) {
    RouteArgs b = a;
    for (b.first = 0; b.first < a.T; b.first += most) {
      const int64_t n = std::min(a.T - b.first, most);
      launch_kernel(kern, dim3((unsigned)((n + tokens - 1) / tokens)), dim3(64 * kRouteWaves), 0, s, b);
    }
  };
  if (a.k <= 2) go(route_kernel<LPT, NCH, 2, GROUPS>);
  else if (a.k <= 4) go(route_kernel<LPT, NCH, 4, GROUPS>);
  else if (a.k <= 8) go(route_kernel<LPT, NCH, 8, GROUPS>);
  else go(route_kernel<LPT, NCH, 16, GROUPS>);
}

void launch_route(const moe_route_cfg& c, const float* logits, const float* bias, int32_t* idx, float* w,
                  int32_t* load, hipStream_t s) {
  if (c.T == 0) return;
  const RouteArgs a{logits, bias, idx, w, c.T, c.E, c.k, c.score, c.renorm, c.groups, c.top_groups, c.scale, 0};
  // E < 4 has no whole load; groups that are no whole chunks or more than a team's lanes
  // have no place in it.  (All in double: E 64, k 8, 64 tokens 4.5 us where it takes 3.1,
  // 65536 71 where it takes 9.4.)
  if (c.E < 4 || (c.groups > 1 && (c.groups > kRouteGroupsFast || (c.E / c.groups) % 4 != 0))) {
    const unsigned blocks = (unsigned)std::min<int64_t>((c.T + 3) / 4, 8 * num_cus());
    auto go = [&](auto kern) { launch_kernel(kern, dim3(blocks), dim3(256), 0, s, a); };
    if (c.E <= 64) go(route_exact_kernel<1>);
    else if (c.E <= 128) go(route_exact_kernel<2>);
    else if (c.E <= 256) go(route_exact_kernel<4>);
    else go(route_exact_kernel<8>);
  } else if (c.groups > 1) {
    if (c.E <= 64) launch_route_n<16, 1, true>(a, s);
    else if (c.E <= 128) launch_route_n<16, 2, true>(a, s);
    else if (c.E <= 256) launch_route_n<16, 4, true>(a, s);
    else launch_route_n<16, 8, true>(a, s);
  } else {
    // Teams of 4 take fewer instructions a token, teams of 16 have shorter chains.  Up to 16
    // experts 4 lanes hold a row in a load each (top-2, us, 4 and 16 lanes: 64 tokens 2.4 and
    // 2.7, 65536 3.4 and 6.7); up to 64 it is 16 lanes until a CU's waves are many (E 64, k 8:
    // 8192 tokens 6.5 and 5.0, 24000 6.8 and 6.5, 32768 7.2 and 7.6, 65536 9.4 and 10.7); above
    // it is 16 (E 128, k 8: 64 tokens 4.1 and 3.3, 65536 16.1 and 13.8).
    if (c.E <= 16) launch_route_n<4, 1, false>(a, s);
    else if (c.E <= 64 && c.T > 96 * num_cus()) launch_route_n<4, 4, false>(a, s);
    else if (c.E <= 64) launch_route_n<16, 1, false>(a, s);
    else if (c.E <= 128) launch_route_n<16, 2, false>(a, s);
    else if (c.E <= 256) launch_route_n<16, 4, false>(a, s);
    else launch_route_n<16, 8, false>(a, s);
  }
  if (load) {
    const int64_t n = c.T * c.k;
    const unsigned blocks = (unsigned)std::min<int64_t>((n + 4 * kLoadThreads - 1) / (4 * kLoadThreads), 64);
    launch_kernel(route_load_kernel, dim3(blocks), dim3(kLoadThreads), 0, s, (const int32_t*)idx, n, c.E, load);
  }
}

// ------------------------------------------------------------------- gradient
// Bound by writing dlogits, most of it zeros (a plain softmax also reads the logits, a sigmoid
// those of the choices, with 8 of 256 most lines of a row).  A wavefront builds its tokens' rows in LDS and stores them as one run
// (32768 tokens, 256 experts, k 8: 8.8 us; k shuffles a token and scattered stores 16.8).
struct RouteBwdArgs {
  const float* logits;
  const int32_t* idx;
  const float *w, *dw;
  float* dlogits;
  int64_t T;
  int32_t E, k, score, renorm;
  float scale;
  int64_t first;
};
constexpr int kBwdWaves = 4;
constexpr int kBwdLds = 2048;   // floats of a wave

// Lane (token i / KP, choice i % KP) of the wave's tokens: its part of the gradient, and G
// (renorm: G / scale, from shares, which no scale takes past float's range).
template <int KP>
__device__ __forceinline__ float choice_grad(const RouteBwdArgs& a, int64_t t, int r, bool on, int& e, float& G) {
  e = -1;
  float w = 0.f, g = 0.f;
  if (on && r < a.k) {
    e = a.idx[t * a.k + r];
    if (e < 0 || e >= a.E) e = -1;
    if (e >= 0) {
      w = a.w[t * a.k + r];
      g = a.dw[t * a.k + r];
    }
  }
  G = (a.renorm ? w / a.scale : w) * g;
  if constexpr (KP >= 2) G += dpp_f<0xB1>(G);
  if constexpr (KP >= 4) G += dpp_f<0x4E>(G);
  if constexpr (KP >= 8) G += dpp_f<0x141>(G);    // row_half_mirror
  if constexpr (KP >= 16) G += dpp_f<0x140>(G);   // row_mirror
  float v = w * (a.renorm ? g - G : g);
  if (a.score == MOE_SCORE_SIGMOID && e >= 0) v *= 1.f / (1.f + expf(a.logits[t * a.E + e]));   // 1 - s
  return v;
}

// Every score but the plain softmax: k elements of a row are not zero.
template <int KP>
__global__ __launch_bounds__(64 * kBwdWaves) void route_bwd_kernel(RouteBwdArgs a, int tokens) {
  __shared__ __attribute__((aligned(16))) float rows[kBwdWaves][kBwdLds];
  const int lane = threadIdx.x & 63;
  float* mine = rows[threadIdx.x >> 6];
  const int64_t tb = a.first + ((int64_t)blockIdx.x * kBwdWaves + (threadIdx.x >> 6)) * tokens;   // (a multiple of 4)
  if (tb >= a.T) return;
  const int64_t left = (a.T - tb) * a.E;
  const int n = (int)(left < tokens * a.E ? left : tokens * a.E);   // elements of the wave's rows
  int e;
  float G;
  const int tok = lane / KP;
  const float v = choice_grad<KP>(a, tb + tok, lane % KP, tok < tokens && tb + tok < a.T, e, G);
  for (int i = 4 * lane; i < n; i += 256) *reinterpret_cast<f32x4*>(mine + i) = f32x4{0.f, 0.f, 0.f, 0.f};
  wave_lds_fence();
  if (e >= 0) unsafeAtomicAdd(mine + tok * a.E + e, v);   // (a row may name an expert twice)
  wave_lds_fence();
  float* out = a.dlogits + tb * a.E;
  for (int i = 4 * lane; i < (n & ~3); i += 256) *reinterpret_cast<f32x4*>(out + i) = *reinterpret_cast<const f32x4*>(mine + i);
  if (lane < (n & 3)) out[(n & ~3) + lane] = mine[(n & ~3) + lane];
}

// The plain softmax: 16 lanes per token, lane j experts j, j + 16, ...
template <int NV>
__global__ __launch_bounds__(64 * kBwdWaves) void route_bwd_softmax_kernel(RouteBwdArgs a) {
  __shared__ float rows[kBwdWaves][4][16 * NV];
  const int lane = threadIdx.x & 63, j = lane & 15, team = lane >> 4;
  float* mine = rows[threadIdx.x >> 6][team];
  const int64_t t = a.first + ((int64_t)blockIdx.x * kBwdWaves + (threadIdx.x >> 6)) * 4 + team;
  const bool on = t < a.T;
  const float* row = a.logits + (on ? t : a.T - 1) * a.E;
  float l[NV], m = -INFINITY, z = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int x = j + 16 * i;
    l[i] = x < a.E ? row[x] : -INFINITY;
  }
  int e;
  float G;
  const float v = choice_grad<16>(a, t, j, on, e, G);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    l[i] = l[i] > -INFINITY ? l[i] : -INFINITY;   // (a NaN compares false)
    m = fmaxf(m, l[i]);
    mine[j + 16 * i] = 0.f;
  }
  m = from_order_key(team_max<16>(order_key(m)));
  float p[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    p[i] = l[i] == -INFINITY ? 0.f : l[i] == m ? 1.f : expf(l[i] - m);   // (+inf logits: an even share)
    z += p[i];
  }
  z = team_sum<16>(z);
  const float f = z > 0.f ? -G / z : 0.f;
  wave_lds_fence();
  if (e >= 0) unsafeAtomicAdd(mine + e, v);
  wave_lds_fence();
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int x = j + 16 * i;
    if (on && x < a.E) a.dlogits[t * a.E + x] = mine[x] + f * p[i];
  }
}

void launch_route_bwd(const moe_route_cfg& c, const float* logits, const int32_t* idx, const float* w,
                      const float* dw, float* dlogits, hipStream_t s) {
  if (c.T == 0) return;
  const RouteBwdArgs a{logits, idx, w, dw, dlogits, c.T, c.E, c.k, c.score, c.renorm, c.scale, 0};
  auto slices = [&](int tokens, auto launch) {   // tokens of a wave; a launch's thread count is 32 bits
    const int64_t per = (int64_t)kBwdWaves * tokens, most = per << 23;
    RouteBwdArgs b = a;
    for (b.first = 0; b.first < c.T; b.first += most)
      launch(b, dim3((unsigned)((std::min(c.T - b.first, most) + per - 1) / per)));
  };
  if (c.score == MOE_SCORE_SOFTMAX && !c.renorm) {
    auto go = [&](auto kern) {
      slices(4, [&](const RouteBwdArgs& b, dim3 grid) { launch_kernel(kern, grid, dim3(64 * kBwdWaves), 0, s, b); });
    };
    if (c.E <= 16) go(route_bwd_softmax_kernel<1>);
    else if (c.E <= 64) go(route_bwd_softmax_kernel<4>);
    else if (c.E <= 128) go(route_bwd_softmax_kernel<8>);
    else if (c.E <= 256) go(route_bwd_softmax_kernel<16>);
    else go(route_bwd_softmax_kernel<32>);
    return;
  }
  // As many tokens a wave as its choices have lanes and its rows have room in LDS.
  int kp = 1, tokens = 4;
  while (kp < c.k) kp *= 2;
  while (tokens * 2 * kp <= kWave && tokens * 2 * c.E <= kBwdLds) tokens *= 2;
  auto go = [&](auto kern) {
    slices(tokens, [&](const RouteBwdArgs& b, dim3 grid) {
      launch_kernel(kern, grid, dim3(64 * kBwdWaves), 0, s, b, tokens);
    });
  };
  if (kp == 1) go(route_bwd_kernel<1>);
  else if (kp == 2) go(route_bwd_kernel<2>);
  else if (kp == 4) go(route_bwd_kernel<4>);
  else if (kp == 8) go(route_bwd_kernel<8>);
  else go(route_bwd_kernel<16>);
}

}  // namespace lmoe
