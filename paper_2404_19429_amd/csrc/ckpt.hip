// 8-bit checkpoint of the expert buffers: 64 columns of a row share a float step =
// max|x| / 127, a value is the integer nearest to 127 x / max|x|.
//
// One pass over the data, memory-bound: a wavefront takes units of 16 rows x 64
// columns.  Lane l holds 16 values of row l / 4 (16-byte pieces), so a group is four neighbouring
// lanes and its maximum two cross-lane steps; the codes of a unit are 1 KiB in lane
// order (16 bytes a lane), its steps 16 floats.  In the 16 x 32-block layout a unit
// is two neighbouring blocks, 2 KiB in a run; in a row-major buffer 16 row pieces.
// 16384 tokens top-2, d 2048, f 8192: saved in 246 us, restored in 332, 5.2 and 5.5 TB/s,
// what a copy of that size reaches.
//
// A checkpoint is the three buffers in turn (send_buf, H, expert_out), each its codes
// [E][rows / 16][columns / 64][1024] and then its steps [E][rows / 16][columns / 64][16].
#include "internal.h"

namespace lmoe {

constexpr int64_t kUnitRows = 16, kUnitCols = 64, kUnitCodes = kUnitRows * kUnitCols;
// Units of one wave: their loads are all on their way before the first is used (8192 rows,
// d 1024, f 4096, save and load, us: 1 unit 78 and 80, 2 units 70 and 78, 4 units 74 and 80).
constexpr int kCkptUnits = 2;

// One buffer of the checkpoint.
struct CkptPart {
  void* buf;         // the caller's (saving: only read); null: left out
  void* act;         // loading H: act(H) (null: not wanted)
  int8_t* codes;
  float* steps;
  int32_t X, ucols;  // columns; units across them
  int32_t first;     // first unit column of the part among all parts'
  int32_t blocked;   // 1: 16 x 32 blocks
};
struct CkptArgs {
  CkptPart part[3];
  const int32_t *rb, *re;
  int32_t E, C, rows, urows, ucols;   // rows per expert in the buffers; units down; unit columns of all parts
  int32_t strips;                     // blocks across the unit columns
  int64_t blocks;                     // E * urows * strips
};

static int ckpt_rows(const moe_cfg& c) { return c.dtype == MOE_BF16 ? (int)pad16(c.C) : c.C; }

static size_t part_bytes(const moe_cfg& c, int X) {
  const size_t units = (size_t)c.E * ((ckpt_rows(c) + 15) / 16) * ((X + 63) / 64);
  return units * (kUnitCodes + 4 * kUnitRows);
}
size_t ckpt_bytes(const moe_cfg& c) { return 2 * part_bytes(c, c.d_model) + part_bytes(c, c.d_ff); }

// Column of 16-byte piece h (bf16: two, float: four) of the lane's 16 values in unit column
// uc: four neighbouring lanes' pieces are 64 bytes in a run.
template <typename T>
__device__ __forceinline__ int piece_col(int uc, int h) {
  constexpr int V = Vec<T>::N;
  return uc * 64 + 4 * V * h + V * (int)(threadIdx.x & 3);
}
template <typename T>
__device__ __forceinline__ int64_t piece_off(const CkptPart& p, int64_t base, int64_t row, int64_t col) {
  return base + (sizeof(T) == 2 && p.blocked ? blk_off(row, col, p.X) : row * p.X + col);
}

// The integers nearest to 127 x / amax, ties to even, from q = x * RN(127 / amax), which
// is off by less than 2^-23 of itself.
// bfloat16: X and A being the 8-bit significands of x and amax and s the difference of
// their exponents, |127 x / amax - (n + 1/2)| = |254 X - (2n + 1) 2^s A| / (2^(s+1) A) is 0
// or at least 2^-s / 510, and a q in [2^m, 2^(m+1)) has m <= 7 - s: a quotient is half way,
// or further than 2^(m-16) from it.  Rounding q to 19 bits after the first moves it by less
// than 2^(m-19) and brings it back to a half that it should be.
// float: within 2e-5 of a half (127 * 2^-23 is less) the quotient in double decides; its
// rounding cannot reach the half unless the exact quotient is it, both operands having at
// most 31 bits.
template <typename T> __device__ __forceinline__ void round_codes(const float (&x)[16], float amax, float (&q)[16]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i] = rintf(__uint_as_float((__float_as_uint(q[i]) + 8u) & ~15u));
  } else {
    float far = 0.f;
    float r[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      r[i] = rintf(q[i]);
      far = fmaxf(far, fabsf(q[i] - r[i]));
    }
    if (far > 0.49998f) {   // (a lane in 1600)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (fabsf(q[i] - r[i]) > 0.49998f) r[i] = (float)rint((double)x[i] * 127.0 / (double)amax);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) q[i] = r[i];
  }
}

// The rows and units of a wave in strip b: expert, row and the first of its unit columns.
struct CkptWave {
  int e, ur, row, u0;
  bool live;   // the lane's row is in the range
};
// false: no row of the strip is.
__device__ __forceinline__ bool ckpt_wave(const CkptArgs& a, int64_t b, CkptWave& w) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int64_t er = b / a.strips;
  w.e = (int)(er / a.urows);
  w.ur = (int)(er % a.urows);
  const int lo = a.rb ? max(a.rb[w.e], 0) : 0, hi = min(a.re[w.e], a.C);
  w.row = w.ur * 16 + (lane >> 2);
  w.live = w.row >= lo && w.row < hi;
  w.u0 = ((int)(b % a.strips) * 4 + wv) * kCkptUnits;
  return w.ur * 16 < hi && w.ur * 16 + 16 > lo;
}
__device__ __forceinline__ const CkptPart& ckpt_part(const CkptArgs& a, int u) {
  return a.part[u >= a.part[2].first ? 2 : u >= a.part[1].first ? 1 : 0];
}

template <typename T>
__global__ __launch_bounds__(256) void ckpt_save_kernel(CkptArgs a) {
  constexpr int V = Vec<T>::N, NP = 16 / V;
  const int lane = threadIdx.x & 63;
  for (int64_t b = blockIdx.x; b < a.blocks; b += gridDim.x) {
    CkptWave w;
    if (!ckpt_wave(a, b, w)) continue;
    // Every load of the wave's units ahead of the first code.
    u32x4 raw[kCkptUnits][NP];
#pragma unroll
    for (int n = 0; n < kCkptUnits; ++n) {
      const int u = w.u0 + n;
#pragma unroll
      for (int h = 0; h < NP; ++h) raw[n][h] = u32x4{0u, 0u, 0u, 0u};
      if (u >= a.ucols) continue;
      const CkptPart& p = ckpt_part(a, u);
      if (!p.buf || !w.live) continue;
      const T* src = (const T*)p.buf;
      const int64_t base = (int64_t)w.e * a.rows * p.X;
#pragma unroll
      for (int h = 0; h < NP; ++h) {
        const int col = piece_col<T>(u - p.first, h);
        if (sizeof(T) == 2 || col < p.X)   // (bf16 buffers have whole units)
          raw[n][h] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + piece_off<T>(p, base, w.row, col)));
      }
    }
#pragma unroll
    for (int n = 0; n < kCkptUnits; ++n) {
      const int u = w.u0 + n;
      if (u >= a.ucols) break;
      const CkptPart& p = ckpt_part(a, u);
      if (!p.buf) continue;
      float v[16];
#pragma unroll
      for (int h = 0; h < NP; ++h) Vec<T>::load(&raw[n][h], v + h * V);
      // the largest magnitude by its bits: infinities and NaN are above every finite value
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
      m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, true));   // lanes 1, 0, 3, 2 of four
      m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, true));   // lanes 2, 3, 0, 1
      const float amax = __uint_as_float(m);
      const bool bad = m >= 0x7f800000u, tiny = amax < 1e-30f;
      const float inv = bad || tiny ? 0.f : 127.f / amax;
      // (of the largest float the quotient rounds up to a step of which 127 are infinite)
      const float step = bad ? __uint_as_float(0x7fc00000u) : tiny ? 0.f : fminf(amax / 127.f, 0x1.020406p+121f);
      float q[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) q[i] = bad ? 0.f : v[i] * inv;
      round_codes<T>(v, amax, q);
      u32x4 out;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t word = 0;
        // (a code and 2^23 + 2^22: its integer in the low bits)
#pragma unroll
        for (int i = 0; i < 4; ++i) word |= (__float_as_uint(q[4 * j + i] + 12582912.f) & 0xffu) << (8 * i);
        out[j] = word;
      }
      const int64_t unit = ((int64_t)w.e * a.urows + w.ur) * p.ucols + (u - p.first);
      if (w.live) {
        *reinterpret_cast<u32x4*>(p.codes + unit * kUnitCodes + lane * 16) = out;
        if ((lane & 3) == 0) p.steps[unit * kUnitRows + (lane >> 2)] = step;
      }
    }
  }
}

template <typename T, int ACT>
__device__ __forceinline__ float ckpt_act(float h) {
  if constexpr (sizeof(T) == 2 && ACT != MOE_ACT_RELU) return act_fwd_t<ACT>(h);
  else return act_fwd_nan(h, ACT);
}

template <typename T, int ACT>
__global__ __launch_bounds__(256) void ckpt_load_kernel(CkptArgs a) {
  constexpr int V = Vec<T>::N, NP = 16 / V;
  const int lane = threadIdx.x & 63;
  for (int64_t b = blockIdx.x; b < a.blocks; b += gridDim.x) {
    CkptWave w;
    if (!ckpt_wave(a, b, w) || !w.live) continue;
    u32x4 code[kCkptUnits];
    float step[kCkptUnits];
#pragma unroll
    for (int n = 0; n < kCkptUnits; ++n) {
      const int u = w.u0 + n;
      code[n] = u32x4{0u, 0u, 0u, 0u};
      step[n] = 0.f;
      if (u >= a.ucols) continue;
      const CkptPart& p = ckpt_part(a, u);
      if (!p.buf && !p.act) continue;
      const int64_t unit = ((int64_t)w.e * a.urows + w.ur) * p.ucols + (u - p.first);
      code[n] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p.codes + unit * kUnitCodes + lane * 16));
      step[n] = p.steps[unit * kUnitRows + (lane >> 2)];
    }
#pragma unroll
    for (int n = 0; n < kCkptUnits; ++n) {
      const int u = w.u0 + n;
      if (u >= a.ucols) break;
      const CkptPart& p = ckpt_part(a, u);
      if (!p.buf && !p.act) continue;
      const int64_t base = (int64_t)w.e * a.rows * p.X;
      float v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = (float)(int8_t)(code[n][i >> 2] >> (8 * (i & 3))) * step[n];
#pragma unroll
      for (int h = 0; h < NP; ++h) {
        const int col = piece_col<T>(u - p.first, h);
        if (sizeof(T) == 2 || col < p.X) {
          const int64_t off = piece_off<T>(p, base, w.row, col);
          if (p.buf) Vec<T>::store((T*)p.buf + off, v + h * V);
          if (p.act) {
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = ckpt_act<T, ACT>(v[h * V + i]);
            Vec<T>::store((T*)p.act + off, o);
          }
        }
      }
    }
  }
}

static CkptArgs ckpt_args(const moe_cfg& c, const void* send, const void* H, const void* A, const void* O,
                          const int32_t* rb, const int32_t* re, const void* ckpt) {
  CkptArgs a;
  a.rb = rb;
  a.re = re;
  a.E = c.E;
  a.C = c.C;
  a.rows = ckpt_rows(c);
  a.urows = (a.rows + 15) / 16;
  a.ucols = 0;
  const void* buf[3] = {send, H, O};
  const int X[3] = {c.d_model, c.d_ff, c.d_model};
  int8_t* at = (int8_t*)ckpt;
  for (int i = 0; i < 3; ++i) {
    CkptPart& p = a.part[i];
    p.buf = const_cast<void*>(buf[i]);
    p.act = i == 1 ? const_cast<void*>(A) : nullptr;
    p.X = X[i];
    p.ucols = (X[i] + 63) / 64;
    p.first = a.ucols;
    p.blocked = c.dtype == MOE_BF16 && i < 2;
    const size_t units = (size_t)c.E * a.urows * p.ucols;
    p.codes = at;
    p.steps = (float*)(at + units * kUnitCodes);
    at += part_bytes(c, X[i]);
    a.ucols += p.ucols;
  }
  a.strips = (a.ucols + 4 * kCkptUnits - 1) / (4 * kCkptUnits);
  a.blocks = (int64_t)a.E * a.urows * a.strips;
  return a;
}
static dim3 ckpt_grid(const CkptArgs& a) { return dim3((unsigned)std::min<int64_t>(a.blocks, 1 << 20)); }

void launch_ckpt_save(const moe_cfg& c, const void* send, const void* H, const void* O, const int32_t* rb,
                      const int32_t* re, void* ckpt, hipStream_t s) {
  const CkptArgs a = ckpt_args(c, send, H, nullptr, O, rb, re, ckpt);
  if (c.dtype == MOE_BF16) hipLaunchKernelGGL(ckpt_save_kernel<uint16_t>, ckpt_grid(a), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(ckpt_save_kernel<float>, ckpt_grid(a), dim3(256), 0, s, a);
}

void launch_ckpt_load(const moe_cfg& c, const void* ckpt, const int32_t* rb, const int32_t* re, void* send, void* H,
                      void* A, void* O, hipStream_t s) {
  const CkptArgs a = ckpt_args(c, send, H, A, O, rb, re, ckpt);
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, ckpt_grid(a), dim3(256), 0, s, a); };
  auto pick = [&](auto tag) {
    using T = decltype(tag);
    switch (c.act) {
      case MOE_ACT_RELU: go(ckpt_load_kernel<T, MOE_ACT_RELU>); break;
      case MOE_ACT_GELU_TANH: go(ckpt_load_kernel<T, MOE_ACT_GELU_TANH>); break;
      case MOE_ACT_GELU_ERF: go(ckpt_load_kernel<T, MOE_ACT_GELU_ERF>); break;
      default: go(ckpt_load_kernel<T, MOE_ACT_IDENTITY>); break;
    }
  };
  if (c.dtype == MOE_BF16) pick(uint16_t{});
  else pick(float{});
}

}  // namespace lmoe
