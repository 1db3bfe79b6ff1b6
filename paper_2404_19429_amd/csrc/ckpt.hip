// 8-bit checkpoint of the expert buffers: 64 columns of a row share a float step =
// max|x| / 127, a value is the integer nearest to 127 x / max|x|.
//
// One pass over the data, memory-bound: a wavefront takes units of 16 rows x 64
// columns.  Lane l holds 16 values of row l / 4, so a group is four neighbouring
// lanes and its maximum two cross-lane steps; the codes of a unit are 1 KiB in lane
// order (16 bytes a lane), its steps 16 floats.  In the 16 x 32-block layout a unit
// is two neighbouring blocks, 2 KiB in a run; in a row-major buffer 16 row pieces.
//
// A checkpoint is the three buffers in turn (send_buf, H, expert_out), each its codes
// [E][rows / 16][columns / 64][1024] and then its steps [E][rows / 16][columns / 64][16].
#include "internal.h"

namespace lmoe {

constexpr int64_t kUnitRows = 16, kUnitCols = 64, kUnitCodes = kUnitRows * kUnitCols;
constexpr int kCkptUnits = 8;   // units of one wave

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

// The lane's 16 values of a unit: addresses of their 16-byte pieces (bf16: two, float: four).
template <typename T>
__device__ __forceinline__ int64_t piece_off(const CkptPart& p, int64_t base, int64_t row, int64_t col, int h) {
  // base: the expert's first element.  Blocked: piece h is the lane's part of block h of
  // the unit's two; row-major: pieces follow each other.
  if constexpr (sizeof(T) == 2) {
    if (p.blocked) return base + blk_off(row, (col & ~63) + 32 * h + ((col & 63) >> 1), p.X);
    return base + row * p.X + col + 8 * h;
  } else {
    return base + row * p.X + col + 4 * h;
  }
}

// The integer nearest to 127 x / amax.  x * (127 / amax) is within 2^-23 * 127 of it;
// next to a half the quotient in double decides (its rounding cannot reach the half
// unless the exact quotient is it: both operands have at most 31 bits).
__device__ __forceinline__ float nearest_code(float x, float inv, float amax) {
  const float t = x * inv;
  float q = rintf(t);
  if (fabsf(t - q) > 0.4999f) q = (float)rint((double)x * 127.0 / (double)amax);
  return q;
}

template <typename T>
__global__ __launch_bounds__(256) void ckpt_save_kernel(CkptArgs a) {
  constexpr int V = Vec<T>::N, NP = 16 / V;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  for (int64_t b = blockIdx.x; b < a.blocks; b += gridDim.x) {
    const int64_t er = b / a.strips;
    const int e = (int)(er / a.urows), ur = (int)(er % a.urows);
    const int lo = a.rb ? max(a.rb[e], 0) : 0, hi = min(a.re[e], a.C);
    if (ur * 16 >= hi || ur * 16 + 16 <= lo) continue;
    const int row = ur * 16 + (lane >> 2);
    const bool live = row >= lo && row < hi;
    const int u0 = ((int)(b % a.strips) * 4 + wv) * kCkptUnits;
    for (int u = u0; u < min(u0 + kCkptUnits, a.ucols); ++u) {
      const CkptPart& p = a.part[u >= a.part[2].first ? 2 : u >= a.part[1].first ? 1 : 0];
      if (!p.buf) continue;
      const int uc = u - p.first;
      const int col = uc * 64 + 16 * (lane & 3);
      const T* src = (const T*)p.buf;
      const int64_t base = (int64_t)e * a.rows * p.X;
      float v[16];
#pragma unroll
      for (int h = 0; h < NP; ++h) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[h * V + i] = 0.f;
        if (live && (sizeof(T) == 2 || col + h * V < p.X)) Vec<T>::load(src + piece_off<T>(p, base, row, col, h), v + h * V);
      }
      // the largest magnitude by its bits: infinities and NaN are above every finite value
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
      m = max(m, (uint32_t)__shfl_xor((int)m, 1, kWave));
      m = max(m, (uint32_t)__shfl_xor((int)m, 2, kWave));
      const float amax = __uint_as_float(m);
      const bool bad = m >= 0x7f800000u, tiny = amax < 1e-30f;
      const float inv = bad || tiny ? 0.f : 127.f / amax;
      const float step = bad ? __uint_as_float(0x7fc00000u) : tiny ? 0.f : amax / 127.f;
      u32x4 out;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float q = bad || tiny ? 0.f : nearest_code(v[4 * j + i], inv, amax);
          word |= ((uint32_t)(int)q & 0xffu) << (8 * i);
        }
        out[j] = word;
      }
      const int64_t unit = ((int64_t)e * a.urows + ur) * p.ucols + uc;
      if (live) {
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
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  for (int64_t b = blockIdx.x; b < a.blocks; b += gridDim.x) {
    const int64_t er = b / a.strips;
    const int e = (int)(er / a.urows), ur = (int)(er % a.urows);
    const int lo = a.rb ? max(a.rb[e], 0) : 0, hi = min(a.re[e], a.C);
    if (ur * 16 >= hi || ur * 16 + 16 <= lo) continue;
    const int row = ur * 16 + (lane >> 2);
    const bool live = row >= lo && row < hi;
    const int u0 = ((int)(b % a.strips) * 4 + wv) * kCkptUnits;
    for (int u = u0; u < min(u0 + kCkptUnits, a.ucols); ++u) {
      const CkptPart& p = a.part[u >= a.part[2].first ? 2 : u >= a.part[1].first ? 1 : 0];
      if ((!p.buf && !p.act) || !live) continue;
      const int uc = u - p.first;
      const int col = uc * 64 + 16 * (lane & 3);
      const int64_t unit = ((int64_t)e * a.urows + ur) * p.ucols + uc;
      const u32x4 code = *reinterpret_cast<const u32x4*>(p.codes + unit * kUnitCodes + lane * 16);
      const float step = p.steps[unit * kUnitRows + (lane >> 2)];
      const int64_t base = (int64_t)e * a.rows * p.X;
      float v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = (float)(int8_t)(code[i >> 2] >> (8 * (i & 3))) * step;
#pragma unroll
      for (int h = 0; h < NP; ++h)
        if (sizeof(T) == 2 || col + h * V < p.X) {
          const int64_t off = piece_off<T>(p, base, row, col, h);
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
