// Grouped expert GEMMs over the [E][C][*] dispatch layout.
//
// One launch covers every expert.  Two raggedness modes:
//   ragged-M (forward and dX products): expert e owns buffer rows
//     [rb_e, re_e); C(m, n) = sum_k A(rb_e + m, k) B(k, n) with A row-major
//     (K contiguous).  Tiles past the expert's row count exit at once, so no
//     host read-back of the counts is needed.
//   ragged-K (dW products): C_e = A_e^T B_e reduced over the expert's rows
//     [rb_e, re_e); both operands are row-major in the token dimension, i.e.
//     MN contiguous.  An expert with no rows stores exact zeros.
//
// bf16 path: a persistent kernel with v_mfma_f32_16x16x32_bf16 and float
// accumulation; operand tiles stream global -> LDS asynchronously through a
// multi-stage ring (details below).  Epilogues: plain store, (H, act(H))
// store, dA * act'(H) for the backward, a residual add, and float partials of
// a K-split dense weight gradient.
// The same kernel serves dense products (one group, no row ranges): the
// block's projections and, with row-major operands split into token ranges,
// their weight gradients.
// f32 path: LDS-tiled float MFMAs with the same addressing.
#include "internal.h"
#include "gemm_wide.h"

#include <cmath>
#include <utility>
#include <vector>

namespace lmoe {

// ------------------------------------------------------------------ f32 path
// v_mfma_f32_16x16x4_f32 over LDS tiles, float in, float accumulation.  Bound:
// the matrix cores' float rate (157 TFLOP/s nominal; 119 reached on 4096 x 16384
// x 2048); an MFMA takes 32 cycles for two 4-byte operands per lane, so plain
// loads (global -> registers -> LDS, one stage ahead) and LDS reads hide under
// it where a wave's own MFMAs stand between them and their use: with reads, then
// MFMAs, stage by stage, waves of a SIMD in turn had them busy 72 % of the time
// (113 TFLOP/s).  Unpadded LDS rows for five blocks a CU in place of four need
// more addresses than 96 registers hold (108).  Training step of 2000 tokens
// (d 512, f 2048, 8 experts, one MI355X), against a 64 x 64 tile of vector
// multiply-adds: H 191 -> 113 us, expert_out 358 -> 125, each dW 146 -> 104 (81
// TFLOP/s); a 128-tile was slower on all but dW (its ragged rows and rounds).
//
// A block is 2 x 2 waves of WT x WT fragments of 16 x 16: a tile of 32 WT on a
// side, 64 / WT of K per stage (the same 16 KB of LDS and four 16-byte loads
// per thread and stage for either WT).  The MFMA adds its four products to the
// accumulator one fused multiply-add at a time in K order (measured: the same
// bits as a loop of fmaf), and every element takes its K in ascending order, so
// results do not depend on WT and are those of the plain sum.
// The product is computed transposed: a lane ends with four consecutive output
// columns of one row.
template <int WT, bool KC>
struct F32Tile {
  static constexpr int ROWS = 32 * WT, BK = 64 / WT;   // rows or columns of the operand; K per stage
  static constexpr int LD = KC ? BK + 4 : ROWS + 16;   // padded LDS row: a wave's reads spread over the banks
  static constexpr int ELEMS = (KC ? ROWS : BK) * LD;
  static constexpr int NLD = ROWS * BK / 4 / 256;      // 16-byte loads per thread and stage
  static constexpr int W = KC ? BK / 4 : ROWS / 4;     // chunks per LDS row
  const float* rp[NLD];                                // the thread's row (KC) or column of chunk i, at K = 0
  // KC: [ROWS][K] from row r0 < rlim; else [K][ROWS] from column r0.  Rows or
  // columns past the limit repeat the last (their outputs are not stored).
  __device__ void plan(const float* base, int64_t ld, int r0, int rlim) {
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      const int c = threadIdx.x + 256 * i;
      if constexpr (KC) rp[i] = base + min(r0 + c / W, rlim - 1) * ld;
      else rp[i] = base + min(r0 + 4 * (c % W), rlim - 4);
    }
  }
  __device__ static int kofs(int i) { return KC ? 4 * ((threadIdx.x + 256 * i) % W) : (threadIdx.x + 256 * i) / W; }
  // The stage at k0, from addresses clamped into K (klim > 0): without a branch
  // every load of the stage is in flight together.
  __device__ void load(f32x4 (&v)[NLD], int64_t ld, int k0, int klim) const {
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      const int k = min(k0 + kofs(i), klim - (KC ? 4 : 1));
      v[i] = *reinterpret_cast<const f32x4*>(rp[i] + (KC ? k : k * ld));
    }
  }
  // To LDS, K at and past klim as zeros.  KC: within 16 of K, k = 4 s + q goes
  // to place 4 q + s, so that a lane's elements of four MFMAs are one 16-byte read.
  template <bool WHOLE>
  __device__ static void store(const f32x4 (&v)[NLD], float* st, int k0, int klim) {
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      const int c = threadIdx.x + 256 * i;
      const f32x4 x = WHOLE || k0 + kofs(i) < klim ? v[i] : f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (KC) {
        float* o = st + c / W * LD + (c % W >> 2) * 16 + (c & 3);
#pragma unroll
        for (int q = 0; q < 4; ++q) o[4 * q] = x[q];
      } else {
        *reinterpret_cast<f32x4*>(st + c / W * LD + 4 * (c % W)) = x;
      }
    }
  }
  // The lane's elements of the four MFMAs of the stage's 16-K block kb (K 4 s + lane / 16
  // for MFMA s) for row or column r16 + lane % 16.
  __device__ static f32x4 frag(const float* st, int r16, int kb, int lane) {
    const int r = r16 + (lane & 15), q = lane >> 4;
    if constexpr (KC) {
      return *reinterpret_cast<const f32x4*>(st + r * LD + 16 * kb + 4 * q);
    } else {
      const float* o = st + (16 * kb + q) * LD + r;
      return f32x4{o[0], o[4 * LD], o[8 * LD], o[12 * LD]};
    }
  }
};

template <int EPI>
__device__ __forceinline__ void f32_store(const KernParams<EPI>& p, int64_t off, const f32x4& v) {
  f32x4 o = v;
  if constexpr (EPI == EPI_DACT) {
    const f32x4 h = *reinterpret_cast<const f32x4*>((const float*)p.Aux + off);
#pragma unroll
    for (int u = 0; u < 4; ++u) o[u] = v[u] * act_bwd(h[u], p.act);
  }
  if constexpr (EPI == EPI_ADD) {
    if (p.Aux) o += *reinterpret_cast<const f32x4*>((const float*)p.Aux + off);   // (Aux may be C)
  }
  *reinterpret_cast<f32x4*>((float*)p.C + off) = o;
  if constexpr (EPI == EPI_FWD1) {
#pragma unroll
    for (int u = 0; u < 4; ++u) o[u] = act_fwd(v[u], p.act);
    *reinterpret_cast<f32x4*>((float*)p.C2 + off) = o;
  }
}

// Ragged-M: the tiles of the rows that are there, n fastest, fall into eight
// contiguous ranges, one per XCD (block index modulo 8), so an XCD's L2 holds
// the operands its blocks share and every XCD has the same number of tiles.
// Ragged-K (tiles as long as their group): rows of tn tiles are dealt to the
// XCDs in turn, so a few large experts still spread over the chip.
template <int WT, bool B_K, bool RAGGED_K, int EPI>
__global__ __launch_bounds__(256, 4) void gemm_f32_kernel(KernParams<EPI> p, int tm, int tn, int groups) {
  using TA = F32Tile<WT, !RAGGED_K>;
  using TB = F32Tile<WT, B_K && !RAGGED_K>;
  constexpr int BM = TA::ROWS, BK = TA::BK;
  __shared__ __attribute__((aligned(16))) float As[2][TA::ELEMS];
  __shared__ __attribute__((aligned(16))) float Bs[2][TB::ELEMS];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int xcd = blockIdx.x % 8, local = blockIdx.x / 8;
  int g, m0, n0, lo, span;
  if constexpr (RAGGED_K) {
    const int tr = (local / tn) * 8 + xcd;
    if (tr >= groups * tm) return;
    g = tr / tm;
    m0 = (tr - g * tm) * BM;
    n0 = (local % tn) * BM;
    group_rows(p, g, lo, span);
  } else {
    const WPrefix P = wide_tile_prefix<BM, false, false>(p, lane, groups, tm, tn);
    const int per = (P.NF + 7) / 8, t = xcd * per + local;
    if (local >= per || t >= P.NF) return;
    g = __builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < groups && P.incl <= t)));
    const int q = t - __builtin_amdgcn_readlane(P.excl, g);
    m0 = q / tn * BM;
    n0 = q % tn * BM;
    lo = __builtin_amdgcn_readlane(P.lo, g);
    span = __builtin_amdgcn_readlane(P.span, g);
  }
  // The cross entropy: the gradient at the logits has padding columns (zeros) that W has no rows for; its product
  // with W may be in groups, each a slice of p.ksplit classes.
  const int k0g = EPI == EPI_ADD ? g * p.ksplit : 0;
  const int Mlim = RAGGED_K ? p.M : span, Klim = RAGGED_K ? span : EPI == EPI_ADD ? min(p.ksplit, p.K - k0g) : p.K;
  const int Alim = RAGGED_K ? (Mlim + 3) & ~3 : Mlim;
  int Blim = p.N;
  if constexpr (EPI == EPI_DL) Blim = p.x.cols;
  const int KlimB = EPI == EPI_ADD ? min(p.ksplit, p.M - k0g) : Klim;
  if (m0 >= Mlim) return;
  const float* Ab = (const float*)p.A + g * p.sA + (int64_t)lo * p.lda;
  const float* Bb = (const float*)p.B + g * p.sB + (RAGGED_K ? (int64_t)lo * p.ldb : 0);
  const int wm = (wid >> 1) * 16 * WT, wn = (wid & 1) * 16 * WT;
  f32x4 acc[WT][WT];
#pragma unroll
  for (int i = 0; i < WT; ++i)
#pragma unroll
    for (int j = 0; j < WT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  f32x4 va[TA::NLD], vb[TB::NLD];
  TA ta;
  TB tb;
  ta.plan(Ab, p.lda, m0, Alim);
  tb.plan(Bb, p.ldb, n0, Blim);
  auto load = [&](int k0) {
    ta.load(va, p.lda, k0, Klim);
    tb.load(vb, p.ldb, k0, KlimB);
  };
  auto store = [&](int k0, int buf) {
    if (k0 + BK <= KlimB) {   // (not the last of either operand)
      TA::template store<true>(va, As[buf], k0, Klim);
      TB::template store<true>(vb, Bs[buf], k0, KlimB);
    } else {
      TA::template store<false>(va, As[buf], k0, Klim);
      TB::template store<false>(vb, Bs[buf], k0, KlimB);
    }
  };
  constexpr int KB = BK / 16;
  f32x4 fa[2][WT], fb[2][WT];
  auto frags = [&](int kb, int buf) {
#pragma unroll
    for (int i = 0; i < WT; ++i) fa[kb & 1][i] = TA::frag(As[buf], wm + 16 * i, kb, lane);
#pragma unroll
    for (int j = 0; j < WT; ++j) fb[kb & 1][j] = TB::frag(Bs[buf], wn + 16 * j, kb, lane);
  };
  auto half = [&](int kb, int h) {
#pragma unroll
    for (int s = 2 * h; s < 2 * h + 2; ++s)
#pragma unroll
      for (int i = 0; i < WT; ++i)
#pragma unroll
        for (int j = 0; j < WT; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[kb & 1][j][s], fa[kb & 1][i][s], acc[i][j], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  if (Klim > 0) {
    load(0);
    store(0, 0);
    load(BK);
    __syncthreads();
    frags(0, 0);
  }
  // Nothing is waited for next to what asks for it: under the MFMAs of 16 of K the fragments of the next 16 come from
  // LDS, under the first the next stage goes there and the one after it is asked for (one past the last is not stored),
  // and the barrier (the next stage is in LDS; every wave is past its reads of the stage before this) stands ahead of the
  // last eight, with the next stage's first fragments.
  for (int k0 = 0, buf = 0; k0 < Klim; k0 += BK, buf ^= 1) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      if (kb + 1 < KB) frags(kb + 1, buf);
      __builtin_amdgcn_sched_barrier(0);
      half(kb, 0);
      if (kb == 0 && k0 + BK < Klim) {
        store(k0 + BK, buf ^ 1);
        load(k0 + 2 * BK);
      }
      if (kb == KB - 1 && k0 + BK < Klim) {
        __syncthreads();
        frags(0, buf ^ 1);
      }
      __builtin_amdgcn_sched_barrier(0);
      half(kb, 1);
    }
  }
  if constexpr (EPI == EPI_LSE) {
    xent_lse_rows<WT, WT>(p.x, acc, m0 + wm, n0 + wn, Mlim, p.x.block0 + n0 / BM * 2 + (wid & 1), lane);
    return;
  }
  if constexpr (EPI == EPI_DL) {
#pragma unroll
    for (int i = 0; i < WT; ++i) {
      const XentRow r = xent_row(p.x, m0 + wm + 16 * i + (lane & 15), Mlim);
#pragma unroll
      for (int j = 0; j < WT; ++j) {
        float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
        xent_dl4(p.x, r, v, n0 + wn + 16 * j + 4 * (lane >> 4), true, false);
        acc[i][j] = f32x4{v[0], v[1], v[2], v[3]};
      }
    }
  }
  const int64_t cbase = (int64_t)g * p.sC + (RAGGED_K ? 0 : (int64_t)lo * p.ldc);
#pragma unroll
  for (int i = 0; i < WT; ++i) {
    const int row = m0 + wm + 16 * i + (lane & 15);
    if (row >= Mlim) continue;
#pragma unroll
    for (int j = 0; j < WT; ++j) {
      const int col = n0 + wn + 16 * j + 4 * (lane >> 4);
      if (col < p.N)   // (N is a multiple of 8)
        f32_store<EPI>(p, cbase + (int64_t)row * p.ldc + col, acc[i][j]);
    }
  }
}

template <int WT, bool B_K, bool RAGGED_K, int EPI>
static void launch_f32(const KernParams<EPI>& p, int groups, int64_t rows, int cols, hipStream_t s, int64_t all_rows = 0) {
  // (ragged-M: with up to 15 alignment rows, as wide_tile_prefix counts them; all_rows: the groups' rows together
  // are at most so many)
  const int tm = (int)((rows + (RAGGED_K ? 0 : 15) + 32 * WT - 1) / (32 * WT)), tn = (cols + 32 * WT - 1) / (32 * WT);
  const int64_t mt = all_rows > 0 ? (all_rows + 15 * groups) / (32 * WT) + groups : (int64_t)groups * tm;
  const int64_t blocks = RAGGED_K ? ((int64_t)groups * tm + 7) / 8 * 8 * tn : (mt * tn + 7) / 8 * 8;
  launch_kernel((gemm_f32_kernel<WT, B_K, RAGGED_K, EPI>), dim3((unsigned)blocks), dim3(256), 0, s, p, tm, tn,
                groups);
}

// --------------------------------------------------------------- launchers

// Workspace of the ragged-M bf16 expert products: a partial float tile per
// block, for a K-split last round.
size_t expert_sk_ws_bytes(const moe_cfg& c) { return c.dtype == MOE_BF16 ? (size_t)kSkPartElems * sizeof(float) : 0; }

// Tile choice of the wide kernel's ragged-M products.  A product's blocks
// advance in rounds of per_cu tiles per CU.  A tile takes K / 32 steps of `full`
// ns when the round fills the chip, `part` ns when at most one block is on a CU,
// and `store` ns for its epilogue (two outputs, or an output and H).  The
// larger tile moves fewer bytes per flop (its step is the cheapest per output
// element); the smaller one wastes less on ragged rows and on rounds that leave
// CUs idle.  The constants are measured (whole products on one MI355X divided
// by their steps); the shape with the least modelled time runs.  The rows are
// taken as spread evenly over the groups: how a routing is skewed shows on the
// device only.
// Where the line lies, 256-tiles against the choice: expert_out of 1531 tokens (d
// 768, f 3072, 8 experts) 68 -> 26 us, of 48 tokens (d 1024, f 4096, 16 experts) 75 -> 44,
// of 2048 tokens (d 768) 73 -> 40, of 3108 tokens 78 -> 65; at 4096 tokens
// (d 1024, 16 experts) 128-tiles lose (128 against 110), and the fused products
// keep 256-tiles from 2048 tokens on (37 against 41).  192-row tiles, for rows
// that end just past a multiple of 256: expert_out of 4096 tokens (d 2048, 16
// experts, no K-split) 372 -> 328, of 6000 tokens (d 1536, 32 experts) 178 -> 145;
// of 16384 tokens (8 experts) 256-tiles stay, 948 against 971.
struct TileCost {
  int bm, bn, per_cu;   // per_cu: blocks of this shape on a CU, so a round is per_cu tiles per CU
  double full, part, store;
  void (*run)(const WideCall&, hipStream_t);
  void (*run_rows)(const WideCall&, hipStream_t);
  int wtn;              // columns of a wave's tile
};
static const TileCost kTilesM[] = {{256, 256, 1, 650., 650., 8000., run_wide_256x256, run_rows_256x256, 64},
                                   {192, 256, 1, 560., 560., 7000., run_wide_192x256, run_rows_192x256, 64},
                                   {128, 128, 2, 520., 330., 4500., run_wide_128x128, run_rows_128x128, 64},
                                   {64, 128, 2, 390., 230., 3000., run_wide_64x128, run_rows_64x128, 64},
                                   {64, 64, 2, 300., 190., 2000., run_wide_64x64, run_rows_64x64, 32}};
constexpr int kTileCount = sizeof kTilesM / sizeof kTilesM[0];
static double tile_cost(const TileCost& t, const WideCall& w, int cus) {
  // M-tiles of a group: a mean over the routed rows' spread.
  const double tm = 0.25 * std::ceil(std::max(1., w.expect - w.spread) / t.bm) + 0.5 * std::ceil(w.expect / t.bm) +
                    0.25 * std::ceil((w.expect + w.spread) / t.bm);
  const double tiles = std::ceil(w.groups * tm * std::ceil((double)w.cols / t.bn));
  const double slots = (double)t.per_cu * cus;
  const double rounds = std::floor(tiles / slots), rem = tiles - rounds * slots;
  const double steps = w.p.K / 32., store = w.kind == WK_NK || w.kind == WK_NK_RES || w.kind == WK_KN || w.kind == WK_KN_RM ? t.store / 2 : t.store;
  double last = rem <= 0 ? 0. : steps * (rem <= cus ? t.part : t.full) + store;
  // A K-split last round: its share of a round, and the partial tiles' write and sum.
  if (t.bm == 256 && w.p.ksplit && (w.kind == WK_NK || w.kind == WK_KN) && rounds > 0 && rem > 0 && 4 * rem <= slots)
    last = steps * t.full * rem / slots + 15000.;
  return rounds * (steps * t.full + store) + last;
}
// The tile of a ragged-M product (index into kTilesM).
static int tile_m(const WideCall& w, int cus, int tiles = kTileCount) {
  int best = 0;
  for (int i = 1; i < tiles; ++i)
    if (tile_cost(kTilesM[i], w, cus) < tile_cost(kTilesM[best], w, cus)) best = i;
  return best;
}
// The tile of a ragged-K product: 128 or 256 wide.  A tile is as long as its group
// and its blocks stay on the CUs, so whole rounds decide: 256-tiles one per CU,
// 128-tiles three.  Modelled, in ns per 32 rows of a group: a round of 256-tiles 720
// to half full, 900 full; of 128-tiles 440 where no CU has more than one, 620 two, 850
// three in several rounds and 1000 in a single one (780 with at most 128 operand
// slices of 128, which the L2s then share); 4000 and 2000 for a round's stores, 8000
// and 7000 once, 3000 for an idle launch.  Below 512 rows per group the choice is
// worth 2 us at most, and 128-tiles run.
//
// Measured on one MI355X, one product, 128- against 256-tiles: 128 large tiles of
// 2048 rows (d 512, f 2048, 8 experts) 46 and 57 us; 160 of 11506 rows (d 192, f 2560,
// 16 experts) 350 and 297; 192 (d 768) of 512 rows 25 and 27, of 4096 132 and 119, (d
// 2048, 3 experts) of 2048 55 and 60; 240 (d 640, f 1280, 16 experts) of 2048 122 and 81; 256 (d
// 1024) of 200 20 and 19, of 1024 50 and 41, of 8192 343 and 239; 288 (d 768, f 3072)
// of 512 34 and 38, of 8192 387 and 405; 384 of 512 39 and 40, of 8192 449 and 409;
// 512 of 1024 88 and 73.  Past two rounds of 256-tiles they win or tie at any length.
//
// Routed groups may be skewed, which shows on the device only; there the longest
// group's tiles are the time, and smaller ones share them between CUs (Zipf 1.2,
// capacity twice the mean of 4096 rows: 256 large tiles of 8 experts 152 and 191 us,
// of 64 experts 174 and 194; 512 large tiles 239 and 245, of 1024 rows 72 and 74; 64
// experts of d 832, f 512, 512 large tiles in part-filled columns, 182 and 218).  So up
// to one and a half rounds, and up to two where an idle launch (3 us) is little
// against the product, both shapes are launched and the row counts pick the one that
// runs.
// A single group is as long as it is: no second launch.  Where the model has 256-tiles up
// to 3 us ahead, they are for long groups, and 128-tiles stay for short ones, up to twice as
// long where the operands are few slices.  128- against 256-tiles: 2048 rows (d 1280, f 6656) 54 and 60 us, (d 1536, f
// 14080) 111 and 112; 3000 (d 768, f 12032) 79 and 78; 4096 (d 1792, f 5120) 94 and 101, (d 2816, f 3328) 97 and 102, (d 768,
// f 12800) 106 and 102; 8192 (d 1024, f 10240) 210 and 192; 16384 (d 768, f 14080) 434 and 375.
// The dense weight gradients' groups are token ranges of one length (w.expect): where
// they are not short, 128-tiles take 3/4 of the time of a 256-tile round for the work
// of 192 large tiles.  dW of 256 large tiles and 8192 rows each, 128- against
// 256-tiles (two launches) 645 and 505 us, of 416 tiles and 1260 rows 191 and 170; of
// 512 tiles and 75 rows 45 and 50.
//
// Where other work runs beside the product (the block's weight stream), it fills the
// CUs that a part-filled round leaves idle, and the tile with the least CU time wins:
// 256-tiles from three quarters of a round on.  Block backward on three streams, the choice above
// against 256-tiles: 6 x 2501 tokens (d 1536, f 3072, 4 experts; 288 large tiles, dWo
// 144, dWqkv 432) 2561 and 2296 us, 8 x 2048 (d 1024, f 4096, 8 experts; 512, 64, 192)
// 1877 and 1762; with all products below a full round 128-tiles stay ahead (4 x 500
// tokens, d 512, f 2048, 8 experts; 128, 16, 48) 208 and 244.  (Nor is an idle launch
// little there: its blocks wait for CUs that the other work holds.)
enum TileK { kTileK128, kTileK256, kTileKByRows };
static TileK tile_k(const WideCall& w, int cus) {
  const auto tiles = [&](int t) { return (w.rows + t - 1) / t * ((w.cols + t - 1) / t) * w.groups; };
  const int64_t large = tiles(256);
  if (large > 2 * cus) return kTileK256;
  if (w.beside && 4 * large >= 3 * cus) return kTileK256;
  if (w.kind == WK_WGF32) {
    const int64_t three = cus * 3 / 4;
    return w.expect >= 512. && 3 * ((large + three - 1) / three) >= 4 * ((large + cus - 1) / cus) ? kTileK256
                                                                                                  : kTileK128;
  }
  if (w.expect < 512.) return kTileK128;
  const double steps = w.expect / 32.;
  auto cost = [&](int64_t n, int64_t per, double full, double store, double last) {
    return n / per * (steps * full + store) + (n % per ? steps * last + store : 0.);
  };
  const double fill = (double)(large % cus) / cus;
  const double c256 = 8000. + cost(large, cus, 900., 4000., fill <= 0.5 ? 720. : 540. + 360. * fill);
  const int64_t small = tiles(128), per = 3 * cus, rem = small % per;
  const int64_t slices = ((w.rows + 127) / 128 + (w.cols + 127) / 128) * w.groups;
  const double three = small > per ? 850. : slices <= 128 ? 780. : 1000.;
  const double c128 = 7000. + cost(small, per, three, 2000., rem <= cus ? 440. : rem <= 2 * cus ? 620. : three);
  if (w.groups == 1) return c128 <= c256 + (w.expect <= (slices <= 72 ? 4096. : 2048.) ? 3000. : 0.) ? kTileK128 : kTileK256;
  if (c128 <= c256 + 3000.) return kTileK128;
  return 2 * large <= 3 * cus || c256 >= 1e5 ? kTileKByRows : kTileK256;
}
static void run_wide_any(const WideCall& w, hipStream_t s) {
  if (w.rows <= 0 || w.cols <= 0 || w.groups <= 0) return;
  const bool rows = w.shared || (w.kind >= WK_LSE && w.kind < WK_DW) || w.kind == WK_DW_SCALED;
  if (w.kind < WK_DW) {
    const TileCost& t = kTilesM[tile_m(w, num_cus())];
    return (rows ? t.run_rows : t.run)(w, s);
  }
  const TileK t = tile_k(w, num_cus());
  WideCall q = w;
  q.p.only = t == kTileKByRows ? 1 : 0;
  if (t != kTileK128) (rows ? run_rows_256x256 : run_wide_256x256)(q, s);
  q.p.only = t == kTileKByRows ? 2 : 0;
  if (t != kTileK256) (rows ? run_rows_128x128 : run_wide_128x128)(q, s);
}

// Rows a group is expected to hold, and their standard deviation: the call's
// assignments spread evenly (T is only a hint here: rows may come from elsewhere).
static WideCall expert_call(const moe_cfg& c, WideKind kind, const GemmParams& p, int64_t rows, int cols, bool later) {
  const double expect = c.T > 0 ? std::min<double>(c.C, (double)c.T * c.k / c.E) : c.C;
  const double spread = std::sqrt(expect * (1. - (double)c.k / c.E));
  // A later partition's rows start anywhere in a 16-row block.
  return WideCall{kind, c.act, c.E, rows, cols, expect + (later ? 7.5 : 0.), spread, p};
}
// The tile of a float product: the one whose busiest CU has the least work, tiles
// per CU times area, the 32-tile's extra loads per flop counted as 30 %.
// Measured, 64-tile against 32-tile: expert_out of 2000 tokens (d 512, f 2048, 8
// experts) 136 and 125 us, its H 113 and 123; dW of 63 tokens (d 640, f 1280, 8
// experts) 15 and 23, its H 24 and 15.
static int f32_tile(const WideCall& w, int cus) {
  auto cost = [&](int t, double f) {
    const double n = w.kind >= WK_DW ? std::ceil((double)w.rows / t)
                                     : 0.5 * (std::ceil(std::max(1., w.expect - w.spread) / t) +
                                              std::ceil((w.expect + w.spread) / t));
    return std::ceil(w.groups * n * std::ceil((double)w.cols / t) / cus) * t * t * f;
  };
  const bool fits = (double)w.groups * ((w.rows + 46) / 32) * ((w.cols + 31) / 32) <= 1 << 22;   // bounds the grid
  return fits && cost(32, 1.3) < cost(64, 1.) ? 32 : 64;
}

// Expert products.  bf16: blocked operands, wide tiles; outputs that a later
// product reads (H, A, dH) blocked, the others (expert_out, dXe, which only
// the gathers read, and the dW products) row-major.  float: the float MFMA
// kernel, row-major.
// rows: rows of the output per group (ragged-M: the capacity C, with up to 15
// alignment rows; ragged-K: M); cols: N.
template <bool B_K, bool RAGGED_K, int EPI>
static void run_expert(const moe_cfg& c, WideKind kind, const GemmParams& p, int64_t rows, int cols, hipStream_t s,
                       bool later = false, bool beside = false) {
  if (rows <= 0 || cols <= 0 || c.E <= 0) return;
  WideCall w = expert_call(c, kind, p, rows, cols, later);
  w.beside = beside;
  if (c.dtype != MOE_BF16) {
    if (f32_tile(w, num_cus()) == 32) launch_f32<1, B_K, RAGGED_K, EPI>(p, c.E, rows, cols, s);
    else launch_f32<2, B_K, RAGGED_K, EPI>(p, c.E, rows, cols, s);
    return;
  }
  run_wide_any(w, s);
}

// Rows per expert block of an [E][C][*] buffer (C rounded up to 16 for bf16).
static int64_t rows_alloc(const moe_cfg& c) { return c.dtype == MOE_BF16 ? pad16(c.C) : c.C; }

// Per-product timing (moe_product_timing): while on, each expert product
// launch of this thread is bracketed by a pair of events on its stream (the
// K-split fix-up launch inside the pair); product_times sums them per product.
namespace {
struct ProductTimer {
  bool on = false;
  int dev = -1;
  bool failed = false;
  std::vector<hipEvent_t> pool;      // events of this device, reused after each readout
  size_t next = 0;
  std::vector<std::pair<int, size_t>> rec;   // (product, index of its first event)
};
thread_local ProductTimer g_ptimer;

hipEvent_t ptimer_event() {
  ProductTimer& t = g_ptimer;
  if (t.next == t.pool.size()) {
    hipEvent_t e = nullptr;
    if (hipEventCreate(&e) != hipSuccess) {
      t.failed = true;
      return nullptr;
    }
    t.pool.push_back(e);
  }
  return t.pool[t.next++];
}
// Records the opening event of product `prod` on s; returns false when timing is off.
bool ptimer_begin(int prod, hipStream_t s) {
  ProductTimer& t = g_ptimer;
  if (!t.on) return false;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev != t.dev) {   // events belong to the device timing was started on
    t.failed = true;
    return false;
  }
  const size_t i = t.next;
  hipEvent_t a = ptimer_event(), b = ptimer_event();
  if (!a || !b || hipEventRecord(a, s) != hipSuccess) {
    t.failed = true;
    return false;
  }
  t.rec.push_back({prod, i});
  return true;
}
void ptimer_end(bool begun, hipStream_t s) {
  if (!begun) return;
  ProductTimer& t = g_ptimer;
  if (hipEventRecord(t.pool[t.rec.back().second + 1], s) != hipSuccess) t.failed = true;
}
}  // namespace

hipError_t product_timing(bool on) {
  ProductTimer& t = g_ptimer;
  int dev = 0;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev != t.dev) {   // a different device: the pool's events belong to the old one (left, not destroyed)
    t.pool.clear();
    t.dev = dev;
  }
  t.on = on;
  t.failed = false;
  t.next = 0;
  t.rec.clear();
  return hipSuccess;
}

hipError_t product_times(double* ms, int32_t* counts) {
  ProductTimer& t = g_ptimer;
  for (int q = 0; q < kProducts; ++q) {
    ms[q] = 0.0;
    counts[q] = 0;
  }
  if (t.failed) return hipErrorUnknown;
  for (const auto& r : t.rec) {
    hipError_t e = hipEventSynchronize(t.pool[r.second + 1]);
    float v = 0.f;
    if (e == hipSuccess) e = hipEventElapsedTime(&v, t.pool[r.second], t.pool[r.second + 1]);
    if (e != hipSuccess) return e;
    ms[r.first] += v;
    counts[r.first] += 1;
  }
  t.next = 0;
  t.rec.clear();
  return hipSuccess;
}

void launch_expert_fwd(const moe_cfg& c, const void* X, const int32_t* rb, const int32_t* re, const void* W1,
                       const void* W2, void* H, void* A, void* O, void* ws, hipStream_t s, bool later) {
  const int64_t d = c.d_model, f = c.d_ff, C = c.C, Cp = rows_alloc(c);
  GemmParams p1{X, d, Cp * d, W1, d, f * d, H, f, Cp * f, A, nullptr, rb, re, 0, (int)f, (int)d, c.act, (int)C};
  p1.part = (float*)ws;
  p1.ksplit = c.ksplit;
  bool tb = ptimer_begin(kProdFwd1, s);
  run_expert<true, false, EPI_FWD1>(c, WK_FWD1, p1, C, (int)f, s, later);
  ptimer_end(tb, s);
  GemmParams p2{A, f, Cp * f, W2, f, d * f, O, d, Cp * d, nullptr, nullptr, rb, re, 0, (int)d, (int)f, c.act, (int)C};
  p2.part = (float*)ws;
  p2.ksplit = c.ksplit;
  tb = ptimer_begin(kProdFwd2, s);
  run_expert<true, false, EPI_STORE>(c, WK_NK, p2, C, (int)d, s, later);   // expert_out row-major
  ptimer_end(tb, s);
}

void launch_expert_bwd_dx(const moe_cfg& c, const void* dO, const int32_t* rb, const int32_t* re, const void* H,
                          const void* W1, const void* W2, void* dH, void* dXe, void* ws, hipStream_t s) {
  const int64_t d = c.d_model, f = c.d_ff, C = c.C, Cp = rows_alloc(c);
  // dA = dO W2_e  (B(k=i, n=j) = W2[e][i][j], N contiguous), epilogue dH = dA * act'(H)
  GemmParams p1{dO, d, Cp * d, W2, f, d * f, dH, f, Cp * f, nullptr, H, rb, re, 0, (int)f, (int)d, c.act, (int)C};
  p1.part = (float*)ws;
  p1.ksplit = c.ksplit;
  bool tb = ptimer_begin(kProdDA, s);
  run_expert<false, false, EPI_DACT>(c, WK_DACT, p1, C, (int)f, s);
  ptimer_end(tb, s);
  // dXe = dH W1_e  (B(k=i, n=j) = W1[e][i][j])
  GemmParams p2{dH, f, Cp * f, W1, d, f * d, dXe, d, Cp * d, nullptr, nullptr, rb, re, 0, (int)d, (int)f, c.act, (int)C};
  p2.part = (float*)ws;
  p2.ksplit = c.ksplit;
  tb = ptimer_begin(kProdDXe, s);
  run_expert<false, false, EPI_STORE>(c, WK_KN, p2, C, (int)d, s);   // dXe row-major
  ptimer_end(tb, s);
}

void launch_expert_bwd_dw(const moe_cfg& c, const void* X, const void* A, const void* dO, const void* dH,
                          const int32_t* rb, const int32_t* re, void* dW1, void* dW2, hipStream_t s, bool beside) {
  const int64_t d = c.d_model, f = c.d_ff, C = c.C, Cp = rows_alloc(c);
  // dW2_e [d][f] = dO_e^T A_e : A-operand(m, k) = dO[e][k][m], B(k, n) = A[e][k][n]
  // (wpacked: written in the blocked layout of the packed weights)
  GemmParams p2{dO, d, Cp * d, A, f, Cp * f, dW2, f, d * f, nullptr, nullptr, rb, re, (int)d, (int)f, 0, c.act, (int)C};
  // dW1_e [f][d] = dH_e^T X_e
  GemmParams p1{dH, f, Cp * f, X, d, Cp * d, dW1, d, f * d, nullptr, nullptr, rb, re, (int)f, (int)d, 0, c.act, (int)C};
  const bool blk = c.wpacked && c.dtype == MOE_BF16;
  bool tb = ptimer_begin(kProdDW2, s);
  run_expert<false, true, EPI_STORE>(c, blk ? WK_DW_BLK : WK_DW, p2, d, (int)f, s, false, beside);
  ptimer_end(tb, s);
  tb = ptimer_begin(kProdDW1, s);
  run_expert<false, true, EPI_STORE>(c, blk ? WK_DW_BLK : WK_DW, p1, f, (int)d, s, false, beside);
  ptimer_end(tb, s);
}

// ------------------------------------------------- experts over sorted rows
// The same products over one buffer of rows that the experts share (moe_sorted_*):
// groups without a stride (SharedRows), each on its range of rows, which in bf16 starts at a
// 16-row block; up to kMaxE experts a launch.
namespace {
struct Part {   // experts [e0, e0 + n) of a call
  int e0, n;
};
template <typename F>
void each_part(const moe_sorted_cfg& c, F&& f) {
  for (int e = 0; e < c.E; e += kMaxE) f(Part{e, std::min(kMaxE, c.E - e)});
}

// One product: C rows or, ragged-K, C_e = A_e^T B_e.  X elements a row of A; wide operands as for run_expert.
template <bool B_K, bool RAGGED_K, int EPI>
void run_sorted(const moe_sorted_cfg& c, const Part& part, int prod, WideKind kind, GemmParams p, int64_t rows, int cols,
                void* ws, hipStream_t s) {
  const int64_t R = sorted_rows(c);
  p.cap = (int)R;
  p.act = c.act;
  p.part = (float*)ws;
  p.ksplit = 1;
  p.rb += part.e0;
  p.re += part.e0;
  const double expect = (double)c.T * c.k / c.E;
  WideCall w{kind, c.act, part.n, rows, cols, expect, std::sqrt(expect * std::max(0., 1. - (double)c.k / c.E)), p};
  w.shared = true;
  const bool tb = ptimer_begin(prod, s);
  if (c.dtype == MOE_BF16) {
    run_wide_any(w, s);
  } else {
    WideCall q = w;
    if (!RAGGED_K) q.rows = R / part.n + 32;   // (the bound on the grid that f32_tile looks at)
    const int64_t all = RAGGED_K ? 0 : R;
    if (f32_tile(q, num_cus()) == 32) launch_f32<1, B_K, RAGGED_K, EPI>(p, part.n, rows, cols, s, all);
    else launch_f32<2, B_K, RAGGED_K, EPI>(p, part.n, rows, cols, s, all);
  }
  ptimer_end(tb, s);
}
// Element e of the experts' matrices of n elements each.
const void* mat(const moe_sorted_cfg& c, const void* W, int64_t e, int64_t n) {
  return (const char*)W + e * n * (c.dtype == MOE_BF16 ? 2 : 4);
}
}  // namespace

size_t sorted_ffn_ws_bytes(const moe_sorted_cfg& c) {
  return c.dtype == MOE_BF16 ? (size_t)kSkPartElems * sizeof(float) : 0;
}

void launch_sorted_fwd(const moe_sorted_cfg& c, const void* X, const int32_t* rb, const int32_t* re, const void* W1,
                       const void* W2, void* H, void* A, void* O, void* ws, hipStream_t s) {
  const int64_t d = c.d_model, f = c.d_ff, R = sorted_rows(c);
  if (R == 0) return;
  each_part(c, [&](const Part& q) {
    GemmParams p{X, d, 0, mat(c, W1, q.e0, f * d), d, f * d, H, f, 0, A, nullptr, rb, re, 0, (int)f, (int)d};
    run_sorted<true, false, EPI_FWD1>(c, q, kProdFwd1, WK_FWD1, p, R, (int)f, ws, s);
  });
  each_part(c, [&](const Part& q) {
    GemmParams p{A, f, 0, mat(c, W2, q.e0, d * f), f, d * f, O, d, 0, nullptr, nullptr, rb, re, 0, (int)d, (int)f};
    run_sorted<true, false, EPI_STORE>(c, q, kProdFwd2, WK_NK, p, R, (int)d, ws, s);
  });
}

void launch_sorted_bwd_dx(const moe_sorted_cfg& c, const int32_t* rb, const int32_t* re, const void* H, const void* W1,
                          const void* W2, const void* dO, void* dH, void* dXe, void* ws, hipStream_t s) {
  const int64_t d = c.d_model, f = c.d_ff, R = sorted_rows(c);
  if (R == 0) return;
  each_part(c, [&](const Part& q) {
    GemmParams p{dO, d, 0, mat(c, W2, q.e0, d * f), f, d * f, dH, f, 0, nullptr, H, rb, re, 0, (int)f, (int)d};
    run_sorted<false, false, EPI_DACT>(c, q, kProdDA, WK_DACT, p, R, (int)f, ws, s);
  });
  each_part(c, [&](const Part& q) {
    GemmParams p{dH, f, 0, mat(c, W1, q.e0, f * d), d, f * d, dXe, d, 0, nullptr, nullptr, rb, re, 0, (int)d, (int)f};
    run_sorted<false, false, EPI_STORE>(c, q, kProdDXe, WK_KN, p, R, (int)d, ws, s);
  });
}

void launch_sorted_bwd_dw(const moe_sorted_cfg& c, const int32_t* rb, const int32_t* re, const void* X, const void* A,
                          const void* dO, const void* dH, void* dW1, void* dW2, hipStream_t s) {
  const int64_t d = c.d_model, f = c.d_ff, R = sorted_rows(c);
  const WideKind kind = c.wpacked && c.dtype == MOE_BF16 ? WK_DW_BLK : WK_DW;
  each_part(c, [&](const Part& q) {
    GemmParams p{dO, d, 0, A, f, 0, (void*)mat(c, dW2, q.e0, d * f), f, d * f, nullptr, nullptr, rb, re, (int)d, (int)f};
    run_sorted<false, true, EPI_STORE>(c, q, kProdDW2, kind, p, d, (int)f, nullptr, s);
  });
  each_part(c, [&](const Part& q) {
    GemmParams p{dH, f, 0, X, d, 0, (void*)mat(c, dW1, q.e0, f * d), d, f * d, nullptr, nullptr, rb, re, (int)f, (int)d};
    run_sorted<false, true, EPI_STORE>(c, q, kProdDW1, kind, p, f, (int)d, nullptr, s);
  });
}

// --------------------------------------------------------------- cross entropy
// Logits over a piece of the vocabulary (see XentParams), and the products of the
// gradient at them.  bf16: the wide kernel, W (and in the forward x) as the caller has
// it, row-major, x in the backward and dl blocked; float: the float kernel, row-major.
static GemmParams xent_params(int64_t T, int N, int K, const void* A, int64_t lda, int64_t sA, const void* B, int64_t ldb,
                              int64_t sB, void* C, int64_t ldc) {
  GemmParams p{A, lda, sA, B, ldb, sB, C, ldc, 0, nullptr, nullptr, nullptr, nullptr, 0, N, K, 0, (int)T};
  return p;
}
static WideCall xent_call(WideKind kind, int64_t T, int cols, const GemmParams& p) {
  return WideCall{kind, MOE_ACT_IDENTITY, 1, T, cols, (double)T, 0., p};
}
// Many tokens: no tile whose waves have narrow runs of columns (the partial sums are one for each).
constexpr int64_t kXentNarrow = 1024;
int xent_run_columns(int dtype, int64_t T) { return dtype == MOE_BF16 ? (T <= kXentNarrow ? 32 : 64) : (T <= kXentNarrow ? 16 : 32); }

// Columns of a product of T rows that fill whole rounds of 256-tiles (a multiple of 256; all of them if there is no
// whole round, or nothing is left past the last).  The columns left run as a product of their own on the tiles that
// suit them, where that takes less: a last round of a few 256-tiles takes as long as a full one.  2048 tokens, width
// 1024, 50257 classes: 1576 tiles, six rounds and 40 tiles.
static int whole_rounds(const WideCall& w, int cus) {
  const int64_t tm = (w.rows + 255) / 256, tn = (w.cols + 255) / 256;
  const int64_t main = tm * tn / cus * cus / tm * 256;
  if (main <= 0 || main >= w.cols) return w.cols;
  WideCall a = w, b = w;
  a.cols = (int)main;
  b.cols = w.cols - (int)main;
  const double apart = tile_cost(kTilesM[tile_m(a, cus)], a, cus) + tile_cost(kTilesM[tile_m(b, cus)], b, cus) + 3000.;
  return apart < tile_cost(kTilesM[tile_m(w, cus)], w, cus) ? (int)main : w.cols;
}

static int launch_lse_part(int dtype, int form, int64_t T, int d, const void* x, const void* W, const XentParams& xp,
                           hipStream_t s) {
  GemmParams p = xent_params(T, xp.cols, d, x, d, form >= kXentX ? pad16(T) * d : T * d, W, d,
                             (form == kXentBlocked ? pad16(xp.cols) : (int64_t)xp.cols) * d, nullptr, 0);
  WideCall w = xent_call(form == kXentBlocked ? WK_LSE_BLK : form == kXentX ? WK_LSE_X : WK_LSE, T, xp.cols, p);
  w.x = xp;
  if (dtype == MOE_BF16) {
    const TileCost& t = kTilesM[tile_m(w, num_cus(), T <= kXentNarrow ? kTileCount : kTileCount - 1)];
    t.run_rows(w, s);
    return (xp.cols + t.bn - 1) / t.bn * (t.bn / t.wtn);
  }
  if (T <= kXentNarrow && f32_tile(w, num_cus()) == 32) {
    launch_f32<1, true, false, EPI_LSE>(XentGemmParams{p, xp}, 1, T, xp.cols, s);
    return (xp.cols + 31) / 32 * 2;
  }
  launch_f32<2, true, false, EPI_LSE>(XentGemmParams{p, xp}, 1, T, xp.cols, s);
  return (xp.cols + 63) / 64 * 2;
}
// Returns the runs of columns written from xp.block0 on.
int launch_xent_lse(int dtype, int form, int64_t T, int d, const void* x, const void* W, const XentParams& xp,
                    hipStream_t s) {
  if (dtype != MOE_BF16) return launch_lse_part(dtype, kXentRows, T, d, x, W, xp, s);
  GemmParams p{};
  p.K = d;
  const int main = whole_rounds(xent_call(WK_LSE, T, xp.cols, p), num_cus());
  XentParams a = xp, b = xp;
  a.cols = main;
  int n = launch_lse_part(dtype, form, T, d, x, W, a, s);
  if (main < xp.cols) {   // (whole 16-row blocks of W come before the rest)
    b.col0 += main;
    b.cols -= main;
    b.block0 += n;
    n += launch_lse_part(dtype, form, T, d, x, (const uint16_t*)W + (int64_t)main * d, b, s);
  }
  return n;
}

// dl [T][ld] (bf16: blocked, pad16(T) rows), ld >= xp.cols a multiple of 64 (float: 8); x: bf16 blocked.
void launch_xent_dl(int dtype, int form, int64_t T, int d, const void* x, const void* W, const XentParams& xp, void* dl,
                    int ld, hipStream_t s) {
  auto extent = [&](int cols) { return (form == kXentBlocked ? pad16(cols) : (int64_t)cols) * d; };
  GemmParams p = xent_params(T, ld, d, x, d, pad16(T) * d, W, d, extent(xp.cols), dl, ld);
  WideCall w = xent_call(form == kXentBlocked ? WK_DL_BLK : WK_DL, T, ld, p);
  w.x = xp;
  if (dtype != MOE_BF16) {
    if (f32_tile(w, num_cus()) == 32) launch_f32<1, true, false, EPI_DL>(XentGemmParams{p, xp}, 1, T, ld, s);
    else launch_f32<2, true, false, EPI_DL>(XentGemmParams{p, xp}, 1, T, ld, s);
    return;
  }
  const int main = whole_rounds(w, num_cus());
  if (main < w.cols) {   // (the columns left, in a dl that begins further right: 32 columns are a block)
    WideCall b = w;
    b.cols = b.p.N = ld - main;
    b.x.col0 += main;
    b.x.cols -= main;
    b.p.B = (const uint16_t*)W + (int64_t)main * d;
    b.p.sB = extent(b.x.cols);
    b.p.C = (uint16_t*)dl + (int64_t)main / 32 * 512;
    run_wide_any(b, s);
    w.cols = w.p.N = w.x.cols = main;
    w.p.sB = extent(main);
  }
  run_wide_any(w, s);
}

// dx over one piece: acc_in (NULL = 0) + dl W -> acc_out (float), or times *scale rounded to dx (bf16).
//
// float: few tiles with long sums are cut into slices of the classes (each a group of the launch, its sums in `part`),
// enough of them for four blocks a CU, which a launch adds in order.  500 tokens, 10007 classes, width 512: 109 us in
// one, the product of the same size that has tiles enough 63.
static int xent_slices(int64_t T, int d, int cols) {
  const int64_t tiles = (T + 63) / 64 * ((d + 63) / 64);
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(16, 1024 / tiles), cols / 256));
}
size_t xent_slices_bytes(int64_t T, int d, int cols) {
  const int n = xent_slices(T, d, cols);
  return n > 1 ? (size_t)n * T * d * sizeof(float) : 0;
}
// (in may be out: a thread reads its four values of it before it writes them)
__global__ __launch_bounds__(256) void xent_slices_kernel(const float* __restrict__ part, int n, int64_t size,
                                                          const float* in, float* out) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= size) return;
  f32x4 v[16];
#pragma unroll
  for (int q = 0; q < 16; ++q)
    if (q < n) v[q] = *reinterpret_cast<const f32x4*>(part + q * size + i);
  f32x4 a = v[0];
#pragma unroll
  for (int q = 1; q < 16; ++q)
    if (q < n) a += v[q];
  if (in) a += *reinterpret_cast<const f32x4*>(in + i);
  *reinterpret_cast<f32x4*>(out + i) = a;
}

void launch_xent_dx(int dtype, int64_t T, int d, int cols, const void* dl, int ld, const void* W, const float* acc_in,
                    float* acc_out, void* dx, const float* scale, void* part, hipStream_t s) {
  GemmParams p = xent_params(T, d, ld, dl, ld, pad16(T) * ld, W, d, (int64_t)cols * d, acc_out, d);
  p.Aux = acc_in;
  if (dtype == MOE_BF16) p.part = (float*)scale;
  p.C2 = dx;
  p.M = cols;
  WideCall w = xent_call(WK_ADD, T, d, p);
  if (dtype == MOE_BF16) return run_wide_any(w, s);
  int n = xent_slices(T, d, cols);
  p.ksplit = n > 1 ? ((cols + n - 1) / n + 15) / 16 * 16 : ld;
  n = (cols + p.ksplit - 1) / p.ksplit;
  p.sA = p.ksplit;
  p.sB = (int64_t)p.ksplit * d;
  if (n > 1) {
    p.sC = T * d;
    p.C = part;
    p.Aux = nullptr;
  }
  w.groups = n;
  if (n == 1 && f32_tile(w, num_cus()) == 32) launch_f32<1, false, false, EPI_ADD>(p, n, T, d, s);
  else launch_f32<2, false, false, EPI_ADD>(p, n, T, d, s);
  if (n > 1)
    launch_kernel(xent_slices_kernel, dim3((unsigned)((T * d / 4 + 255) / 256)), dim3(256), 0, s, (const float*)part, n,
                  T * d, acc_in, acc_out);
}

// dx where the vocabulary is one piece (bf16): no float sums to keep, and where the
// result has few tiles, their long sums over the vocabulary are split over the CUs
// (part: sorted_ffn_ws_bytes-sized).
size_t xent_part_bytes() { return (size_t)kSkPartElems * sizeof(float); }
void launch_xent_dx_whole(int64_t T, int d, int cols, const void* dl, int ld, const void* W, void* dx, const float* scale,
                          void* part, hipStream_t s) {
  GemmParams p = xent_params(T, d, ld, dl, ld, pad16(T) * ld, W, d, (int64_t)cols * d, dx, d);
  p.Aux = scale;
  p.part = (float*)part;
  const int64_t large = (T + 255) / 256 * ((d + 255) / 256);
  WideCall w = xent_call(WK_KN_RM, T, d, p);
  // (the split: its share of a 256-tile's steps, and 30 us for 64 MB of partial tiles written, read and summed; with few
  // classes smaller whole tiles take less.  Whole backward, us, never split and always: 2000 classes of 1024 tokens of
  // width 512 49 and 82, 5000 90 and 109, 10000 117 and 111; of 2048 of width 2048 362 and 322; 20000 of 64 157 and 74)
  const int cus = num_cus();
  const double split = ld / 32. * 650. * large / cus + 30000.;
  if (4 * large <= cus && split < tile_cost(kTilesM[tile_m(w, cus)], w, cus)) {
    w.p.ksplit = 2;
    return run_rows_256x256(w, s);
  }
  run_wide_any(w, s);
}

// Sum of the token ranges' partials in range order, times *scale: 8 consecutive elements a thread.
__global__ __launch_bounds__(256) void xent_ranges_kernel(const float* __restrict__ part, int n, int64_t size,
                                                          const float* __restrict__ scale, uint16_t* __restrict__ out) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= size) return;
  f32x4 a = *reinterpret_cast<const f32x4*>(part + i), b = *reinterpret_cast<const f32x4*>(part + i + 4);
  for (int q = 1; q < n; ++q) {
    a += *reinterpret_cast<const f32x4*>(part + q * size + i);
    b += *reinterpret_cast<const f32x4*>(part + q * size + i + 4);
  }
  const float k = *scale, v[8] = {a[0] * k, a[1] * k, a[2] * k, a[3] * k, b[0] * k, b[1] * k, b[2] * k, b[3] * k};
  Vec<uint16_t>::store(out + i, v);
}

// Token ranges of a dW product that has too few tiles for the chip: it is one 128-tile a CU at most, as long as the
// batch, so its tokens are cut into ranges (float partials, joined in order) until there are three a CU.  Backward of
// 16384 tokens over 1000 classes of width 512: 296 us in one range, 139 in up to four, 123 in up to eight; of 4096 over
// 5000 165 and 157.
static int dw_ranges(int64_t T, int rows, int d, int cus) {
  const int64_t tiles = (int64_t)((rows + 127) / 128) * ((d + 127) / 128);
  if (tiles > cus) return 1;
  const int64_t n = std::min<int64_t>(std::min<int64_t>(8, 3 * cus / tiles), T / 256);
  return (int)std::max<int64_t>(1, std::min<int64_t>(n, kSkPartElems / ((int64_t)rows * d)));
}

// dW [cols][d] = dl^T x (bf16: times *scale); x as dl (bf16: blocked).  Whole rounds of 256-tiles, and what is left
// past them on smaller ones (as whole_rounds, with the rows in the columns' place).  part: xent_part_bytes.
void launch_xent_dw(int dtype, int64_t T, int d, int cols, const void* dl, int ld, const void* x, void* dW,
                    const float* scale, void* part, hipStream_t s) {
  GemmParams p{dl, ld, pad16(T) * ld, x, d, pad16(T) * d, dW, d, 0, nullptr, nullptr, nullptr, nullptr, cols, d, 0, 0, (int)T};
  p.Aux = scale;
  WideCall w = xent_call(WK_DW_SCALED, cols, d, p);
  w.expect = (double)T;
  if (dtype != MOE_BF16) {
    if (f32_tile(w, num_cus()) == 32) launch_f32<1, false, true, EPI_STORE>(p, 1, cols, d, s);
    else launch_f32<2, false, true, EPI_STORE>(p, 1, cols, d, s);
    return;
  }
  const int cus = num_cus();
  auto run = [&](WideCall q) {
    const int n = dw_ranges(T, q.p.M, d, cus);
    if (n == 1) return run_wide_any(q, s);
    const int64_t size = (int64_t)q.p.M * d;
    uint16_t* const out = (uint16_t*)q.p.C;
    q.kind = WK_DW_PART;
    q.groups = n;
    q.p.kchunk = (int)(((T + n - 1) / n + 31) / 32 * 32);
    q.p.sA = q.p.sB = 0;
    q.p.C = part;
    q.p.sC = size;
    q.p.Aux = nullptr;
    run_rows_128x128(q, s);
    launch_kernel(xent_ranges_kernel, dim3((unsigned)((size / 8 + 255) / 256)), dim3(256), 0, s, (const float*)part, n,
                  size, scale, out);
  };
  const int64_t tn = (d + 255) / 256, tm = (cols + 255) / 256, main = tm * tn / cus * cus / tn * 256;
  // (half a round or more left: it is as well spent on 256-tiles)
  if (main > 0 && main < cols && 2 * (tm * tn % cus) < cus) {
    WideCall b = w;
    b.rows = b.p.M = cols - (int)main;
    b.p.A = (const uint16_t*)dl + main / 32 * 512;
    b.p.sA = p.sA - main / 32 * 512;
    b.p.C = (uint16_t*)dW + main * d;
    run(b);
    w.rows = w.p.M = (int)main;
  }
  run(w);
}

// Sum of the S float partials of a K-split weight gradient, in group order,
// rounded once to bf16: 8 consecutive elements per thread.
__global__ __launch_bounds__(256) void gemm_wgrad_reduce_kernel(const float* __restrict__ part, int S, int64_t MN,
                                                                 uint16_t* __restrict__ C) {
  const int64_t i = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * 8;
  if (i >= MN) return;
  f32x4 a0 = *reinterpret_cast<const f32x4*>(part + i), a1 = *reinterpret_cast<const f32x4*>(part + i + 4);
  for (int g = 1; g < S; ++g) {
    a0 += *reinterpret_cast<const f32x4*>(part + (int64_t)g * MN + i);
    a1 += *reinterpret_cast<const f32x4*>(part + (int64_t)g * MN + i + 4);
  }
  const float v0[4] = {a0[0], a0[1], a0[2], a0[3]}, v1[4] = {a1[0], a1[1], a1[2], a1[3]};
  const u32x2 lo = pack4_bf16(v0), hi = pack4_bf16(v1);
  *reinterpret_cast<u32x4*>(C + i) = u32x4{lo[0], lo[1], hi[0], hi[1]};
}

// Token ranges of the dense weight gradients: the block's 2048 x 2048 and
// 6144 x 2048 products have 64 and 192 tiles of 256 x 256, so four ranges give
// every CU work (256 and 768 tile-ranges).
constexpr int kWgradSplit = 4;
size_t wgrad_ws_bytes(int M, int N) { return (size_t)kWgradSplit * M * N * sizeof(float); }

// Weight gradient C[M][N] = A^T B of the block's dense projections, A [K][M]
// and B [K][N] row-major bf16 (K = tokens), C bf16: the wide kernel's ragged-K
// product with K split into wgrad_ksplit(M, N) token ranges of equal length
// (multiples of 32), one float partial per range in `part`
// (wgrad_ws_bytes(M, N) bytes), then their sum in range order.
void launch_dense_wgrad(int M, int N, int64_t K, const void* A, const void* B, void* C, void* part, hipStream_t s,
                        bool beside) {
  if (M <= 0 || N <= 0) return;
  const int S = kWgradSplit;
  const int64_t MN = (int64_t)M * N;
  GemmParams p{A, M, 0, B, N, 0, part, N, MN, nullptr, nullptr, nullptr, nullptr, M, N, 0, 0, (int)K};
  p.kchunk = (int)(((K + S - 1) / S + 31) / 32 * 32);
  run_wide_any(WideCall{WK_WGF32, MOE_ACT_IDENTITY, S, M, N, (double)std::min<int64_t>(K, p.kchunk), 0., p, beside},
               s);
  launch_kernel(gemm_wgrad_reduce_kernel, dim3((unsigned)((MN / 8 + 255) / 256)), dim3(256), 0, s,
                (const float*)part, S, MN, (uint16_t*)C);
}

// Row-major [M][K] bf16 -> the blocked layout with pad16(M) rows (rows past M
// zero).  One wave per 16 x 32 block: each lane reads 16 bytes of one row and
// the wave writes the block's 1 KiB as one contiguous run.
__global__ __launch_bounds__(256) void pack_rows_kernel(const uint16_t* __restrict__ src, uint16_t* __restrict__ dst,
                                                        int64_t M, int K) {
  const int64_t b = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 6;
  const int lane = threadIdx.x & 63;
  const int kb = K >> 5;
  const int64_t rb = b / kb;
  if (rb * 16 >= pad16(M)) return;
  const int cb = (int)(b - rb * kb);
  const int64_t row = rb * 16 + (lane >> 2);
  const int col = cb * 32 + (lane & 3) * 8;
  u32x4 v = u32x4{0u, 0u, 0u, 0u};
  if (row < M) v = *reinterpret_cast<const u32x4*>(src + row * K + col);
  *reinterpret_cast<u32x4*>(dst + b * 512 + lane * 8) = v;
}

void launch_pack_rows(const void* src, void* dst, int64_t M, int K, hipStream_t s) {
  if (M <= 0 || K <= 0) return;
  const int64_t blocks = pad16(M) / 16 * (K / 32);
  launch_kernel(pack_rows_kernel, dim3((unsigned)((blocks * 64 + 255) / 256)), dim3(256), 0, s,
                (const uint16_t*)src, (uint16_t*)dst, M, K);
}

// Dense products on the wide MFMA kernel: one group of M rows, both operands
// blocked (A [pad16(M)][K]; B [N][K] if b_nk else [K][N]), output row-major,
// + resid (row-major like C) if given.  Every output element is one in-order
// K sum (no K-split), so a product over a batch partition's rows gives the
// same bits as over the whole batch.
void launch_dense_wide(int64_t M, int N, int K, const void* A, const void* B, bool b_nk, void* C, int64_t ldc,
                       const void* resid, hipStream_t s) {
  if (M <= 0 || N <= 0 || K <= 0) return;
  GemmParams p{A, K, pad16(M) * K, B, b_nk ? K : N, (int64_t)N * K, C, ldc, M * ldc, nullptr, resid, nullptr, nullptr,
               0, N, K, 0, (int)M};
  p.ksplit = 0;
  run_wide_any(WideCall{b_nk ? (resid ? WK_NK_RES : WK_NK) : WK_KN, MOE_ACT_IDENTITY, 1, M, N, (double)M, 0., p}, s);
}

// The tile, (rows << 16) + columns, that the choices above give an expert product
// (kProd*) of a call, or a dense product, on `cus` compute units (0: by the
// row counts).
int expert_tile(const moe_cfg& c, int product, bool later, int cus) {
  static const WideKind kinds[kProducts] = {WK_FWD1, WK_NK, WK_DACT, WK_KN, WK_DW, WK_DW};
  const bool to_f = product == kProdFwd1 || product == kProdDA || product == kProdDW2;   // N = f (else d)
  GemmParams p{};
  p.K = to_f ? c.d_model : c.d_ff;
  p.ksplit = c.ksplit;
  const bool dw = product == kProdDW2 || product == kProdDW1;
  const WideCall w = expert_call(c, kinds[product], p, dw ? (to_f ? c.d_model : c.d_ff) : c.C,
                                 to_f ? c.d_ff : c.d_model, later);
  if (c.dtype != MOE_BF16) return f32_tile(w, cus) * ((1 << 16) + 1);
  if (dw) {
    const TileK t = tile_k(w, cus);
    return t == kTileKByRows ? 0 : t == kTileK256 ? (256 << 16) + 256 : (128 << 16) + 128;
  }
  const TileCost& t = kTilesM[tile_m(w, cus)];
  return (t.bm << 16) + t.bn;
}
int dense_tile(int64_t M, int N, int K, int cus) {
  GemmParams p{};
  p.K = K;
  const TileCost& t = kTilesM[tile_m(WideCall{WK_NK, MOE_ACT_IDENTITY, 1, M, N, (double)M, 0., p}, cus)];
  return (t.bm << 16) + t.bn;
}

}  // namespace lmoe
