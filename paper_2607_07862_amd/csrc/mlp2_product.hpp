// Tile products of the training operators: C[m][n] = sum over k of R(m, k) C(n, k)
// for column operands of either storage order, with a fused epilogue.
//
// The forward kernels of the library multiply activations [M, K] by weights
// [K, N].  Training needs other orders too: dZ = dY W2^T reads weights whose K
// is contiguous, dW = X^T dP has K as the slow index of both operands, of which
// the row side is transposed beforehand.  Here the column side is staged
// through LDS in panels of its own order, the row side in inner ones:
//
//   inner panel (K contiguous in memory): [rows][k], read
//     by ds_read_b128 (8 consecutive k per lane);
//   outer panel (K is the slow index): [k][columns], read transposed by
//     ds_read_b64_tr_b16.
//
// Both are XOR-swizzled in 16-byte chunks and filled by direct-to-LDS buffer
// loads, whose range check supplies zeros past an operand's end: ragged rows
// and a K that is not a multiple of 64 (the token count of a weight gradient)
// need no masks in the loop.  Offsets inside a tile's stage are 32 bits wide;
// the base of every stage is carried in 64.
//
// As in the forward kernels the MFMA takes the column side as its A operand
// and the row side as its B operand, so a lane ends up with 8 consecutive
// columns of one row for each pair of 16 x 16 blocks.
#pragma once

#include <cmath>

#include "mlp2_device.hpp"
#include "mlp2_host.h"

namespace mlp2 {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4_t;

// Element types of the operands: both are 16 bits wide and accumulate in fp32.
struct Bf16 {
  __device__ static f32x4 mfma(u32x4 w, u32x4 x, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0, 0, 0);
  }
};
struct Fp16 {
  __device__ static f32x4 mfma(u32x4 w, u32x4 x, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w), __builtin_bit_cast(f16x8, x), c, 0, 0, 0);
  }
};

// One side of a product: element (i, k) is p[i * ld + k] (inner) or p[k * ld + i] (outer).
struct Side {
  const uint16_t* p;
  int64_t ld;
  int64_t bytes;   // from p to the end of the matrix (outer: of its last matrix); what lies past it reads as zero
  int64_t panel;   // outer: elements from a tile's first panel to its second, in another matrix; 0: the next columns
  int64_t jump;    // inner: elements added to the base from unit `jump_at` of K on (K runs on in a second matrix)
  int jump_at;     // in units of 64 k; 0: no second matrix
  int64_t batch;   // elements between the matrices of a batch
};

// A work-group tile: ROWP row panels of ER rows and COLP column panels of EC
// columns, WM x WN waves, a ring of NS stages, each BK deep.  Every wave owns
// 32 columns of every column panel (so that the two panels of a gated product,
// gate and up weights, meet in one lane) and 16 * TM rows.
template <int ER_, int ROWP_, int EC_, int COLP_, int WM_, int WN_, int NS_>
struct PTile {
  static constexpr int ER = ER_, ROWP = ROWP_, EC = EC_, COLP = COLP_, WM = WM_, WN = WN_, NS = NS_;
  static constexpr int BK = 64;
  static constexpr int NWAVES = WM * WN, THREADS = 64 * NWAVES;
  static constexpr int BM = ER * ROWP, BN = EC * COLP;
  static constexpr int TM = BM / WM / 16;             // 16-row blocks of a wave
  static constexpr int KS = BK / 32;                  // MFMA steps of a stage
  static constexpr int RPANEL = ER * BK * 2, CPANEL = EC * BK * 2;  // bytes of a panel's stage
  static constexpr int STAGE = ROWP * RPANEL + COLP * CPANEL;
  static constexpr int LOADS = STAGE / 1024 / NWAVES;  // 1 KB loads per wave and stage
  static constexpr int LDS = NS * STAGE;
  static_assert(EC == 32 * WN, "a wave owns 32 columns of every column panel");
  static_assert(RPANEL % (1024 * NWAVES) == 0 && CPANEL % (1024 * NWAVES) == 0, "every wave loads whole 1 KB pieces");
  // Wave wm's row block tm: in the quadrant tile its rows lie in both halves, elsewhere together.
  static constexpr bool QUAD = NWAVES == 8 && COLP * EC == 256;
  __device__ static constexpr int row_of(int wm, int tm) {
    return QUAD ? 64 * wm + 16 * (tm & 3) + 128 * (tm >> 2) : wm * (BM / WM) + 16 * tm;
  }
};
using Tile64 = PTile<64, 1, 64, 1, 2, 2, 4>;    // 64 x 64
using Tile64G = PTile<64, 1, 64, 2, 2, 2, 3>;   // 64 x (64 + 64): gated
using Tile128 = PTile<64, 2, 64, 2, 2, 2, 2>;   // 128 x 128, gated 128 x (64 + 64)
using Tile256 = PTile<128, 2, 128, 2, 2, 4, 2>;  // 256 x 256, gated 256 x (128 + 128): the ping-pong loop

// ------------------------------------------------------------------ panel loads

// One direct-to-LDS buffer load: lane i moves 16 bytes from base + voff to
// lds_addr + 16 i, zeros where voff is past the descriptor's range.  The wait
// states ahead of it cover a scalar operand that a vector instruction has just
// written (5; the compiler keeps them for its own instructions, not for an
// asm's) and the write of M0 (1).
template <int STATES>
__device__ __forceinline__ void dma16_buffer(u32x4 rsrc, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_nop %3\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "{m0}"(lds_addr), "n"(STATES - 1) : "memory");
}

// The chunk swizzle of a panel's row.  Inner: rows of 8 chunks, so that the 16
// rows of one ds_read_b128 group lie in different banks.  Outer: k rows
// of E / 8 chunks, so that the 4 k rows of one ds_read_b64_tr_b16 group do.
__device__ __forceinline__ int swz_inner(int row) { return (row >> 1) & 7; }
template <int E>
__device__ __forceinline__ int swz_outer(int k) {
  return E == 128 ? (4 * (k & 3)) ^ (2 * ((k >> 3) & 1)) : (4 * ((k >> 1) & 1)) ^ (2 * ((k >> 3) & 1));
}

// Loads of one panel, stage by stage.  COL: the column side, whose inner panels
// hold their rows permuted within every 32 (LDS row 16 t + i is matrix row
// 8 (i / 4) + 4 t + i % 4), so that a pair of blocks gives a lane 8 consecutive
// columns; outer panels get the same from the fragment addresses.
//
// The base moves on by one stage a load; the range is kept as follows.
//   inner: every stage may read the rows that exist, rows * ld elements from
//     the panel's first row; the columns of a stage always exist (K is a
//     multiple of 64), so the range does not change.
//   outer: a stage may read its own BK rows of k, the last one those that are
//     left.  Columns past the matrix's width read the next row's, or zeros;
//     either way they belong to results that are not stored.
template <class T, bool OUTER, bool COL, bool JUMP>
struct PanelLoad {
  static constexpr int E = COL ? T::EC : T::ER, BK = T::BK, BYTES = COL ? T::CPANEL : T::RPANEL;
  static constexpr int PIECES = BYTES / 1024 / T::NWAVES;
  static_assert(!JUMP || !OUTER, "a second matrix along K is inner");
  static_assert(!OUTER || COL, "K is contiguous on the row side");
  const char* base;
  uint32_t range, tail;  // of every stage; outer: of the last stage
  uint32_t step;
  int64_t jump;
  int left;              // outer: stages before the last; inner: before the second matrix
  uint32_t voff[PIECES];
  uint32_t lds;          // of this wave's first piece, from the stage's base

  __device__ static __forceinline__ uint32_t clamp(int64_t v) { return v <= 0 ? 0u : v > 0xFFFFFFFFll ? 0xFFFFFFFFu : (uint32_t)v; }

  // Stages stage0 .. stage0 + nk - 1 (of BK) of the panel of rows (columns) from i0 + panel * E on.
  __device__ __forceinline__ PanelLoad(const Side& s, int64_t batch, int i0, int panel, int stage0, int nk, uint32_t lds_off) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63, wave = uniform(tid >> 6);
    uint32_t piece_step;
    if constexpr (OUTER) {
      const int col = i0 + (s.panel ? 0 : panel * E);
      const int64_t first = batch * s.batch + (s.panel ? panel * s.panel : 0) + col + (int64_t)stage0 * BK * s.ld;
      base = (const char*)(s.p + first);
      step = (uint32_t)(BK * s.ld * 2);
      range = clamp((int64_t)step - 2 * col);
      tail = min(range, clamp(s.bytes - 2 * (first + (int64_t)(nk - 1) * BK * s.ld)));
      left = nk - 1;
      if (left == 0) range = tail;
      constexpr int CPR = E / 8, RPP = 64 / CPR;  // chunks per k row, k rows per piece
      const int row = RPP * wave + lane / CPR;
      static_assert(T::NWAVES * RPP % 16 == 0, "the swizzle repeats from piece to piece");
      const int chunk = (lane % CPR) ^ swz_outer<E>(row);
      piece_step = (uint32_t)(T::NWAVES * RPP * s.ld * 2);
      voff[0] = (uint32_t)((row * s.ld + 8 * chunk) * 2);
    } else {
      const int64_t rows = batch * s.batch + (int64_t)(i0 + panel * E) * s.ld;
      base = (const char*)(s.p + rows + (int64_t)stage0 * BK);
      step = BK * 2;
      // the end of this batch's matrix: the next one's start, or the end of all
      range = clamp((s.batch ? (batch + 1) * s.batch * 2 : s.bytes) - 2 * rows);
      if constexpr (JUMP) {
        jump = s.jump * 2;
        left = s.jump_at - stage0;
        if (left <= 0) base += jump;
      }
      constexpr int CPR = BK / 8, RPP = 64 / CPR;  // chunks per row, rows per piece
      const int row = RPP * wave + lane / CPR;
      static_assert(T::NWAVES * RPP % 32 == 0, "so do swizzle and permutation");
      const int chunk = (lane % CPR) ^ swz_inner(row);
      const int i = row & 15;
      const int at = COL ? (row & ~31) + 8 * (i >> 2) + 4 * ((row >> 4) & 1) + (i & 3) : row;
      piece_step = (uint32_t)(T::NWAVES * RPP * s.ld * 2);
      voff[0] = (uint32_t)((at * s.ld + 8 * chunk) * 2);
    }
#pragma unroll
    for (int j = 1; j < PIECES; ++j) voff[j] = voff[0] + j * piece_step;
    lds = lds_off + (uint32_t)wave * 1024u;
  }
  // The next stage, into the ring slot at stage_lds.
  __device__ __forceinline__ void load(uint32_t stage_lds) {
    const uint64_t b = (uint64_t)base;  // 48 bits
    const u32x4 r = {(uint32_t)b, (uint32_t)(b >> 32), range, 0x00027000u};
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      const uint32_t to = uniform(stage_lds + lds + (uint32_t)(j * T::NWAVES * 1024));
      if (j == 0) dma16_buffer<5>(r, voff[j], to);
      else dma16_buffer<1>(r, voff[j], to);
    }
    base += step;
    if constexpr (OUTER) range = --left == 0 ? tail : range;
    if constexpr (JUMP) base += --left == 0 ? jump : 0;
  }
};

// ------------------------------------------------------------------ fragments

__device__ __forceinline__ u32x4 read_tr(const char* p, int upper) {
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(p));
  const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(p + upper));
  typedef short i16x8 __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(u32x4, (i16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Row side: lane holds row (lane % 16) of a 16-row block, k = 8 (lane / 16) .. + 7 of a 32-deep slice.
template <class T>
struct RowFrag {
  static constexpr int E = T::ER;
  uint32_t off[T::KS];  // one per K slice
  __device__ __forceinline__ RowFrag(int wm) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63;
    const int first = T::row_of(wm, 0), r0 = first % E;
    const uint32_t panel = (uint32_t)(first / E * T::RPANEL);
    const int row = r0 + (lane & 15);
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks)
      off[ks] = panel + (uint32_t)(row * (2 * T::BK) + (((4 * ks + (lane >> 4)) ^ swz_inner(row)) << 4));
  }
  // Block tm of K slice ks; `stage` is the address of the stage's row panels.
  __device__ __forceinline__ u32x4 read(const char* stage, int ks, int tm) const {
    const int half = T::QUAD ? tm >> 2 : 0, blk = T::QUAD ? tm & 3 : tm;
    return *reinterpret_cast<const u32x4*>(stage + half * T::RPANEL + off[ks] + blk * 32 * T::BK);
  }
};

// Column side: block i of the pair that covers the wave's 32 columns of a panel.
template <class T, bool OUTER>
struct ColFrag {
  static constexpr int E = T::EC;
  uint32_t off[T::KS];
  __device__ __forceinline__ ColFrag(int wn) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63;
    if constexpr (OUTER) {
      // columns 8 c + 4 i .. + 3 of the pair: the interleave that leaves 8 consecutive columns in a lane
      const int k = 8 * (lane >> 4) + ((lane & 15) >> 2);
      off[0] = (uint32_t)(k * (2 * E) + (((4 * wn + (lane & 3)) ^ swz_outer<E>(k)) << 4));
    } else {
      const int row = 32 * wn + (lane & 15);
#pragma unroll
      for (int ks = 0; ks < T::KS; ++ks)
        off[ks] = (uint32_t)(row * (2 * T::BK) + (((4 * ks + (lane >> 4)) ^ swz_inner(row)) << 4));
    }
  }
  __device__ __forceinline__ u32x4 read(const char* panel, int ks, int i) const {
    if constexpr (OUTER) return read_tr(panel + off[0] + 8 * i + ks * 64 * E, 8 * E);
    else return *reinterpret_cast<const u32x4*>(panel + off[ks] + i * 32 * T::BK);
  }
};

// ------------------------------------------------------------------ mainloops

template <class T>
using Acc = f32x4[T::COLP][2][T::TM];

// The plain loop.  st0 and nk count stages of BK.
//
// A stage's fragments are read from LDS while the stage before it is
// multiplied (two register sets that swap roles, two stages a trip): the
// latency of the reads, which one or two waves to a SIMD would otherwise wait
// out once a stage, passes behind the products.  Stage it's ring slot is free
// once every wave holds its fragments, at the barrier for stage it + 1, and
// takes the loads of stage it + NS.
//
// LDS bounds it: a 64 x 64 x 64 unit reads 32 KB of fragments and takes in 16
// KB, 384 clocks at 128 bytes each, and measures 0.2 us on a CU of its own; twice
// the stages gained nothing (the Gram matrices of 2 x 512 x 2048 9.8 -> 10.4 us).
template <class T, class Elem, bool CO, bool JUMP>
__device__ __forceinline__ void product_loop(const Side& rs, const Side& cs, int64_t batch, int m0, int n0, int st0, int nk,
                                             Acc<T>& acc, char* lds) {
  const int wave = uniform((int)threadIdx.x >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM;
#pragma unroll
  for (int p = 0; p < T::COLP; ++p)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < T::TM; ++j) acc[p][i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (nk <= 0) return;
  const uint32_t lds_base = (uint32_t)(uintptr_t)lds;
  constexpr int C0 = T::ROWP * T::RPANEL;  // the column panels of a stage
  PanelLoad<T, false, false, false> r0(rs, batch, m0, 0, st0, nk, 0), r1(rs, batch, m0, T::ROWP - 1, st0, nk, (T::ROWP - 1) * T::RPANEL);
  PanelLoad<T, CO, true, JUMP> c0(cs, batch, n0, 0, st0, nk, C0),
      c1(cs, batch, n0, T::COLP - 1, st0, nk, C0 + (T::COLP - 1) * T::CPANEL);
  uint32_t to = lds_base;  // the ring slot that is requested next
  auto issue = [&]() {
    r0.load(to);
    if constexpr (T::ROWP == 2) r1.load(to);
    c0.load(to);
    if constexpr (T::COLP == 2) c1.load(to);
    to = to == lds_base + (T::NS - 1) * T::STAGE ? lds_base : to + T::STAGE;
  };
  const RowFrag<T> rf(wm);
  const ColFrag<T, CO> cf(wn);
  struct Frags {
    u32x4 x[T::KS][T::TM], w[T::KS][T::COLP][2];
  };
  const char* stage = lds;  // the ring slot that is read next
  auto read = [&](Frags& f) {
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) {
#pragma unroll
      for (int tm = 0; tm < T::TM; ++tm) f.x[ks][tm] = rf.read(stage, ks, tm);
#pragma unroll
      for (int p = 0; p < T::COLP; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i) f.w[ks][p][i] = cf.read(stage + C0 + p * T::CPANEL, ks, i);
    }
    stage = stage == lds + (T::NS - 1) * T::STAGE ? lds : stage + T::STAGE;
  };
  auto mma = [&](const Frags& f) {
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks)
#pragma unroll
      for (int p = 0; p < T::COLP; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int tm = 0; tm < T::TM; ++tm) acc[p][i][tm] = Elem::mfma(f.w[ks][p][i], f.x[ks][tm], acc[p][i][tm]);
  };
  // Every wave's loads of stage st have arrived, and every wave holds the fragments of the stages before it.
  auto resident = [&](int st) {
    wait_stages_behind<T::LOADS, T::NS - 2>(min(T::NS - 2, nk - 1 - st));
    __syncthreads();
  };
#pragma unroll
  for (int st = 0; st < T::NS - 1; ++st)
    if (st < nk) issue();
  resident(0);
  if (T::NS - 1 < nk) issue();
  Frags fa, fb;
  read(fa);
  auto advance = [&](int it, Frags& now, Frags& next) {  // stage it is multiplied, stage it + 1 (< nk) read
    resident(it + 1);
    if (it + T::NS < nk) issue();
    read(next);
    mma(now);
  };
  int it = 0;
  for (; it + 2 < nk; it += 2) {
    advance(it, fa, fb);
    advance(it + 1, fb, fa);
  }
  if (it + 1 < nk) {
    advance(it, fa, fb);
    mma(fb);
  } else {
    mma(fa);
  }
  __syncthreads();
}

// The ping-pong loop of the 256 x 256 tile, eight waves, two to a SIMD.
//
// What bounds a large tile: a 64-deep stage is 2048 cycles of MFMA per SIMD
// and its fragment reads and LDS writes take about three quarters of that, so
// the two must overlap.  As in the forward kernels' quadrant loop the two
// waves of a SIMD alternate (waves 0-3 run half a phase ahead of 4-7): while one
// multiplies, the other reads its next fragments and requests loads.  A stage
// is four phases of one output quadrant each, (A0, B0), (A0, B1), (A1, B1),
// (A1, B0) with A the row panels and B the column panels, and a phase is a
// memory slot and a product slot, each ended by a barrier.
//   memory slot 0 of stage it: request A1 of stage it + 1, read B0 of stage it
//               1:             request A0 of it + 2,       read B1 of it
//               2:             request B0 of it + 2,       read A1 of it
//               3:             request B1 of it + 2,       read A0 of it + 1
//   * Visibility: a wave waits for its own pieces of a panel at the end of the
//     memory slot before the one that reads it; a barrier lies between, and the
//     trailing waves reach that wait one slot before the leading waves read.
//   * Reuse: a panel read in memory slot p is complete in registers at product
//     slot p (lgkmcnt(0)) and its ring slot is requested again in memory slot
//     p + 2, after the barrier that ends the trailing waves' product slot p.
// Here the column side may have either storage order, and every panel carries
// its own 64-bit base and range.  8192 x 8192 x 8192 in bf16: K contiguous on both
// sides 731 us (1.50 PFLOP/s), on the row side alone 749 (1.47).  (With outer
// panels on both sides it took 926 (1.19), so no product has them.)
template <class T, class Elem, bool CO, bool JUMP>
__device__ __forceinline__ void product_pingpong(const Side& rs, const Side& cs, int64_t batch, int m0, int n0, int st0, int nk,
                                                 Acc<T>& acc, char* lds) {
  static_assert(T::ER == 128 && T::EC == 128 && T::ROWP == 2 && T::COLP == 2 && T::NWAVES == 8 && T::BK == 64 && T::NS == 2 && T::TM == 8, "256 x 256 tile");
  const int wave = uniform((int)threadIdx.x >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM;
  const bool trailing = wave >= 4;
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[p][i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (nk <= 0) return;

  const uint32_t lds_base = (uint32_t)(uintptr_t)lds;
  PanelLoad<T, false, false, false> pa[2] = {{rs, batch, m0, 0, st0, nk, 0}, {rs, batch, m0, 1, st0, nk, T::RPANEL}};
  PanelLoad<T, CO, true, JUMP> pb[2] = {{cs, batch, n0, 0, st0, nk, 2 * T::RPANEL},
                                        {cs, batch, n0, 1, st0, nk, 2 * T::RPANEL + T::CPANEL}};
  auto load_a = [&](int half, int st) { pa[half].load(lds_base + (uint32_t)(st & 1) * T::STAGE); };  // a panel's stages come in order
  auto load_b = [&](int half, int st) { pb[half].load(lds_base + (uint32_t)(st & 1) * T::STAGE); };

  const RowFrag<T> rf(wm);
  const ColFrag<T, CO> cf(wn);
  u32x4 xa[2][4], xb[2][4], w0[2][2], w1[2][2];
  auto read_a = [&](u32x4 (&x)[2][4], int half, int st) {
    const char* stage = lds + (st & 1) * T::STAGE;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int tm = 0; tm < 4; ++tm) x[ks][tm] = rf.read(stage, ks, 4 * half + tm);
  };
  auto read_b = [&](u32x4 (&w)[2][2], int half, int st) {
    const char* panel = lds + (st & 1) * T::STAGE + 2 * T::RPANEL + half * T::CPANEL;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < 2; ++i) w[ks][i] = cf.read(panel, ks, i);
  };
  auto mma = [&](const u32x4 (&w)[2][2], const u32x4 (&x)[2][4], auto bh, auto ah) {
    constexpr int b = decltype(bh)::value, a = 4 * decltype(ah)::value;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int tm = 0; tm < 4; ++tm) acc[b][i][a + tm] = Elem::mfma(w[ks][i], x[ks][tm], acc[b][i][a + tm]);
  };
  using Lo = int_constant<0>;
  using Hi = int_constant<1>;

  auto slot_end = [&]() {  // a barrier that neither the compiler's memory operations nor its products cross
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto vm_wait = [&](auto n) { wait_vm<decltype(n)::value>(); };
  auto products_begin = [&]() {  // this wave's fragment reads are complete
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
  };
  auto products_end = [&]() {
    __builtin_amdgcn_s_setprio(0);
    slot_end();
  };

  // One stage.  LEFT: stages after it, counted up to 2 (fewer loads to request
  // and to leave in flight).
  auto stage = [&](int it, auto left_) {
    constexpr int LEFT = decltype(left_)::value;
    read_b(w0, 0, it);
    if constexpr (LEFT >= 1) load_a(1, it + 1);
    vm_wait(int_constant<LEFT >= 1 ? 10 : 2>());  // B1 of this stage
    slot_end();
    products_begin();
    mma(w0, xa, Lo(), Lo());
    products_end();

    read_b(w1, 1, it);
    if constexpr (LEFT >= 2) load_a(0, it + 2);
    vm_wait(int_constant<LEFT >= 2 ? 10 : LEFT == 1 ? 8 : 0>());  // A1 of this stage
    slot_end();
    products_begin();
    mma(w1, xa, Hi(), Lo());
    products_end();

    read_a(xb, 1, it);
    if constexpr (LEFT >= 2) load_b(0, it + 2);
    if constexpr (LEFT >= 1) vm_wait(int_constant<LEFT >= 2 ? 10 : 6>());  // A0 of the next stage
    slot_end();
    products_begin();
    mma(w1, xb, Hi(), Hi());
    products_end();

    if constexpr (LEFT >= 1) read_a(xa, 0, it + 1);
    if constexpr (LEFT >= 2) load_b(1, it + 2);
    if constexpr (LEFT >= 1) {
      vm_wait(int_constant<LEFT >= 2 ? 10 : 4>());  // B0 of the next stage
    }
    slot_end();
    products_begin();
    mma(w0, xb, Lo(), Hi());
    products_end();
  };

  // Prologue: the first stage and all of the second but A1.
  const bool two = nk > 1;
  load_a(0, 0);
  load_b(0, 0);
  load_b(1, 0);
  load_a(1, 0);
  if (two) {
    load_a(0, 1);
    load_b(0, 1);
    load_b(1, 1);
    wait_vm<10>();  // A0, B0
  } else {
    wait_vm<4>();
  }
  slot_end();
  read_a(xa, 0, 0);
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)

  if (trailing) slot_end();
  for (int it = 0; it < nk - 2; ++it) stage(it, int_constant<2>());
  if (two) stage(nk - 2, int_constant<1>());
  stage(nk - 1, int_constant<0>());
  if (!trailing) slot_end();
  __syncthreads();  // every wave is done reading the ring before it is reused
}

// ------------------------------------------------------------------ one product of a launch

// Output tiles in launch order.  Work-groups land on the XCDs round-robin, so
// item i runs on XCD i % 8 (up to a rotation): every XCD takes a contiguous
// range of an order that goes down `band` row tiles before the next column
// tile, and so shares operand panels in its L2.  `sym`: the tiles on and above
// the diagonal only.
struct TileWalk {
  int tiles_m, tiles_n, band, sym;
  __host__ __device__ int total() const { return sym ? tiles_m * (tiles_m + 1) / 2 : tiles_m * tiles_n; }
  __device__ __forceinline__ void at(int item, int& tm, int& tn) const {
    const int n = total(), q = n / 8, r = n % 8, x = item % 8;
    int t = x * q + min(x, r) + item / 8;
    if (!sym) {
      const int per = band * tiles_n, g = t / per, in = t - g * per;
      const int rows = min(band, tiles_m - g * band);
      tn = in / rows;
      tm = g * band + (in - tn * rows);
      return;
    }
    // a band of rows i0 .. : its triangle on the diagonal, column by column, then whole columns
    for (int i0 = 0;; i0 += band) {
      const int rows = min(band, tiles_m - i0), tri = rows * (rows + 1) / 2, all = tri + rows * (tiles_m - i0 - rows);
      if (t >= all) {
        t -= all;
        continue;
      }
      if (t < tri) {
        int j = 0;
        while (t > j) t -= ++j;
        tn = i0 + j;
        tm = i0 + t;
      } else {
        t -= tri;
        tn = i0 + rows + t / rows;
        tm = i0 + t % rows;
      }
      return;
    }
  }
};

struct Nothing {};  // an epilogue's Read where it reads nothing

// CO: an outer column side; JUMP: the column side runs on in a second matrix.
template <bool CO_, class Epi_, bool JUMP_ = false>
struct Problem {
  static constexpr bool CO = CO_, JUMP = JUMP_;
  using Epi = Epi_;
  Side r, c;
  int M, N;          // rows and columns of the result (of each matrix of a gated product)
  int nk;            // K in units of 64
  int split, per;    // parts of K, units of each (the last one may have fewer)
  float* part;       // the parts' sums, fragment by fragment (split > 1)
  uint32_t* arrived; // parts of a tile that are done, one counter a line; zero between launches
  TileWalk walk;
  Epi epi;
  __host__ __device__ int items() const { return walk.total() * split; }
};

// 8 consecutive values of a lane: block pair (p, tm).
template <class T>
__device__ __forceinline__ void lane_values(const Acc<T>& acc, int p, int tm, float (&v)[8]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    v[r] = acc[p][0][tm][r];
    v[4 + r] = acc[p][1][tm][r];
  }
}

// Split K: every part stores its fp32 sums "fragment by fragment" (1 KB runs
// of a wave), written through to the device's point of coherence, and counts
// its arrival; the part that arrives last adds all parts in the order 0, 1, ...
// and goes on to the epilogue, so the bits do not depend on which one it is,
// and no part waits.  Row blocks from `rows` on hold nothing.  Returns whether
// this work-group goes on.
template <class T>
__device__ __forceinline__ bool join_parts(Acc<T>& acc, float* part, uint32_t* arrived, int64_t tile, int split, int s, int rows,
                                           char* lds) {
  constexpr int BLOCKS = T::COLP * 2 * T::TM, ITEM = T::NWAVES * BLOCKS * 256;  // floats of a part
  constexpr int kSc1 = 16;  // device scope: stores written through, loads past this XCD's L2 (it may hold lines of an earlier launch)
  const int tid = thread_here(), lane = tid & 63, wave = uniform(tid >> 6);
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(part + tile * split * ITEM, 0, split * ITEM * 4, 0x00027000);
  // Row blocks that hold nothing get an offset past the range: their stores are dropped, their loads return zeros.
  uint32_t off[T::TM];
#pragma unroll
  for (int tm = 0; tm < T::TM; ++tm)
    off[tm] = T::row_of(wave % T::WM, tm) < rows ? (uint32_t)(wave * BLOCKS * 1024 + lane * 16) : 0x80000000u;
  const int mine = s * ITEM * 4;
#pragma unroll
  for (int c = 0; c < T::COLP * 2; ++c)
#pragma unroll
    for (int tm = 0; tm < T::TM; ++tm)
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[c / 2][c % 2][tm]), rsrc, (int)(off[tm] + mine + (c * T::TM + tm) * 1024),
                                             0, kSc1);
  wait_all_mem();
  __syncthreads();
  uint32_t* seen = reinterpret_cast<uint32_t*>(lds);
  uint32_t* count = arrived + tile * kLine;
  if (tid == 0) *seen = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  const uint32_t before = uniform(*seen);
  if (before != (uint32_t)(split - 1)) return false;
  if (tid == 0) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // as the next launch expects it
#pragma unroll
  for (int c = 0; c < T::COLP * 2; ++c)
#pragma unroll
    for (int tm = 0; tm < T::TM; ++tm) acc[c / 2][c % 2][tm] = f32x4{0.f, 0.f, 0.f, 0.f};
  // Loads in flight together: those of 8 row blocks with the largest tile, of a whole part or of several with the others
  // (a part a round trip past the L2 takes about 0.35 us; 27 parts of a 64 x 64 tile 15.2 us).
  constexpr int AHEAD = BLOCKS >= 16 ? 1 : 32 / BLOCKS, COLS = BLOCKS > 16 ? 1 : T::COLP * 2;
  for (int q = 0; q < split; q += AHEAD) {
#pragma unroll
    for (int c0 = 0; c0 < T::COLP * 2; c0 += COLS) {
      u32x4 v[AHEAD][COLS][T::TM] = {};
#pragma unroll
      for (int d = 0; d < AHEAD; ++d)
        if (q + d < split)
#pragma unroll
          for (int c = 0; c < COLS; ++c)
#pragma unroll
            for (int tm = 0; tm < T::TM; ++tm)
              v[d][c][tm] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(off[tm] + (q + d) * (ITEM * 4) + ((c0 + c) * T::TM + tm) * 1024), 0, kSc1);
#pragma unroll
      for (int d = 0; d < AHEAD; ++d)
#pragma unroll
        for (int c = 0; c < COLS; ++c)
#pragma unroll
          for (int tm = 0; tm < T::TM; ++tm) acc[(c0 + c) / 2][(c0 + c) % 2][tm] += __builtin_bit_cast(f32x4, v[d][c][tm]);
    }
  }
  return true;
}

template <class T>
constexpr int mirror_pitch() { return T::BM * 2 + 16; }  // bytes of a column of the tile, kept apart in banks
template <class T, class P>
constexpr int lds_of() {
  constexpr int mirror = P::Epi::kMirror ? T::BN * mirror_pitch<T>() : 0;
  return mirror > T::LDS ? mirror : T::LDS;
}

// Epi::read: what the epilogue has to read for 8 values of a row; Epi::Read
// goes back to it with the sums.
// Epi::kGated: the two column panels are the same columns of two matrices and
// the epilogue takes both values; otherwise they are consecutive columns.
// Epi::kMirror: the epilogue returns 16-bit values whose transpose goes out too,
// through LDS and Epi::mirror, in 16-byte pieces of 8 rows.
// Epi::kSymmetric (with kMirror): the result is symmetric and only the tiles on
// and above the diagonal are computed; those on it are not mirrored.
// The transpose goes out for rows below Epi's `rows`: M, or M padded, where
// zeros go out for the rows past M.
template <class T, class P>
__device__ __forceinline__ void finish_product(const P& a, Acc<T>& acc, int batch, int tile, int s, int tm_, int tn_, char* lds) {
  using Epi = typename P::Epi;
  static_assert(!Epi::kSymmetric || (Epi::kMirror && T::BM == T::BN), "square tiles on the diagonal");
  constexpr int COLS = Epi::kGated ? T::EC : T::BN;  // result columns of a tile
  const int total = a.walk.total(), m0 = tm_ * T::BM, n0 = tn_ * COLS;
  int go = 1;
  if (a.split > 1) go = join_parts<T>(acc, a.part, a.arrived, (int64_t)batch * total + tile, a.split, s, a.M - m0, lds);
  if (uniform(go) == 0) return;  // a scalar branch: barriers follow
  const int tid = thread_here(), lane = tid & 63, wave = uniform(tid >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM;
  const bool mirrored = !Epi::kSymmetric || tm_ != tn_;
  if constexpr (Epi::kMirror) __syncthreads();  // join_parts' flag is read before the LDS is written again
  // Units: block pair p of row block tm.  What an epilogue reads for a group
  // of units is requested before the group ahead of it is stored: a load
  // behind a store of unknown address would otherwise wait for it, one round
  // trip a unit.
  constexpr int PAIRS = Epi::kGated ? 1 : T::COLP, UNITS = PAIRS * T::TM, GROUP = UNITS < 4 ? UNITS : 4;
  auto row_at = [&](int u) { return T::row_of(wm, u / PAIRS) + (lane & 15); };
  auto block_at = [&](int u) { return u % PAIRS * T::EC + 32 * wn; };
  auto inside = [&](int u) { return n0 + block_at(u) < a.N && m0 + row_at(u) < a.M; };
  typename Epi::Read read[2][GROUP];
  auto request = [&](int g) {
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
      const int u = g * GROUP + i;
      if (inside(u)) read[g & 1][i] = a.epi.read(batch, m0 + row_at(u), n0 + block_at(u) + 8 * (lane >> 4));
    }
  };
  request(0);
#pragma unroll
  for (int g = 0; g < UNITS / GROUP; ++g) {
    if (g + 1 < UNITS / GROUP) request(g + 1);
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
      const int u = g * GROUP + i, p = u % PAIRS, tm = u / PAIRS;
      const int row = m0 + row_at(u), col = n0 + block_at(u) + 8 * (lane >> 4);
      float v[8];
      lane_values<T>(acc, p, tm, v);
      if constexpr (Epi::kGated) {
        float w[8];
        lane_values<T>(acc, 1, tm, w);
        if (inside(u)) a.epi(batch, row, col, v, w);
      } else if constexpr (Epi::kMirror) {
        u32x4 q = {0, 0, 0, 0};
        if (inside(u)) q = a.epi(batch, row, col, v, read[g & 1][i]);
        uint16_t* to = reinterpret_cast<uint16_t*>(lds + (block_at(u) + 8 * (lane >> 4)) * mirror_pitch<T>()) + row_at(u);
        if (mirrored)
#pragma unroll
          for (int e = 0; e < 8; ++e) to[e * (mirror_pitch<T>() / 2)] = (uint16_t)(q[e / 2] >> (16 * (e & 1)));
      } else {
        if (inside(u)) a.epi(batch, row, col, v, read[g & 1][i]);
      }
    }
  }
  if constexpr (Epi::kMirror) {
    if (!mirrored) return;
    __syncthreads();
    constexpr int CH = T::BM / 8;  // 16-byte pieces of a column of the tile
    static_assert(T::BN * CH % T::THREADS == 0, "whole rounds");
    for (int j = 0; j < T::BN * CH / T::THREADS; ++j) {
      const int i = tid + j * T::THREADS, col = i / CH, piece = i % CH;
      if (n0 + col < a.N && m0 + 8 * piece < a.epi.rows)
        a.epi.mirror(batch, n0 + col, m0 + 8 * piece, *reinterpret_cast<const u32x4*>(lds + col * mirror_pitch<T>() + 16 * piece));
    }
  }
}

template <class T, class Elem, class P>
__device__ __forceinline__ void run_product(const P& a, int item, int batch, char* lds) {
  constexpr int COLS = P::Epi::kGated ? T::EC : T::BN;  // result columns of a tile
  static_assert(T::BK == 64, "a stage is a unit of K");
  const int total = a.walk.total(), s = item / total, tile = item - s * total;
  int tm_, tn_;
  a.walk.at(tile, tm_, tn_);
  const int m0 = tm_ * T::BM, n0 = tn_ * COLS;
  const int st0 = s * a.per, nk = min(a.per, a.nk - st0);
  Acc<T> acc;
  if constexpr (T::QUAD) product_pingpong<T, Elem, P::CO, P::JUMP>(a.r, a.c, batch, m0, n0, st0, nk, acc, lds);
  else product_loop<T, Elem, P::CO, P::JUMP>(a.r, a.c, batch, m0, n0, st0, nk, acc, lds);
  finish_product<T>(a, acc, batch, tile, s, tm_, tn_, lds);
}

template <class T, class Elem, class P>
__global__ __launch_bounds__(T::THREADS) __attribute__((amdgpu_waves_per_eu(2))) void k_product(const P a) {
  __shared__ __align__(1024) char lds[lds_of<T, P>()];
  run_product<T, Elem>(a, blockIdx.x, blockIdx.y, lds);
}

// Three products in one launch: the items of a, b and c, from item `first` of
// that order on and round to it (the longest items go first).
template <class T, class Elem, class PA, class PB, class PC>
__global__ __launch_bounds__(T::THREADS) __attribute__((amdgpu_waves_per_eu(2))) void k_products(const PA a, const PB b, const PC c,
                                                                                                   int first) {
  __shared__ __align__(1024) char lds[T::LDS];
  static_assert(!PA::Epi::kMirror && !PB::Epi::kMirror && !PC::Epi::kMirror, "no room for a transpose");
  const int na = a.items(), nb = b.items(), all = gridDim.x, from = blockIdx.x + first, item = from < all ? from : from - all;
  if (item < na) run_product<T, Elem>(a, item, 0, lds);
  else if (item < na + nb) run_product<T, Elem>(b, item - na, 0, lds);
  else run_product<T, Elem>(c, item - na - nb, 0, lds);
}

// ------------------------------------------------------------------ host side

inline Side make_side(const void* p, int64_t ld, int64_t bytes) {
  Side s{};
  s.p = (const uint16_t*)p;
  s.ld = ld;
  s.bytes = bytes;
  return s;
}

// What a plan lends its products for split K.
struct SplitSpace {
  float* part;
  int64_t part_floats;
  uint32_t* arrived;
  int64_t counters;
};

constexpr int kMaxSplit = 32;
constexpr int64_t kSplitCounters = 4096;

// Floats of the parts of any product with up to M x N results: all that the
// splits can ask for, but 96 MB at most (a part and slot of the largest tile is
// 64 MB; a launch of several products holds the parts of each).
inline int64_t split_floats(int64_t M, int64_t N, int64_t batches) {
  const int64_t most = (int64_t)24 << 20, all = kMaxSplit * batches * round_up(M, 256) * round_up(N, 256);
  return all < most ? all : most;
}

enum { TILE_64, TILE_128, TILE_256, TILES };

// The sizes that tile and split are chosen by.
struct Shape {
  int64_t M, N, K;  // N: columns of a result (of each of a gated product's two)
  int batches;
  bool gated, symmetric;
};

// What a tile costs a work-group, in microseconds: `unit` for 64 of K with every
// slot of the chip taken, `alone` with at most one work-group to a CU, `item`
// once (prologue and epilogue), `join` for meeting the other parts of K beside
// the traffic of their sums, and `part` for each of them.  Measured with the
// products of 2048 x 4096 x 14336 (every slot taken), 24 x 4096 x 14336, 64 x 512 x
// 2048, and by their parts of K: the Gram matrices of 4 x 37 x 5081 (64 x 64 tiles;
// 2, 4, 8, 16 and 27 parts 12.8, 9.6, 8.0, 9.0 and 11.9 us) and of 1664 x 6656 (128 x
// 128; 1, 2, 4 and 5 parts 69, 45, 38 and 38), 2063 x 768 with K = 8192 (256 x 256;
// 1, 2, 3, 4, 6 and 8 parts 131, 81, 65, 60, 62 and 65).
struct TileCost {
  int rows, cols, slots;  // slots: work-groups to a CU
  double unit, alone, item, join, part;
};
// `once`: every weight is read by one row of tiles, from memory and not from an
// L2 (23 rows of 7104 by 2 x 18944, 296 tiles: 153 us, in two parts of K 111).
inline TileCost tile_cost(int tile, bool gated, bool once) {
  if (tile == TILE_256) return {256, gated ? 128 : 256, 1, 1.40, 1.20, 12.0, 1.0, 1.5};
  if (tile == TILE_128) return {128, gated ? 64 : 128, 2, 1.20, 0.65, 4.0, 2.5, 0.8};
  if (gated) return {64, 64, 2, once ? 1.30 : 0.80, once ? 0.58 : 0.45, 3.0, 0.5, 0.5};
  return {64, 64, 2, 0.50, 0.25, 3.0, 0.5, 0.3};
}
constexpr double kBytesPerUs = 6.0e6;   // what parts are written and read at (most stay in the last-level cache)
constexpr double kStreamPerUs = 5.2e6;  // what a product reads its operands at

struct Choice {
  int tile, split;
};

inline int64_t tiles_of(const Shape& s, const TileCost& t) {
  const int64_t m = (s.M + t.rows - 1) / t.rows, n = (s.N + t.cols - 1) / t.cols;
  return s.batches * (s.symmetric ? m * (m + 1) / 2 : m * n);
}
inline int64_t units_of(const Shape& s) { return (s.K + 63) / 64; }

// The most parts that the workspace has room for.
inline int64_t split_room(const Shape& s, const TileCost& t, const SplitSpace& ws) {
  const int64_t tiles = tiles_of(s, t);
  if (tiles < 1 || tiles > ws.counters) return 1;
  const int64_t room = ws.part_floats / (tiles * t.rows * t.cols * (s.gated ? 2 : 1));
  return room < 1 ? 1 : room;
}

// Microseconds for the parts' sums, written and read.
inline double join_time(const Shape& s, const TileCost& t, int64_t split) {
  const int64_t rows = s.M < t.rows ? round_up(s.M, 16) : t.rows;
  return split > 1 ? t.join + t.part * split + 8.0 * tiles_of(s, t) * split * rows * t.cols * (s.gated ? 2 : 1) / kBytesPerUs : 0.0;
}

// Time of the tiles' items, whole rounds of the chip's slots, then the rest, and
// of the operands' traffic; where both are alike they hold each other up.  (24
// rows of 14336 by 14336 x 4096 in 64 tiles, two to six parts of K: 40, 30, 27, 37
// and 33 us; the estimates 36, 30, 28, 33 and 30.)
inline double product_time(const Shape& s, const TileCost& t, int64_t split, int num_cus) {
  const int64_t items = tiles_of(s, t) * split, slots = (int64_t)num_cus * t.slots, per = (units_of(s) + split - 1) / split;
  const int64_t rest = items % slots;
  double time = (double)(items / slots) * (per * t.unit + t.item);
  if (rest) time += per * (rest <= num_cus ? t.alone : t.unit) + t.item;
  const double bytes = 2.0 * s.batches * ((double)s.M * s.K + (s.symmetric ? 0.0 : (double)s.N * s.K * (s.gated ? 2 : 1)));
  const double stream = bytes / kStreamPerUs + t.item;
  return std::cbrt(time * time * time + stream * stream * stream) + join_time(s, t, split);
}

// The tile and split of one product: the least of the estimates.  (Splitting
// only the tiles of a last round that leaves half of the CUs idle was tried:
// 441 -> 463 us for the forward pass's first product of 2048 x 4096 x 14336,
// 454 -> 437 us for an orthogonalisation's update; busy halves clock higher.)
inline Choice choose(const Shape& s, const SplitSpace& ws, int num_cus) {
  Choice best{TILE_64, 1};
  double least = 1e30;
  for (int tile = 0; tile < TILES; ++tile) {
    TileCost t = tile_cost(tile, s.gated, s.M <= 64);
    if (s.symmetric && tile == TILE_128) t.unit = 1.0, t.alone = 0.6;  // K is contiguous on both sides
    const int64_t units = units_of(s), room = split_room(s, t, ws), most = units < kMaxSplit ? units : kMaxSplit;
    for (int64_t split = 1; split <= most && split <= room; ++split) {
      const double time = product_time(s, t, split, num_cus);
      if (time < least) {
        least = time;
        best = Choice{tile, (int)split};
      }
    }
  }
  return best;
}

// One tile for products that share a launch, and the split of each: every
// slot gets about the same work, so no item should last longer than that.
// The weights of the terms below (three fifths of a share, three times the fixed
// cost, half of a join, three tenths of the shorter time) were set by trying,
// and the operands' stream is left out.  Against every tile with 1 to 32 parts
// of dX (and 1, 2 and 4 of the weight gradients up to 1000 rows), us for whole
// backward passes, the choice, the best, and the best of each other tile:
//   64 x 512 x 2048 SwiGLU      17.4 (64, 3 parts)   15.2 (64, 8 parts)   128: 22.9   256: 36.8
//   24 x 4096 x 14336 SwiGLU    185 (128, 5)         179 (256, 8)         64: 261     128: 184
//   128 x 1024 x 4096 GELU      25.0 (64, 3)         24.4 (64, 2)         128: 28.1   256: 40.4
//   300 x 2048 x 5440 SwiGLU    70-73 (128, 5)       65 (128, 4)          64: 87      256: 77
//   777 x 2112 x 5440 GELU      108 (256, 3)         100 (128, 1)         64: 126     256: 107
//   1500 x 2048 x 5632 SwiGLU   222 (256, 3)         218 (256, 4)         64: 315     128: 222
//   2048 x 4096 x 14336 SwiGLU  1100 (256, 1)        1097 (the same)      64: 2040    128: 1415
template <int N>
int choose_shared(const Shape (&s)[N], const SplitSpace& ws, int num_cus, int (&split)[N]) {
  int best = TILE_64;
  double least = 1e30;
  for (int tile = 0; tile < TILES; ++tile) {
    int parts[N];
    double work = 0.0;
    const TileCost t = tile_cost(tile, false, false);
    int64_t items = 0;
    for (int i = 0; i < N; ++i) {
      items += tiles_of(s[i], t);
      work += tiles_of(s[i], t) * (units_of(s[i]) * t.unit + t.item);
    }
    const double slots = (double)num_cus * t.slots, share = work / slots;
    double longest = 0.0, extra = 0.0;
    for (int i = 0; i < N; ++i) {
      const int64_t tiles = tiles_of(s[i], t), units = units_of(s[i]);
      parts[i] = 1;
      if (!tiles) continue;
      // (a long item shares its CU with short ones that mostly move data)
      const double unit = items <= num_cus ? t.alone : 0.5 * (t.alone + t.unit);
      // An item longer than its slot's share is cut to three fifths of it, or to where overheads would outweigh the work.
      const double whole = units * unit + t.item, limit = 0.6 * share > 3 * t.item ? 0.6 * share : 3 * t.item;
      int64_t want = whole > share ? (int64_t)(units * unit / limit + 0.999) : 1;
      const int64_t room = split_room(s[i], t, ws);
      if (want > room) want = room;
      if (want > units) want = units;
      if (want > kMaxSplit) want = kMaxSplit;
      if (want > 1) parts[i] = (int)want;
      const double one = (double)((units + parts[i] - 1) / parts[i]) * unit + t.item + (parts[i] > 1 ? t.join + t.part * parts[i] : 0.0);
      if (one > longest) longest = one;
      if (parts[i] > 1) extra += (double)tiles * (parts[i] - 1) * t.item / slots + 0.5 * join_time(s[i], t, parts[i]);
    }
    const double even = share + extra, time = even > longest ? even + 0.3 * longest : longest + 0.3 * even;
    if (time < least) {
      least = time;
      best = tile;
      for (int i = 0; i < N; ++i) split[i] = parts[i];
    }
  }
  return best;
}

template <class T, class P>
P make_problem(const decltype(P::r)& r, const decltype(P::c)& c, int64_t M, int64_t N, int64_t K, int batches, const typename P::Epi& epi, int parts,
               const SplitSpace& ws) {
  constexpr int COLS = P::Epi::kGated ? T::EC : T::BN;
  P a{};
  a.r = r;
  a.c = c;
  a.M = (int)M;
  a.N = (int)N;
  a.nk = (int)((K + 63) / 64);
  a.part = ws.part;
  a.arrived = ws.arrived;
  a.walk.tiles_m = (int)((M + T::BM - 1) / T::BM);
  a.walk.tiles_n = (int)((N + COLS - 1) / COLS);
  a.walk.band = P::Epi::kSymmetric ? 4 : 8;
  a.walk.sym = P::Epi::kSymmetric;
  // No part is empty, and every part of every tile has its place in the workspace.
  const int64_t tiles = (int64_t)a.walk.total() * batches;
  const int64_t room = tiles >= 1 && tiles <= ws.counters ? ws.part_floats / (tiles * T::BM * T::BN) : 1;
  int64_t split = parts < room ? parts : room;
  if (split > a.nk) split = a.nk;
  a.per = split > 1 ? (int)((a.nk + split - 1) / split) : a.nk;
  a.split = split > 1 ? (a.nk + a.per - 1) / a.per : 1;
  a.epi = epi;
  return a;
}

// What is left of the workspace behind a product's parts.
template <class T, class P>
SplitSpace behind(const SplitSpace& ws, const P& a) {
  if (a.split == 1) return ws;
  const int64_t tiles = a.walk.total(), floats = tiles * a.split * T::BM * T::BN;
  return {ws.part + floats, ws.part_floats - floats, ws.arrived + tiles * kLine, ws.counters - tiles};
}

template <class T, class Elem, class P>
hipError_t launch_product(const P& a, int batches, hipStream_t stream) {
  k_product<T, Elem, P><<<dim3((unsigned)a.items(), (unsigned)batches), T::THREADS, 0, stream>>>(a);
  return hipGetLastError();
}

// Calls f with the tile type of a choice.
template <class Epi, class F>
auto with_tile(int tile, F&& f) {
  if (tile == TILE_256) return f(Tile256{});
  if (tile == TILE_128) return f(Tile128{});
  if constexpr (Epi::kGated) return f(Tile64G{});
  else return f(Tile64{});
}

// One product with the tile and split that suit it.
template <class Elem, bool CO, class Epi>
hipError_t product(const Side& r, const Side& c, int64_t M, int64_t N, int64_t K, int batches, const Epi& epi, const SplitSpace& ws,
                   int num_cus, hipStream_t stream) {
  const Choice ch = choose({M, N, K, batches, Epi::kGated, Epi::kSymmetric}, ws, num_cus);
  return with_tile<Epi>(ch.tile, [&](auto tile) {
    using T = decltype(tile);
    return launch_product<T, Elem>(make_problem<T, Problem<CO, Epi>>(r, c, M, N, K, batches, epi, ch.split, ws), batches, stream);
  });
}

}  // namespace mlp2
