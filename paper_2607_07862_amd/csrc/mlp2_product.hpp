// Tile products of the training operators: C[m][n] = sum over k of R(m, k) C(n, k)
// for operands of either storage order, with a fused epilogue.
//
// The forward kernels of the library multiply activations [M, K] by weights
// [K, N].  Training needs every other order too: dZ = dY W2^T reads weights
// whose K is contiguous, dW = X^T dP reads both operands with K as the slow
// index.  Here each side of the product is staged through LDS in panels of
// its own order:
//
//   inner panel (K contiguous in memory): [rows][64 k], 128-byte rows, read
//     by ds_read_b128 (8 consecutive k per lane);
//   outer panel (K is the slow index): [64 k][columns], read transposed by
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

#include "mlp2_device.hpp"

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
  int64_t bytes;   // readable bytes from p; anything past them reads as zero
  int64_t panel;   // elements from a tile's first panel to its second; 0: the next rows (columns) of the same matrix
  int64_t jump;    // elements added to the base from stage `jump_at` on (K runs through a second matrix)
  int jump_at;     // stage of 64 k, or INT_MAX
  int64_t batch;   // elements between the matrices of a batch
};

// A work-group tile: ROWP row panels and COLP column panels of E rows
// (columns) each, WM x WN waves, an NS-deep ring of 64-deep stages.  Every
// wave owns 32 columns of every column panel (so that the two panels of a
// gated product, gate and up weights, meet in one lane) and 16 * TM rows.
template <int E_, int ROWP_, int COLP_, int WM_, int WN_, int NS_>
struct PTile {
  static constexpr int E = E_, ROWP = ROWP_, COLP = COLP_, WM = WM_, WN = WN_, NS = NS_;
  static constexpr int NWAVES = WM * WN, THREADS = 64 * NWAVES;
  static constexpr int BM = E * ROWP, BN = E * COLP;
  static constexpr int TM = BM / WM / 16;             // 16-row blocks of a wave
  static constexpr int PANEL = E * 128;               // bytes of a panel's stage
  static constexpr int STAGE = (ROWP + COLP) * PANEL;
  static constexpr int PIECES = PANEL / 1024 / NWAVES;  // 1 KB loads per wave and panel
  static constexpr int LOADS = (ROWP + COLP) * PIECES;  // and per stage
  static constexpr int LDS = NS * STAGE;
  static_assert(E == 32 * WN, "a wave owns 32 columns of every column panel");
  // Wave wm's row block tm.  Two row panels: the wave's rows lie in both halves
  // of an eight-wave tile, in panel wm of a four-wave one.
  __device__ static constexpr int row_of(int wm, int tm) {
    return NWAVES == 8 ? 64 * wm + 16 * (tm & 3) + 128 * (tm >> 2) : wm * (BM / WM) + 16 * tm;
  }
};
using Tile64 = PTile<64, 1, 1, 2, 2, 8>;    // 64 x 64
using Tile64G = PTile<64, 1, 2, 2, 2, 5>;   // 64 x (64 + 64): gated, or 64 x 128
using Tile128 = PTile<64, 2, 2, 2, 2, 4>;   // 128 x 128, gated 128 x (64 + 64)

// ------------------------------------------------------------------ panel loads

__device__ __forceinline__ u32x4 panel_rsrc(const char* base, int64_t left) {
  const uint64_t b = (uint64_t)base;
  const uint32_t n = left <= 0 ? 0u : left > 0xFFFFFFFFll ? 0xFFFFFFFFu : (uint32_t)left;
  return u32x4{(uint32_t)b, (uint32_t)(b >> 32) & 0xFFFFu, n, 0x00027000u};
}

// One direct-to-LDS buffer load: lane i moves 16 bytes from base + voff to
// lds_addr + 16 i, zeros where voff is past the descriptor's range.  The wait
// states ahead of it cover a scalar operand that a vector instruction has just
// written (the compiler keeps them for its own instructions, not for an asm's).
__device__ __forceinline__ void dma16_buffer(u32x4 rsrc, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "{m0}"(lds_addr) : "memory");
}

// The chunk swizzle of a panel's row (inner: row of 8 chunks; outer: k row of E / 8 chunks).
__device__ __forceinline__ int swz_inner(int row) { return (row >> 1) & 7; }
template <int E>
__device__ __forceinline__ int swz_outer(int k) {
  return E == 128 ? (4 * (k & 3)) ^ (2 * ((k >> 3) & 1)) : (4 * ((k >> 1) & 1)) ^ (2 * ((k >> 3) & 1));
}

// Loads of one panel, stage by stage.  COL: the column side, whose inner panels
// hold their rows permuted within every 32 (LDS row 16 t + i is matrix row
// 8 (i / 4) + 4 t + i % 4), so that a pair of blocks gives a lane 8 consecutive
// columns; outer panels get the same from the fragment addresses.
template <class T, bool OUTER, bool COL>
struct PanelLoad {
  const char* base;
  int64_t left, step, jump;
  int to_jump;
  uint32_t voff, piece_step;
  uint32_t lds;  // of this wave's first piece, from the stage's base

  __device__ __forceinline__ PanelLoad(const Side& s, int64_t batch, int i0, int panel, int stage0, uint32_t lds_off) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63, wave = uniform(tid >> 6);
    constexpr int E = T::E;
    int64_t first = batch * s.batch + (int64_t)panel * (s.panel ? s.panel : OUTER ? E : E * s.ld);
    first += OUTER ? i0 + (int64_t)stage0 * 64 * s.ld : (int64_t)i0 * s.ld + (int64_t)stage0 * 64;
    step = (OUTER ? 64 * s.ld : 64) * 2;
    jump = s.jump * 2;
    to_jump = s.jump_at - stage0;
    if (to_jump <= 0) first += s.jump;
    base = (const char*)(s.p + first);
    left = s.bytes - 2 * first;
    int row, chunk;
    if constexpr (OUTER) {
      constexpr int CPR = E / 8, RPP = 64 / CPR;  // chunks per k row, k rows per piece
      row = RPP * wave + lane / CPR;
      chunk = (lane % CPR) ^ swz_outer<E>(row);
      piece_step = (uint32_t)(T::NWAVES * RPP * s.ld * 2);
      voff = (uint32_t)((row * s.ld + 8 * chunk) * 2);
    } else {
      row = 8 * wave + lane / 8;
      chunk = (lane & 7) ^ swz_inner(row);
      const int i = row & 15;
      const int at = COL ? (row & ~31) + 8 * (i >> 2) + 4 * ((row >> 4) & 1) + (i & 3) : row;
      piece_step = (uint32_t)(T::NWAVES * 8 * s.ld * 2);
      voff = (uint32_t)((at * s.ld + 8 * chunk) * 2);
    }
    lds = lds_off + (uint32_t)wave * 1024u;
  }
  __device__ __forceinline__ void load(uint32_t stage_lds) {
    const u32x4 r = panel_rsrc(base, left);
#pragma unroll
    for (int j = 0; j < T::PIECES; ++j)
      dma16_buffer(r, voff + j * piece_step, uniform(stage_lds + lds + (uint32_t)(j * T::NWAVES * 1024)));
    const int64_t by = --to_jump == 0 ? step + jump : step;
    base += by;
    left -= by;
  }
};

// ------------------------------------------------------------------ fragments

// Row side: lane holds row (lane % 16) of a 16-row block, k = 8 (lane / 16) .. + 7 of a 32-deep slice.
template <class T, bool OUTER>
struct RowFrag {
  uint32_t off[2];  // inner: one per K slice; outer: one
  __device__ __forceinline__ RowFrag(int wm) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63;
    const int r0 = T::NWAVES == 8 ? 64 * wm : (wm * (T::BM / T::WM)) % T::E;
    const uint32_t panel = T::NWAVES == 8 ? 0u : (uint32_t)((wm * (T::BM / T::WM)) / T::E * T::PANEL);
    if constexpr (OUTER) {
      // lane 4 r + c of group g addresses k row 8 g + r, columns 4 c .. + 3 of the block
      const int k = 8 * (lane >> 4) + ((lane & 15) >> 2), c = lane & 3;
      off[0] = panel + (uint32_t)(k * (2 * T::E) + ((((r0 >> 3) + (c >> 1)) ^ swz_outer<T::E>(k)) << 4) + 8 * (c & 1));
      off[1] = 0;
    } else {
      const int row = r0 + (lane & 15);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) off[ks] = panel + (uint32_t)(row * 128 + (((4 * ks + (lane >> 4)) ^ swz_inner(row)) << 4));
    }
  }
  // block tm of K slice ks; `stage` is the address of the stage's row panels
  __device__ __forceinline__ u32x4 read(const char* stage, int ks, int tm) const;
};

__device__ __forceinline__ u32x4 read_tr(const char* p, int upper) {
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(p));
  const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(p + upper));
  typedef short i16x8 __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(u32x4, (i16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <class T, bool OUTER>
__device__ __forceinline__ u32x4 RowFrag<T, OUTER>::read(const char* stage, int ks, int tm) const {
  const int half = T::NWAVES == 8 ? tm >> 2 : 0, blk = T::NWAVES == 8 ? tm & 3 : tm;
  if constexpr (OUTER) {
    // Block blk is 2 blk chunks further on; the swizzle touches chunk bits 1 to 3, so the offset is XORed, not added.
    return read_tr(stage + half * T::PANEL + (off[0] ^ (uint32_t)(32 * blk)) + ks * 64 * T::E, 8 * T::E);
  } else {
    return *reinterpret_cast<const u32x4*>(stage + half * T::PANEL + off[ks] + blk * 2048);
  }
}

// Column side: block i of the pair that covers the wave's 32 columns of a panel.
template <class T, bool OUTER>
struct ColFrag {
  uint32_t off[2];
  __device__ __forceinline__ ColFrag(int wn) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63;
    if constexpr (OUTER) {
      // columns 8 c + 4 i .. + 3 of the pair: the interleave that leaves 8 consecutive columns in a lane
      const int k = 8 * (lane >> 4) + ((lane & 15) >> 2);
      off[0] = (uint32_t)(k * (2 * T::E) + (((4 * wn + (lane & 3)) ^ swz_outer<T::E>(k)) << 4));
      off[1] = 0;
    } else {
      const int row = 32 * wn + (lane & 15);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) off[ks] = (uint32_t)(row * 128 + (((4 * ks + (lane >> 4)) ^ swz_inner(row)) << 4));
    }
  }
  __device__ __forceinline__ u32x4 read(const char* panel, int ks, int i) const {
    if constexpr (OUTER) return read_tr(panel + off[0] + 8 * i + ks * 64 * T::E, 8 * T::E);
    else return *reinterpret_cast<const u32x4*>(panel + off[ks] + i * 2048);
  }
};

// ------------------------------------------------------------------ mainloops

template <class T>
using Acc = f32x4[T::COLP][2][T::TM];

// The plain loop: NS - 1 stages in flight, one barrier a stage.
template <class T, class Elem, bool RO, bool CO>
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
  PanelLoad<T, RO, false> r0(rs, batch, m0, 0, st0, 0), r1(rs, batch, m0, T::ROWP - 1, st0, (T::ROWP - 1) * T::PANEL);
  PanelLoad<T, CO, true> c0(cs, batch, n0, 0, st0, T::ROWP * T::PANEL),
      c1(cs, batch, n0, T::COLP - 1, st0, (T::ROWP + T::COLP - 1) * T::PANEL);
  auto issue = [&](int st) {
    const uint32_t dst = lds_base + (uint32_t)((st % T::NS) * T::STAGE);
    r0.load(dst);
    if constexpr (T::ROWP == 2) r1.load(dst);
    c0.load(dst);
    if constexpr (T::COLP == 2) c1.load(dst);
  };
  const RowFrag<T, RO> rf(wm);
  const ColFrag<T, CO> cf(wn);
#pragma unroll
  for (int st = 0; st < T::NS - 1; ++st)
    if (st < nk) issue(st);
  for (int it = 0; it < nk; ++it) {
    wait_stages_behind<T::LOADS, T::NS - 2>(min(T::NS - 2, nk - 1 - it));
    __syncthreads();
    if (it + T::NS - 1 < nk) issue(it + T::NS - 1);
    const char* stage = lds + (it % T::NS) * T::STAGE;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      u32x4 x[T::TM], w[T::COLP][2];
#pragma unroll
      for (int tm = 0; tm < T::TM; ++tm) x[tm] = rf.read(stage, ks, tm);
#pragma unroll
      for (int p = 0; p < T::COLP; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i) w[p][i] = cf.read(stage + (T::ROWP + p) * T::PANEL, ks, i);
#pragma unroll
      for (int p = 0; p < T::COLP; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int tm = 0; tm < T::TM; ++tm) acc[p][i][tm] = Elem::mfma(w[p][i], x[tm], acc[p][i][tm]);
    }
  }
  __syncthreads();
}

// ------------------------------------------------------------------ the kernel

// Output tiles of M x N (COLS columns of every column panel's matrix), walked
// so that an XCD's work-groups (blockIdx % 8) share operand panels: each XCD
// takes a contiguous range of an order that goes down `band` row tiles before
// the next column tile.
struct TileWalk {
  int tiles_m, tiles_n, band;
  __device__ __forceinline__ void at(int item, int& tm, int& tn) const {
    const int total = tiles_m * tiles_n, q = total / 8, r = total % 8, x = item % 8;
    const int t = x * q + min(x, r) + item / 8;
    const int per = band * tiles_n, g = t / per, in = t - g * per;
    const int rows = min(band, tiles_m - g * band);
    tn = in / rows;
    tm = g * band + (in - tn * rows);
  }
};

template <class Epi>
struct ProductArgs {
  Side r, c;
  int M, N;          // rows and columns of the result (of each matrix of a gated product)
  int nk;            // 64-deep stages of K
  TileWalk walk;
  Epi epi;
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

// Epi::kGated: the two column panels are the same columns of two matrices and
// the epilogue takes both values; otherwise they are consecutive columns.
template <class T, class Elem, bool RO, bool CO, class Epi>
__global__ __launch_bounds__(T::THREADS) void k_product(const ProductArgs<Epi> a) {
  __shared__ __align__(1024) char lds[T::LDS];
  constexpr int COLS = Epi::kGated ? T::E : T::BN;  // result columns of a tile
  int tm_, tn_;
  a.walk.at(blockIdx.x, tm_, tn_);
  const int m0 = tm_ * T::BM, n0 = tn_ * COLS;
  const int batch = blockIdx.y;
  Acc<T> acc;
  product_loop<T, Elem, RO, CO>(a.r, a.c, batch, m0, n0, 0, a.nk, acc, lds);
  const int tid = thread_here(), lane = tid & 63, wave = uniform(tid >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM;
#pragma unroll
  for (int tm = 0; tm < T::TM; ++tm) {
    const int row = m0 + T::row_of(wm, tm) + (lane & 15);
    if constexpr (Epi::kGated) {
      const int block = n0 + 32 * wn;
      float g[8], u[8];
      lane_values<T>(acc, 0, tm, g);
      lane_values<T>(acc, 1, tm, u);
      if (block < a.N && row < a.M) a.epi(batch, row, block + 8 * (lane >> 4), g, u);
    } else {
#pragma unroll
      for (int p = 0; p < T::COLP; ++p) {
        const int block = n0 + p * T::E + 32 * wn;
        float v[8];
        lane_values<T>(acc, p, tm, v);
        if (block < a.N && row < a.M) a.epi(batch, row, block + 8 * (lane >> 4), v);
      }
    }
  }
}

inline Side make_side(const void* p, int64_t ld, int64_t bytes) {
  Side s{};
  s.p = (const uint16_t*)p;
  s.ld = ld;
  s.bytes = bytes;
  s.jump_at = 0x7FFFFFFF;
  return s;
}

template <class T, class Elem, bool RO, bool CO, class Epi>
hipError_t launch_product(const Side& r, const Side& c, int64_t M, int64_t N, int64_t K, int batches, const Epi& epi,
                          hipStream_t stream) {
  constexpr int COLS = Epi::kGated ? T::E : T::BN;
  ProductArgs<Epi> a;
  a.r = r;
  a.c = c;
  a.M = (int)M;
  a.N = (int)N;
  a.nk = (int)((K + 63) / 64);
  a.walk.tiles_m = (int)((M + T::BM - 1) / T::BM);
  a.walk.tiles_n = (int)((N + COLS - 1) / COLS);
  a.walk.band = 8;
  a.epi = epi;
  auto kernel = k_product<T, Elem, RO, CO, Epi>;
  kernel<<<dim3((unsigned)(a.walk.tiles_m * a.walk.tiles_n), (unsigned)batches), T::THREADS, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace mlp2
