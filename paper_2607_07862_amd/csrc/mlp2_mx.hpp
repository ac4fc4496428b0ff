// Products of two MXFP4 matrices: C[m][n] = sum over k of A(m, k) W(n, k), K contiguous on both sides.
//
// MXFP4: 32 neighbours along K share a scale 2^(s - 127); the values are 0, 0.5,
// 1, 1.5, 2, 3, 4, 6 and their negatives, two to a byte.  Codes lie row-major,
// K padded to a multiple of 128 with zeros; scales as [K / 128][row][4], so that
// the scales of one row and 128 of K are one word and those of a tile's rows lie
// together.
//
// The matrix instruction takes 16 x 16 x 128 at a time, 16 bytes of codes a lane
// and operand: the same bytes, lanes and cycles as 16 x 16 x 32 of bf16.  So the
// tiles, rings and slots are those of the 16-bit products (a stage of 64 16-bit
// elements holds 256 of K) and the estimates that choose tile and split count K in
// units of 64 x 16 bits.  (Of 14 products from 1 x 4096 x 14336 to 4096 cubed the
// choice was the best of every tile with 1 to 16 parts, or within 12 % of it: 7.3
// against 6.6 us for 16 x 4096 x 4096, 8.7 against 8.1 for 128 rows of it.)  What
// comes on top are the scales: two words a row and stage, one more direct-to-LDS
// load (4 bytes a lane) for each wave and side.
//
// Few rows are bound by the weights (64 x 14336 x 4096, gated: 64 MB in 12.6 us, partly
// out of the caches; 15.0 from memory), many by the matrix cores and their power (4096 x
// 14336 x 4096, gated: 239 to 250 us on several machines, 3.85 to 4.0 PFLOP/s; matrix cores
// busy for 44 % of the clocks, at 2 GHz).  Between them waits do: 777 x 2111 x 5441 takes
// 15.6 us with LDS busy for 11 % of the clocks and the matrix cores for 9 %, its waves
// waiting for 40 % of theirs.
//
// K is dealt to the lanes so that a lane's two 16-byte chunks of a stage are
// neighbours, chunks 2 g and 2 g + 1 for lane group g = lane / 16: their scales are
// neighbouring bytes of one word, of which the instruction picks one by itself.
#pragma once

#include "mlp2_product.hpp"

namespace mlp2 {

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kMxBlock = 32;   // elements that share a scale
constexpr int kMxGroup = 128;  // elements whose scales share a word
__host__ __device__ constexpr int64_t mx_padded(int64_t k) { return (k + kMxGroup - 1) / kMxGroup * kMxGroup; }

typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
// A scale as the float that the conversion instructions take: they use its exponent field alone, 0 standing for 2^-127 and 255 for NaN.
__device__ __forceinline__ float mx_unit(uint32_t s) {
  return __builtin_bit_cast(float, s << 23);
}

constexpr int kFp4 = 4;  // the operand format of the scaled matrix instruction

// c += W X for 16 columns (w) by 16 rows (x) and 128 of K; the scales of this lane's 32 are bytes BW of sw and BX of sx.
template <int BW, int BX>
__device__ __forceinline__ f32x4 mfma_mx(u32x4 w, u32x4 x, f32x4 c, int sw, int sx) {
  const i32x8 a = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0}, b = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, kFp4, kFp4, BW, sw, BX, sx);
}

// Two by two blocks, chunk KS of the stage: w0 and w1 with the two halves of sw, x0 and x1 with those of sx.
template <int KS>
__device__ __forceinline__ void mx_block(f32x4& c00, f32x4& c01, f32x4& c10, f32x4& c11, u32x4 w0, u32x4 w1, u32x4 x0, u32x4 x1, int sw, int sx) {
  c00 = mfma_mx<KS, KS>(w0, x0, c00, sw, sx);
  c01 = mfma_mx<KS, 2 + KS>(w0, x1, c01, sw, sx);
  c10 = mfma_mx<2 + KS, KS>(w1, x0, c10, sw, sx);
  c11 = mfma_mx<2 + KS, 2 + KS>(w1, x1, c11, sw, sx);
}

// One side of a product.  Matrix i of several (the gate and up weights) starts i * rows * ld bytes on.
struct MxSide {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t rows;   // of one matrix
  int64_t ld;     // bytes of a row of codes: padded K / 2
  bool gated;     // a tile's second panel is the same rows of the next matrix
};

// A stage in LDS: the panels' codes, rows of 128 bytes; then the scales of the rows, a word for each 128 of K, and of the columns.
template <class T>
struct MxTile {
  static constexpr int RPANEL = T::ER * 128, CPANEL = T::EC * 128, C0 = T::ROWP * RPANEL;
  // the second 128's words lie 16 banks on, so that one read of both halves' words meets no bank twice
  static constexpr int RPITCH = T::BM * 4 + 64, CPITCH = T::BN * 4 + 64;
  static constexpr int RSCALES = C0 + T::COLP * CPANEL, CSCALES = RSCALES + 2 * RPITCH;
  static constexpr int STAGE = (CSCALES + 2 * CPITCH + 1023) / 1024 * 1024;
  static constexpr int LOADS = T::LOADS + 2;  // of a wave and stage
  static constexpr int LDS = T::NS * STAGE;
};

// One direct-to-LDS buffer load of 4 bytes a lane: lane i's to lds_addr + 4 i, zeros past the range.
__device__ __forceinline__ void dma4_buffer(u32x4 rsrc, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "{m0}"(lds_addr) : "memory");
}

// Loads of one panel's codes, stage by stage: rows past the matrix's end read as zeros, and so do the chunks that do not exist in a last
// stage of 128 of K.  Every panel of a side has the same offsets in its lanes; bases and ranges are scalars.
//
// Chunk c = 2 g + ks of row r lies at (4 ks + g) ^ swz_inner(r): the reads of one ks meet no bank twice, as those of the 16-bit panels.
template <class T, bool COL>
struct MxLanes {
  static constexpr int E = COL ? T::EC : T::ER, PIECES = E * 128 / 1024 / T::NWAVES;
  uint32_t voff[PIECES];
  bool upper;  // this lane's chunk lies in the upper half of a stage
  __device__ __forceinline__ explicit MxLanes(const MxSide& s) {
    const int tid = thread_here(), lane = tid & 63, wave = uniform(tid >> 6);
    const int row = 8 * wave + lane / 8, place = (lane % 8) ^ swz_inner(row), chunk = 2 * (place & 3) + (place >> 2), i = row & 15;
    static_assert(T::NWAVES * 8 % 32 == 0, "swizzle and permutation repeat from piece to piece");
    const int at = COL ? (row & ~31) + 8 * (i >> 2) + 4 * ((row >> 4) & 1) + (i & 3) : row;
    upper = chunk >= 4;
    voff[0] = (uint32_t)(at * s.ld + 16 * chunk);
#pragma unroll
    for (int j = 1; j < PIECES; ++j) voff[j] = voff[0] + (uint32_t)(j * T::NWAVES * 8 * s.ld);
  }
};

template <class T, bool COL>
struct MxPanelLoad {
  using Lanes = MxLanes<T, COL>;
  static constexpr int E = Lanes::E;
  const char* base;
  uint32_t range, lds;
  int rest;       // stages that have not been requested
  bool ragged;    // of the last one only half exists

  __device__ __forceinline__ MxPanelLoad(const MxSide& s, int i0, int panel, int stage0, int nk, uint32_t lds_off) {
    const int wave = uniform((int)threadIdx.x >> 6);
    const int which = s.gated ? panel : 0, first = i0 + (s.gated ? 0 : panel * E);
    const int64_t there = s.rows - first, rows = there < 0 ? 0 : there > E ? E : there;
    base = (const char*)(s.codes + (which * s.rows + first) * s.ld + (int64_t)stage0 * 128);
    range = (uint32_t)(rows * s.ld);  // the same for every stage: the base moves on inside the rows
    rest = rows > 0 ? nk : 0;
    ragged = (stage0 + nk) * 2 > s.ld / 64;
    lds = lds_off + (uint32_t)wave * 1024u;
  }
  // The next stage, into the ring slot at stage_lds; zeros, from nowhere, behind the last one.
  __device__ __forceinline__ void load(const Lanes& l, uint32_t stage_lds) {
    const uint64_t b = (uint64_t)base;  // 48 bits
    const u32x4 r = {(uint32_t)b, (uint32_t)(b >> 32), rest > 0 ? range : 0u, 0x00027000u};
    const bool half = ragged && rest == 1;
#pragma unroll
    for (int j = 0; j < Lanes::PIECES; ++j) {
      const uint32_t to = uniform(stage_lds + lds + (uint32_t)(j * T::NWAVES * 1024));
      const uint32_t from = half && l.upper ? 0x80000000u : l.voff[j];
      if (j == 0) dma16_buffer<5>(r, from, to);
      else dma16_buffer<1>(r, from, to);
    }
    base += 128;
    --rest;
  }
};

// Loads of a side's scales: a wave brings 64 rows' words of one half of the stage (the smallest tiles have fewer pieces than waves: two
// waves bring the same).  What lies past the matrix's scales, the second half of a ragged last stage, reads as zeros: 2^-127, never NaN.
template <class T, bool COL>
struct MxScaleLoad {
  static constexpr int ROWS = COL ? T::BN : T::BM, E = COL ? T::EC : T::ER, PIECES = 2 * ROWS / 64;
  static_assert(T::NWAVES % PIECES == 0, "every piece has its waves");
  const char* base;
  uint32_t left, step, voff, lds;  // left: bytes from base to the end of the matrix's scales (those of 2^18 by 2^18 are 2^31)
  int rest;                        // stages whose words exist
  __device__ __forceinline__ MxScaleLoad(const MxSide& s, int i0, int stage0, int nk) {
    const int tid = thread_here(), wave = uniform(tid >> 6), piece = wave % PIECES, k = piece / (ROWS / 64), r = 64 * (piece % (ROWS / 64));
    const int panel = s.gated ? r / E : 0, first = i0 + (s.gated ? r % E : r);
    const int64_t kb = s.ld / 64;  // groups of 128
    const int64_t words = (2 * (int64_t)stage0 + k) * s.rows + first;
    base = (const char*)(s.scales + (panel * s.rows * kb + words) * 4);
    left = (uint32_t)((kb * s.rows - words) * 4);
    step = (uint32_t)(8 * s.rows);
    voff = (uint32_t)((tid & 63) * 4);
    lds = (COL ? MxTile<T>::CSCALES + k * MxTile<T>::CPITCH : MxTile<T>::RSCALES + k * MxTile<T>::RPITCH) + 4 * r;
    rest = first < s.rows ? min(nk, ((int)kb - k + 1) / 2 - stage0) : 0;
  }
  __device__ __forceinline__ void load(uint32_t stage_lds) {
    const uint64_t b = (uint64_t)base;
    const u32x4 r = {(uint32_t)b, (uint32_t)(b >> 32), rest > 0 ? left : 0u, 0x00027000u};
    dma4_buffer(r, voff, uniform(stage_lds + lds));
    base += step;
    left -= step;
    --rest;
  }
};

// Fragments: block tm of the row side, block i of the column side; both chunks of a stage and their scales.
template <class T>
struct MxRowFrag {
  uint32_t off[2], soff, halves;
  __device__ __forceinline__ MxRowFrag(int wm) {
    const int lane = thread_here() & 63, g = lane >> 4;
    const int first = T::row_of(wm, 0), row = first % T::ER + (lane & 15);
    const uint32_t panel = (uint32_t)(first / T::ER * MxTile<T>::RPANEL);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) off[ks] = panel + (uint32_t)(row * 128 + (((4 * ks + g) ^ swz_inner(row)) << 4));
    soff = (uint32_t)(MxTile<T>::RSCALES + (g >> 1) * MxTile<T>::RPITCH + (first + (lane & 15)) * 4);
    halves = g & 1 ? 0x07060302u : 0x05040100u;
  }
  static constexpr int half(int tm) { return (T::QUAD ? tm >> 2 : 0) * MxTile<T>::RPANEL; }
  static constexpr int blk(int tm) { return T::QUAD ? tm & 3 : tm; }
  __device__ __forceinline__ u32x4 read(const char* stage, int ks, int tm) const {
    return *reinterpret_cast<const u32x4*>(stage + half(tm) + off[ks] + blk(tm) * 16 * 128);
  }
  // The scales of blocks tm and tm + 1: bytes 0 and 1, 2 and 3, one for each chunk.
  __device__ __forceinline__ int scales(const char* stage, int tm) const {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(stage + soff + ((T::QUAD ? tm >> 2 : 0) * 128 + blk(tm) * 16) * 4);
    return (int)__builtin_amdgcn_perm(p[16], p[0], halves);
  }
};
template <class T>
struct MxColFrag {
  uint32_t off[2], soff, halves;
  __device__ __forceinline__ MxColFrag(int wn) {
    const int lane = thread_here() & 63, g = lane >> 4, i = lane & 15, row = 32 * wn + i;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) off[ks] = (uint32_t)(MxTile<T>::C0 + row * 128 + (((4 * ks + g) ^ swz_inner(row)) << 4));
    // LDS row 16 t + i holds matrix row 8 (i / 4) + 4 t + i % 4 of every 32; the scales are in the matrix's order
    soff = (uint32_t)(MxTile<T>::CSCALES + (g >> 1) * MxTile<T>::CPITCH + (32 * wn + 8 * (i >> 2) + (i & 3)) * 4);
    halves = g & 1 ? 0x07060302u : 0x05040100u;
  }
  __device__ __forceinline__ u32x4 read(const char* stage, int panel, int ks, int t) const {
    return *reinterpret_cast<const u32x4*>(stage + panel * MxTile<T>::CPANEL + off[ks] + t * 16 * 128);
  }
  // The scales of both blocks of a panel.
  __device__ __forceinline__ int scales(const char* stage, int panel) const {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(stage + soff + panel * T::EC * 4);
    return (int)__builtin_amdgcn_perm(p[4], p[0], halves);
  }
};

// The plain loop: as product_loop, a stage's fragments read while the stage before it is multiplied.
template <class T>
__device__ __forceinline__ void mx_loop(const MxSide& rs, const MxSide& cs, int m0, int n0, int st0, int nk, Acc<T>& acc, char* lds) {
  using X = MxTile<T>;
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
  const MxLanes<T, false> rl(rs);
  const MxLanes<T, true> cl(cs);
  MxPanelLoad<T, false> r0(rs, m0, 0, st0, nk, 0), r1(rs, m0, T::ROWP - 1, st0, nk, (T::ROWP - 1) * X::RPANEL);
  MxPanelLoad<T, true> c0(cs, n0, 0, st0, nk, X::C0), c1(cs, n0, T::COLP - 1, st0, nk, X::C0 + (T::COLP - 1) * X::CPANEL);
  MxScaleLoad<T, false> rsc(rs, m0, st0, nk);
  MxScaleLoad<T, true> csc(cs, n0, st0, nk);
  uint32_t to = lds_base;  // the ring slot that is requested next
  auto issue = [&]() {
    r0.load(rl, to);
    if constexpr (T::ROWP == 2) r1.load(rl, to);
    rsc.load(to);
    c0.load(cl, to);
    if constexpr (T::COLP == 2) c1.load(cl, to);
    csc.load(to);
    to = to == lds_base + (T::NS - 1) * X::STAGE ? lds_base : to + X::STAGE;
  };
  const MxRowFrag<T> rf(wm);
  const MxColFrag<T> cf(wn);
  struct Frags {
    u32x4 x[2][T::TM], w[2][T::COLP][2];
    int sx[T::TM / 2], sw[T::COLP];
  };
  const char* stage = lds;  // the ring slot that is read next
  auto read = [&](Frags& f) {
#pragma unroll
    for (int tm = 0; tm < T::TM; tm += 2) f.sx[tm / 2] = rf.scales(stage, tm);
#pragma unroll
    for (int p = 0; p < T::COLP; ++p) f.sw[p] = cf.scales(stage, p);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int tm = 0; tm < T::TM; ++tm) f.x[ks][tm] = rf.read(stage, ks, tm);
#pragma unroll
      for (int p = 0; p < T::COLP; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i) f.w[ks][p][i] = cf.read(stage, p, ks, i);
    }
    stage = stage == lds + (T::NS - 1) * X::STAGE ? lds : stage + X::STAGE;
  };
  auto mma = [&](const Frags& f) {
    auto chunk = [&](auto ks_) {
      constexpr int ks = decltype(ks_)::value;
#pragma unroll
      for (int p = 0; p < T::COLP; ++p)
#pragma unroll
        for (int tm = 0; tm < T::TM; tm += 2)
          mx_block<ks>(acc[p][0][tm], acc[p][0][tm + 1], acc[p][1][tm], acc[p][1][tm + 1], f.w[ks][p][0], f.w[ks][p][1], f.x[ks][tm], f.x[ks][tm + 1],
                       f.sw[p], f.sx[tm / 2]);
    };
    chunk(int_constant<0>());
    chunk(int_constant<1>());
  };
  // Every wave's loads of stage st have arrived, and every wave holds the fragments of the stages before it.
  auto resident = [&](int st) {
    wait_stages_behind<X::LOADS, T::NS - 2>(min(T::NS - 2, nk - 1 - st));
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

// (Tried for it: four waves of 128 x 128 each, which read a third less from LDS, 300 us for the case above; requests between the
// products in place of between the slots, 248; both against 239 as it is.)
//
// The ping-pong loop of the 256 x 256 tile: the slots, visibility and reuse of product_pingpong.  The scales of all rows come with panel A0
// (its load is three of a wave, two of codes and one of scales) and are read with it, those of all columns with B0; so they are requested
// again where those panels are, two slots after they were read.  The waits count the loads of the five panels behind the one waited for.
template <class T>
struct MxPingPong {
  using X = MxTile<T>;
  static_assert(T::ER == 128 && T::EC == 128 && T::ROWP == 2 && T::COLP == 2 && T::NWAVES == 8 && T::NS == 2 && T::TM == 8, "256 x 256 tile");
  MxPanelLoad<T, false> pa[2];
  MxPanelLoad<T, true> pb[2];
  MxScaleLoad<T, false> sa;
  MxScaleLoad<T, true> sb;
  int nk;

  __device__ __forceinline__ void load_a(const MxLanes<T, false>& rl, uint32_t ring, int half, int st) {  // a panel's stages come in order
    pa[half].load(rl, ring + (uint32_t)(st & 1) * X::STAGE);
    if (half == 0) sa.load(ring + (uint32_t)(st & 1) * X::STAGE);
  }
  __device__ __forceinline__ void load_b(const MxLanes<T, true>& cl, uint32_t ring, int half, int st) {
    pb[half].load(cl, ring + (uint32_t)(st & 1) * X::STAGE);
    if (half == 0) sb.load(ring + (uint32_t)(st & 1) * X::STAGE);
  }
  // Requests a tile's first stage and all of its second but A1; the ring is free.
  __device__ __forceinline__ MxPingPong(const MxSide& rs, const MxSide& cs, const MxLanes<T, false>& rl, const MxLanes<T, true>& cl, int m0, int n0, int st0,
                                        int nk_, char* lds)
      : pa{{rs, m0, 0, st0, nk_, 0}, {rs, m0, 1, st0, nk_, X::RPANEL}},
        pb{{cs, n0, 0, st0, nk_, X::C0}, {cs, n0, 1, st0, nk_, X::C0 + X::CPANEL}},
        sa(rs, m0, st0, nk_),
        sb(cs, n0, st0, nk_),
        nk(nk_) {
    const uint32_t ring = (uint32_t)(uintptr_t)lds;
    load_a(rl, ring, 0, 0);
    load_b(cl, ring, 0, 0);
    load_b(cl, ring, 1, 0);
    load_a(rl, ring, 1, 0);
    load_a(rl, ring, 0, 1);
    load_b(cl, ring, 0, 1);
    load_b(cl, ring, 1, 1);
  }

  __device__ __forceinline__ void run(const MxLanes<T, false>& rl, const MxLanes<T, true>& cl, Acc<T>& acc, char* lds) {
    const int wave = uniform((int)threadIdx.x >> 6);
    const int wm = wave % T::WM, wn = wave / T::WM;
    const bool trailing = wave >= 4;
    const uint32_t ring = (uint32_t)(uintptr_t)lds;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[p][i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const MxRowFrag<T> rf(wm);
    const MxColFrag<T> cf(wn);
    u32x4 xa[2][4], xb[2][4], w0[2][2], w1[2][2];
    int sx[2][2], sw[2], next[2];  // scales, two blocks a word; `next`: of the next stage's panel A1, read with A0
    auto read_a = [&](u32x4 (&x)[2][4], int half, int st) {
      const char* stage = lds + (st & 1) * X::STAGE;
      if (half == 0) {
  #pragma unroll
        for (int i = 0; i < 2; ++i) {
          sx[0][i] = rf.scales(stage, 2 * i);
          next[i] = rf.scales(stage, 4 + 2 * i);
        }
      } else {
  #pragma unroll
        for (int i = 0; i < 2; ++i) sx[1][i] = next[i];
      }
  #pragma unroll
      for (int ks = 0; ks < 2; ++ks)
  #pragma unroll
        for (int tm = 0; tm < 4; ++tm) x[ks][tm] = rf.read(stage, ks, 4 * half + tm);
    };
    auto read_b = [&](u32x4 (&w)[2][2], int half, int st) {
      const char* stage = lds + (st & 1) * X::STAGE;
      if (half == 0)
  #pragma unroll
        for (int p = 0; p < 2; ++p) sw[p] = cf.scales(stage, p);
  #pragma unroll
      for (int ks = 0; ks < 2; ++ks)
  #pragma unroll
        for (int i = 0; i < 2; ++i) w[ks][i] = cf.read(stage, half, ks, i);
    };
    auto mma = [&](const u32x4 (&w)[2][2], const u32x4 (&x)[2][4], auto bh, auto ah) {
      constexpr int b = decltype(bh)::value, h = decltype(ah)::value, a = 4 * h;
      auto chunk = [&](auto ks_) {
        constexpr int ks = decltype(ks_)::value;
  #pragma unroll
        for (int tm = 0; tm < 4; tm += 2)
          mx_block<ks>(acc[b][0][a + tm], acc[b][0][a + tm + 1], acc[b][1][a + tm], acc[b][1][a + tm + 1], w[ks][0], w[ks][1], x[ks][tm], x[ks][tm + 1],
                       sw[b], sx[h][tm / 2]);
      };
      chunk(int_constant<0>());
      chunk(int_constant<1>());
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

    // One stage.  It requests two stages ahead to the end: what lies behind the last stage arrives as zeros that are not read.  (With
    // the last two stages as copies of their own, which request less, 256 registers did not hold the sums.)
    auto stage = [&](int it) {
      read_b(w0, 0, it);
      load_a(rl, ring, 1, it + 1);
      vm_wait(int_constant<12>());  // B1 of this stage
      slot_end();
      products_begin();
      mma(w0, xa, Lo(), Lo());
      products_end();

      read_b(w1, 1, it);
      load_a(rl, ring, 0, it + 2);
      vm_wait(int_constant<13>());  // A1 of this stage
      slot_end();
      products_begin();
      mma(w1, xa, Hi(), Lo());
      products_end();

      read_a(xb, 1, it);
      load_b(cl, ring, 0, it + 2);
      vm_wait(int_constant<13>());  // A0 of the next stage
      slot_end();
      products_begin();
      mma(w1, xb, Hi(), Hi());
      products_end();

      read_a(xa, 0, it + 1);
      load_b(cl, ring, 1, it + 2);
      vm_wait(int_constant<12>());  // B0 of the next stage
      slot_end();
      products_begin();
      mma(w0, xb, Lo(), Hi());
      products_end();
    };

    wait_vm<12>();  // A0, B0 (what was stored since they were requested makes the wait longer, never shorter)
    slot_end();
    read_a(xa, 0, 0);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)

    if (trailing) slot_end();
    for (int it = 0; it < nk; ++it) stage(it);
    if (!trailing) slot_end();
    wait_vm<0>();
    __syncthreads();  // every wave is done with the ring, its loads among them, before it is reused
  }
};

template <class Epi_>
struct MxProblem {
  using Epi = Epi_;
  MxSide r, c;
  int M, N;
  int nk;            // K in stages of 256
  int split, per;    // parts of K, stages of each
  float* part;
  uint32_t* arrived;
  TileWalk walk;
  Epi epi;
  __host__ __device__ int items() const { return walk.total() * split; }
};

template <class T, class P>
__global__ __launch_bounds__(T::THREADS) __attribute__((amdgpu_waves_per_eu(2))) void k_mx_product(const P a) {
  __shared__ __align__(1024) char lds[MxTile<T>::LDS];
  constexpr int COLS = P::Epi::kGated ? T::EC : T::BN;  // result columns of a tile
  const int total = a.walk.total();
  struct Place {
    int s, tile, tm, tn, st0, nk;
  };
  auto place_of = [&](int item) {
    Place p;
    p.s = item / total;
    p.tile = item - p.s * total;
    a.walk.at(p.tile, p.tm, p.tn);
    p.st0 = p.s * a.per;
    p.nk = min(a.per, a.nk - p.st0);
    return p;
  };
  Acc<T> acc;
  if constexpr (T::QUAD) {
    // One work-group to a CU goes through several whole tiles, and requests the next tile's first stages before it stores this one's results
    // (267 us for 4096 x 14336 x 4096 gated with a launch's work-group for each tile, 239 so).  Parts of K, which meet through LDS, have a
    // work-group each.
    const MxLanes<T, false> rl(a.r);
    const MxLanes<T, true> cl(a.c);
    const int items = a.items();
    int item = blockIdx.x;
    Place p = place_of(item);
    MxPingPong<T> loop(a.r, a.c, rl, cl, p.tm * T::BM, p.tn * COLS, p.st0, p.nk, lds);
    for (;;) {
      loop.run(rl, cl, acc, lds);
      const int next = item + gridDim.x;
      const bool more = next < items;
      const Place q = more ? place_of(next) : p;
      if (more) loop = MxPingPong<T>(a.r, a.c, rl, cl, q.tm * T::BM, q.tn * COLS, q.st0, q.nk, lds);
      finish_product<T>(a, acc, 0, p.tile, p.s, p.tm, p.tn, lds);
      if (!more) return;
      item = next;
      p = q;
    }
  } else {
    const Place p = place_of(blockIdx.x);
    mx_loop<T>(a.r, a.c, p.tm * T::BM, p.tn * COLS, p.st0, p.nk, acc, lds);
    finish_product<T>(a, acc, 0, p.tile, p.s, p.tm, p.tn, lds);
  }
}

}  // namespace mlp2
