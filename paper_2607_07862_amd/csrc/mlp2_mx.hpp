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
// units of 64 x 16 bits.  What comes on top are the scales: each panel's stage
// carries two words a row behind its codes, one more direct-to-LDS load (4 bytes a
// lane) for every wave.
//
// K is dealt to the lanes so that a lane's two 16-byte chunks of a stage are
// neighbours, chunks 2 g and 2 g + 1 for lane group g = lane / 16: their scales are
// the two halves of one 16-bit LDS read, which the instruction picks by itself.
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

// Where a panel's stage lies in LDS: E rows of 128 bytes of codes, then two times E words of scales.
template <int E>
constexpr int mx_panel() { return E * 136; }

template <class T>
struct MxTile {
  static constexpr int RPANEL = mx_panel<T::ER>(), CPANEL = mx_panel<T::EC>();
  static constexpr int STAGE = T::ROWP * RPANEL + T::COLP * CPANEL;
  static constexpr int LOADS = T::LOADS + T::ROWP + T::COLP;  // of a wave and stage
  static constexpr int LDS = T::NS * STAGE;
};

// One direct-to-LDS buffer load of 4 bytes a lane: lane i's to lds_addr + 4 i, zeros past the range.
__device__ __forceinline__ void dma4_buffer(u32x4 rsrc, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(voff), "s"(rsrc), "{m0}"(lds_addr) : "memory");
}

// Loads of one panel, stage by stage: each wave 1 KB pieces of the codes and one
// piece of 64 rows of the scales (with fewer pieces than waves, two waves load
// the same one).
// The ranges: rows past the matrix's end read as zeros.  A last stage of which
// only 128 of K exist has its other chunks asked for from past the range; their
// scales lie past the end of the matrix's scales (zeros: 2^-127, never NaN).
// Every panel of a side has the same offsets in its lanes; bases and ranges are scalars.
template <class T, bool COL>
struct MxLanes {
  static constexpr int E = COL ? T::EC : T::ER, PIECES = E * 128 / 1024 / T::NWAVES;
  uint32_t voff[PIECES], soff;
  bool upper;  // this lane's chunk lies in the upper half of a stage
  __device__ __forceinline__ explicit MxLanes(const MxSide& s) {
    const int tid = thread_here(), lane = tid & 63, wave = uniform(tid >> 6);
    const int row = 8 * wave + lane / 8, chunk = (lane % 8) ^ swz_inner(row), i = row & 15;
    static_assert(T::NWAVES * 8 % 32 == 0, "swizzle and permutation repeat from piece to piece");
    const int at = COL ? (row & ~31) + 8 * (i >> 2) + 4 * ((row >> 4) & 1) + (i & 3) : row;
    upper = chunk >= 4;
    voff[0] = (uint32_t)(at * s.ld + 16 * chunk);
#pragma unroll
    for (int j = 1; j < PIECES; ++j) voff[j] = voff[0] + (uint32_t)(j * T::NWAVES * 8 * s.ld);
    soff = (uint32_t)((scale_k(wave) * s.rows + scale_row(wave) + lane) * 4);
  }
  static constexpr int SP = 2 * E / 64;  // pieces of the scales
  static_assert(T::NWAVES % SP == 0, "every piece of the scales has its waves");
  static __device__ __forceinline__ int scale_k(int wave) { return wave % SP / (E / 64); }
  static __device__ __forceinline__ int scale_row(int wave) { return 64 * (wave % SP % (E / 64)); }
};

template <class T, bool COL>
struct MxPanelLoad {
  using Lanes = MxLanes<T, COL>;
  static constexpr int E = Lanes::E;
  const char *base, *sbase;
  uint32_t range;
  uint32_t sleft;  // bytes of scales from sbase on (the scales of 2^18 by 2^18 are 2^31)
  uint32_t sstep;
  int rest;       // stages that have not been requested
  bool ragged;    // of the last one only half exists
  uint32_t lds, slds;

  __device__ __forceinline__ MxPanelLoad(const MxSide& s, int i0, int panel, int stage0, int nk, uint32_t lds_off) {
    const int wave = uniform((int)threadIdx.x >> 6);
    const int which = s.gated ? panel : 0, first = i0 + (s.gated ? 0 : panel * E);
    const int64_t matrix = which * s.rows, there = s.rows - first;
    const int64_t rows = there < 0 ? 0 : there > E ? E : there;
    base = (const char*)(s.codes + (matrix + first) * s.ld + (int64_t)stage0 * 128);
    range = (uint32_t)(rows * s.ld);  // the same for every stage: the base moves on inside the rows
    const int64_t kb = s.ld / 64;     // groups of 128
    rest = rows > 0 ? nk : 0;
    ragged = (stage0 + nk) * 2 > kb;
    sbase = (const char*)(s.scales + (matrix * kb + 2 * (int64_t)stage0 * s.rows + first) * 4);
    sleft = (uint32_t)(((kb - 2 * (int64_t)stage0) * s.rows - first) * 4);
    sstep = (uint32_t)(8 * s.rows);
    lds = lds_off + (uint32_t)wave * 1024u;
    slds = lds_off + (uint32_t)(E * 128 + (Lanes::scale_k(wave) * E + Lanes::scale_row(wave)) * 4);
  }
  // The next stage, into the ring slot at stage_lds; zeros, from nowhere, behind the last one.
  __device__ __forceinline__ void load(const Lanes& l, uint32_t stage_lds) {
    const uint64_t b = (uint64_t)base, sb = (uint64_t)sbase;  // 48 bits
    const u32x4 r = {(uint32_t)b, (uint32_t)(b >> 32), rest > 0 ? range : 0u, 0x00027000u};
    const u32x4 sr = {(uint32_t)sb, (uint32_t)(sb >> 32), rest > 0 ? sleft : 0u, 0x00027000u};
    const bool half = ragged && rest == 1;
#pragma unroll
    for (int j = 0; j < Lanes::PIECES; ++j) {
      const uint32_t to = uniform(stage_lds + lds + (uint32_t)(j * T::NWAVES * 1024));
      const uint32_t from = half && l.upper ? 0x80000000u : l.voff[j];
      if (j == 0) dma16_buffer<5>(r, from, to);
      else dma16_buffer<1>(r, from, to);
    }
    dma4_buffer(sr, l.soff, uniform(stage_lds + slds));
    base += 128;
    sbase += sstep;
    sleft -= sstep;
    --rest;
  }
};

__device__ __forceinline__ int pair_of(const char* lo, const char* hi) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  const u16x2 v = {*reinterpret_cast<const uint16_t*>(lo), *reinterpret_cast<const uint16_t*>(hi)};
  return __builtin_bit_cast(int, v);
}

// Fragments: block tm of the row side, block i of the column side; both chunks of a stage and their scales.
template <class T>
struct MxRowFrag {
  uint32_t off[2], soff;
  __device__ __forceinline__ MxRowFrag(int wm) {
    const int lane = thread_here() & 63, g = lane >> 4;
    const int first = T::row_of(wm, 0), row = first % T::ER + (lane & 15);
    const uint32_t panel = (uint32_t)(first / T::ER * MxTile<T>::RPANEL);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) off[ks] = panel + (uint32_t)(row * 128 + (((2 * g + ks) ^ swz_inner(row)) << 4));
    soff = panel + (uint32_t)(T::ER * 128 + ((g >> 1) * T::ER + row) * 4 + 2 * (g & 1));
  }
  static constexpr int half(int tm) { return (T::QUAD ? tm >> 2 : 0) * MxTile<T>::RPANEL; }
  static constexpr int blk(int tm) { return T::QUAD ? tm & 3 : tm; }
  __device__ __forceinline__ u32x4 read(const char* stage, int ks, int tm) const {
    return *reinterpret_cast<const u32x4*>(stage + half(tm) + off[ks] + blk(tm) * 16 * 128);
  }
  // The scales of blocks tm and tm + 1: bytes 0 and 1, 2 and 3 (one for each chunk).
  __device__ __forceinline__ int scales(const char* stage, int tm) const {
    const char* p = stage + half(tm) + soff + blk(tm) * 16 * 4;
    return pair_of(p, p + 16 * 4);
  }
};
template <class T>
struct MxColFrag {
  uint32_t off[2], soff;
  __device__ __forceinline__ MxColFrag(int wn) {
    const int lane = thread_here() & 63, g = lane >> 4, i = lane & 15, row = 32 * wn + i;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) off[ks] = (uint32_t)(row * 128 + (((2 * g + ks) ^ swz_inner(row)) << 4));
    // LDS row 16 t + i holds matrix row 8 (i / 4) + 4 t + i % 4 of every 32; the scales are in the matrix's order
    soff = (uint32_t)(T::EC * 128 + ((g >> 1) * T::EC + 32 * wn + 8 * (i >> 2) + (i & 3)) * 4 + 2 * (g & 1));
  }
  __device__ __forceinline__ u32x4 read(const char* panel, int ks, int t) const {
    return *reinterpret_cast<const u32x4*>(panel + off[ks] + t * 16 * 128);
  }
  // The scales of both blocks.
  __device__ __forceinline__ int scales(const char* panel) const { return pair_of(panel + soff, panel + soff + 16); }
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
  constexpr int C0 = T::ROWP * X::RPANEL;  // the column panels of a stage
  const MxLanes<T, false> rl(rs);
  const MxLanes<T, true> cl(cs);
  MxPanelLoad<T, false> r0(rs, m0, 0, st0, nk, 0), r1(rs, m0, T::ROWP - 1, st0, nk, (T::ROWP - 1) * X::RPANEL);
  MxPanelLoad<T, true> c0(cs, n0, 0, st0, nk, C0), c1(cs, n0, T::COLP - 1, st0, nk, C0 + (T::COLP - 1) * X::CPANEL);
  uint32_t to = lds_base;  // the ring slot that is requested next
  auto issue = [&]() {
    r0.load(rl, to);
    if constexpr (T::ROWP == 2) r1.load(rl, to);
    c0.load(cl, to);
    if constexpr (T::COLP == 2) c1.load(cl, to);
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
    for (int p = 0; p < T::COLP; ++p) f.sw[p] = cf.scales(stage + C0 + p * X::CPANEL);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int tm = 0; tm < T::TM; ++tm) f.x[ks][tm] = rf.read(stage, ks, tm);
#pragma unroll
      for (int p = 0; p < T::COLP; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i) f.w[ks][p][i] = cf.read(stage + C0 + p * X::CPANEL, ks, i);
    }
    stage = stage == lds + (T::NS - 1) * X::STAGE ? lds : stage + X::STAGE;
  };
  auto mma = [&](const Frags& f) {
#pragma unroll
    for (int p = 0; p < T::COLP; ++p)
#pragma unroll
      for (int tm = 0; tm < T::TM; tm += 2) {
        mx_block<0>(acc[p][0][tm], acc[p][0][tm + 1], acc[p][1][tm], acc[p][1][tm + 1], f.w[0][p][0], f.w[0][p][1], f.x[0][tm], f.x[0][tm + 1],
                    f.sw[p], f.sx[tm / 2]);
        mx_block<1>(acc[p][0][tm], acc[p][0][tm + 1], acc[p][1][tm], acc[p][1][tm + 1], f.w[1][p][0], f.w[1][p][1], f.x[1][tm], f.x[1][tm + 1],
                    f.sw[p], f.sx[tm / 2]);
      }
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

// The ping-pong loop of the 256 x 256 tile: the slots, visibility and reuse of product_pingpong.  A panel's stage is three
// loads of a wave here (two of codes, one of scales), so the waits count three where those count two.
template <class T>
__device__ __forceinline__ void mx_pingpong(const MxSide& rs, const MxSide& cs, int m0, int n0, int st0, int nk, Acc<T>& acc, char* lds) {
  using X = MxTile<T>;
  static_assert(T::ER == 128 && T::EC == 128 && T::ROWP == 2 && T::COLP == 2 && T::NWAVES == 8 && T::NS == 2 && T::TM == 8, "256 x 256 tile");
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
  const MxLanes<T, false> rl(rs);
  const MxLanes<T, true> cl(cs);
  MxPanelLoad<T, false> pa[2] = {{rs, m0, 0, st0, nk, 0}, {rs, m0, 1, st0, nk, X::RPANEL}};
  MxPanelLoad<T, true> pb[2] = {{cs, n0, 0, st0, nk, 2 * X::RPANEL}, {cs, n0, 1, st0, nk, 2 * X::RPANEL + X::CPANEL}};
  auto load_a = [&](int half, int st) { pa[half].load(rl, lds_base + (uint32_t)(st & 1) * X::STAGE); };  // a panel's stages come in order
  auto load_b = [&](int half, int st) { pb[half].load(cl, lds_base + (uint32_t)(st & 1) * X::STAGE); };

  const MxRowFrag<T> rf(wm);
  const MxColFrag<T> cf(wn);
  struct XFrag {
    u32x4 v[2][4];
    int s[2];
  };
  struct WFrag {
    u32x4 v[2][2];
    int s;
  };
  XFrag xa, xb;
  WFrag w0, w1;
  auto read_a = [&](XFrag& x, int half, int st) {
    const char* stage = lds + (st & 1) * X::STAGE;
#pragma unroll
    for (int tm = 0; tm < 4; tm += 2) x.s[tm / 2] = rf.scales(stage, 4 * half + tm);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int tm = 0; tm < 4; ++tm) x.v[ks][tm] = rf.read(stage, ks, 4 * half + tm);
  };
  auto read_b = [&](WFrag& w, int half, int st) {
    const char* panel = lds + (st & 1) * X::STAGE + 2 * X::RPANEL + half * X::CPANEL;
    w.s = cf.scales(panel);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < 2; ++i) w.v[ks][i] = cf.read(panel, ks, i);
  };
  auto mma = [&](const WFrag& w, const XFrag& x, auto bh, auto ah) {
    constexpr int b = decltype(bh)::value, a = 4 * decltype(ah)::value;
    auto both = [&](auto ks_) {
      constexpr int ks = decltype(ks_)::value;
#pragma unroll
      for (int tm = 0; tm < 4; tm += 2)
        mx_block<ks>(acc[b][0][a + tm], acc[b][0][a + tm + 1], acc[b][1][a + tm], acc[b][1][a + tm + 1], w.v[ks][0], w.v[ks][1], x.v[ks][tm],
                     x.v[ks][tm + 1], w.s, x.s[tm / 2]);
    };
    both(int_constant<0>());
    both(int_constant<1>());
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
    load_a(1, it + 1);
    vm_wait(int_constant<15>());  // B1 of this stage
    slot_end();
    products_begin();
    mma(w0, xa, Lo(), Lo());
    products_end();

    read_b(w1, 1, it);
    load_a(0, it + 2);
    vm_wait(int_constant<15>());  // A1 of this stage
    slot_end();
    products_begin();
    mma(w1, xa, Hi(), Lo());
    products_end();

    read_a(xb, 1, it);
    load_b(0, it + 2);
    vm_wait(int_constant<15>());  // A0 of the next stage
    slot_end();
    products_begin();
    mma(w1, xb, Hi(), Hi());
    products_end();

    read_a(xa, 0, it + 1);
    load_b(1, it + 2);
    vm_wait(int_constant<15>());  // B0 of the next stage
    slot_end();
    products_begin();
    mma(w0, xb, Lo(), Hi());
    products_end();
  };

  // Prologue: the first stage and all of the second but A1.
  load_a(0, 0);
  load_b(0, 0);
  load_b(1, 0);
  load_a(1, 0);
  load_a(0, 1);
  load_b(0, 1);
  load_b(1, 1);
  wait_vm<15>();  // A0, B0
  slot_end();
  read_a(xa, 0, 0);
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)

  if (trailing) slot_end();
  for (int it = 0; it < nk; ++it) stage(it);
  if (!trailing) slot_end();
  wait_vm<0>();
  __syncthreads();  // every wave is done with the ring, its loads among them, before it is reused
}

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
  const int item = blockIdx.x, total = a.walk.total(), s = item / total, tile = item - s * total;
  int tm_, tn_;
  a.walk.at(tile, tm_, tn_);
  const int m0 = tm_ * T::BM, n0 = tn_ * COLS;
  const int st0 = s * a.per, nk = min(a.per, a.nk - st0);
  Acc<T> acc;
  if constexpr (T::QUAD) mx_pingpong<T>(a.r, a.c, m0, n0, st0, nk, acc, lds);
  else mx_loop<T>(a.r, a.c, m0, n0, st0, nk, acc, lds);
  finish_product<T>(a, acc, 0, tile, s, tm_, tn_, lds);
}

}  // namespace mlp2
