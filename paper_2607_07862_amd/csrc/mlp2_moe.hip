// A mixture-of-experts layer for a few tokens: router, the two-layer MLPs of each token's experts, their weighted sum.
//
//   logits = X Wr;  ids, gates = the k largest of a token and the softmax over them
//   Y[t] = sum over j of gates[t][j] * (act(X[t] W1[e]) W2[e]),  e = ids[t][j]
//
// Three launches: the router, the first products with the activation, the second products with the weighted sum.  A few tokens
// reach few rows of every expert, so the products are bound by the stream of the experts' weights.  In bf16 they go from memory to
// registers without LDS: a wave takes 128 columns and every fourth (of four waves) step of K, 16 bytes a lane and load, eight loads
// a step, the next step's in flight while this one is multiplied; the waves' sums meet in LDS at the end.  In 4 bits they go through
// LDS.
//
// A row here is a slot: row r = t k + j is token t with its j-th expert.  Every work-group counts the slots of each expert by
// itself, from ids (at most 8192 words), and finds the items of work from that: an item is an expert with at least one slot, up to
// 16 MT of its rows, a block of columns and a part of K.
#include <new>
#include <type_traits>

#include "mlp2_host.h"
#include "mlp2_mx.hpp"

namespace mlp2 {

constexpr int kMostExperts = 512, kMostSlots = 8192, kMostChosen = 16;
constexpr int kWaves = 4;
constexpr int kRoutePart = 512;  // the most of K in a part of the router
constexpr int kMostParts = 16;   // of K in the experts' products

// ------------------------------------------------------------------ memory that other XCDs write and read in the same launch

// (Buffer accesses with the device-scope bit: stores are written through, loads go past this XCD's L2.  Unlike atomic loads, which the
// compiler waits for one by one, these are in flight together.)
constexpr int kSc1 = 16;
constexpr int kNt = 2;  // streamed: read once
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void store_far(double* p, double v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
struct Far {
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ __forceinline__ explicit Far(const void* p) : rsrc(__builtin_amdgcn_make_buffer_rsrc((void*)p, 0, -1, 0x00027000)) {}
  __device__ __forceinline__ void store16(uint32_t off, f32x4 v) const {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), rsrc, (int)off, 0, kSc1);
  }
  __device__ __forceinline__ f32x4 load16(uint32_t off) const {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)off, 0, kSc1));
  }
  __device__ __forceinline__ double load_double(uint32_t off) const {
    return __builtin_bit_cast(double, __builtin_amdgcn_raw_buffer_load_b64(rsrc, (int)off, 0, kSc1));
  }
};

// An offset past the range of every buffer here but Far's: zeros, and no memory is read.  Rows that do not exist are read there.
constexpr uint32_t kNowhere = 0x80000000u;

// dma16_buffer for what is read once.
__device__ __forceinline__ void dma16_stream(u32x4 rsrc, uint32_t voff, uint32_t lds_addr) {
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen nt lds" ::"v"(voff), "s"(rsrc), "{m0}"(lds_addr) : "memory");
}

// ------------------------------------------------------------------ router

struct Route {
  const uint16_t* X;
  const void* Wr;   // [H, E]
  double* part;     // [splits, T, E]
  uint32_t* arrived;  // one counter for each group of tokens, a line each; zero between launches
  int32_t* ids;     // [T, k]
  float* gates;
  int T, H, E, k, splits, per;  // per: K of a split, a multiple of 64
  int width;        // threads that share a row of Wr: 2^width, at least E where that is at most 256
};

__device__ __forceinline__ double widen(uint16_t v) { return (double)__builtin_bit_cast(float, (uint32_t)v << 16); }
__device__ __forceinline__ double widen(float v) { return (double)v; }

// The largest of a wave's values, in a scalar register: inside rows of 16 lanes by data-parallel moves, then across the four rows.
template <int CTRL>
__device__ __forceinline__ double moved(double v) {
  const u32x2 w = __builtin_bit_cast(u32x2, v);
  const u32x2 m = {(uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[0], CTRL, 0xF, 0xF, true), (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[1], CTRL, 0xF, 0xF, true)};
  return __builtin_bit_cast(double, m);
}
__device__ __forceinline__ double lane_value(double v, int lane) {
  const u32x2 w = __builtin_bit_cast(u32x2, v);
  const u32x2 m = {(uint32_t)__builtin_amdgcn_readlane((int)w[0], lane), (uint32_t)__builtin_amdgcn_readlane((int)w[1], lane)};
  return __builtin_bit_cast(double, m);
}
__device__ __forceinline__ double largest_of(double a, double b) { return a > b ? a : b; }
__device__ __forceinline__ double wave_largest(double v) {
  v = largest_of(v, moved<0xB1>(v));   // quad_perm 1 0 3 2
  v = largest_of(v, moved<0x4E>(v));   // quad_perm 2 3 0 1
  v = largest_of(v, moved<0x141>(v));  // row_half_mirror
  v = largest_of(v, moved<0x140>(v));  // row_mirror
  return largest_of(largest_of(lane_value(v, 0), lane_value(v, 16)), largest_of(lane_value(v, 32), lane_value(v, 48)));
}

// The k largest of a token's logits (in LDS; ties: the lowest index; NaN counts as larger than infinity) and the softmax over them, by one
// wave.  Finite logits stay below 2^272 (at most 2^15 products of a bf16 and an fp32 number), so 2^1000 stands for infinity in the
// comparisons and infinity for NaN.
__device__ __forceinline__ void choose_experts(const double* logits, int E, int k, int32_t* ids, float* gates) {
  const int lane = threadIdx.x & 63;
  constexpr int PER = kMostExperts / 64;
  double v[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = lane + 64 * i;
    v[i] = e < E ? logits[e] : 0.0;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (64 * i < E) v[i] = v[i] != v[i] ? __builtin_huge_val() : v[i] == __builtin_huge_val() ? 0x1p1000 : v[i];
  uint32_t gone = 0;  // of this lane's experts, those that are chosen already or do not exist
#pragma unroll
  for (int i = 0; i < PER; ++i) gone |= lane + 64 * i >= E ? 1u << i : 0u;
  int mine = 0;
  for (int j = 0; j < k; ++j) {
    double best = -__builtin_huge_val();
    int at = kMostExperts;  // this lane's best expert
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (64 * i < E && !(gone >> i & 1) && (v[i] > best || at == kMostExperts)) {
        best = v[i];
        at = lane + 64 * i;
      }
    const double top = wave_largest(best);
    int chosen = kMostExperts;
    for (uint64_t m = __ballot(best == top && at < kMostExperts); m; m &= m - 1) chosen = min(chosen, __builtin_amdgcn_readlane(at, __builtin_ctzll(m)));
    if ((chosen & 63) == lane) gone |= 1u << (chosen >> 6);
    if (lane == j) mine = chosen;
  }
  // lane j: the j-th expert; the exponentials' sum is at least 1
  const double top = logits[uniform(__builtin_amdgcn_readlane(mine, 0))];
  float e = 0.f;
  if (lane < k) e = __builtin_amdgcn_exp2f((float)((logits[mine] - top) * 1.4426950408889634));
  float sum = e;
#pragma unroll
  for (int d = 1; d < 16; d *= 2) sum += __shfl_xor(sum, d);
  if (lane < k) {
    ids[lane] = mine;
    gates[lane] = e / sum;
  }
}

// Logits of TT tokens over one part of K, in fp64: which experts are chosen hangs on logits next to each other, and fp32 sums would
// put some of them in another order.  256 threads are `width` experts by 256 / width rows of K.  Latencies bound it: the part's X and
// the first weights are requested together, the parts' sums are read all at once.  (6.2 us for one token of 4096 and eight experts, 8.4
// for 16 of 2048 and 64, 10.2 for nine of 1024 and 251, 35 for 128 of 7168 and 256, there by the reads of X from LDS.)
template <class W, int TT>
__global__ __launch_bounds__(256) void k_moe_route(const Route a) {
  constexpr int MOST = TT * kMostExperts > TT * kRoutePart ? TT * kMostExperts : TT * kRoutePart;
  __shared__ __align__(16) double lds[256 * TT > MOST ? 256 * TT : MOST];
  __shared__ int seen;
  constexpr int AHEAD = 16, GROUP = 4;  // rows of K of a thread that are requested and multiplied at a time
  const int tid = threadIdx.x, t0 = blockIdx.x * TT, split = blockIdx.y;
  const int width = 1 << a.width, sub = tid >> a.width, subs = 256 >> a.width, e0 = tid & (width - 1);
  const int from = split * a.per, deep = min(a.H - from, a.per);
  const auto wr = __builtin_amdgcn_make_buffer_rsrc((void*)((const W*)a.Wr + (int64_t)from * a.E), 0, deep * a.E * (int)sizeof(W), 0x00027000);
  const int chunks = (a.E + width - 1) >> a.width;  // of experts; one but for E > 256
  for (int c = 0; c < chunks; ++c) {
    const int e = (c << a.width) + e0;
    // from this thread's first row on; zeros past the part and for the experts past the last
    const uint32_t first = e < a.E ? (uint32_t)((sub * a.E + e) * (int)sizeof(W)) : kNowhere;
    W w[AHEAD];
    auto request = [&](int k0) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int off = (int)(first + (uint32_t)((k0 + i * subs) * a.E * (int)sizeof(W)));
        if constexpr (sizeof(W) == 4) w[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(wr, off, 0, 0));
        else w[i] = __builtin_amdgcn_raw_buffer_load_b16(wr, off, 0, 0);
      }
    };
    request(0);
    if (c) __syncthreads();
    // (rows of K behind the part's last: zeros, as their weights are, so that the products need no branch; behind one, each row waited for
    // its own read of LDS, 190 clocks)
    const int padded = (deep + GROUP * subs - 1) / (GROUP * subs) * (GROUP * subs);
    for (int kk = tid & 63; kk < padded; kk += 64)
#pragma unroll
      for (int t = tid >> 6; t < TT; t += 4) lds[kk * TT + t] = t0 + t < a.T && kk < deep ? widen(a.X[(int64_t)(t0 + t) * a.H + from + kk]) : 0.0;
    __syncthreads();
    double acc[TT] = {};
    for (int k0 = 0; k0 < deep; k0 += AHEAD * subs) {
      W now[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) now[i] = w[i];
      if (k0 + AHEAD * subs < deep) request(k0 + AHEAD * subs);
#pragma unroll
      for (int g = 0; g < AHEAD; g += GROUP) {
        if (k0 + g * subs >= deep) break;
        const double* x = lds + (k0 + g * subs + sub) * TT;
#pragma unroll
        for (int i = 0; i < GROUP; ++i) {
          const double v = widen(now[g + i]);
#pragma unroll
          for (int t = 0; t < TT; ++t) acc[t] = __builtin_fma(v, x[i * subs * TT + t], acc[t]);
        }
      }
    }
    // the rows of K meet
    __syncthreads();
#pragma unroll
    for (int t = 0; t < TT; ++t) lds[((sub * TT + t) << a.width) + e0] = acc[t];
    __syncthreads();
    for (int i = tid; i < TT << a.width; i += 256) {
      const int t = i >> a.width, en = (c << a.width) + (i & (width - 1));
      double sum = 0.0;
#pragma unroll 8
      for (int s = 0; s < subs; ++s) sum += lds[((s * TT + t) << a.width) + (i & (width - 1))];
      if (t0 + t < a.T && en < a.E) store_far(a.part + ((int64_t)split * a.T + t0 + t) * a.E + en, sum);
    }
  }
  wait_all_mem();
  __syncthreads();
  if (tid == 0) seen = (int)__hip_atomic_fetch_add(a.arrived + blockIdx.x * kLine, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (uniform(seen) != a.splits - 1) return;
  if (tid == 0) __hip_atomic_store(a.arrived + blockIdx.x * kLine, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // The parts, 32 in flight; all in the order 0, 1, ... whichever came last.
  constexpr int ALL = 32;
  const Far part(a.part);
  const int here = min(TT, a.T - t0) * a.E;
  for (int i = tid; i < here; i += 256) {
    const uint32_t first = (uint32_t)((t0 * a.E + i) * 8), pitch = (uint32_t)(a.T * a.E * 8);
    double sum = 0.0;
    for (int s = 0; s < a.splits; s += ALL) {
      double v[ALL];
#pragma unroll
      for (int d = 0; d < ALL; ++d) v[d] = part.load_double(first + min(s + d, a.splits - 1) * pitch);
#pragma unroll
      for (int d = 0; d < ALL; ++d)
        if (s + d < a.splits) sum += v[d];
    }
    lds[i] = sum;
  }
  __syncthreads();
  for (int t = tid / 64; t < TT; t += 4)
    if (t0 + t < a.T) choose_experts(lds + t * a.E, a.E, a.k, a.ids + (int64_t)(t0 + t) * a.k, a.gates + (int64_t)(t0 + t) * a.k);
}

// ------------------------------------------------------------------ the experts' products

struct Experts {
  const uint16_t* X;   // first: [T, H]; second: Z [2, T k, F]
  const int32_t* ids;
  const float* gates;
  const char* W;       // bf16 [E, nb, K, N], or MXFP4 codes of E nb matrices [N, K]
  const char* scales;
  uint16_t* out;       // first: Z; second: Y [T, H]
  float* part;         // parts of K: first [splits, T k, nb, N], second [splits, T k, N]; below 4 GB
  uint32_t* arrived;   // zero between launches; first: one counter for each slot and block of columns, second: for each token and block
  int T, E, k, K, N;
  int blocks;          // of columns
  int steps;           // of K
  float item;          // what an item costs beside its steps, in steps
  float join;          // and a part of K where there are several
  int most;            // parts of K
};

// An item of work: up to `tile` slots of an expert, a block of columns, a part of K.
struct Item {
  int expert, block, split, first, rows;
  int* slots;  // `rows` of them
};

// Weights as they lie in the rest of the library, [K, N] in bf16.  A lane loads 8 columns of 8 consecutive k; taken by columns,
// with one byte permute for each pair, those are the 8 operands (16 columns, 8 k a lane) of eight instructions, the columns of
// instruction j being j, 8 + j, 16 + j, ...
//
// 470 MB of first weights stream in 83 us (5.6 TB/s; one token, two experts of 4096 x 14336), 577 MB in 102 (16 tokens, 50 experts of
// 2048 x 1408); without the mark that the weights are read once, 113 us there.  The second products, with the sum over experts behind them,
// 235 MB in 45 and 288 in 60: there 800 items meet 768 places of work-groups, or a multiple.  Two or four steps in registers and ITEM of 4
// to 32 were all the same.
struct Bf16Weights {
  static constexpr int STEP = 32;  // K of a step (of one wave)
  static constexpr int ITEM = 8;   // what an item costs beside its steps
  static constexpr int FEWEST = 16;  // steps of a part of K: four of each wave
  static constexpr int NARROW = 2;  // slots an expert up to which items have one block of 16 rows
  static constexpr int most(bool second) { return second ? 2 : 4; }  // blocks of 16 rows that one pass over the weights serves
  static constexpr int WAVES = kWaves, COPIES = 4, ROWS = 64;  // copies of sums in LDS; rows of an item, at most
  static constexpr int RING = 2;   // steps in registers
  static constexpr int cols(bool) { return 128; }     // result columns of an item
  static constexpr int UP_WAVE = 2, UP_COL = 0;       // where the second matrix's sums are
  static constexpr int J = 8;                         // instruction groups of a wave: 16 columns each
  static constexpr int resident(int most) { return most == 1 ? 3 : 2; }  // work-groups of a CU, by their registers
  template <int XT>  // blocks of 16 rows of X; of Z two for each
  struct Regs {
    u32x4 w[8], x[XT];
  };
  uint32_t off, row;  // of this lane's first row, and from row to row
  __device__ __forceinline__ Bf16Weights(const Experts& a, int col) {
    const int lane = thread_here() & 63;
    row = (uint32_t)(2 * a.N);
    // columns past the last are read as the last eight
    off = (uint32_t)(2 * (min(col + 8 * (lane & 15), a.N - 8) + 8 * (lane >> 4) * a.N));
  }
  __device__ static __forceinline__ int64_t matrix(const Experts& a) { return (int64_t)a.K * a.N * 2; }
  // Steps from `end` on load zeros, from nowhere.
  template <int XT>
  __device__ __forceinline__ void load(Regs<XT>& r, const char* w, const uint16_t* x, const uint32_t (&xo)[XT], const Experts& a, int step, int end) const {
    const int range = step < end ? 0x7FFFFFFF : 0;
    const auto wr = __builtin_amdgcn_make_buffer_rsrc((void*)(w + (int64_t)step * STEP * a.N * 2), 0, range, 0x00027000);
    const auto xr = __builtin_amdgcn_make_buffer_rsrc((void*)(x + step * STEP), 0, range, 0x00027000);
#pragma unroll
    for (int i = 0; i < 8; ++i) r.w[i] = __builtin_amdgcn_raw_buffer_load_b128(wr, (int)off, (int)(i * row), kNt);
#pragma unroll
    for (int m = 0; m < XT; ++m) r.x[m] = __builtin_amdgcn_raw_buffer_load_b128(xr, (int)xo[m], 0, 0);
  }
  template <int MT, int XT>
  __device__ __forceinline__ void multiply(const Regs<XT>& r, f32x4 (&acc)[MT][8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      u32x4 f;
#pragma unroll
      for (int d = 0; d < 4; ++d) f[d] = __builtin_amdgcn_perm(r.w[2 * d + 1][j / 2], r.w[2 * d][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int m = 0; m < XT; ++m) acc[m * MT / XT][j] = Bf16::mfma(f, r.x[m], acc[m * MT / XT][j]);
    }
  }
  // Sums over this wave's steps of from .. end - 1: every fourth, with a gate every second one of the wave's matrix.
  template <int MT, bool GATED, bool SECOND>
  __device__ static __forceinline__ void stream(const Item& it, const Experts& a, int from, int end, f32x4 (&acc)[MT][8]) {
    constexpr int SHARE = GATED ? 2 : kWaves;
    const Bf16Weights w(a, 128 * it.block);
    const int lane = thread_here() & 63, wave = uniform((int)threadIdx.x >> 6);
    constexpr int XT = SECOND ? 2 * MT : MT;
    uint32_t xo[XT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int r = 16 * m + (lane & 15), slot = it.slots[r < it.rows ? r : 0];
      const uint32_t to = (uint32_t)(((int64_t)(SECOND ? slot : slot / a.k) * a.K + 8 * (lane >> 4)) * 2);
      xo[m * XT / MT] = r < it.rows ? to : kNowhere;
      if constexpr (SECOND) xo[2 * m + 1] = r < it.rows ? to + (uint32_t)((int64_t)a.T * a.k * a.K * 2) : kNowhere;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const char* base = a.W + ((int64_t)it.expert * (GATED ? 2 : 1) + wave / SHARE) * matrix(a);
    // A ring of steps in registers: while one is multiplied the others are in flight.  What is requested behind the last step arrives
    // as zeros, so that every request is unconditional and the waits count the same loads on every path.  (Four steps in place of two
    // streamed no faster.)
    Regs<XT> ring[RING];
    int step = from + wave % SHARE;
#pragma unroll
    for (int d = 0; d < RING - 1; ++d) w.load<XT>(ring[d], base, a.X, xo, a, step + d * SHARE, end);
    for (; step < end; step += RING * SHARE) {
#pragma unroll
      for (int d = 0; d < RING; ++d) {
        w.load<XT>(ring[(d + RING - 1) % RING], base, a.X, xo, a, step + (d + RING - 1) * SHARE, end);
        __builtin_amdgcn_sched_barrier(0);
        w.multiply<MT, XT>(ring[d], acc);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // Where the four sums of instruction j lie: columns 8 (4 g + i) + j.
  template <class Sums>
  __device__ static __forceinline__ void put(Sums& sum, const f32x4 (&c)[8]) {
    const int lane = threadIdx.x & 63, g = lane >> 4;
    float* to = sum[uniform((int)threadIdx.x >> 6)][lane & 15];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 lo, hi;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        lo[j] = c[j][i];
        hi[j] = c[4 + j][i];
      }
      *reinterpret_cast<f32x4*>(to + 8 * (4 * g + i)) = lo;
      *reinterpret_cast<f32x4*>(to + 8 * (4 * g + i) + 4) = hi;
    }
  }
};

// MXFP4 weights [N, K], K contiguous.  A memory line is 256 k of one row, the matrix instruction's operand 8 k of 16 rows: loads
// straight into registers would take a row's line in 64-byte pieces, and stream at 4 TB/s (pieces of a whole line: 6.9).  So the weights
// go through LDS, and X with them: a stage is 128 rows (with a gate 64 of either matrix) by 256 k of codes, two words of scales a row
// and 512 bytes of each X row, brought by direct-to-LDS loads of whole lines into a ring of stages.  Every wave multiplies a quarter
// of the stage's k with half of its rows.  A lane turns 16 codes of a row into two bf16 operands (exactly: two significant bits and a power of
// two).  Two waves of a work-group to a SIMD, as one's reads, conversions and products wait for each other (3.8 TB/s with one).
//
// 570 MB of first weights stream in 105 us (5.4 TB/s; 48 tokens, four each of 32 experts, 4096 x 4096), 285 of second ones in 64: Z's two
// numbers are twice the products and reads of X there, which cost a sixth of the time.
struct MxWeights {
  static constexpr int WAVES = 8, COPIES = 2, ROWS = 32;
  static constexpr int STEP = 256;  // (of all waves)
  static constexpr int ITEM = 2, FEWEST = 2;
  static constexpr int NARROW = 8;
  static constexpr int most(bool second) { return second ? 1 : 2; }
  static constexpr int resident(int) { return 2; }
  static constexpr int cols(bool gated) { return gated ? 64 : 128; }   // result columns of an item
  static constexpr int UP_WAVE = 0, UP_COL = 64;                       // where the second matrix's sums are
  static constexpr int J = 4;                                          // instruction groups of a wave: 16 columns each
  static constexpr int CODES = 16384, X0 = CODES + 1024;
  // by blocks of 16 rows of X (of Z two for each)
  static constexpr int stage(int xt) { return X0 + 8192 * xt; }
  static constexpr int DEPTH = 2;  // stages of the ring
  static constexpr int loads(int xt) { return 2 + 1 + xt; }  // of a wave and stage
  __device__ static __forceinline__ int64_t matrix(const Experts& a) { return a.N * (mx_padded(a.K) / 2); }

  // The stages of an item, one by one.
  template <int MT, bool GATED, bool SECOND>
  struct Requests {
    static constexpr int XT = SECOND ? 2 * MT : MT;
    const char *base, *sbase;
    int step, rest, last, length, groups;  // the next step, how many are left, the part's last one and length
    uint32_t wo[2], so, xo[XT];
    __device__ __forceinline__ void begin(const Item& it, const Experts& a, int from, int to) {
      const int lane = thread_here() & 63, wave = uniform((int)threadIdx.x >> 6), col = it.block * cols(GATED);
      const int64_t ld = mx_padded(a.K) / 2;
      groups = (int)(ld / 64);
      // Blocks start at different steps of their part and come round: rows lie a multiple of 2 KB apart, so that a step's lines are all in
      // one of an L2's channels, and work-groups that went through the steps together would all ask the same one.
      length = to - from;
      rest = length;
      last = to - 1;
      step = from + it.block % length;
      const int64_t first = (int64_t)it.expert * (GATED ? 2 : 1) * matrix(a);
      base = a.W + first;
      sbase = a.scales + first / 16;
      // Row r of the stage's 128 in its matrices (past the last column: the last).
      auto row_of = [&](int r) { return GATED ? (r >= 64 ? a.N : 0) + min(col + (r & 63), a.N - 1) : min(col + r, a.N - 1); };
      // codes: lane l brings 16 bytes of row l / 8 of eight
#pragma unroll
      for (int i = 0; i < 2; ++i) wo[i] = (uint32_t)(row_of(16 * wave + 8 * i + (lane >> 3)) * ld + 16 * chunk(lane, i));
      // scales: a word of 64 rows, of the stage's first or second 128 k (two waves bring the same)
      const int sr = row_of(64 * (wave & 1) + lane);
      so = (uint32_t)(((GATED && sr >= a.N ? (int64_t)(groups - 1) * a.N : 0) + (int64_t)(wave >> 1 & 1) * a.N + sr) * 4);
      // X: lane l brings 16 bytes of row l / 32 of two
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int r = 2 * (wave + 8 * i) + (lane >> 5), slot = it.slots[r < it.rows ? r : 0];
        const uint32_t at = (uint32_t)((int64_t)(SECOND ? slot : slot / a.k) * a.K * 2 + 16 * x_chunk(lane, wave));
        xo[i * XT / MT] = r < it.rows ? at : kNowhere;
        if constexpr (SECOND) xo[2 * i + 1] = r < it.rows ? at + (uint32_t)((int64_t)a.T * a.k * a.K * 2) : kNowhere;
      }
    }
    // Chunk c of row r of the codes lies at c ^ (r / 2 % 8), chunk c of row r of X at c ^ (r % 16).
    __device__ static __forceinline__ int chunk(int lane, int i) { return (lane & 7) ^ ((lane >> 4) & 3) ^ (4 * (i & 1)); }
    __device__ static __forceinline__ int x_chunk(int lane, int wave) { return (lane & 31) ^ (2 * wave + (lane >> 5)); }
    __device__ __forceinline__ void issue(const Experts& a, uint32_t to) {
      const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
      const uint32_t range = rest > 0 ? 0x7FFFFFFFu : 0u;
      const uint64_t b = (uint64_t)(base + (int64_t)step * 128), sb = (uint64_t)(sbase + (int64_t)step * a.N * 8), xb = (uint64_t)(a.X + (int64_t)step * STEP);
      const u32x4 wr = {uniform((uint32_t)b), uniform((uint32_t)(b >> 32)), range, 0x00027000u};
      // the last step may have 128 k only: zeros for the others' codes and scales, from past the range
      const bool half = 2 * step + 1 >= groups;
      const u32x4 sr = {uniform((uint32_t)sb), uniform((uint32_t)(sb >> 32)), half && (wave >> 1 & 1) ? 0u : range, 0x00027000u};
      const u32x4 xr = {uniform((uint32_t)xb), uniform((uint32_t)(xb >> 32)), range, 0x00027000u};
#pragma unroll
      for (int i = 0; i < 2; ++i) dma16_stream(wr, half && chunk(lane, i) >= 4 ? kNowhere : wo[i], uniform(to + 2048u * wave + 1024 * i));
      dma4_buffer(sr, so, uniform(to + CODES + 256u * (wave & 3)));
      const int deep = (a.K - step * STEP) / 8;  // chunks of X that exist
#pragma unroll
      for (int i = 0; i < XT; ++i) dma16_buffer<5>(xr, x_chunk(lane, wave) >= deep ? kNowhere : xo[i], uniform(to + X0 + 1024u * (wave + 8 * i)));
      step = step == last ? step + 1 - length : step + 1;
      --rest;
    }
  };

  // One stage: a quarter of its k, one half of its rows; the first HERE blocks of X's rows, of Z both numbers.  Lane group g has 16 k of every row, two
  // operands; everything that the stage holds for this lane is read before the first product.
  template <int MT, int HERE, bool SECOND>
  __device__ static __forceinline__ void multiply(const char* stage, f32x4 (&acc)[MT][J]) {
    constexpr int EACH = SECOND ? 2 : 1;
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), g = lane >> 4, i16 = lane & 15, k = wave % 4, upper = wave / 4;
    const char* codes = stage + 8192 * upper + 128 * i16 + 16 * ((2 * k + (g >> 1)) ^ (i16 >> 1)) + 8 * (g & 1);
    const char* scales = stage + CODES + 512 * (k >> 1) + 256 * upper + 4 * i16 + 2 * (k & 1) + (g >> 1);
    const char* xs = stage + X0 + 512 * i16;
    u32x4 x[HERE * EACH][2];
    u32x2 c[J];
    uint32_t sc[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      c[j] = *reinterpret_cast<const u32x2*>(codes + 2048 * j);
      sc[j] = *reinterpret_cast<const uint8_t*>(scales + 64 * j);
    }
#pragma unroll
    for (int m = 0; m < HERE * EACH; ++m)
#pragma unroll
      for (int p = 0; p < 2; ++p) x[m][p] = *reinterpret_cast<const u32x4*>(xs + 8192 * m + 16 * ((8 * k + 2 * g + p) ^ i16));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const float scale = mx_unit(sc[j]);
        u32x4 f;
        f[0] = __builtin_bit_cast(uint32_t, (mx_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j][p], scale, 0));
        f[1] = __builtin_bit_cast(uint32_t, (mx_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j][p], scale, 1));
        f[2] = __builtin_bit_cast(uint32_t, (mx_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j][p], scale, 2));
        f[3] = __builtin_bit_cast(uint32_t, (mx_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[j][p], scale, 3));
#pragma unroll
        for (int m = 0; m < HERE * EACH; ++m) acc[m / EACH][j] = Bf16::mfma(f, x[m][p], acc[m / EACH][j]);
      }
  }
  // Where the four sums of instruction group j lie: columns 16 j + 4 g + i of the wave's half.  Two copies, to which two quarters of k each
  // are added: four would not fit a place of the ring.
  template <class Sums>
  __device__ static __forceinline__ void put(Sums& sum, const f32x4 (&c)[J]) {
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), k = wave % 4;
    float* to = sum[k % 2][lane & 15] + 64 * (wave / 4) + 4 * (lane >> 4);
    if (k >= 2)
#pragma unroll
      for (int j = 0; j < J; ++j) *reinterpret_cast<f32x4*>(to + 16 * j) = c[j];
    __syncthreads();
    if (k < 2)
#pragma unroll
      for (int j = 0; j < J; ++j) *reinterpret_cast<f32x4*>(to + 16 * j) += c[j];
  }
};

constexpr int kIdsInLds = 2048;
template <class Weights, int RING>
struct MoeShared {
  static constexpr int kWave = Weights::WAVES, kThreads = 64 * kWave;
  // (4-bit weights) the ring of stages, and the slots' experts: reading those from memory would wait for every stage in flight
  static constexpr bool kIds = RING > 0;
  using Sums = float[Weights::COPIES][16][128 + 4];  // the waves' sums; behind the last item, tokens that are complete
  alignas(1024) char ring[RING ? RING : sizeof(Sums)];
  int16_t ids[kIds ? kIdsInLds : 1];
  int count[kMostExperts];  // slots of an expert
  int start[kMostExperts];  // its first unit (an expert's chunk of rows and a block of columns)
  int rows[2][kWave][Weights::ROWS];  // slots of an item and of the next one, a copy for each wave
  int total, found;
  // The sums: in the place of the ring whose stage was multiplied last.
  __device__ __forceinline__ Sums& sums(int place) { return *reinterpret_cast<Sums*>(ring + place); }
};

// Items, from ids.  Up to 64 slots every wave keeps them in its lanes, an expert's units with the first of its slots; beyond, the
// work-group counts the slots of every expert in LDS.  Either way a wave finds its item and rows without a barrier.
template <int TILE>
struct Items {
  int id, count, unit0, unit1;  // few slots: this lane's, its expert's slots and units, where it is the expert's first
  bool few;
  int units, splits, per;  // per: steps of a part
  __device__ __forceinline__ static int chunks(int slots) { return (slots + TILE - 1) / TILE; }
  template <class Shared>
  __device__ __forceinline__ Items(Shared& s, const Experts& a) {
    const int tid = threadIdx.x, lane = tid & 63, slots = a.T * a.k;
    few = slots <= 64;
    id = -1;
    count = unit0 = unit1 = 0;
    if (few) {
      if (lane < slots) id = a.ids[lane];
      if (id >= a.E) id = -1;
      bool first = id >= 0;
      for (int i = 0; i < slots; ++i) {
        const bool same = id == __builtin_amdgcn_readlane(id, i);
        count += same;
        first &= !same || i >= lane;
      }
      const int mine = first ? chunks(count) * a.blocks : 0;
      unit1 = mine;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int v = __shfl_up(unit1, d);
        if (lane >= d) unit1 += v;
      }
      unit0 = unit1 - mine;
      units = __builtin_amdgcn_readlane(unit1, 63);
    } else {
      for (int e = tid; e < a.E; e += Shared::kThreads) s.count[e] = 0;
      __syncthreads();
      for (int i = tid; i < slots; i += Shared::kThreads) {
        const int e = a.ids[i];
        const bool here = e >= 0 && e < a.E;
        if (here) atomicAdd(&s.count[e], 1);
        if (Shared::kIds && slots <= kIdsInLds) s.ids[i] = (int16_t)(here ? e : -1);
      }
      __syncthreads();
      if (tid < 64) {
        int before = 0;
        for (int e0 = 0; e0 < a.E; e0 += 64) {
          const int e = e0 + tid, n = e < a.E ? chunks(s.count[e]) * a.blocks : 0;
          int sum = n;
#pragma unroll
          for (int d = 1; d < 64; d *= 2) {
            const int v = __shfl_up(sum, d);
            if (tid >= d) sum += v;
          }
          if (e < a.E) s.start[e] = before + sum - n;
          before += __shfl(sum, 63);
        }
        if (tid == 0) s.total = before;
      }
      __syncthreads();
      units = uniform(s.total);
    }
    // Parts of K: as many as make the work-groups' shares alike, each item costing about as much as a.item steps more than it streams, and
    // joining the parts a.join.  (A CU takes in at most 40 to 50 GB/s, whatever its loads in flight, so the last round of a few items is as
    // long as a whole one.)  In floats: integer divisions, one after the other, took 3 us.
    float least = 1e30f;
    splits = 1;
    const float rounds1 = (float)units / (float)gridDim.x;
#pragma unroll
    for (int n = 1; n <= kMostParts; ++n) {
      const float steps = __builtin_ceilf((float)a.steps * (1.0f / n) - 1e-3f);
      const float cost = __builtin_ceilf(rounds1 * n - 1e-3f) * (steps + a.item) + (n > 1 ? a.join * n : 0.f);
      if (n <= a.most && cost < least) {
        least = cost;
        splits = n;
      }
    }
    splits = uniform(splits);
    per = (a.steps + splits - 1) / splits;
    splits = (a.steps + per - 1) / per;
  }
  __device__ __forceinline__ int total() const { return units * splits; }
  __device__ __forceinline__ int from(const Item& it) const { return it.split * per; }
  __device__ __forceinline__ int end(const Experts& a, const Item& it) const { return min(a.steps, (it.split + 1) * per); }

  // Item `n`; its slots go to this wave's s.rows[copy].
  template <class Shared>
  __device__ __forceinline__ Item find(Shared& s, const Experts& a, int n, int copy) const {
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), slots = a.T * a.k;
    // consecutive items: the blocks of columns, then the next rows, then the next expert, then the next part of K
    Item it;
    it.slots = s.rows[copy][wave];
    it.split = n / units;
    int in = n - it.split * units, total;
    it.expert = 0;
    if (few) {
      const int first = __builtin_ctzll(__ballot(in >= unit0 && in < unit1));
      it.expert = __builtin_amdgcn_readlane(id, first);
      total = __builtin_amdgcn_readlane(count, first);
      in -= __builtin_amdgcn_readlane(unit0, first);
    } else {
      for (int e0 = 0; e0 < a.E; e0 += 64) {
        const int e = e0 + lane;
        const bool here = e < a.E && in >= s.start[e] && in < s.start[e] + chunks(s.count[e]) * a.blocks;
        const uint64_t m = __ballot(here);
        if (m) {
          it.expert = e0 + __builtin_ctzll(m);
          break;
        }
      }
      it.expert = uniform(it.expert);
      in -= uniform(s.start[it.expert]);
      total = uniform(s.count[it.expert]);
    }
    it.block = in % a.blocks;
    it.first = in / a.blocks * TILE;
    it.rows = min(TILE, total - it.first);
    int before = -it.first;
    for (int i0 = 0; i0 < slots; i0 += 64) {
      const int i = i0 + lane;
      bool here = few ? id == it.expert : i < slots;
      if (!few && here) here = Shared::kIds && slots <= kIdsInLds ? s.ids[i] == it.expert : a.ids[i] == it.expert;
      const uint64_t all = __ballot(here);
      const int at = before + __builtin_popcountll(all & ((1ull << lane) - 1));
      if (here && at >= 0 && at < it.rows) it.slots[at] = i;
      before += __builtin_popcountll(all);
      if (before >= it.rows) break;
    }
    return it;
  }
};

// The waves' sums of one block of rows meet in LDS.
template <class Weights, class Sums>
__device__ __forceinline__ void meet(Sums& sum, const f32x4 (&acc)[Weights::J]) {
  __syncthreads();  // the sums before these have been read
  Weights::put(sum, acc);
  __syncthreads();
}
// Thread 16 r + c / 8 (of the first 256) gets eight columns of row r: v those from column c on, and with a gate u those of the second
// matrix.
template <class Weights, bool GATED, class Sums>
__device__ __forceinline__ void collect(Sums& sum, const f32x4 (&acc)[Weights::J], float (&v)[8], float (&u)[8]) {
  constexpr int SHARE = GATED && Weights::UP_WAVE ? Weights::UP_WAVE : Weights::COPIES;
  const int tid = thread_here(), r = tid / 16, c = 8 * (tid % 16);
  meet<Weights>(sum, acc);
  if (tid >= 256 || c >= Weights::cols(GATED)) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = u[e] = 0.f;
#pragma unroll
  for (int i = 0; i < SHARE; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] += sum[i][r][c + e];
      if (GATED) u[e] += sum[Weights::UP_WAVE + i][r][Weights::UP_COL + c + e];
    }
}

// act of eight columns of a slot's row, to Z.  Z is held as two bf16 numbers, the nearest one and what that leaves: 16 significant bits.
// So the second product adds no rounding of its own to that of Y: with one bf16 number, Y's error against 64 bits was 1.4 times that of
// rounding Y alone.  It costs two instructions and two reads of Z for each of one, where the weights' stream is what bounds it.
template <int ACT>
__device__ __forceinline__ void store_z(const Experts& a, int slot, int col, const float (&v)[8], const float (&u)[8]) {
  float z[8], low[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = ACT == ACT_SWIGLU ? silu(v[e]) * u[e] : ACT == ACT_GELU_TANH ? gelu_tanh(v[e]) : v[e];
  const u32x4 high = pack_bf16x8(z);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float h = __builtin_bit_cast(float, e & 1 ? high[e / 2] & 0xFFFF0000u : high[e / 2] << 16);
    low[e] = __builtin_isfinite(h) ? z[e] - h : 0.f;  // infinities and NaN stand in the first number alone
  }
  uint16_t* to = a.out + (int64_t)slot * a.N + col;
  *reinterpret_cast<u32x4*>(to) = high;
  *reinterpret_cast<u32x4*>(to + (int64_t)a.T * a.k * a.N) = pack_bf16x8(low);
}

// Z = act(X W1) of the item's rows, or a part of X W1, from the waves' sums.
template <class Weights, int ACT, int MT, int TILE, class Sums>
__device__ __forceinline__ void finish_first(Sums& sum, const Experts& a, const Items<TILE>& items, const Item& it, const f32x4 (&acc)[MT][Weights::J]) {
  constexpr bool GATED = ACT == ACT_SWIGLU;
  constexpr int NB = GATED ? 2 : 1, COLS = Weights::cols(GATED);
  const int tid = thread_here(), r = tid / 16, c = 8 * (tid % 16), col = it.block * COLS + c;
  const int64_t slots = (int64_t)a.T * a.k;
  const Far part(a.part);
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    if (16 * m >= it.rows) break;
    float v[8], u[8];
    collect<Weights, GATED>(sum, acc[m], v, u);
    if (tid >= 256 || c >= COLS || col >= a.N || 16 * m + r >= it.rows) continue;
    const int slot = it.slots[16 * m + r];
    if (items.splits == 1) {
      store_z<ACT>(a, slot, col, v, u);
    } else {
      const uint32_t to = (uint32_t)((it.split * slots + slot) * NB * a.N + col) * 4;
      part.store16(to, f32x4{v[0], v[1], v[2], v[3]});
      part.store16(to + 16, f32x4{v[4], v[5], v[6], v[7]});
      if (GATED) {
        part.store16(to + 4 * a.N, f32x4{u[0], u[1], u[2], u[3]});
        part.store16(to + 4 * a.N + 16, f32x4{u[4], u[5], u[6], u[7]});
      }
    }
  }
}

// Z of the items whose parts of K are all in memory.  A work-group's own parts are, once every wave has waited for its stores; then each
// wave counts the arrivals of some of its items, and where it was the last one adds all parts, in the order 0, 1, ...  So no item waits
// for its stores, and the counts' latencies pass side by side.
template <class Weights, int ACT, int TILE, class Shared>
__device__ __forceinline__ void join_first(Shared& s, const Experts& a, const Items<TILE>& items) {
  if (items.splits == 1) return;
  constexpr int NB = ACT == ACT_SWIGLU ? 2 : 1, COLS = Weights::cols(ACT == ACT_SWIGLU), LANES = COLS / 8;
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), total = items.total();
  const int64_t slots = (int64_t)a.T * a.k;
  const Far part(a.part);
  wait_all_mem();
  __syncthreads();
  for (int n = blockIdx.x + wave * gridDim.x; n < total; n += gridDim.x * Shared::kWave) {
    const Item it = items.find(s, a, n, 0);
    uint32_t* count = a.arrived + (int64_t)it.slots[0] * a.blocks + it.block;
    int last = 0;
    if (lane == 0) {
      last = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(items.splits - 1);
      if (last) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // as the next launch expects it
    }
    if (!uniform(last)) continue;
    const int col = it.block * COLS + 8 * (lane % LANES);
    if (col >= a.N) continue;
    for (int r = lane / LANES; r < it.rows; r += 64 / LANES) {
      const int slot = it.slots[r];
      const uint32_t first = (uint32_t)(slot * (int64_t)NB * a.N + col) * 4, pitch = (uint32_t)(slots * NB * a.N * 4);
      float v[8] = {}, u[8] = {};
      for (int q = 0; q < items.splits; q += 4) {
        f32x4 x[4][2 * NB];
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int i = 0; i < 2 * NB; ++i) x[d][i] = part.load16(first + min(q + d, items.splits - 1) * pitch + (i / 2) * 4 * a.N + 16 * (i % 2));
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[e] += q + d < items.splits ? x[d][e / 4][e % 4] : 0.f;
            if (NB == 2) u[e] += q + d < items.splits ? x[d][2 * NB - 2 + e / 4][e % 4] : 0.f;
          }
      }
      store_z<ACT>(a, slot, col, v, u);
    }
  }
}

// The item's part of Z W2, to memory: 32 threads to a row, so that a store covers whole lines (with 32 bytes a thread in two stores, 9.6 us
// in place of 8.4 for one token's two of eight experts of 512 x 2048, 63 in place of 60.5 for six of 64 of 2048 x 1408 and 16 tokens).
template <class Weights, int MT, class Sums>
__device__ __forceinline__ void finish_second(Sums& sum, const Experts& a, const Item& it, const f32x4 (&acc)[MT][Weights::J]) {
  const int tid = thread_here(), c = 4 * (tid % 32), col = it.block * 128 + c;
  const int64_t slots = (int64_t)a.T * a.k;
  const Far part(a.part);
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    if (16 * m >= it.rows) break;
    meet<Weights>(sum, acc[m]);
    if (col >= a.N) continue;
    for (int r = tid / 32; r < min(16, it.rows - 16 * m); r += 2 * Weights::WAVES) {
      f32x4 v = *reinterpret_cast<const f32x4*>(&sum[0][r][c]);
#pragma unroll
      for (int i = 1; i < Weights::COPIES; ++i) v += *reinterpret_cast<const f32x4*>(&sum[i][r][c]);
      part.store16((uint32_t)((it.split * slots + it.slots[16 * m + r]) * a.N + col) * 4, v);
    }
  }
}

// Y of one token's block of columns from its slots' parts, by 32 lanes: slots in order, a slot's parts of K in order; sixteen loads in
// flight.
__device__ __forceinline__ void sum_token(const Experts& a, int splits, int token, uint32_t valid, int block) {
  constexpr int AHEAD = 16;
  const int col = block * 128 + 4 * (threadIdx.x & 31), terms = a.k * splits;
  if (col >= a.N) return;
  const Far part(a.part);
  const uint32_t pitch = (uint32_t)((int64_t)a.T * a.k * a.N * 4);
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  int j = 0, q = 0;  // the next term
  for (int t = 0; t < terms; t += AHEAD) {
    f32x4 v[AHEAD];
    float gate[AHEAD];
    bool there[AHEAD];
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) {
      there[d] = t + d < terms && (valid >> j & 1);
      const int slot = token * a.k + min(j, a.k - 1);
      gate[d] = a.gates[slot];
      v[d] = part.load16(there[d] ? (uint32_t)(slot * a.N + col) * 4 + q * pitch : 0u);
      if (++q == splits) {
        q = 0;
        ++j;
      }
    }
#pragma unroll
    for (int d = 0; d < AHEAD; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = there[d] ? __builtin_fmaf(gate[d], v[d][i], y[i]) : y[i];
  }
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  bf16x4 b;
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = (__bf16)y[i];
  *reinterpret_cast<bf16x4*>(a.out + (int64_t)token * a.N + col) = b;
}

// Y of the tokens whose parts are all in memory, counted as in join_first, but by tokens: every slot's part of a block of columns counts
// for its token.  Whoever completes a count notes the token, and all threads of the work-group add up what was noted.
template <int TILE, class Shared>
__device__ __forceinline__ void join_second(Shared& s, const Experts& a, const Items<TILE>& items) {
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), total = items.total();
  struct Done {
    uint32_t token, valid;  // token: its block of columns in the upper half
  };
  constexpr int ROOM = sizeof(typename Shared::Sums) / sizeof(Done);
  Done* done = reinterpret_cast<Done*>(s.ring);
  wait_all_mem();
  if (tid == 0) s.found = 0;
  __syncthreads();
  for (int n = blockIdx.x + wave * gridDim.x; n < total; n += gridDim.x * Shared::kWave) {
    const Item it = items.find(s, a, n, 0);
    const int mine = it.slots[lane < it.rows ? lane : 0] / a.k;  // lane r: the token of row r
    uint32_t valid = 0;  // its slots that have an expert
    if (items.few) {
      valid = (uint32_t)(__ballot(items.id >= 0) >> (mine * a.k)) & ((1u << a.k) - 1);
    } else {
      int e[kMostChosen];
#pragma unroll
      for (int j = 0; j < kMostChosen; ++j) e[j] = a.ids[mine * a.k + min(j, a.k - 1)];
#pragma unroll
      for (int j = 0; j < kMostChosen; ++j) valid |= j < a.k && e[j] >= 0 && e[j] < a.E ? 1u << j : 0u;
    }
    bool over = false;  // complete, but there is no room to note it
    if (lane < it.rows) {
      uint32_t* count = a.arrived + (int64_t)mine * a.blocks + it.block;
      if (__hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(__builtin_popcount(valid) * items.splits - 1)) {
        __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // as the next launch expects it
        const int at = atomicAdd(&s.found, 1);
        over = at >= ROOM;
        if (!over) done[at] = Done{(uint32_t)(mine | it.block << 16), valid};
      }
    }
    for (uint64_t left = __ballot(over); left; left &= left - 1) {
      const int r = __builtin_ctzll(left), token = __shfl(mine, r);
      const uint32_t mask = (uint32_t)__shfl((int)valid, r);
      if (lane < 32) sum_token(a, items.splits, token, mask, it.block);
    }
  }
  __syncthreads();
  const int found = min(uniform(s.found), ROOM);
  for (int i = tid / 32; i < found; i += Shared::kThreads / 32) sum_token(a, items.splits, (int)(done[i].token & 0xFFFFu), done[i].valid, (int)(done[i].token >> 16));
}

// Zeros for the tokens without an expert.
__device__ __forceinline__ void clear_idle(const Experts& a) {
  for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
    int valid = 0;
    for (int j = 0; j < a.k; ++j) {
      const int e = a.ids[t * a.k + j];
      valid += e >= 0 && e < a.E;
    }
    if (valid == 0)
      for (int c = 8 * threadIdx.x; c < a.N; c += 8 * blockDim.x) *reinterpret_cast<u32x4*>(a.out + (int64_t)t * a.N + c) = u32x4{0, 0, 0, 0};
  }
}

// Items of bf16 weights, one after the other.  MOST: the most blocks of 16 rows that an item has; SECOND: of the second product.
template <int ACT, int MOST, bool SECOND>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(Bf16Weights::resident(MOST)))) void k_moe_bf16(const Experts a) {
  __shared__ MoeShared<Bf16Weights, 0> s;
  const Items<16 * MOST> items(s, a);
  for (int n = blockIdx.x; n < items.total(); n += gridDim.x) {
    const Item it = items.find(s, a, n, 0);
    auto run = [&](auto mt) {
      constexpr int MT = decltype(mt)::value;
      f32x4 acc[MT][8];
      Bf16Weights::stream<MT, ACT == ACT_SWIGLU && !SECOND, SECOND>(it, a, items.from(it), items.end(a, it), acc);
      if constexpr (SECOND) finish_second<Bf16Weights, MT>(s.sums(0), a, it, acc);
      else finish_first<Bf16Weights, ACT, MT>(s.sums(0), a, items, it, acc);
    };
    if (MOST == 1 || it.rows <= 16) run(int_constant<1>());
    else if (MOST > 2 && it.rows <= 32) run(int_constant<2>());
    else run(int_constant<MOST>());
  }
  if constexpr (SECOND) {
    join_second(s, a, items);
    clear_idle(a);
  } else {
    join_first<Bf16Weights, ACT>(s, a, items);
  }
}

// Items of 4-bit weights.  Requests run on into the next item's stages while one ends (an item with fewer stages than are in flight is
// filled up with empty ones, so that requests are never more than one item ahead), and one of two work-groups to a CU streams while the
// other multiplies or ends an item: with one, of four stages, the first products above took 120 us in place of 107, those of 54 slots of 251
// experts of 1024 x 2112 41 in place of 33.
template <int ACT, int MT, bool SECOND>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(4))) void k_moe_mx(const Experts a) {
  using W = MxWeights;
  constexpr int XT = SECOND ? 2 * MT : MT, NS = W::DEPTH, STAGE = W::stage(XT);
  constexpr bool GATED = ACT == ACT_SWIGLU && !SECOND;
  __shared__ MoeShared<W, STAGE * NS> s;
  const Items<16 * MT> items(s, a);
  const int total = items.total();
  if ((int)blockIdx.x < total) {
    int ahead = blockIdx.x, copy = 0, left;  // the item that is being requested; its stages left
    Item next = items.find(s, a, ahead, copy);
    W::Requests<MT, GATED, SECOND> ask;
    auto begin = [&]() {
      ask.begin(next, a, items.from(next), items.end(a, next));
      left = max(NS - 1, ask.length);
    };
    begin();
    uint32_t to = 0, at = 0;  // places of the ring: of the next request, of the next products
    auto request = [&]() {
      if (left == 0 && ahead + (int)gridDim.x < total) {
        ahead += gridDim.x;
        copy ^= 1;
        next = items.find(s, a, ahead, copy);
        begin();
      }
      ask.issue(a, (uint32_t)(uintptr_t)s.ring + to * STAGE);  // behind the last item: zeros, from nowhere
      left = max(left - 1, 0);
      to = to == NS - 1 ? 0 : to + 1;
    };
    Item it = next;
    for (int i = 0; i < NS - 1; ++i) request();
    for (int n = blockIdx.x; n < total; n += gridDim.x) {
      f32x4 acc[MT][W::J];
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < W::J; ++j) acc[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      const int steps = items.end(a, it) - items.from(it), stages = max(NS - 1, steps);
      for (int i = 0; i < stages; ++i) {
        wait_vm<(NS - 2) * W::loads(XT)>();
        __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): this wave holds what it read of the stage before
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        request();  // into the place of the stage before
        if (i < steps) {
          const char* stage = s.ring + at * STAGE;
          if (MT == 1 || it.rows > 16) W::multiply<MT, MT, SECOND>(stage, acc);
          else W::multiply<MT, 1, SECOND>(stage, acc);
        }
        at = at == NS - 1 ? 0 : at + 1;
      }
      auto& sums = s.sums((at == 0 ? NS - 1 : at - 1) * STAGE);  // requested into again behind the next barrier
      if constexpr (SECOND) finish_second<W, MT>(sums, a, it, acc);
      else finish_first<W, ACT, MT>(sums, a, items, it, acc);
      it = next;  // (the last item's requests stay with it)
    }
    wait_vm<0>();  // no load is left that writes LDS
  }
  if constexpr (SECOND) {
    join_second(s, a, items);
    clear_idle(a);
  } else {
    join_first<W, ACT>(s, a, items);
  }
}

}  // namespace mlp2

using namespace mlp2;

struct mlp2_moe_s {
  int64_t tokens = 0, H = 0, F = 0;  // tokens: the most of a call
  int E = 0, k = 0, act = 0, dtype = 0, device = -1, num_cus = 0, nb = 1;
  char* ws = nullptr;
  uint16_t* Z = nullptr;
  float* part = nullptr;
  int64_t part_floats = 0;
  double* logits = nullptr;
  uint32_t *arrived = nullptr, *joined = nullptr, *routed = nullptr;
};

namespace {

int status(hipError_t e) { return e == hipSuccess ? MLP2_OK : record_error(MLP2_ERR_HIP); }

constexpr int kRouteGroups = 1024;
// K of a part of the router: 32 parts, of 64 to 512 each (more than 32 only for H > 16384).
int route_part(int64_t H) {
  const int64_t per = round_up((H + 31) / 32, 64);
  return (int)(per > kRoutePart ? kRoutePart : per);
}

template <class W>
hipError_t route(const mlp2_moe_s* p, int64_t T, const void* X, const void* Wr, int32_t* ids, float* gates, hipStream_t s) {
  Route a{(const uint16_t*)X, Wr, p->logits, p->routed, ids, gates, (int)T, (int)p->H, p->E, p->k, 1, 0, 0};
  a.width = 3;  // 8 experts at least: the padded rows of K (four of a thread) fit the room for the most of K
  while (1 << a.width < p->E && a.width < 8) ++a.width;
  a.per = route_part(p->H);
  a.splits = (int)((p->H + a.per - 1) / a.per);
  // Tokens of a work-group share the reads of Wr, but follow each other in its sums: as few as keep the work-groups down to kRouteGroups.
  // (us, fp32 or bf16 router, one, two and four tokens: 9 x 1024, 251 experts 10.2, 12.5, 16.8; 48 x 4096, 32 experts 8.8, 7.8, 8.2;
  // 128 x 4096, 128 experts 21.1, 17.5, 17.0; eight were slower than four throughout.)
  const int tokens = T * a.splits <= kRouteGroups ? 1 : T * a.splits <= 2 * kRouteGroups ? 2 : 4;
  const int64_t groups = (T + tokens - 1) / tokens;
  const dim3 grid((unsigned)groups, (unsigned)a.splits);
  if (tokens == 1) k_moe_route<W, 1><<<grid, 256, 0, s>>>(a);
  else if (tokens == 2) k_moe_route<W, 2><<<grid, 256, 0, s>>>(a);
  else k_moe_route<W, 4><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

// Whether items hold up to 16 rows of an expert only: with few slots an expert, more rows than that are rare (they make a second item,
// which streams the weights again), and the smaller kernel leaves more work-groups to a CU.  (us, narrow and not, swiglu: 64 bf16 experts of
// 1024 x 1408, three slots each 102 and 97, six 113 and 105, 12 138 and 118; 16 of 2048 x 4096 16 each 188 and 161; 217 of 768 x 768 with one
// each 63 and 71.  4 bits: 64 experts, three each 52 and 53; 32 of 4096 x 4096, eight each 170 and 174; 16 of 2048 x 4096, 16 each 84 and 73.)
template <class Weights>
bool narrow(int64_t slots, int E) { return slots <= (int64_t)Weights::NARROW * E; }

template <class Weights, int ACT, bool SECOND>
void launch(const Experts& a, unsigned grid, hipStream_t s) {
  const bool few = narrow<Weights>((int64_t)a.T * a.k, a.E);
  if constexpr (std::is_same_v<Weights, Bf16Weights>) {
    if (few) k_moe_bf16<ACT, 1, SECOND><<<grid, 256, 0, s>>>(a);
    else k_moe_bf16<ACT, Weights::most(SECOND), SECOND><<<grid, 256, 0, s>>>(a);
  } else {
    if (few) k_moe_mx<ACT, 1, SECOND><<<grid, 512, 0, s>>>(a);
    else k_moe_mx<ACT, Weights::most(SECOND), SECOND><<<grid, 512, 0, s>>>(a);
  }
}

template <class Weights>
hipError_t experts(const mlp2_moe_s* p, int64_t T, const void* X, const int32_t* ids, const float* gates, const void* W1, const void* W1s, const void* W2,
                   const void* W2s, void* Y, hipStream_t s) {
  const int64_t slots = T * p->k, active = slots < p->E ? slots : p->E;  // experts that have a slot, at most
  auto fill = [&](Experts& a, bool second, int64_t K, int64_t N, int64_t width, bool gated, float join) {  // width: floats of a slot's part
    const int most_blocks = narrow<Weights>(slots, p->E) ? 1 : Weights::most(second);
    const int64_t resident = (int64_t)Weights::resident(most_blocks) * p->num_cus;  // work-groups that the chip holds at once
    const int64_t tile = 16 * most_blocks, room = p->part_floats / (slots * width);
    a.K = (int)K;
    a.N = (int)N;
    a.blocks = (int)((N + Weights::cols(gated) - 1) / Weights::cols(gated));
    a.item = Weights::ITEM;
    // a part's sums go to memory and back: 8 bytes each at the stream's rate, where a step of all work-groups takes 0.85 us.  (Without this
    // term and with parts of four steps in bf16: 85 tokens x 1536 x 960, seven of 16 experts, 102 us in place of 90; 14 x 768 x 2624, three of
    // six, 49 in place of 38; over 44 such calls 5 % more, in 4 bits 1 %.)
    a.join = join + 1.5e-6f * Weights::ITEM * (float)(slots * width);
    a.steps = (int)((K + Weights::STEP - 1) / Weights::STEP);
    a.most = (int)(room < 1 ? 1 : room > kMostParts ? kMostParts : room);
    if (a.most > a.steps / Weights::FEWEST) a.most = a.steps < Weights::FEWEST ? 1 : a.steps / Weights::FEWEST;
    const int64_t most = (active + slots / tile) * a.blocks * a.most;
    return (unsigned)(most < resident ? most : resident);
  };
  Experts a{};
  a.X = (const uint16_t*)X;
  a.ids = ids;
  a.gates = gates;
  a.T = (int)T;
  a.E = p->E;
  a.k = p->k;
  a.part = p->part;
  Experts b = a;
  a.W = (const char*)W1;
  a.scales = (const char*)W1s;
  a.out = p->Z;
  a.arrived = p->joined;
  const unsigned g1 = fill(a, false, p->H, p->F, p->nb * p->F, p->nb == 2, 0.5f * Weights::ITEM);
  if (p->act == MLP2_ACT_SWIGLU) launch<Weights, ACT_SWIGLU, false>(a, g1, s);
  else if (p->act == MLP2_ACT_GELU_TANH) launch<Weights, ACT_GELU_TANH, false>(a, g1, s);
  else launch<Weights, ACT_IDENTITY, false>(a, g1, s);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  b.X = p->Z;
  b.W = (const char*)W2;
  b.scales = (const char*)W2s;
  b.out = (uint16_t*)Y;
  b.arrived = p->arrived;
  const unsigned g2 = fill(b, true, p->F, p->H, p->H, false, 0.03f * Weights::ITEM * p->k);
  launch<Weights, ACT_IDENTITY, true>(b, g2, s);
  return hipGetLastError();
}

// What forward and experts check alike; the sizes in bytes of the weights.
int check_call(mlp2_moe_t p, int64_t T, const void* X, const void* ids, const void* gates, const void* W1, const void* W1s, const void* W2,
               const void* W2s, const void* Y, int64_t (&w)[4]) {
  if (!X || !ids || !gates || !W1 || !W2 || !Y) return MLP2_ERR_INVALID_ARG;
  const bool mx = p->dtype == MLP2_DTYPE_MXFP4;
  if (mx != (W1s != nullptr) || mx != (W2s != nullptr)) return MLP2_ERR_INVALID_ARG;
  if ((((uintptr_t)X | (uintptr_t)W1 | (uintptr_t)W1s | (uintptr_t)W2 | (uintptr_t)W2s | (uintptr_t)Y) & 15u) || ((uintptr_t)ids | (uintptr_t)gates) & 3u)
    return MLP2_ERR_ALIGNMENT;
  const int64_t n1 = (int64_t)p->E * p->nb, kp = mx_padded(p->H), fp = mx_padded(p->F);
  w[0] = mx ? n1 * p->F * kp / 2 : n1 * p->H * p->F * 2;
  w[1] = mx ? n1 * p->F * kp / kMxBlock : 0;
  w[2] = mx ? p->E * p->H * fp / 2 : p->E * p->H * p->F * 2;
  w[3] = mx ? p->E * p->H * fp / kMxBlock : 0;
  return MLP2_OK;
}

int run_experts(mlp2_moe_t p, int64_t T, const void* X, const void* ids, const void* gates, const void* W1, const void* W1s, const void* W2,
                const void* W2s, void* Y, hipStream_t s) {
  return status(p->dtype == MLP2_DTYPE_MXFP4 ? experts<MxWeights>(p, T, X, (const int32_t*)ids, (const float*)gates, W1, W1s, W2, W2s, Y, s)
                                            : experts<Bf16Weights>(p, T, X, (const int32_t*)ids, (const float*)gates, W1, W1s, W2, W2s, Y, s));
}

}  // namespace

extern "C" {

mlp2_moe_t mlp2_moe_plan(int64_t max_tokens, int64_t H, int64_t F, int64_t E, int64_t k, int act, int w_dtype) {
  clear_error();
  if (max_tokens < 1 || H < 1 || F < 1 || E < 1 || k < 1 || k > E || act < MLP2_ACT_IDENTITY || act > MLP2_ACT_SWIGLU ||
      (w_dtype != MLP2_DTYPE_BF16 && w_dtype != MLP2_DTYPE_MXFP4)) {
    record_error(MLP2_ERR_INVALID_ARG);
    return nullptr;
  }
  if (H % 64 || F % 64 || H > 32768 || F > 32768 || E > kMostExperts || k > kMostChosen || max_tokens > kMostSlots || max_tokens * k > kMostSlots) {
    record_error(MLP2_ERR_UNSUPPORTED);
    return nullptr;
  }
  int device = -1, cus = 0;
  if (const int rc = current_device(&device, &cus)) {
    record_error(rc);
    return nullptr;
  }
  auto* p = new (std::nothrow) mlp2_moe_s();
  if (!p) {
    record_error(MLP2_ERR_HIP);
    return nullptr;
  }
  p->tokens = max_tokens;
  p->H = H;
  p->F = F;
  p->E = (int)E;
  p->k = (int)k;
  p->act = act;
  p->dtype = w_dtype;
  p->nb = act == MLP2_ACT_SWIGLU ? 2 : 1;
  p->device = device;
  p->num_cus = cus;
  const int64_t slots = max_tokens * k, groups = max_tokens < kRouteGroups ? max_tokens : max_tokens / 4 + kRouteGroups;
  // room for 16 parts of K of either product while they are small; one part of the second always fits
  const int64_t wide = p->nb * F > H ? p->nb * F : H, all = kMostParts * slots * wide, few = (int64_t)16 << 20, one = slots * H;
  p->part_floats = all < few ? all : one > few ? one : few;
  const int64_t z = round_up(2 * slots * F * 2, 256), part = round_up(p->part_floats * 4, 256);
  const int64_t logits = round_up(max_tokens * ((H + route_part(H) - 1) / route_part(H)) * E * 8, 256);
  const int64_t tokens_blocks = max_tokens * ((H + 127) / 128), slots_blocks = slots * (F / 64);
  const int64_t counters = (tokens_blocks + slots_blocks + groups * kLine) * 4;
  if (hipMalloc((void**)&p->ws, (size_t)(z + part + logits + counters)) != hipSuccess ||
      hipMemset(p->ws + z + part + logits, 0, (size_t)counters) != hipSuccess ||
      hipStreamSynchronize(nullptr) != hipSuccess) {  // calls may come on any stream
    (void)hipGetLastError();
    (void)hipFree(p->ws);
    delete p;
    record_error(MLP2_ERR_HIP);
    return nullptr;
  }
  p->Z = (uint16_t*)p->ws;
  p->part = (float*)(p->ws + z);
  p->logits = (double*)(p->ws + z + part);
  p->routed = (uint32_t*)(p->ws + z + part + logits);
  p->arrived = p->routed + groups * kLine;
  p->joined = p->arrived + tokens_blocks;
  return p;
}

int mlp2_moe_experts(mlp2_moe_t p, int64_t T, const void* X, const void* ids, const void* gates, const void* W1, const void* W1_scales, const void* W2,
                     const void* W2_scales, void* Y, void* stream) {
  if (!p || T < 0 || T > p->tokens) return record_error(MLP2_ERR_INVALID_ARG);
  if (T == 0) return MLP2_OK;
  int64_t w[4];
  if (const int rc = check_call(p, T, X, ids, gates, W1, W1_scales, W2, W2_scales, Y, w)) return record_error(rc);
  const Span in[] = {{X, T * p->H * 2}, {ids, T * p->k * 4}, {gates, T * p->k * 4}, {W1, w[0]}, {W1_scales, w[1]}, {W2, w[2]}, {W2_scales, w[3]}};
  const Span out[] = {{Y, T * p->H * 2}};
  if (outputs_overlap(in, out)) return record_error(MLP2_ERR_INVALID_ARG);
  if (!on_device(p->device)) return record_error(MLP2_ERR_DEVICE);
  return run_experts(p, T, X, ids, gates, W1, W1_scales, W2, W2_scales, Y, (hipStream_t)stream);
}

int mlp2_moe_forward(mlp2_moe_t p, int64_t T, const void* X, const void* Wr, int wr_dtype, const void* W1, const void* W1_scales, const void* W2,
                     const void* W2_scales, void* Y, void* ids, void* gates, void* stream) {
  if (!p || T < 0 || T > p->tokens || (wr_dtype != MLP2_DTYPE_BF16 && wr_dtype != MLP2_DTYPE_F32)) return record_error(MLP2_ERR_INVALID_ARG);
  if (T == 0) return MLP2_OK;
  const int64_t size = wr_dtype == MLP2_DTYPE_F32 ? 4 : 2;
  if (!Wr) return record_error(MLP2_ERR_INVALID_ARG);
  int64_t w[4];
  if (const int rc = check_call(p, T, X, ids, gates, W1, W1_scales, W2, W2_scales, Y, w)) return record_error(rc);
  if ((uintptr_t)Wr % size) return record_error(MLP2_ERR_ALIGNMENT);
  const Span in[] = {{X, T * p->H * 2}, {Wr, p->H * p->E * size}, {W1, w[0]}, {W1_scales, w[1]}, {W2, w[2]}, {W2_scales, w[3]}};
  const Span out[] = {{Y, T * p->H * 2}, {ids, T * p->k * 4}, {gates, T * p->k * 4}};
  if (outputs_overlap(in, out)) return record_error(MLP2_ERR_INVALID_ARG);
  if (!on_device(p->device)) return record_error(MLP2_ERR_DEVICE);
  hipStream_t s = (hipStream_t)stream;
  const hipError_t e = size == 4 ? route<float>(p, T, X, Wr, (int32_t*)ids, (float*)gates, s) : route<uint16_t>(p, T, X, Wr, (int32_t*)ids, (float*)gates, s);
  if (e != hipSuccess) return status(e);
  return run_experts(p, T, X, ids, gates, W1, W1_scales, W2, W2_scales, Y, s);
}

void mlp2_moe_destroy(mlp2_moe_t p) {
  if (!p) return;
  release_on(p->device, p->ws);
  delete p;
}

}  // extern "C"
