// A mixture-of-experts layer for a few tokens: router, the two-layer MLPs of each token's experts, their weighted sum.
//
//   logits = X Wr;  ids, gates = the k largest of a token and the softmax over them
//   Y[t] = sum over j of gates[t][j] * (act(X[t] W1[e]) W2[e]),  e = ids[t][j]
//
// Three launches: the router, the first products with the activation, the second products with the weighted sum.  A few tokens
// reach few rows of every expert, so the products are bound by the stream of the experts' weights.  They go from memory to
// registers without LDS: a wave takes 128 columns and every fourth (of four waves) step of K, 16 bytes a lane and load, eight loads
// a step, the next step's in flight while this one is multiplied; the waves' sums meet in LDS at the end.
//
// A row here is a slot: row r = t k + j is token t with its j-th expert.  Every work-group counts the slots of each expert by
// itself, from ids (at most 8192 words), and finds the items of work from that: an item is an expert with at least one slot, up to
// 16 MT of its rows, a block of columns and a part of K.
#include <new>

#include "mlp2_host.h"
#include "mlp2_mx.hpp"

namespace mlp2 {

constexpr int kMostExperts = 512, kMostSlots = 8192, kMostChosen = 16;
constexpr int kWaves = 4;

// ------------------------------------------------------------------ memory that other XCDs write and read in the same launch

__device__ __forceinline__ void store_far(double* p, double v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ double load_far(const double* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void store_far(float* p, float a, float b) {
  const f32x2 v = {a, b};
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 load_far(const float* p) {
  return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
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
  int width;        // threads that share a row of Wr: a power of two, at least E where that is at most 256
};

__device__ __forceinline__ double widen(uint16_t v) { return (double)__builtin_bit_cast(float, (uint32_t)v << 16); }
__device__ __forceinline__ double widen(float v) { return (double)v; }

// The k largest of a token's logits (in LDS; ties: the lowest index; NaN counts as the largest) and the softmax over them, by one wave.
__device__ __forceinline__ void choose_experts(const double* logits, int E, int k, int32_t* ids, float* gates) {
  const int lane = threadIdx.x & 63;
  constexpr int PER = kMostExperts / 64;
  double v[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = lane + 64 * i;
    v[i] = e < E ? logits[e] : 0.0;
    if (v[i] != v[i]) v[i] = __builtin_huge_val();
  }
  uint32_t gone = 0;  // of this lane's experts, those that are chosen already
  int mine = 0;
  for (int j = 0; j < k; ++j) {
    double best = -__builtin_huge_val();
    int at = kMostExperts;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = lane + 64 * i;
      if (e < E && !(gone >> i & 1) && (v[i] > best || at == kMostExperts)) {
        best = v[i];
        at = e;
      }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const double other = __shfl_xor(best, d);
      const int other_at = __shfl_xor(at, d);
      if (other > best || (other == best && other_at < at)) {
        best = other;
        at = other_at;
      }
    }
    if ((at & 63) == lane) gone |= 1u << (at >> 6);
    if (lane == j) mine = at;
  }
  // lane j: the j-th expert; the exponentials' sum is at least 1
  const double top = logits[__shfl(mine, 0)];
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
// put some of them in another order.  256 threads are `width` experts by 256 / width rows of K.
template <class W, int TT>
__global__ __launch_bounds__(256) void k_moe_route(const Route a) {
  __shared__ __align__(16) double lds[256 * TT > TT * kMostExperts ? 256 * TT : TT * kMostExperts];
  __shared__ int seen;
  const int tid = threadIdx.x, t0 = blockIdx.x * TT, split = blockIdx.y;
  const int sub = tid / a.width, subs = 256 / a.width, e0 = tid % a.width;
  const int from = split * a.per, to = min(a.H, from + a.per);
  const W* Wr = (const W*)a.Wr;
  const int chunks = (a.E + a.width - 1) / a.width;  // of experts; one but for E > 256
  for (int c = 0; c < chunks; ++c) {
    const int e = c * a.width + e0;
    double acc[TT] = {};
    for (int k0 = from; k0 < to; k0 += 64) {
      // 64 of K of the tokens' rows
      if (c || k0 > from) __syncthreads();
      for (int i = tid; i < 64 * TT; i += 256) {
        const int t = i / 64, kk = i % 64;
        lds[kk * TT + t] = t0 + t < a.T ? widen(a.X[(int64_t)(t0 + t) * a.H + k0 + kk]) : 0.0;
      }
      __syncthreads();
      if (e < a.E) {
        const W* w = Wr + (int64_t)k0 * a.E + e;
#pragma unroll 8
        for (int kk = sub; kk < 64; kk += subs) {
          const double v = widen(w[(int64_t)kk * a.E]);
#pragma unroll
          for (int t = 0; t < TT; ++t) acc[t] = __builtin_fma(v, lds[kk * TT + t], acc[t]);
        }
      }
    }
    // the rows of K meet
    __syncthreads();
#pragma unroll
    for (int t = 0; t < TT; ++t) lds[(sub * TT + t) * a.width + e0] = acc[t];
    __syncthreads();
    for (int i = tid; i < TT * a.width; i += 256) {
      const int t = i / a.width, en = c * a.width + i % a.width;
      double sum = 0.0;
      for (int s = 0; s < subs; ++s) sum += lds[(s * TT + t) * a.width + i % a.width];
      if (t0 + t < a.T && en < a.E) store_far(a.part + ((int64_t)split * a.T + t0 + t) * a.E + en, sum);
    }
  }
  wait_all_mem();
  __syncthreads();
  if (tid == 0) seen = (int)__hip_atomic_fetch_add(a.arrived + blockIdx.x * kLine, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (uniform(seen) != a.splits - 1) return;
  if (tid == 0) __hip_atomic_store(a.arrived + blockIdx.x * kLine, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  for (int i = tid; i < TT * a.E; i += 256) {
    const int t = i / a.E;
    double sum = 0.0;
    if (t0 + t < a.T)
      for (int s = 0; s < a.splits; ++s) sum += load_far(a.part + ((int64_t)s * a.T + t0) * a.E + i);
    lds[i] = sum;
  }
  __syncthreads();
  for (int t = tid / 64; t < TT; t += 4)
    if (t0 + t < a.T) choose_experts(lds + t * a.E, a.E, a.k, a.ids + (int64_t)(t0 + t) * a.k, a.gates + (int64_t)(t0 + t) * a.k);
}

// ------------------------------------------------------------------ the experts' products

struct Experts {
  const uint16_t* X;   // first: [T, H]; second: Z [T k, F]
  const int32_t* ids;
  const float* gates;
  const char* W;       // bf16 [E, nb, K, N], or MXFP4 codes of E nb matrices [N, K]
  const char* scales;
  uint16_t* out;       // first: Z; second: Y [T, H]
  float* part;         // second: [splits, T k, N]
  uint32_t* arrived;   // second: one counter for each token and block of columns; zero between launches
  int T, E, k, K, N;
  int blocks;          // of columns
  int splits, per;     // parts of K, steps of each
};

// Weights as they lie in the rest of the library, [K, N] in bf16.  A lane loads 8 columns of 8 consecutive k; taken by columns,
// with one byte permute for each pair, those are the 8 operands (16 columns, 8 k a lane) of eight instructions, the columns of
// instruction j being j, 8 + j, 16 + j, ...
struct Bf16Weights {
  static constexpr int STEP = 32;  // K of a step
  static constexpr int MOST = 4;   // blocks of 16 rows that one pass over the weights serves
  template <int MT>
  struct Regs {
    u32x4 w[8], x[MT];
  };
  uint32_t off, row;  // of this lane's first row, and from row to row
  __device__ __forceinline__ Bf16Weights(const Experts& a, int col, int64_t second) {
    const int lane = threadIdx.x & 63, c = lane & 15;
    // columns past the last are read as the last eight
    const int mine = second ? col + 8 * (c & 7) : col + 8 * c;
    row = (uint32_t)(2 * a.N);
    off = (uint32_t)((second && c >= 8 ? second : 0) + 2 * (min(mine, a.N - 8) + (int64_t)(8 * (lane >> 4)) * a.N));
  }
  __device__ static __forceinline__ int64_t matrix(const Experts& a) { return (int64_t)a.K * a.N * 2; }
  template <int MT>
  __device__ __forceinline__ void load(Regs<MT>& r, const char* w, const char*, const uint16_t* x, const uint32_t (&xo)[MT], const Experts& a, int step) const {
    const auto wr = __builtin_amdgcn_make_buffer_rsrc((void*)(w + (int64_t)step * STEP * a.N * 2), 0, -1, 0x00027000);
    const auto xr = __builtin_amdgcn_make_buffer_rsrc((void*)(x + step * STEP), 0, -1, 0x00027000);
#pragma unroll
    for (int i = 0; i < 8; ++i) r.w[i] = __builtin_amdgcn_raw_buffer_load_b128(wr, (int)off, (int)(i * row), 0);
#pragma unroll
    for (int m = 0; m < MT; ++m) r.x[m] = __builtin_amdgcn_raw_buffer_load_b128(xr, (int)xo[m], 0, 0);
  }
  __device__ static __forceinline__ int x_lane() { return 8 * ((threadIdx.x & 63) >> 4); }  // this lane's first k
  template <int MT>
  __device__ __forceinline__ void multiply(const Regs<MT>& r, f32x4 (&acc)[MT][8], const Experts&, int) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      u32x4 f;
#pragma unroll
      for (int d = 0; d < 4; ++d) f[d] = __builtin_amdgcn_perm(r.w[2 * d + 1][j / 2], r.w[2 * d][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[m][j] = Bf16::mfma(f, r.x[m], acc[m][j]);
    }
  }
  // Where the four sums of instruction j lie: columns 8 (4 g + i) + j.
  __device__ static __forceinline__ void put(float* to, const f32x4 (&c)[8]) {
    const int g = (threadIdx.x & 63) >> 4;
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

// MXFP4 weights [N, K]: a lane loads the codes of 32 k of one row, 16 rows an instruction group, and turns them into bf16 operands
// (exactly: two significant bits and a power of two), four instructions to a load.
struct MxWeights {
  static constexpr int STEP = 128;
  static constexpr int MOST = 2;
  template <int MT>
  struct Regs {
    u32x4 w[8], x[MT][4];
    uint32_t s[8];
  };
  uint32_t off[8], soff[8];
  __device__ __forceinline__ MxWeights(const Experts& a, int col, int64_t second) {
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int64_t ld = mx_padded(a.K) / 2, groups = ld / 64;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int up = second && j >= 4, n = min(col + 16 * (up ? j - 4 : j) + (lane & 15), a.N - 1);
      off[j] = (uint32_t)(((int64_t)up * a.N + n) * ld + 16 * g);
      soff[j] = (uint32_t)((up * groups * a.N + n) * 4 + g);
    }
  }
  __device__ static __forceinline__ int64_t matrix(const Experts& a) { return a.N * (mx_padded(a.K) / 2); }
  template <int MT>
  __device__ __forceinline__ void load(Regs<MT>& r, const char* w, const char* s, const uint16_t* x, const uint32_t (&xo)[MT], const Experts& a, int step) const {
    const auto wr = __builtin_amdgcn_make_buffer_rsrc((void*)(w + step * 64), 0, -1, 0x00027000);
    const auto sr = __builtin_amdgcn_make_buffer_rsrc((void*)(s + (int64_t)step * a.N * 4), 0, -1, 0x00027000);
    const auto xr = __builtin_amdgcn_make_buffer_rsrc((void*)(x + step * STEP), 0, -1, 0x00027000);
#pragma unroll
    for (int j = 0; j < 8; ++j) r.s[j] = __builtin_amdgcn_raw_buffer_load_b8(sr, (int)soff[j], 0, 0);
#pragma unroll
    for (int j = 0; j < 8; ++j) r.w[j] = __builtin_amdgcn_raw_buffer_load_b128(wr, (int)off[j], 0, 0);
    // K may end inside the last step (it is a multiple of 64): the lanes past it read the step's first k and are cleared
    const bool past = step * STEP + 32 * (int)((threadIdx.x & 63) >> 4) >= a.K;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int q = 0; q < 4; ++q) r.x[m][q] = __builtin_amdgcn_raw_buffer_load_b128(xr, (int)(xo[m] + 16 * q - (past ? 64 * ((threadIdx.x & 63) >> 4) : 0)), 0, 0);
  }
  __device__ static __forceinline__ int x_lane() { return 32 * ((threadIdx.x & 63) >> 4); }
  template <int MT>
  __device__ __forceinline__ void multiply(Regs<MT>& r, f32x4 (&acc)[MT][8], const Experts& a, int step) const {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    if ((step + 1) * STEP > a.K) {
      const bool past = step * STEP + x_lane() >= a.K;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int d = 0; d < 4; ++d) r.x[m][q][d] = past ? 0u : r.x[m][q][d];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // 2^(s - 127) as a float; 2^-127 is a subnormal one
      const float scale = __builtin_bit_cast(float, r.s[j] == 0 ? 0x00400000u : r.s[j] == 255 ? 0x7FC00000u : r.s[j] << 23);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        u32x4 f;
        f[0] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.w[j][q], scale, 0));
        f[1] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.w[j][q], scale, 1));
        f[2] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.w[j][q], scale, 2));
        f[3] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(r.w[j][q], scale, 3));
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[m][j] = Bf16::mfma(f, r.x[m][q], acc[m][j]);
      }
    }
  }
  __device__ static __forceinline__ void put(float* to, const f32x4 (&c)[8]) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int j = 0; j < 8; ++j) *reinterpret_cast<f32x4*>(to + 16 * j + 4 * g) = c[j];
  }
};

constexpr int kPitch = 128 + 4;  // floats of a row of sums in LDS
struct MoeShared {
  float sums[kWaves][16][kPitch];
  int count[kMostExperts];  // slots of an expert
  int start[kMostExperts];  // its first item
  int rows[64];             // slots of the item
  int total, expert, found;
  int done[64];             // second: tokens of the item that are complete
};

// Items of every expert: start[] and their total, from the counts.
__device__ __forceinline__ void place_items(MoeShared& s, const Experts& a, int tile) {
  const int tid = threadIdx.x;
  for (int e = tid; e < a.E; e += 256) s.count[e] = 0;
  __syncthreads();
  for (int i = tid; i < a.T * a.k; i += 256) {
    const int e = a.ids[i];
    if (e >= 0 && e < a.E) atomicAdd(&s.count[e], 1);
  }
  __syncthreads();
  if (tid < 64) {
    int before = 0;
    for (int e0 = 0; e0 < a.E; e0 += 64) {
      const int e = e0 + tid, n = e < a.E ? (s.count[e] + tile - 1) / tile * a.blocks * a.splits : 0;
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
}

// The item's expert, and the slots of its chunk of rows: their number, and the slots in s.rows.
__device__ __forceinline__ int find_rows(MoeShared& s, const Experts& a, int item, int tile, int& expert, int& block, int& split) {
  const int tid = threadIdx.x;
  __syncthreads();  // the last item's rows are no longer read
  for (int e = tid; e < a.E; e += 256) {
    const int n = (s.count[e] + tile - 1) / tile * a.blocks * a.splits;
    if (item >= s.start[e] && item < s.start[e] + n) s.expert = e;
  }
  __syncthreads();
  expert = uniform(s.expert);
  const int in = item - uniform(s.start[expert]);
  // consecutive items: the blocks of columns, then the parts of K, then the next rows
  block = in % a.blocks;
  split = in / a.blocks % a.splits;
  const int first = in / (a.blocks * a.splits) * tile, rows = min(tile, uniform(s.count[expert]) - first);
  if (tid < 64) {
    int before = 0;
    for (int i0 = 0; i0 < a.T * a.k; i0 += 64) {
      const int i = i0 + tid;
      const bool here = i < a.T * a.k && a.ids[i] == expert;
      const uint64_t all = __ballot(here);
      const int at = before + __builtin_popcountll(all & ((1ull << tid) - 1)) - first;
      if (here && at >= 0 && at < rows) s.rows[at] = i;
      before += __builtin_popcountll(all);
    }
  }
  __syncthreads();
  return rows;
}

// Sums over this wave's steps of the split, for 16 MT rows.
template <class Weights, int MT, bool SECOND>
__device__ __forceinline__ void stream_weights(const MoeShared& s, const Experts& a, const Weights& w, int expert, int nb, int rows, int split,
                                               f32x4 (&acc)[MT][8]) {
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  uint32_t xo[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int r = 16 * m + (lane & 15), slot = s.rows[r < rows ? r : 0];
    xo[m] = (uint32_t)(((int64_t)(SECOND ? slot : slot / a.k) * a.K + Weights::x_lane()) * 2);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int64_t matrix = Weights::matrix(a);
  const char* base = a.W + (int64_t)expert * nb * matrix;
  const char* sbase = a.scales + (int64_t)expert * nb * (matrix / 16);
  const int all = (a.K + Weights::STEP - 1) / Weights::STEP, end = min(all, (split + 1) * a.per);
  typename Weights::template Regs<MT> p, q;
  int step = split * a.per + wave;
  if (step >= end) return;
  w.template load<MT>(p, base, sbase, a.X, xo, a, step);
  for (;;) {
    const int next = step + kWaves;
    if (next < end) w.template load<MT>(q, base, sbase, a.X, xo, a, next);
    w.template multiply<MT>(p, acc, a, step);
    if (next >= end) break;
    step = next + kWaves;
    if (step < end) w.template load<MT>(p, base, sbase, a.X, xo, a, step);
    w.template multiply<MT>(q, acc, a, next);
    if (step >= end) break;
  }
}

// Z = act(X W1) of the item's rows.
template <class Weights, int ACT, int MT>
__device__ __forceinline__ void run_first(MoeShared& s, const Experts& a, int expert, int block, int rows) {
  constexpr bool GATED = ACT == ACT_SWIGLU;
  constexpr int COLS = GATED ? 64 : 128;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col0 = block * COLS;
  const Weights w(a, col0, GATED ? Weights::matrix(a) : 0);
  f32x4 acc[MT][8];
  stream_weights<Weights, MT, false>(s, a, w, expert, GATED ? 2 : 1, rows, 0, acc);
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    if (16 * m >= rows) break;
    if (m) __syncthreads();
    Weights::put(s.sums[wave][lane & 15], acc[m]);
    __syncthreads();
    const int r = tid / 16, c = 8 * (tid % 16);
    if (c < COLS && 16 * m + r < rows && col0 + c < a.N) {
      float v[8] = {}, u[8] = {};
#pragma unroll
      for (int i = 0; i < kWaves; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] += s.sums[i][r][c + e];
          if (GATED) u[e] += s.sums[i][r][64 + c + e];
        }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = GATED ? silu(v[e]) * u[e] : ACT == ACT_GELU_TANH ? gelu_tanh(v[e]) : v[e];
      *reinterpret_cast<u32x4*>(a.out + (int64_t)s.rows[16 * m + r] * a.N + col0 + c) = pack_bf16x8(v);
    }
  }
}

// The item's part of Z W2, to memory; then, for every token of which this was the last part, Y.
template <class Weights, int MT>
__device__ __forceinline__ void run_second(MoeShared& s, const Experts& a, int expert, int block, int split, int rows) {
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), col0 = block * 128;
  const Weights w(a, col0, 0);
  f32x4 acc[MT][8];
  stream_weights<Weights, MT, true>(s, a, w, expert, 1, rows, split, acc);
  const int64_t slots = (int64_t)a.T * a.k;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    if (16 * m >= rows) break;
    if (m) __syncthreads();
    Weights::put(s.sums[wave][lane & 15], acc[m]);
    __syncthreads();
    const int r = tid / 16, c = 8 * (tid % 16);
    if (16 * m + r < rows && col0 + c < a.N) {
      float v[8] = {};
#pragma unroll
      for (int i = 0; i < kWaves; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += s.sums[i][r][c + e];
      float* to = a.part + ((int64_t)split * slots + s.rows[16 * m + r]) * a.N + col0 + c;
#pragma unroll
      for (int e = 0; e < 8; e += 2) store_far(to + e, v[e], v[e + 1]);
    }
  }
  wait_all_mem();
  if (tid == 0) s.found = 0;
  __syncthreads();
  // Every slot's part counts for its token; the part that completes the count finds all of them in memory.
  if (tid < rows) {
    const int t = s.rows[tid] / a.k;
    int valid = 0;
    for (int j = 0; j < a.k; ++j) {
      const int e = a.ids[t * a.k + j];
      valid += e >= 0 && e < a.E;
    }
    uint32_t* count = a.arrived + (int64_t)t * a.blocks + block;
    if (__hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(valid * a.splits - 1)) {
      __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // as the next launch expects it
      s.done[atomicAdd(&s.found, 1)] = t;
    }
  }
  __syncthreads();
  const int found = uniform(s.found), c = col0 + 4 * (tid % 32);
  if (c < a.N)
    for (int i = tid / 32; i < found; i += 8) {
      const int t = s.done[i];
      f32x4 y = {0.f, 0.f, 0.f, 0.f};
      for (int j = 0; j < a.k; ++j) {
        const int e = a.ids[t * a.k + j];
        if (e < 0 || e >= a.E) continue;
        const float gate = a.gates[t * a.k + j];
        const float* p = a.part + ((int64_t)t * a.k + j) * a.N + c;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        for (int q = 0; q < a.splits; ++q) {
          const f32x2 lo = load_far(p + q * slots * a.N), hi = load_far(p + q * slots * a.N + 2);
          sum[0] += lo[0], sum[1] += lo[1], sum[2] += hi[0], sum[3] += hi[1];
        }
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) y[i4] = __builtin_fmaf(gate, sum[i4], y[i4]);
      }
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      bf16x4 b;
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) b[i4] = (__bf16)y[i4];
      *reinterpret_cast<bf16x4*>(a.out + (int64_t)t * a.N + c) = b;
    }
}

// MOST: the most blocks of 16 rows that an item has.
template <class Weights, int ACT, int MOST>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_moe_first(const Experts a) {
  __shared__ MoeShared s;
  place_items(s, a, 16 * MOST);
  const int total = uniform(s.total);
  for (int item = blockIdx.x; item < total; item += gridDim.x) {
    int expert, block, split;
    const int rows = find_rows(s, a, item, 16 * MOST, expert, block, split);
    if (MOST == 1 || rows <= 16) run_first<Weights, ACT, 1>(s, a, expert, block, rows);
    else if (MOST > 2 && rows <= 32) run_first<Weights, ACT, 2>(s, a, expert, block, rows);
    else run_first<Weights, ACT, MOST>(s, a, expert, block, rows);
  }
}

template <class Weights, int MOST>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_moe_second(const Experts a) {
  __shared__ MoeShared s;
  place_items(s, a, 16 * MOST);
  // rows of tokens without an expert
  for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
    int valid = 0;
    for (int j = 0; j < a.k; ++j) {
      const int e = a.ids[t * a.k + j];
      valid += e >= 0 && e < a.E;
    }
    if (valid == 0)
      for (int c = 8 * threadIdx.x; c < a.N; c += 8 * 256) *reinterpret_cast<u32x4*>(a.out + (int64_t)t * a.N + c) = u32x4{0, 0, 0, 0};
  }
  const int total = uniform(s.total);
  for (int item = blockIdx.x; item < total; item += gridDim.x) {
    int expert, block, split;
    const int rows = find_rows(s, a, item, 16 * MOST, expert, block, split);
    if (MOST == 1 || rows <= 16) run_second<Weights, 1>(s, a, expert, block, split, rows);
    else if (MOST > 2 && rows <= 32) run_second<Weights, 2>(s, a, expert, block, split, rows);
    else run_second<Weights, MOST>(s, a, expert, block, split, rows);
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
  int64_t logit_parts = 1;
  uint32_t *arrived = nullptr, *routed = nullptr;
};

namespace {

int status(hipError_t e) { return e == hipSuccess ? MLP2_OK : record_error(MLP2_ERR_HIP); }

constexpr int kRouteTokens = 8;

template <class W>
hipError_t route(const mlp2_moe_s* p, int64_t T, const void* X, const void* Wr, int32_t* ids, float* gates, hipStream_t s) {
  Route a{(const uint16_t*)X, Wr, p->logits, p->routed, ids, gates, (int)T, (int)p->H, p->E, p->k, 1, 0, 1};
  while (a.width < p->E && a.width < 256) a.width *= 2;
  const int tokens = T == 1 ? 1 : kRouteTokens;
  const int64_t groups = (T + tokens - 1) / tokens, units = p->H / 64;
  int64_t splits = p->num_cus / groups;
  if (splits > p->logit_parts) splits = p->logit_parts;
  if (splits > units) splits = units;
  if (splits < 1) splits = 1;
  const int64_t per = (units + splits - 1) / splits;
  a.per = (int)per * 64;
  a.splits = (int)((units + per - 1) / per);
  const dim3 grid((unsigned)groups, (unsigned)a.splits);
  if (tokens == 1) k_moe_route<W, 1><<<grid, 256, 0, s>>>(a);
  else k_moe_route<W, kRouteTokens><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

template <class Weights, int ACT>
void first(const Experts& a, unsigned grid, hipStream_t s) {
  if (a.T <= 16) k_moe_first<Weights, ACT, 1><<<grid, 256, 0, s>>>(a);
  else k_moe_first<Weights, ACT, Weights::MOST><<<grid, 256, 0, s>>>(a);
}

template <class Weights>
hipError_t experts(const mlp2_moe_s* p, int64_t T, const void* X, const int32_t* ids, const float* gates, const void* W1, const void* W1s, const void* W2,
                   const void* W2s, void* Y, hipStream_t s) {
  const int64_t slots = T * p->k, active = slots < p->E ? slots : p->E;  // experts that have a slot, at most
  auto grid_of = [&](const Experts& a) {
    const int64_t tile = T <= 16 ? 16 : 16 * Weights::MOST, most = (active + slots / tile) * a.blocks * a.splits, slots_of_chip = 4ll * p->num_cus;
    return (unsigned)(most < slots_of_chip ? most : slots_of_chip);
  };
  Experts a{};
  a.X = (const uint16_t*)X;
  a.ids = ids;
  a.gates = gates;
  a.W = (const char*)W1;
  a.scales = (const char*)W1s;
  a.out = p->Z;
  a.T = (int)T;
  a.E = p->E;
  a.k = p->k;
  a.K = (int)p->H;
  a.N = (int)p->F;
  a.blocks = (int)(p->nb == 2 ? p->F / 64 : (p->F + 127) / 128);
  a.splits = 1;
  a.per = (int)((p->H + Weights::STEP - 1) / Weights::STEP);
  const unsigned g1 = grid_of(a);
  if (p->act == MLP2_ACT_SWIGLU) first<Weights, ACT_SWIGLU>(a, g1, s);
  else if (p->act == MLP2_ACT_GELU_TANH) first<Weights, ACT_GELU_TANH>(a, g1, s);
  else first<Weights, ACT_IDENTITY>(a, g1, s);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  Experts b = a;
  b.X = p->Z;
  b.W = (const char*)W2;
  b.scales = (const char*)W2s;
  b.out = (uint16_t*)Y;
  b.part = p->part;
  b.arrived = p->arrived;
  b.K = (int)p->F;
  b.N = (int)p->H;
  b.blocks = (int)((p->H + 127) / 128);
  const int64_t steps = (p->F + Weights::STEP - 1) / Weights::STEP, room = p->part_floats / (slots * p->H);
  int64_t splits = (4ll * p->num_cus + active * b.blocks - 1) / (active * b.blocks);
  if (splits > room) splits = room;
  if (splits > steps / 8) splits = steps / 8;
  if (splits < 1) splits = 1;
  b.per = (int)((steps + splits - 1) / splits);
  b.splits = (int)((steps + b.per - 1) / b.per);
  const unsigned g2 = grid_of(b);
  if (T <= 16) k_moe_second<Weights, 1><<<g2, 256, 0, s>>>(b);
  else k_moe_second<Weights, Weights::MOST><<<g2, 256, 0, s>>>(b);
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
  const int64_t slots = max_tokens * k, groups = (max_tokens + kRouteTokens - 1) / kRouteTokens;
  // room for 16 parts of K of the second product while they are small; one always fits
  const int64_t one = slots * H, few = (int64_t)8 << 20;
  p->part_floats = 16 * one < few ? 16 * one : one > few ? one : few;
  p->logit_parts = cus / groups > 32 ? 32 : cus / groups > 1 ? cus / groups : 1;
  const int64_t z = round_up(slots * F * 2, 256), part = round_up(p->part_floats * 4, 256);
  // (a call with fewer tokens may split K further, never into more than 32 parts: those of a call with one token are few)
  int64_t logits = max_tokens * p->logit_parts * E * 8;
  for (int64_t g = 1; g <= groups; ++g) {
    const int64_t parts = cus / g > 32 ? 32 : cus / g > 1 ? cus / g : 1, t = g * kRouteTokens < max_tokens ? g * kRouteTokens : max_tokens;
    if (parts * t * E * 8 > logits) logits = parts * t * E * 8;
  }
  p->logit_parts = 32;
  logits = round_up(logits, 256);
  const int64_t counters = (max_tokens * ((H + 127) / 128) + groups * kLine) * 4;
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
