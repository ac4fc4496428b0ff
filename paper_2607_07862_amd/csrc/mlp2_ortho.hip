// Orthogonalisation of matrices by Newton-Schulz products:
//
//   X = G / (|G|_F + eps), then `steps` times
//   A = X X^T,  B = b A + c A A,  X <- a X + B X
//
// on the short side: a tall matrix is transposed where it is scaled, and its
// result on the way out, so that A = X X^T has K contiguous in both operands
// (the fastest order).  A and B are symmetric: only their tiles on and above the
// diagonal are computed, and stored twice.
//
// The matrix cores bound it: a step of 14336 x 4096 takes 250 to 275 us for A (136 tiles
// of 256 x 256 on 256 CUs; one part of K each, since three parts, 25 us shorter
// alone, left the whole run where it was), 90 to 99 for B and 450 to 476 for X (1.07 PFLOP/s
// with 470 MB of both halves of X read and written in its epilogue).  Small ones
// are bound by the fixed costs of three launches a step: 2 x 512 x 2048 takes 9.2,
// 6.4 and 9.9 us.
//
// Every product runs on the matrix cores in fp16 with fp32 sums.  fp16 rather
// than bf16 because the iteration lifts the small singular values by up to
// a^steps, and with them what rounding leaves there: the values are bounded (the
// singular values stay below about 1.3), so the range of fp16 is enough once each
// matrix has its own power-of-two scale, and its three more bits are needed.
// Three choices keep a bf16 result's error within 1.05 to 1.5 times that of its
// own rounding (1.7e-3 of the norm), whatever the spectrum (Gaussian, power-law,
// low-rank and rank-one matrices against 64 bits; the narrowest matrices are the
// worst):
//   * X is held as two fp16 (22 bits); the products read the upper one, and
//     a X is added from both (but in the last step, after which no error grows
//     any more).  B X rounds only inside B's columns, so the error
//     of a product does not feed the directions that are still small.  (With
//     X in one fp16, a rank-one matrix came out 15 % off.)
//   * A and B are scaled by 2^12 and 2^10, X by about the square root of its
//     long side, which leaves their small elements normal numbers.
//   * In the last three steps the diagonal of B is kept apart in fp32 and
//     applied to both halves of X in the epilogue: there X is nearly
//     orthogonal, B nearly a multiple of the identity, and its rounding would
//     be the largest error left.  (Earlier it would feed the small directions.)
#include <cmath>
#include <new>

#include "mlp2_host.h"
#include "mlp2_product.hpp"
#include "mlp2_vector.hpp"

namespace mlp2 {

constexpr float kOrthoScaleA = 4096.f, kOrthoScaleB = 1024.f;
constexpr int kOrthoDiagSteps = 3;
constexpr int kOrthoParts = 256;  // partial sums of squares of a matrix
constexpr int kOrthoMaxSteps = 64;
constexpr float kOrthoMaxCoeff = 64.f;

__device__ __forceinline__ u32x4 pack_f16x8(const float (&v)[8]) {
  f16x8 h;
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = (_Float16)v[i];
  return __builtin_bit_cast(u32x4, h);
}
__device__ __forceinline__ void unpack_f16x8(u32x4 q, float (&v)[8]) {
  const f16x8 h = __builtin_bit_cast(f16x8, q);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)h[i];
}
// v as upper + lower fp16 (a null `lo`: the upper one alone).
__device__ __forceinline__ void store_split(uint16_t* hi, uint16_t* lo, const float (&v)[8]) {
  u32x4 h = pack_f16x8(v);
  *reinterpret_cast<u32x4*>(hi) = h;
  if (!lo) return;
  // The rest is taken from the bits that are stored: left to itself the compiler converts twice, once from v and once inside the
  // instruction that makes v, which rounds differently in one element of some thousands.
  asm volatile("" : "+v"(h));
  float up[8], rest[8];
  unpack_f16x8(h, up);
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = v[i] - up[i];
  *reinterpret_cast<u32x4*>(lo) = pack_f16x8(rest);
}

__device__ __forceinline__ double block_sum(double v, double* buf) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) v += buf[w];
  return v;
}

// part[matrix][blockIdx.x]: sums of squares of a slice of the matrix, in 64 bits, which hold the square of any fp32 (in 32 bits
// norms from 1.8e19 on and below about 1e-19 were lost).  Bound by the read: fp32 2 x 4096 x 14336 103 us (4.6 TB/s).
template <class T>
__global__ __launch_bounds__(1024) void k_ortho_squares(const T* G, int64_t n, double* part) {
  __shared__ double buf[16];
  const T* g = G + (int64_t)blockIdx.y * n;
  double s = 0.;
#pragma unroll 2
  for (int64_t i = ((int64_t)blockIdx.x * 1024 + threadIdx.x) * 8; i < n; i += (int64_t)gridDim.x * 8192) {
    float v[8];
    load8(g + i, (int)min(n - i, (int64_t)8), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) s += (double)v[e] * (double)v[e];
  }
  s = block_sum(s, buf);
  if (threadIdx.x == 0) part[(int64_t)blockIdx.y * kOrthoParts + blockIdx.x] = s;
}

// The first X [n][m] (n <= m, padded to 64): G, transposed if it is tall, scaled, zeros in the padding.  One 64 x 64 block a work-group.
// Bound by memory traffic: fp32 2 x 4096 x 14336 163 us (5.8 TB/s), 14336 x 4096, through LDS, 90 us (5.2).
template <class T, bool TALL>
__global__ __launch_bounds__(256) void k_ortho_scale(const T* G, int rows, int cols, int n, int m, const double* part, int parts,
                                                     float eps, float scale, uint16_t* hi, uint16_t* lo) {
  __shared__ double buf[4];
  __shared__ float block[64][65];
  const double* mine = part + (int64_t)blockIdx.y * kOrthoParts;
  // |G| + eps is down * [1, 2): neither it nor its reciprocal need be an fp32 number, so G is scaled by 1 / down and by the rest.
  const double norm = sqrt(block_sum((int)threadIdx.x < parts ? mine[threadIdx.x] : 0., buf)) + (double)eps;
  const int down = norm > 0. && norm < INFINITY ? ilogb(norm) : 0;
  const float by = scale / (float)ldexp(norm, -down);
  const T* g = G + (int64_t)blockIdx.y * rows * cols;
  const int64_t base = (int64_t)blockIdx.y * n * m;
  const int across = m / 64, i0 = blockIdx.x / across * 64, j0 = blockIdx.x % across * 64;  // of X
  float v[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = threadIdx.x / 8 + 32 * h, c = threadIdx.x % 8 * 8;
    const int row = (TALL ? j0 : i0) + r, col = (TALL ? i0 : j0) + c;  // of G
#pragma unroll
    for (int e = 0; e < 8; ++e) v[h][e] = 0.f;
    if (row < rows && col < cols) load8(g + (int64_t)row * cols + col, cols - col, v[h]);
    if constexpr (TALL) {
#pragma unroll
      for (int e = 0; e < 8; ++e) block[c + e][r] = v[h][e];
    }
  }
  if constexpr (TALL) __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = threadIdx.x / 8 + 32 * h, c = threadIdx.x % 8 * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[h][e] = ldexpf(TALL ? block[r][c + e] : v[h][e], -down) * by;
    const int64_t at = base + (int64_t)(i0 + r) * m + j0 + c;
    store_split(hi + at, lo + at, v[h]);
  }
}

// A = X X^T in the scale of A.
struct StoreGram {
  using Read = Nothing;
  static constexpr bool kGated = false, kSymmetric = true, kMirror = true;
  uint16_t* A;
  int n, rows;  // rows: n
  float by;
  __device__ __forceinline__ void mirror(int batch, int row, int col, u32x4 q) const {
    *reinterpret_cast<u32x4*>(A + ((int64_t)batch * n + row) * n + col) = q;
  }
  __device__ __forceinline__ Nothing read(int, int, int) const { return {}; }
  __device__ __forceinline__ u32x4 operator()(int batch, int row, int col, const float (&v)[8], Nothing) const {
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = v[i] * by;
    const u32x4 q = pack_f16x8(o);
    mirror(batch, row, col, q);
    return q;
  }
};

// B = b A + c A A, its diagonal apart in the last steps.
struct StorePoly {
  using Read = u32x4;  // A's values
  static constexpr bool kGated = false, kSymmetric = true, kMirror = true;
  const uint16_t* A;
  uint16_t* B;
  float* diag;  // [matrices][n]
  int n, rows;  // rows: n
  float b, c;   // in the scales of the operands
  int apart;
  __device__ __forceinline__ void mirror(int batch, int row, int col, u32x4 q) const {
    *reinterpret_cast<u32x4*>(B + ((int64_t)batch * n + row) * n + col) = q;
  }
  __device__ __forceinline__ u32x4 read(int batch, int row, int col) const {
    return *reinterpret_cast<const u32x4*>(A + ((int64_t)batch * n + row) * n + col);
  }
  __device__ __forceinline__ u32x4 operator()(int batch, int row, int col, const float (&v)[8], u32x4 r) const {
    const int64_t at = ((int64_t)batch * n + row) * n + col;
    float o[8];
    unpack_f16x8(r, o);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      o[i] = b * o[i] + c * v[i];
      if (row == col + i) {
        diag[(int64_t)batch * n + row] = apart ? o[i] * (1.f / kOrthoScaleB) : 0.f;
        if (apart) o[i] = 0.f;
      }
    }
    const u32x4 q = pack_f16x8(o);
    *reinterpret_cast<u32x4*>(B + at) = q;
    return q;
  }
};

// X <- (a + diag B) X + (the rest of B) X.
struct Update {
  const uint16_t *hi, *lo;  // lo: null where X is taken from its upper half alone
  const float* diag;
  int64_t n, m;
  float a, by;
  struct Read {
    u32x4 hi, lo;
    float diag;
  };
  __device__ __forceinline__ Read read(int batch, int row, int col) const {
    const int64_t at = ((int64_t)batch * n + row) * m + col;
    return {*reinterpret_cast<const u32x4*>(hi + at), lo ? *reinterpret_cast<const u32x4*>(lo + at) : u32x4{0, 0, 0, 0},
            diag[batch * n + row]};
  }
  __device__ __forceinline__ void operator()(const float (&v)[8], const Read& r, float (&o)[8]) const {
    float h[8], l[8];
    unpack_f16x8(r.hi, h);
    unpack_f16x8(r.lo, l);
    const float d = a + r.diag;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = d * h[i] + (d * l[i] + by * v[i]);
  }
};
struct StoreUpdate {
  static constexpr bool kGated = false, kSymmetric = false, kMirror = false;
  using Read = Update::Read;
  Update x;
  uint16_t *hi, *lo;
  __device__ __forceinline__ Read read(int batch, int row, int col) const { return x.read(batch, row, col); }
  __device__ __forceinline__ void operator()(int batch, int row, int col, const float (&v)[8], const Read& r) const {
    float o[8];
    x(v, r, o);
    const int64_t at = ((int64_t)batch * x.n + row) * x.m + col;
    store_split(hi + at, lo ? lo + at : nullptr, o);
  }
};

// The last step's result in bf16, transposed back if G is tall.
template <bool TALL>
struct StoreLast {
  static constexpr bool kGated = false, kSymmetric = false, kMirror = TALL;
  using Read = Update::Read;
  Update x;
  uint16_t* O;  // [matrices][g_rows][g_cols]
  int g_rows, g_cols;
  int rows;     // TALL: of X, padded
  float out_by;
  __device__ __forceinline__ void mirror(int batch, int col, int row, u32x4 q) const {
    if (col < g_rows && row < g_cols) store8_packed(O + ((int64_t)batch * g_rows + col) * g_cols + row, g_cols - row, q);
  }
  __device__ __forceinline__ Read read(int batch, int row, int col) const { return x.read(batch, row, col); }
  __device__ __forceinline__ u32x4 operator()(int batch, int row, int col, const float (&v)[8], const Read& r) const {
    float o[8];
    x(v, r, o);
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] *= out_by;
    const u32x4 q = pack_bf16x8(o);
    if constexpr (!TALL) {
      if (row < g_rows && col < g_cols) store8_packed(O + ((int64_t)batch * g_rows + row) * g_cols + col, g_cols - col, q);
    }
    return q;
  }
};

}  // namespace mlp2

using namespace mlp2;

struct mlp2_ortho_s {
  int64_t count = 0, rows = 0, cols = 0;
  int64_t n = 0, m = 0;  // short and long side, padded to 64
  bool tall = false;
  int dtype = 0, device = -1, num_cus = 0;
  float scale = 1.f;  // of X, a power of two near the square root of the long side
  char* ws = nullptr;
  uint16_t* X[2][2] = {};  // [buffer][upper, lower]: [count][n][m]
  uint16_t *A = nullptr, *B = nullptr;  // [count][n][n]
  double* part = nullptr;
  float* diag = nullptr;
  SplitSpace split{};
};

namespace {

hipError_t ortho_step(const mlp2_ortho_s* p, const float* coeff, bool apart, int left, uint16_t* const (&X)[2],
                      uint16_t* const (&out)[2], void* O, hipStream_t s) {
  const int64_t n = p->n, m = p->m;
  const int count = (int)p->count;
  const bool last = left == 0;  // steps after this one
  Side x = make_side(X[0], m, count * n * m * 2), sq = make_side(p->A, n, count * n * n * 2);
  x.batch = n * m;
  sq.batch = n * n;
  const StoreGram gram{p->A, (int)n, (int)n, kOrthoScaleA / (p->scale * p->scale)};
  hipError_t e = product<Fp16, false>(x, x, n, n, m, count, gram, p->split, p->num_cus, s);
  if (e != hipSuccess) return e;
  const StorePoly poly{p->A, p->B, p->diag, (int)n, (int)n, coeff[1] * kOrthoScaleB / kOrthoScaleA,
                       coeff[2] * kOrthoScaleB / (kOrthoScaleA * kOrthoScaleA), apart ? 1 : 0};
  e = product<Fp16, false>(sq, sq, n, n, n, count, poly, p->split, p->num_cus, s);
  if (e != hipSuccess) return e;
  sq.p = p->B;
  const Update update{X[0], last ? nullptr : X[1], p->diag, n, m, coeff[0], 1.f / kOrthoScaleB};
  if (!last) return product<Fp16, true>(sq, x, n, m, n, count, StoreUpdate{update, out[0], left == 1 ? nullptr : out[1]}, p->split, p->num_cus, s);
  const int rows = (int)p->rows, cols = (int)p->cols;
  if (p->tall)
    return product<Fp16, true>(sq, x, n, m, n, count, StoreLast<true>{update, (uint16_t*)O, rows, cols, (int)n, 1.f / p->scale},
                                      p->split, p->num_cus, s);
  return product<Fp16, true>(sq, x, n, m, n, count, StoreLast<false>{update, (uint16_t*)O, rows, cols, (int)n, 1.f / p->scale},
                                    p->split, p->num_cus, s);
}

template <class T>
void ortho_first(const mlp2_ortho_s* p, const void* G, float eps, hipStream_t s) {
  const int64_t n = p->rows * p->cols, slices = (n + 8191) / 8192;
  const int parts = (int)(slices < kOrthoParts ? slices : kOrthoParts);
  k_ortho_squares<T><<<dim3(parts, (unsigned)p->count), 1024, 0, s>>>((const T*)G, n, p->part);
  const dim3 grid((unsigned)(p->n / 64 * (p->m / 64)), (unsigned)p->count);
  if (p->tall)
    k_ortho_scale<T, true><<<grid, 256, 0, s>>>((const T*)G, (int)p->rows, (int)p->cols, (int)p->n, (int)p->m, p->part, parts, eps,
                                                p->scale, p->X[0][0], p->X[0][1]);
  else
    k_ortho_scale<T, false><<<grid, 256, 0, s>>>((const T*)G, (int)p->rows, (int)p->cols, (int)p->n, (int)p->m, p->part, parts, eps,
                                                 p->scale, p->X[0][0], p->X[0][1]);
}

}  // namespace

extern "C" {

mlp2_ortho_t mlp2_ortho_plan(int64_t count, int64_t rows, int64_t cols, int dtype) {
  clear_error();
  if (count < 1 || rows < 1 || cols < 1 || (dtype != MLP2_DTYPE_BF16 && dtype != MLP2_DTYPE_F32)) {
    record_error(MLP2_ERR_INVALID_ARG);
    return nullptr;
  }
  if (count > 4096 || rows > (1 << 16) || cols > (1 << 16)) {
    record_error(MLP2_ERR_UNSUPPORTED);
    return nullptr;
  }
  int device = -1, cus = 0;
  if (const int rc = current_device(&device, &cus)) {
    record_error(rc);
    return nullptr;
  }
  auto* p = new (std::nothrow) mlp2_ortho_s();
  if (!p) {
    record_error(MLP2_ERR_HIP);
    return nullptr;
  }
  p->count = count;
  p->rows = rows;
  p->cols = cols;
  p->tall = rows > cols;
  p->n = round_up(p->tall ? cols : rows, 64);
  p->m = round_up(p->tall ? rows : cols, 64);
  p->dtype = dtype;
  p->device = device;
  p->num_cus = cus;
  p->scale = std::exp2(std::round(0.5f * std::log2((float)(rows > cols ? rows : cols))));
  const int64_t x = round_up(count * p->n * p->m * 2, 256), a = round_up(count * p->n * p->n * 2, 256);
  const int64_t part = round_up(count * kOrthoParts * 8, 256), diag = round_up(count * p->n * 4, 256);
  const int64_t floats = split_floats(p->n, p->m, count), parts = floats * 4, counters = kSplitCounters * kLine * 4;
  const int64_t fixed = 4 * x + 2 * a + part + diag;
  if (hipMalloc((void**)&p->ws, (size_t)(fixed + parts + counters)) != hipSuccess ||
      hipMemset(p->ws + fixed + parts, 0, (size_t)counters) != hipSuccess ||
      hipStreamSynchronize(nullptr) != hipSuccess) {  // calls may come on any stream
    (void)hipGetLastError();
    (void)hipFree(p->ws);
    delete p;
    record_error(MLP2_ERR_HIP);
    return nullptr;
  }
  char* at = p->ws;
  for (int i = 0; i < 4; ++i, at += x) p->X[i / 2][i % 2] = (uint16_t*)at;
  p->A = (uint16_t*)at;
  p->B = (uint16_t*)(at + a);
  p->part = (double*)(at + 2 * a);
  p->diag = (float*)(at + 2 * a + part);
  p->split = SplitSpace{(float*)(p->ws + fixed), floats, (uint32_t*)(p->ws + fixed + parts), kSplitCounters};
  return p;
}

int mlp2_ortho_run(mlp2_ortho_t p, const void* G, void* O, int steps, const float* coeffs, float eps, void* stream) {
  if (!p || !G || !O || !coeffs || steps < 1 || steps > kOrthoMaxSteps || !(eps >= 0.f)) return record_error(MLP2_ERR_INVALID_ARG);
  for (int i = 0; i < 3 * steps; ++i)
    if (!(std::fabs(coeffs[i]) <= kOrthoMaxCoeff)) return record_error(MLP2_ERR_INVALID_ARG);
  if (((uintptr_t)G | (uintptr_t)O) & 15u) return record_error(MLP2_ERR_ALIGNMENT);
  const int64_t n = p->count * p->rows * p->cols;
  const Span in[] = {{G, n * (p->dtype == MLP2_DTYPE_F32 ? 4 : 2)}}, out[] = {{O, n * 2}};
  if (outputs_overlap(in, out)) return record_error(MLP2_ERR_INVALID_ARG);
  if (!on_device(p->device)) return record_error(MLP2_ERR_DEVICE);
  hipStream_t s = (hipStream_t)stream;
  if (p->dtype == MLP2_DTYPE_F32) ortho_first<float>(p, G, eps, s);
  else ortho_first<uint16_t>(p, G, eps, s);
  hipError_t e = hipGetLastError();
  for (int k = 0; k < steps && e == hipSuccess; ++k)
    e = ortho_step(p, coeffs + 3 * k, k >= steps - kOrthoDiagSteps, steps - 1 - k, p->X[k & 1], p->X[~k & 1], O, s);
  return e == hipSuccess ? MLP2_OK : record_error(MLP2_ERR_HIP);
}

void mlp2_ortho_destroy(mlp2_ortho_t p) {
  if (!p) return;
  release_on(p->device, p->ws);
  delete p;
}

}  // extern "C"
