// Orthogonalisation of matrices by Newton-Schulz products:
//
//   X = G / (|G|_F + eps), then `steps` times
//   A = X X^T,  B = b A + c A A,  X <- a X + B X
//
// on the short side: a tall matrix takes A = X^T X and X <- a X + X B, so
// nothing is transposed.  Every product runs on the matrix cores in fp16 with
// fp32 sums.  fp16 rather than bf16 because the iteration lifts the small
// singular values by up to a^steps, and with them what rounding leaves there:
// the values are bounded (the singular values stay below about 1.3), so the
// range of fp16 is enough once each matrix has its own power-of-two scale, and
// its three more bits are needed.  Three choices keep a bf16 result's
// error within 1.05 to 1.5 times that of its own rounding (1.7e-3 of the norm),
// whatever the spectrum (Gaussian, power-law, low-rank and rank-one matrices
// against 64 bits; the narrowest matrices are the worst):
//   * X is held as two fp16 (22 bits); the products read the upper one, and
//     a X is added from both.  B X rounds only inside B's columns, so the error
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
// v as upper + lower fp16.
__device__ __forceinline__ void store_split(uint16_t* hi, uint16_t* lo, const float (&v)[8]) {
  const u32x4 h = pack_f16x8(v);
  float up[8], rest[8];
  unpack_f16x8(h, up);
#pragma unroll
  for (int i = 0; i < 8; ++i) rest[i] = v[i] - up[i];
  *reinterpret_cast<u32x4*>(hi) = h;
  *reinterpret_cast<u32x4*>(lo) = pack_f16x8(rest);
}

__device__ __forceinline__ float load_value(const uint16_t* p) { return __builtin_bit_cast(float, (uint32_t)*p << 16); }
__device__ __forceinline__ float load_value(const float* p) { return *p; }

__device__ __forceinline__ float block_sum(float v, float* buf) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.f;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) v += buf[w];
  return v;
}

// part[matrix][blockIdx.x]: sums of squares of a slice of the matrix.
template <class T>
__global__ __launch_bounds__(256) void k_ortho_squares(const T* G, int64_t n, float* part) {
  __shared__ float buf[4];
  const T* g = G + (int64_t)blockIdx.y * n;
  float s = 0.f;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const float v = load_value(g + i);
    s += v * v;
  }
  s = block_sum(s, buf);
  if (threadIdx.x == 0) part[(int64_t)blockIdx.y * kOrthoParts + blockIdx.x] = s;
}

// The first X: G scaled, zeros in the padding.  One thread an 8-element piece of the padded matrix.
template <class T>
__global__ __launch_bounds__(256) void k_ortho_scale(const T* G, int rows, int cols, int prows, int pcols, const float* part,
                                                     int parts, float eps, float scale, uint16_t* hi, uint16_t* lo) {
  __shared__ float buf[4];
  const float* mine = part + (int64_t)blockIdx.y * kOrthoParts;
  const float norm = sqrtf(block_sum((int)threadIdx.x < parts ? mine[threadIdx.x] : 0.f, buf));
  const float by = scale / (norm + eps);
  const T* g = G + (int64_t)blockIdx.y * rows * cols;
  const int64_t pieces = (int64_t)prows * (pcols / 8), base = (int64_t)blockIdx.y * prows * pcols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * 256) {
    const int row = (int)(i / (pcols / 8)), col = (int)(i % (pcols / 8)) * 8;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = row < rows && col + e < cols ? load_value(g + (int64_t)row * cols + col + e) * by : 0.f;
    store_split(hi + base + 8 * i, lo + base + 8 * i, v);
  }
}

// A = X X^T (or X^T X) in the scale of A.
struct StoreGram {
  static constexpr bool kGated = false;
  uint16_t* A;
  int n;
  float by;
  __device__ __forceinline__ void operator()(int batch, int row, int col, const float (&v)[8]) const {
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = v[i] * by;
    *reinterpret_cast<u32x4*>(A + ((int64_t)batch * n + row) * n + col) = pack_f16x8(o);
  }
};

// B = b A + c A A, its diagonal apart in the last steps.
struct StorePoly {
  static constexpr bool kGated = false;
  const uint16_t* A;
  uint16_t* B;
  float* diag;  // [matrices][n]
  int n;
  float b, c;   // in the scales of the operands
  int apart;
  __device__ __forceinline__ void operator()(int batch, int row, int col, const float (&v)[8]) const {
    const int64_t at = ((int64_t)batch * n + row) * n + col;
    float o[8];
    unpack_f16x8(*reinterpret_cast<const u32x4*>(A + at), o);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      o[i] = b * o[i] + c * v[i];
      if (row == col + i) {
        diag[(int64_t)batch * n + row] = apart ? o[i] * (1.f / kOrthoScaleB) : 0.f;
        if (apart) o[i] = 0.f;
      }
    }
    *reinterpret_cast<u32x4*>(B + at) = pack_f16x8(o);
  }
};

// X <- (a + diag B) X + (the rest of B) X, or the last step's result in bf16.
template <bool TALL, bool LAST>
struct StoreUpdate {
  static constexpr bool kGated = false;
  const uint16_t *hi, *lo;
  uint16_t *hi_out, *lo_out;
  const float* diag;
  int64_t ld, plane;  // of the padded matrices
  int n;
  float a, by;
  uint16_t* O;        // LAST: [matrices][rows][cols]
  int rows, cols;
  float out_by;
  __device__ __forceinline__ void operator()(int batch, int row, int col, const float (&v)[8]) const {
    const int64_t at = batch * plane + row * ld + col;
    float h[8], l[8], d[8], o[8];
    unpack_f16x8(*reinterpret_cast<const u32x4*>(hi + at), h);
    unpack_f16x8(*reinterpret_cast<const u32x4*>(lo + at), l);
    const float* dg = diag + (int64_t)batch * n + (TALL ? col : row);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      d[i] = a + dg[TALL ? i : 0];
      o[i] = d[i] * h[i] + (d[i] * l[i] + by * v[i]);
    }
    if constexpr (!LAST) {
      store_split(hi_out + at, lo_out + at, o);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] *= out_by;
      if (row >= rows) return;
      uint16_t* p = O + ((int64_t)batch * rows + row) * cols + col;
      const u32x4 q = pack_bf16x8(o);
      typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));  // odd widths: rows at any element
      if (col + 8 <= cols) {
        *reinterpret_cast<u32x4_any*>(p) = q;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (col + i < cols) p[i] = (uint16_t)(q[i / 2] >> (16 * (i & 1)));
      }
    }
  }
};

}  // namespace mlp2

using namespace mlp2;

struct mlp2_ortho_s {
  int64_t count = 0, rows = 0, cols = 0;
  int64_t prows = 0, pcols = 0, n = 0;  // padded to 64; n: the short side, padded
  bool tall = false;
  int dtype = 0, device = -1, num_cus = 0;
  float scale = 1.f;  // of X, a power of two near the square root of the long side
  char* ws = nullptr;
  uint16_t* X[2][2] = {};  // [buffer][upper, lower]: [count][prows][pcols]
  uint16_t *A = nullptr, *B = nullptr;  // [count][n][n]
  float *part = nullptr, *diag = nullptr;
};

namespace {

template <class Tile>
hipError_t ortho_step(const mlp2_ortho_s* p, const float* coeff, bool apart, bool last, uint16_t* const (&X)[2],
                      uint16_t* const (&out)[2], void* O, hipStream_t s) {
  const int64_t n = p->n, plane = p->prows * p->pcols, K = p->tall ? p->prows : p->pcols;
  const int count = (int)p->count;
  Side x = make_side(X[0], p->pcols, count * plane * 2), sq = make_side(p->A, n, count * n * n * 2);
  x.batch = plane;
  sq.batch = n * n;
  const StoreGram gram{p->A, (int)n, kOrthoScaleA / (p->scale * p->scale)};
  hipError_t e = p->tall ? launch_product<Tile, Fp16, true, true>(x, x, n, n, K, count, gram, s)
                         : launch_product<Tile, Fp16, false, false>(x, x, n, n, K, count, gram, s);
  if (e != hipSuccess) return e;
  const StorePoly poly{p->A, p->B, p->diag, (int)n, coeff[1] * kOrthoScaleB / kOrthoScaleA,
                       coeff[2] * kOrthoScaleB / (kOrthoScaleA * kOrthoScaleA), apart ? 1 : 0};
  e = launch_product<Tile, Fp16, false, false>(sq, sq, n, n, n, count, poly, s);
  if (e != hipSuccess) return e;
  sq.p = p->B;
  auto update = [&](auto epi) {
    epi.hi = X[0];
    epi.lo = X[1];
    epi.hi_out = out[0];
    epi.lo_out = out[1];
    epi.diag = p->diag;
    epi.ld = p->pcols;
    epi.plane = plane;
    epi.n = (int)n;
    epi.a = coeff[0];
    epi.by = 1.f / kOrthoScaleB;
    epi.O = (uint16_t*)O;
    epi.rows = (int)p->rows;
    epi.cols = (int)p->cols;
    epi.out_by = 1.f / p->scale;
    return epi;
  };
  if (p->tall) {
    if (last) return launch_product<Tile, Fp16, false, false>(x, sq, p->prows, p->pcols, n, count, update(StoreUpdate<true, true>{}), s);
    return launch_product<Tile, Fp16, false, false>(x, sq, p->prows, p->pcols, n, count, update(StoreUpdate<true, false>{}), s);
  }
  if (last) return launch_product<Tile, Fp16, false, true>(sq, x, p->prows, p->pcols, n, count, update(StoreUpdate<false, true>{}), s);
  return launch_product<Tile, Fp16, false, true>(sq, x, p->prows, p->pcols, n, count, update(StoreUpdate<false, false>{}), s);
}

template <class T>
void ortho_first(const mlp2_ortho_s* p, const void* G, float eps, hipStream_t s) {
  const int64_t n = p->rows * p->cols, pieces = p->prows * p->pcols / 8;
  const int parts = (int)((n + 4095) / 4096 < kOrthoParts ? (n + 4095) / 4096 : kOrthoParts);
  k_ortho_squares<T><<<dim3(parts, (unsigned)p->count), 256, 0, s>>>((const T*)G, n, p->part);
  const int64_t blocks = (pieces + 255) / 256, most = 8 * p->num_cus;
  k_ortho_scale<T><<<dim3((unsigned)(blocks < most ? blocks : most), (unsigned)p->count), 256, 0, s>>>(
      (const T*)G, (int)p->rows, (int)p->cols, (int)p->prows, (int)p->pcols, p->part, parts, eps, p->scale, p->X[0][0], p->X[0][1]);
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
  p->prows = round_up(rows, 64);
  p->pcols = round_up(cols, 64);
  p->tall = rows > cols;
  p->n = p->tall ? p->pcols : p->prows;
  p->dtype = dtype;
  p->device = device;
  p->num_cus = cus;
  p->scale = std::exp2(std::round(0.5f * std::log2((float)(rows > cols ? rows : cols))));
  const int64_t x = round_up(count * p->prows * p->pcols * 2, 256), a = round_up(count * p->n * p->n * 2, 256);
  const int64_t part = round_up(count * kOrthoParts * 4, 256), diag = round_up(count * p->n * 4, 256);
  if (hipMalloc((void**)&p->ws, (size_t)(4 * x + 2 * a + part + diag)) != hipSuccess) {
    (void)hipGetLastError();
    delete p;
    record_error(MLP2_ERR_HIP);
    return nullptr;
  }
  char* at = p->ws;
  for (int i = 0; i < 4; ++i, at += x) p->X[i / 2][i % 2] = (uint16_t*)at;
  p->A = (uint16_t*)at;
  p->B = (uint16_t*)(at + a);
  p->part = (float*)(at + 2 * a);
  p->diag = (float*)(at + 2 * a + part);
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
    e = ortho_step<Tile128>(p, coeffs + 3 * k, k >= steps - kOrthoDiagSteps, k == steps - 1, p->X[k & 1], p->X[~k & 1], O, s);
  return e == hipSuccess ? MLP2_OK : record_error(MLP2_ERR_HIP);
}

void mlp2_ortho_destroy(mlp2_ortho_t p) {
  if (!p) return;
  release_on(p->device, p->ws);
  delete p;
}

}  // extern "C"
