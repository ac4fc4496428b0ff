// MXFP4: quantisation along rows or down columns, and the product of two quantised matrices.
//
//   quantise   e = floor(log2 max |x|) - 2 over 32 neighbours, at least -127;  code = nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6
//              to |x| / 2^e (ties to the even code, 6 for what lies above);  scale byte = e + 127
//   product    Y = act(A W^T), SwiGLU: silu(A Wg^T) * (A Wu^T)
//
// A NaN or an infinity in a block makes the block's scale 255, which stands for NaN.
#include <new>

#include "mlp2_host.h"
#include "mlp2_mx.hpp"
#include "mlp2_vector.hpp"

namespace mlp2 {

// The scale byte of a block from the largest |x|, as its fp32 bits (NaN and infinity: 255).
__device__ __forceinline__ uint32_t mx_scale(uint32_t largest) {
  const int e = (int)(largest >> 23);
  return e == 255 ? 255u : (uint32_t)max(e - 2, 0);
}
// Codes of 8 values under a scale.  The values are brought to the codes' range first (exactly; what falls under fp32's range there
// is far below half a step) and rounded by the conversion instruction, which rounds ties to even and saturates.
__device__ __forceinline__ uint32_t mx_codes(const float (&x)[8], uint32_t scale) {
  const int shift = 127 - (int)scale;
  uint32_t q = 0;
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __builtin_ldexpf(x[0], shift), __builtin_ldexpf(x[1], shift), 1.0f, 0);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __builtin_ldexpf(x[2], shift), __builtin_ldexpf(x[3], shift), 1.0f, 1);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __builtin_ldexpf(x[4], shift), __builtin_ldexpf(x[5], shift), 1.0f, 2);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __builtin_ldexpf(x[6], shift), __builtin_ldexpf(x[7], shift), 1.0f, 3);
  return scale == 255u ? 0u : q;
}
// What 8 codes stand for, in bf16 (exact: two significant bits, and 2^-128 is a bf16 number).
__device__ __forceinline__ u32x4 mx_values(uint32_t q, uint32_t scale) {
  float v[8];
  const int shift = (int)scale - 127;
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 1);
  const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 3);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = scale == 255u ? __builtin_nanf("") : __builtin_ldexpf(v[i], shift);
  return pack_bf16x8(v);
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu; }

struct Quantise {
  const void* X;
  int64_t ldx, matrix;  // elements
  uint8_t *codes, *scales;
  uint16_t* values;     // or null
  int rows, cols;       // of X
};

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}

// Blocks along rows.  A work-group takes 32 rows by 128 columns, 16 lanes to a row and 8 elements to a lane: its scales are one
// whole line of 128 bytes.  One row of 4096 takes 2.5 us, a launch; 777 x 2111 of fp32 with the values, 10.7 MB, 4.0.  Larger ones are
// bound by memory, less well the shorter their rows: 4096 x 14336 with the values 60 us in bf16 and 80 in fp32 (4.5 and 4.8 TB/s), 16384 x
// 4096 81 and 98 (3.8 and 4.5), without the values 48 and 71 (3.6 and 4.3).
template <class X>
__global__ __launch_bounds__(256) void k_mx_quantise_rows(const Quantise a) {
  const int lane16 = threadIdx.x & 15, row0 = blockIdx.x * 32, col0 = blockIdx.y * kMxGroup, m = blockIdx.z;
  const X* x = (const X*)a.X + m * a.matrix;
  const int64_t kp = mx_padded(a.cols);
  const int col = col0 + 8 * lane16, left = a.cols - col;
  Piece<X> p[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = row0 + 16 * i + (threadIdx.x >> 4);
    if (row < a.rows && left > 0) p[i].load(x + row * a.ldx + col, left);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = row0 + 16 * i + (threadIdx.x >> 4);
    float v[8];
    p[i].values(v);
    uint32_t largest = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) largest = max(largest, magnitude(v[e]));
    largest = max(largest, dpp<0xB1>(largest));  // quad_perm 1 0 3 2
    largest = max(largest, dpp<0x4E>(largest));  // quad_perm 2 3 0 1
    const uint32_t s = mx_scale(largest), q = mx_codes(v, s);
    uint32_t word = s << (8 * (lane16 >> 2));
    word |= dpp<0x124>(word);  // row_ror 4
    word |= dpp<0x128>(word);  // row_ror 8
    if (row < a.rows) {
      const int64_t r = (int64_t)m * a.rows + row;
      *reinterpret_cast<uint32_t*>(a.codes + (r * kp + col) / 2) = q;
      if (lane16 == 0) *reinterpret_cast<uint32_t*>(a.scales + (((int64_t)m * (kp / kMxGroup) + col0 / kMxGroup) * a.rows + row) * 4) = word;
      if (a.values && left > 0) store8_packed(a.values + r * a.cols + col, left, mx_values(q, s));
    }
  }
}

// The values of codes 2 b and 2 b + 1 of a word, in bf16.
__device__ __forceinline__ uint32_t mx_pair(uint32_t word, float unit, int b) {
  if (b == 0) return __builtin_bit_cast(uint32_t, (mx_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, unit, 0));
  if (b == 1) return __builtin_bit_cast(uint32_t, (mx_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, unit, 1));
  if (b == 2) return __builtin_bit_cast(uint32_t, (mx_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, unit, 2));
  return __builtin_bit_cast(uint32_t, (mx_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, unit, 3));
}
// The first n of C 16-bit values to any element's address.
template <int C>
__device__ __forceinline__ void store_words(uint16_t* p, int n, const uint32_t (&w)[C / 2]) {
  if (n >= C) {
    if constexpr (C == 8) {
      *reinterpret_cast<u32x4_any*>(p) = u32x4{w[0], w[1], w[2], w[3]};
    } else {
      typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
      *reinterpret_cast<u32x2_any*>(p) = u32x2_any{w[0], w[1]};
    }
  } else {
#pragma unroll
    for (int i = 0; i < C; ++i)
      if (i < n) p[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
  }
}

// Blocks down columns: X [K, N] becomes N rows of K.  A lane takes 32 of K by 16 bytes of columns, so that a block's largest element
// is found without another lane; 8 lanes lie beside each other, 8 below, and a store of codes covers 128 bytes of 8 rows.  Memory
// bounds it: 108 us for two bf16 4096 x 14336 and their values, 532 MB, a large copy's rate; one of fp32 53 us, with the values 85 (5.0 and
// 4.5 TB/s).
template <class X>
__global__ __launch_bounds__(256) void k_mx_quantise_down(const Quantise a) {
  constexpr int C = 16 / sizeof(X);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = blockIdx.z;
  const int col = (blockIdx.x * 4 + wave) * (8 * C) + C * (lane & 7), block = blockIdx.y * 8 + (lane >> 3), k0 = block * kMxBlock;
  const int64_t kp = mx_padded(a.rows);
  const int left = a.cols - col, deep = a.rows - k0;
  if (left <= 0 || k0 >= kp) return;
  const X* x = (const X*)a.X + m * a.matrix + col;
  u32x4 raw[kMxBlock];
#pragma unroll
  for (int i = 0; i < kMxBlock; ++i) {
    raw[i] = u32x4{0, 0, 0, 0};
    if (i < deep) {
      const X* from = x + (int64_t)(k0 + i) * a.ldx;
      if (left >= C) {
        raw[i] = *reinterpret_cast<const u32x4_any*>(from);
      } else if constexpr (C == 8) {
        Piece<uint16_t> p;
        p.load(from, left);
        raw[i] = p.q;
      } else {
#pragma unroll
        for (int e = 0; e < C; ++e)
          if (e < left) raw[i][e] = __builtin_bit_cast(uint32_t, from[e]);
      }
    }
  }
  auto value = [&](int i, int c) {
    // (a copy: a bit cast of a vector's element by reference takes the first element)
    const uint32_t word = raw[i][C == 8 ? c / 2 : c];
    return __builtin_bit_cast(float, C == 8 ? c & 1 ? word & 0xFFFF0000u : word << 16 : word);
  };
  u32x4 q[C];
  float unit[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    uint32_t largest = 0;
#pragma unroll
    for (int i = 0; i < kMxBlock; ++i) largest = max(largest, magnitude(value(i, c)));
    const uint32_t s = mx_scale(largest);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = value(8 * j + e, c);
      q[c][j] = mx_codes(v, s);
    }
    unit[c] = mx_unit(s);
    if (c < left) {
      const int64_t row = (int64_t)m * a.cols + col + c;
      *reinterpret_cast<u32x4*>(a.codes + row * (kp / 2) + block * 16) = q[c];
      a.scales[(((int64_t)m * (kp / kMxGroup) + block / 4) * a.cols + col + c) * 4 + block % 4] = (uint8_t)s;
    }
  }
  if (!a.values) return;
  // Two rows of X at a time: a conversion gives two neighbours of a column, a byte permute two columns of a row.
  uint16_t* values = a.values + ((int64_t)m * a.rows + k0) * a.cols + col;
#pragma unroll
  for (int i = 0; i < kMxBlock; i += 2) {
    uint32_t v[C], lo[C / 2], hi[C / 2];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint32_t word = q[c][i / 8];
      v[c] = mx_pair(word, unit[c], i / 2 % 4);
    }
#pragma unroll
    for (int c = 0; c < C; c += 2) {
      lo[c / 2] = __builtin_amdgcn_perm(v[c + 1], v[c], 0x05040100u);
      hi[c / 2] = __builtin_amdgcn_perm(v[c + 1], v[c], 0x07060302u);
    }
    if (i < deep) store_words<C>(values + (int64_t)i * a.cols, left, lo);
    if (i + 1 < deep) store_words<C>(values + (int64_t)(i + 1) * a.cols, left, hi);
  }
}

// ------------------------------------------------------------------ product

// 1 / (1 + e^-t) with the hardware's reciprocal (1 ulp): the division's ten instructions made the epilogue of a 256 x 256 tile last as long
// as three of its sixteen stages.
__device__ __forceinline__ float mx_sigmoid(float t) { return __builtin_amdgcn_rcpf(1.0f + exp_neg(t)); }

// Y of a tile, bf16 or fp32, any width.
template <int ACT, class Y>
struct StoreMx {
  using Read = Nothing;
  static constexpr bool kGated = ACT == ACT_SWIGLU, kSymmetric = false, kMirror = false;
  Y* C;
  int64_t N;
  __device__ __forceinline__ Nothing read(int, int, int) const { return {}; }
  __device__ __forceinline__ void store(int row, int col, const float (&v)[8]) const {
    const int n = (int)N - col;
    if (n > 0) store8(C + (int64_t)row * N + col, n, v);
  }
  __device__ __forceinline__ void operator()(int, int row, int col, const float (&g)[8], const float (&u)[8]) const {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = g[i] * mx_sigmoid(g[i]) * u[i];
    store(row, col, v);
  }
  __device__ __forceinline__ void operator()(int, int row, int col, const float (&p)[8], Nothing) const {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = ACT == ACT_GELU_TANH ? p[i] * mx_sigmoid(1.5957691216057308f * (p[i] + 0.044715f * p[i] * p[i] * p[i])) : p[i];
    store(row, col, v);
  }
};

}  // namespace mlp2

using namespace mlp2;

struct mlp2_mx_s {
  int64_t rows = 0, N = 0, K = 0;  // rows: the most of a call
  int act = 0, dtype = 0, device = -1, num_cus = 0, nb = 1;
  char* ws = nullptr;
  SplitSpace split{};
};

namespace {

int status(hipError_t e) { return e == hipSuccess ? MLP2_OK : record_error(MLP2_ERR_HIP); }

template <int ACT, class Y>
hipError_t mx_product(const mlp2_mx_s* p, const MxSide& r, const MxSide& c, int64_t M, void* out, hipStream_t s) {
  using Epi = StoreMx<ACT, Y>;
  const int64_t K = mx_padded(p->K) / 4;  // in units of 16 bits
  const Epi epi{(Y*)out, p->N};
  const Choice ch = choose({M, p->N, K, 1, Epi::kGated, false}, p->split, p->num_cus);
  return with_tile<Epi>(ch.tile, [&](auto tile) {
    using T = decltype(tile);
    using P = MxProblem<Epi>;
    const P a = make_problem<T, P>(r, c, M, p->N, K, 1, epi, ch.split, p->split);
    const int grid = T::QUAD && a.split == 1 && a.items() > p->num_cus ? p->num_cus : a.items();
    k_mx_product<T, P><<<grid, T::THREADS, 0, s>>>(a);
    return hipGetLastError();
  });
}

template <class Y>
hipError_t mx_product(const mlp2_mx_s* p, const MxSide& r, const MxSide& c, int64_t M, void* out, hipStream_t s) {
  if (p->act == MLP2_ACT_SWIGLU) return mx_product<ACT_SWIGLU, Y>(p, r, c, M, out, s);
  if (p->act == MLP2_ACT_GELU_TANH) return mx_product<ACT_GELU_TANH, Y>(p, r, c, M, out, s);
  return mx_product<ACT_IDENTITY, Y>(p, r, c, M, out, s);
}

}  // namespace

extern "C" {

int mlp2_mx_quantize(int64_t count, int64_t rows, int64_t cols, int down, const void* X, int dtype, int64_t ldx, int64_t matrix_stride,
                     void* codes, void* scales, void* values, void* stream) {
  if (count < 0 || rows < 0 || cols < 0 || (down != 0 && down != 1) || (dtype != MLP2_DTYPE_BF16 && dtype != MLP2_DTYPE_F32))
    return record_error(MLP2_ERR_INVALID_ARG);
  if (count > 65535 || rows > (1 << 20) || cols > (1 << 20) || ldx > (int64_t)1 << 40 || matrix_stride > (int64_t)1 << 40) return record_error(MLP2_ERR_UNSUPPORTED);
  if (count == 0 || rows == 0 || cols == 0) return MLP2_OK;
  // several matrices: one behind the other, or beside each other in the rows of one buffer
  const bool beside = count > 1 && matrix_stride >= cols && (count - 1) * matrix_stride + cols <= ldx;
  if (!X || !codes || !scales || ldx < cols || (count > 1 && !beside && matrix_stride < (rows - 1) * ldx + cols)) return record_error(MLP2_ERR_INVALID_ARG);
  const int64_t size = dtype == MLP2_DTYPE_F32 ? 4 : 2;
  if ((((uintptr_t)codes | (uintptr_t)scales) & 15u) || (uintptr_t)X % size || (uintptr_t)values % 2) return record_error(MLP2_ERR_ALIGNMENT);
  const int64_t out = down ? cols : rows, kp = mx_padded(down ? rows : cols);
  const Span x = beside                                       ? Span{X, ((count - 1) * matrix_stride + cols) * size, rows, ldx * size}
                 : count == 1 || matrix_stride == rows * ldx ? Span{X, cols * size, count * rows, ldx * size}
                                                             : Span{X, ((count - 1) * matrix_stride + (rows - 1) * ldx + cols) * size};
  const Span in[] = {x}, outs[] = {{codes, count * out * kp / 2}, {scales, count * out * kp / kMxBlock}, {values, values ? count * rows * cols * 2 : 0}};
  if (outputs_overlap(in, outs)) return record_error(MLP2_ERR_INVALID_ARG);
  if (const int rc = usable_device()) return record_error(rc);
  const Quantise a{X, ldx, matrix_stride, (uint8_t*)codes, (uint8_t*)scales, (uint16_t*)values, (int)rows, (int)cols};
  // a launch's grid, so that no work-group divides: rows, then columns (down: 512 bytes of columns, then 256 rows), then matrices
  const dim3 grid = down ? dim3((unsigned)((cols * size + 511) / 512), (unsigned)((kp + 255) / 256), (unsigned)count)
                         : dim3((unsigned)((rows + 31) / 32), (unsigned)(kp / kMxGroup), (unsigned)count);
  if ((int64_t)grid.x * grid.y * grid.z >= 1 << 24) return record_error(MLP2_ERR_UNSUPPORTED);  // a launch holds fewer than 2^32 work-items
  hipStream_t s = (hipStream_t)stream;
  if (down && size == 2) k_mx_quantise_down<uint16_t><<<grid, 256, 0, s>>>(a);
  else if (down) k_mx_quantise_down<float><<<grid, 256, 0, s>>>(a);
  else if (size == 2) k_mx_quantise_rows<uint16_t><<<grid, 256, 0, s>>>(a);
  else k_mx_quantise_rows<float><<<grid, 256, 0, s>>>(a);
  return status(hipGetLastError());
}

mlp2_mx_t mlp2_mx_plan(int64_t max_rows, int64_t N, int64_t K, int act, int y_dtype) {
  clear_error();
  if (max_rows < 1 || N < 1 || K < 1 || act < MLP2_ACT_IDENTITY || act > MLP2_ACT_SWIGLU ||
      (y_dtype != MLP2_DTYPE_BF16 && y_dtype != MLP2_DTYPE_F32)) {
    record_error(MLP2_ERR_INVALID_ARG);
    return nullptr;
  }
  if (max_rows > (1 << 18) || N > (1 << 18) || K > (1 << 18)) {
    record_error(MLP2_ERR_UNSUPPORTED);
    return nullptr;
  }
  int device = -1, cus = 0;
  if (const int rc = current_device(&device, &cus)) {
    record_error(rc);
    return nullptr;
  }
  auto* p = new (std::nothrow) mlp2_mx_s();
  if (!p) {
    record_error(MLP2_ERR_HIP);
    return nullptr;
  }
  p->rows = max_rows;
  p->N = N;
  p->K = K;
  p->act = act;
  p->dtype = y_dtype;
  p->nb = act == MLP2_ACT_SWIGLU ? 2 : 1;
  p->device = device;
  p->num_cus = cus;
  const int64_t floats = split_floats(max_rows, N * p->nb, 1), counters = kSplitCounters * kLine * 4;
  if (hipMalloc((void**)&p->ws, (size_t)(floats * 4 + counters)) != hipSuccess ||
      hipMemset(p->ws + floats * 4, 0, (size_t)counters) != hipSuccess ||
      hipStreamSynchronize(nullptr) != hipSuccess) {  // calls may come on any stream
    (void)hipGetLastError();
    (void)hipFree(p->ws);
    delete p;
    record_error(MLP2_ERR_HIP);
    return nullptr;
  }
  p->split = SplitSpace{(float*)p->ws, floats, (uint32_t*)(p->ws + floats * 4), kSplitCounters};
  return p;
}

int mlp2_mx_product(mlp2_mx_t p, int64_t M, const void* A, const void* A_scales, const void* W, const void* W_scales, void* Y, void* stream) {
  if (!p || M < 0 || M > p->rows) return record_error(MLP2_ERR_INVALID_ARG);
  if (M == 0) return MLP2_OK;
  if (!A || !A_scales || !W || !W_scales || !Y) return record_error(MLP2_ERR_INVALID_ARG);
  const int64_t N = p->N, kp = mx_padded(p->K), size = p->dtype == MLP2_DTYPE_F32 ? 4 : 2, nb = p->nb;
  if ((((uintptr_t)A | (uintptr_t)A_scales | (uintptr_t)W | (uintptr_t)W_scales) & 15u) || (uintptr_t)Y % size) return record_error(MLP2_ERR_ALIGNMENT);
  const Span in[] = {{A, M * kp / 2}, {A_scales, M * kp / kMxBlock}, {W, nb * N * kp / 2}, {W_scales, nb * N * kp / kMxBlock}}, out[] = {{Y, M * N * size}};
  if (outputs_overlap(in, out)) return record_error(MLP2_ERR_INVALID_ARG);
  if (!on_device(p->device)) return record_error(MLP2_ERR_DEVICE);
  const MxSide r{(const uint8_t*)A, (const uint8_t*)A_scales, M, kp / 2, false}, c{(const uint8_t*)W, (const uint8_t*)W_scales, N, kp / 2, nb == 2};
  hipStream_t s = (hipStream_t)stream;
  return status(size == 4 ? mx_product<float>(p, r, c, M, Y, s) : mx_product<uint16_t>(p, r, c, M, Y, s));
}

void mlp2_mx_destroy(mlp2_mx_t p) {
  if (!p) return;
  release_on(p->device, p->ws);
  delete p;
}

}  // extern "C"
