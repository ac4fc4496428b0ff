// Training of the two-layer MLP: a forward pass that keeps the pre-activations
// and a backward pass.
//
//   forward    P_i = X W1_i,  Z = act(P),  Y = Z W2
//   backward   dZ = dY W2^T,  dP_i = dZ * d act / d P_i,
//              dW2 = Z^T dY,  dW1_i = X^T dP_i,  dX = sum_i dP_i W1_i^T
//
// with one W1 (identity, GELU) or two (SwiGLU: gate and up).  The activation
// runs in the epilogue of the product in front of it in both directions: the
// forward one stores P and Z from one pass over X and both weights; the
// backward one turns a tile of dZ into dP without storing dZ, and recomputes Z
// from P there, so the forward pass keeps nothing but P.
#include <climits>
#include <new>

#include "mlp2_host.h"
#include "mlp2_product.hpp"

namespace mlp2 {

__device__ __forceinline__ void unpack_bf16x8(u32x4 q, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __builtin_bit_cast(float, q[i] << 16);
    v[2 * i + 1] = __builtin_bit_cast(float, q[i] & 0xFFFF0000u);
  }
}

__device__ __forceinline__ float sigmoid(float t) { return 1.0f / (1.0f + exp_neg(t)); }

// GELU (tanh form) and its derivative at z.  With s = sigmoid(2 y), y the
// argument of the tanh: gelu = z s and gelu' = s + 2 z s (1 - s) y'.  Where s
// has reached 0 or 1 the second term is 0; y' may overflow there.
__device__ __forceinline__ void gelu_and_slope(float z, float& value, float& slope) {
  const float y = 0.7978845608028654f * (z + 0.044715f * z * z * z);
  const float s = sigmoid(2.0f * y), t = s * (1.0f - s);
  value = z * s;
  slope = s + (t == 0.0f ? 0.0f : 2.0f * z * t * (0.7978845608028654f * (1.0f + 0.134145f * z * z)));
}

// P (and Z) of a tile of X W1.  Z is computed from the fp32 sums, before P is rounded.
template <int ACT>
struct StoreForward {
  static constexpr bool kGated = ACT == ACT_SWIGLU;
  uint16_t* P;  // [M, F], gated [2, M, F]
  uint16_t* Z;  // [M, F] (identity: unused, P is Z)
  int64_t plane;  // elements of one P
  int64_t F;
  __device__ __forceinline__ void operator()(int, int row, int col, const float (&g)[8], const float (&u)[8]) const {
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = silu(g[i]) * u[i];
    const int64_t at = (int64_t)row * F + col;
    *reinterpret_cast<u32x4*>(P + at) = pack_bf16x8(g);
    *reinterpret_cast<u32x4*>(P + plane + at) = pack_bf16x8(u);
    *reinterpret_cast<u32x4*>(Z + at) = pack_bf16x8(z);
  }
  __device__ __forceinline__ void operator()(int, int row, int col, const float (&v)[8]) const {
    const int64_t at = (int64_t)row * F + col;
    *reinterpret_cast<u32x4*>(P + at) = pack_bf16x8(v);
    if constexpr (ACT == ACT_GELU_TANH) {
      float z[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = gelu_tanh(v[i]);
      *reinterpret_cast<u32x4*>(Z + at) = pack_bf16x8(z);
    }
  }
};

// dP and Z of a tile of dZ = dY W2^T and the P that the forward pass kept.
template <int ACT>
struct StoreBackward {
  static constexpr bool kGated = false;
  const uint16_t* P;
  uint16_t* dP;   // [M, F], gated [M, 2 F] (gate columns, then up columns)
  uint16_t* Z;    // [M, F] (identity: unused)
  int64_t plane, F;
  __device__ __forceinline__ void operator()(int, int row, int col, const float (&d)[8]) const {
    const int64_t at = (int64_t)row * F + col;
    if constexpr (ACT == ACT_IDENTITY) {
      *reinterpret_cast<u32x4*>(dP + at) = pack_bf16x8(d);
    } else if constexpr (ACT == ACT_GELU_TANH) {
      float p[8], z[8], dp[8];
      unpack_bf16x8(*reinterpret_cast<const u32x4*>(P + at), p);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float slope;
        gelu_and_slope(p[i], z[i], slope);
        dp[i] = d[i] * slope;
      }
      *reinterpret_cast<u32x4*>(dP + at) = pack_bf16x8(dp);
      *reinterpret_cast<u32x4*>(Z + at) = pack_bf16x8(z);
    } else {
      float g[8], u[8], z[8], dg[8], du[8];
      unpack_bf16x8(*reinterpret_cast<const u32x4*>(P + at), g);
      unpack_bf16x8(*reinterpret_cast<const u32x4*>(P + plane + at), u);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float s = sigmoid(g[i]), h = g[i] * s;
        z[i] = h * u[i];
        dg[i] = d[i] * u[i] * (s + h * (1.0f - s));
        du[i] = d[i] * h;
      }
      const int64_t to = (int64_t)row * 2 * F + col;
      *reinterpret_cast<u32x4*>(dP + to) = pack_bf16x8(dg);
      *reinterpret_cast<u32x4*>(dP + to + F) = pack_bf16x8(du);
      *reinterpret_cast<u32x4*>(Z + at) = pack_bf16x8(z);
    }
  }
};

// A bf16 result [M, N], or the two halves of its columns as matrices of their own (dW1 of a gated MLP).
struct StorePlain {
  static constexpr bool kGated = false;
  uint16_t* C;
  int64_t ld;
  int64_t second;  // elements from the first matrix to the second
  int split;       // first column of the second matrix (INT_MAX: none)
  __device__ __forceinline__ void operator()(int, int row, int col, const float (&v)[8]) const {
    uint16_t* p = col >= split ? C + second - split : C;
    *reinterpret_cast<u32x4*>(p + (int64_t)row * ld + col) = pack_bf16x8(v);
  }
};

}  // namespace mlp2

using namespace mlp2;

struct mlp2_train_s {
  int64_t rows = 0, H = 0, F = 0;  // rows: the most of a call
  int act = 0, device = -1, num_cus = 0, nb = 1;
  char* ws = nullptr;
  uint16_t* Z = nullptr;   // [rows, F]
  uint16_t* dP = nullptr;  // [rows, nb F]
};

namespace {

template <class Tile, int ACT>
hipError_t forward_first(const mlp2_train_s* p, int64_t M, const void* X, const void* W1, void* P, hipStream_t s) {
  const int64_t H = p->H, F = p->F;
  StoreForward<ACT> epi{(uint16_t*)P, p->Z, M * F, F};
  const Side r = make_side(X, H, M * H * 2);
  Side c = make_side(W1, F, p->nb * H * F * 2);
  if (p->nb == 2) c.panel = H * F;
  return launch_product<Tile, Bf16, false, true>(r, c, M, F, H, 1, epi, s);
}

template <class Tile, int ACT>
hipError_t backward_first(const mlp2_train_s* p, int64_t M, const void* dY, const void* W2, const void* P, hipStream_t s) {
  const int64_t H = p->H, F = p->F;
  StoreBackward<ACT> epi{(const uint16_t*)P, p->dP, p->Z, M * F, F};
  return launch_product<Tile, Bf16, false, false>(make_side(dY, H, M * H * 2), make_side(W2, H, F * H * 2), M, F, H, 1, epi, s);
}

template <class Tile, bool RO, bool CO>
hipError_t plain(const Side& r, const Side& c, int64_t M, int64_t N, int64_t K, const StorePlain& epi, hipStream_t s) {
  return launch_product<Tile, Bf16, RO, CO>(r, c, M, N, K, 1, epi, s);
}

int status(hipError_t e) { return e == hipSuccess ? MLP2_OK : record_error(MLP2_ERR_HIP); }

}  // namespace

extern "C" {

mlp2_train_t mlp2_train_plan(int64_t max_rows, int64_t H, int64_t F, int act, int dtype) {
  clear_error();
  if (max_rows < 1 || H < 1 || F < 1 || act < MLP2_ACT_IDENTITY || act > MLP2_ACT_SWIGLU || dtype != MLP2_DTYPE_BF16) {
    record_error(MLP2_ERR_INVALID_ARG);
    return nullptr;
  }
  if (max_rows > (1 << 20) || H % 64 || F % 64 || H > (1 << 18) || F > (1 << 18)) {
    record_error(MLP2_ERR_UNSUPPORTED);
    return nullptr;
  }
  int device = -1, cus = 0;
  if (const int rc = current_device(&device, &cus)) {
    record_error(rc);
    return nullptr;
  }
  auto* p = new (std::nothrow) mlp2_train_s();
  if (!p) {
    record_error(MLP2_ERR_HIP);
    return nullptr;
  }
  p->rows = max_rows;
  p->H = H;
  p->F = F;
  p->act = act;
  p->nb = act == MLP2_ACT_SWIGLU ? 2 : 1;
  p->device = device;
  p->num_cus = cus;
  const int64_t z = round_up(max_rows * F * 2, 256), dp = round_up(max_rows * F * 2 * p->nb, 256);
  if (hipMalloc((void**)&p->ws, (size_t)(z + dp)) != hipSuccess) {
    (void)hipGetLastError();
    delete p;
    record_error(MLP2_ERR_HIP);
    return nullptr;
  }
  p->Z = (uint16_t*)p->ws;
  p->dP = (uint16_t*)(p->ws + z);
  return p;
}

int mlp2_train_forward(mlp2_train_t p, int64_t M, const void* X, const void* W1, const void* W2, void* P, void* Y, void* stream) {
  if (!p || M < 0 || M > p->rows) return record_error(MLP2_ERR_INVALID_ARG);
  if (M == 0) return MLP2_OK;
  if (!X || !W1 || !W2 || !P || !Y) return record_error(MLP2_ERR_INVALID_ARG);
  if (((uintptr_t)X | (uintptr_t)W1 | (uintptr_t)W2 | (uintptr_t)P | (uintptr_t)Y) & 15u) return record_error(MLP2_ERR_ALIGNMENT);
  const int64_t H = p->H, F = p->F;
  const Span in[] = {{X, M * H * 2}, {W1, p->nb * H * F * 2}, {W2, F * H * 2}}, out[] = {{P, p->nb * M * F * 2}, {Y, M * H * 2}};
  if (outputs_overlap(in, out)) return record_error(MLP2_ERR_INVALID_ARG);
  if (!on_device(p->device)) return record_error(MLP2_ERR_DEVICE);
  hipStream_t s = (hipStream_t)stream;
  hipError_t e;
  if (p->act == MLP2_ACT_SWIGLU) e = forward_first<Tile128, ACT_SWIGLU>(p, M, X, W1, P, s);
  else if (p->act == MLP2_ACT_GELU_TANH) e = forward_first<Tile128, ACT_GELU_TANH>(p, M, X, W1, P, s);
  else e = forward_first<Tile128, ACT_IDENTITY>(p, M, X, W1, P, s);
  if (e != hipSuccess) return status(e);
  const void* Z = p->act == MLP2_ACT_IDENTITY ? P : p->Z;
  return status(plain<Tile128, false, true>(make_side(Z, F, M * F * 2), make_side(W2, H, F * H * 2), M, H, F,
                                            StorePlain{(uint16_t*)Y, H, 0, INT_MAX}, s));
}

int mlp2_train_backward(mlp2_train_t p, int64_t M, const void* dY, const void* X, const void* W1, const void* W2, const void* P,
                        void* dX, void* dW1, void* dW2, void* stream) {
  if (!p || M < 0 || M > p->rows) return record_error(MLP2_ERR_INVALID_ARG);
  if (!dX && !dW1 && !dW2) return record_error(MLP2_ERR_INVALID_ARG);
  if (M > 0 && (!dY || !X || !W1 || !W2 || !P)) return record_error(MLP2_ERR_INVALID_ARG);
  if (((uintptr_t)dY | (uintptr_t)X | (uintptr_t)W1 | (uintptr_t)W2 | (uintptr_t)P | (uintptr_t)dX | (uintptr_t)dW1 |
       (uintptr_t)dW2) & 15u)
    return record_error(MLP2_ERR_ALIGNMENT);
  const int64_t H = p->H, F = p->F, nb = p->nb;
  const Span in[] = {{dY, M * H * 2}, {X, M * H * 2}, {W1, nb * H * F * 2}, {W2, F * H * 2}, {P, nb * M * F * 2}};
  const Span out[] = {{dX, M * H * 2}, {dW1, nb * H * F * 2}, {dW2, F * H * 2}};
  if (outputs_overlap(in, out)) return record_error(MLP2_ERR_INVALID_ARG);
  if (!on_device(p->device)) return record_error(MLP2_ERR_DEVICE);
  hipStream_t s = (hipStream_t)stream;
  hipError_t e = hipSuccess;
  if (M > 0) {
    if (p->act == MLP2_ACT_SWIGLU) e = backward_first<Tile128, ACT_SWIGLU>(p, M, dY, W2, P, s);
    else if (p->act == MLP2_ACT_GELU_TANH) e = backward_first<Tile128, ACT_GELU_TANH>(p, M, dY, W2, P, s);
    else e = backward_first<Tile128, ACT_IDENTITY>(p, M, dY, W2, P, s);
    if (e != hipSuccess) return status(e);
  }
  // With no rows the weight gradients are sums over nothing: the products run no stage and store zeros.
  if (dW2) {
    const void* Z = p->act == MLP2_ACT_IDENTITY ? P : p->Z;
    e = plain<Tile128, true, true>(make_side(Z, F, M * F * 2), make_side(dY, H, M * H * 2), F, H, M,
                                   StorePlain{(uint16_t*)dW2, H, 0, INT_MAX}, s);
    if (e != hipSuccess) return status(e);
  }
  if (dW1) {
    e = plain<Tile128, true, true>(make_side(X, H, M * H * 2), make_side(p->dP, nb * F, M * nb * F * 2), H, nb * F, M,
                                   StorePlain{(uint16_t*)dW1, F, H * F, nb == 2 ? (int)F : INT_MAX}, s);
    if (e != hipSuccess) return status(e);
  }
  if (dX && M > 0) {
    Side c = make_side(W1, F, nb * H * F * 2);
    if (nb == 2) {
      c.jump_at = (int)(F / 64);
      c.jump = H * F - F;
    }
    e = plain<Tile128, false, false>(make_side(p->dP, nb * F, M * nb * F * 2), c, M, H, nb * F,
                                     StorePlain{(uint16_t*)dX, H, 0, INT_MAX}, s);
  }
  return status(e);
}

void mlp2_train_destroy(mlp2_train_t p) {
  if (!p) return;
  release_on(p->device, p->ws);
  delete p;
}

}  // extern "C"
