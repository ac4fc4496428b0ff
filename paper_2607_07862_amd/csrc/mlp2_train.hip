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
//
// The weight gradients are sums over rows: both operands of Z^T dY and X^T dP
// have K as the slow index.  Read that way on both sides (ds_read_b64_tr_b16
// moves half of what ds_read_b128 does in the same time) they run at 1.19
// PFLOP/s; with K contiguous on the row side at 1.47 (8192 x 8192 x 8192).  So
// Z leaves its epilogue transposed, through LDS, and spare work-groups of the
// same launch transpose X.  The pass is two launches: dZ with both transposes,
// then dX, dW1 and dW2 together, whose items fill each other's last round.
//
// What goes from one product to the next (Z, Z^T from the P that was kept, dP) is
// rounded to bf16: the matrix cores take 16-bit operands, and 32-bit ones would
// run at a sixteenth of the rate.  Outputs are 2.3e-3 of their norm from 64
// bits, where rounding them alone makes 1.7e-3.  All sums are fp32.
//
// Many rows are bound by the matrix cores, few by the stream of weights.  SwiGLU,
// H = 4096, F = 14336, us: 2048 rows forward 390 + 192 (1.23 and 1.25 PFLOP/s),
// backward 248 + 866 (0.97, with 190 MB of P, dP and transposes moved in its
// epilogue, and 1.39); 24 rows forward 48 + 27 (4.9 and 4.3 TB/s of weights).
#include <climits>
#include <new>

#include "mlp2_host.h"
#include "mlp2_product.hpp"
#include "mlp2_vector.hpp"

namespace mlp2 {

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
  using Read = Nothing;
  static constexpr bool kGated = ACT == ACT_SWIGLU, kSymmetric = false, kMirror = false;
  uint16_t* P;  // [M, F], gated [2, M, F]
  uint16_t* Z;  // [M, F] (identity: unused, P is Z)
  int64_t plane;  // elements of one P
  int64_t F;
  __device__ __forceinline__ Nothing read(int, int, int) const { return {}; }
  __device__ __forceinline__ void operator()(int, int row, int col, const float (&g)[8], const float (&u)[8]) const {
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = silu(g[i]) * u[i];
    const int64_t at = (int64_t)row * F + col;
    *reinterpret_cast<u32x4*>(P + at) = pack_bf16x8(g);
    *reinterpret_cast<u32x4*>(P + plane + at) = pack_bf16x8(u);
    *reinterpret_cast<u32x4*>(Z + at) = pack_bf16x8(z);
  }
  __device__ __forceinline__ void operator()(int, int row, int col, const float (&v)[8], Nothing) const {
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

// dP and Z (transposed) of a tile of dZ = dY W2^T and the P that the forward pass kept.
template <int ACT>
struct StoreBackward {
  static constexpr bool kGated = false, kSymmetric = false, kMirror = true;
  const uint16_t* P;
  uint16_t* dP;   // [M, F], gated [M, 2 F] (gate columns, then up columns)
  uint16_t* Zt;   // [F, rows]
  int64_t plane, F;
  int rows;       // M, padded to whole units of K
  __device__ __forceinline__ void mirror(int, int col, int row, u32x4 q) const {
    *reinterpret_cast<u32x4*>(Zt + (int64_t)col * rows + row) = q;
  }
  struct Read {
    u32x4 p[ACT == ACT_SWIGLU ? 2 : 1];
  };
  __device__ __forceinline__ Read read(int, int row, int col) const {
    const int64_t at = (int64_t)row * F + col;
    Read r;
    r.p[0] = *reinterpret_cast<const u32x4*>(P + at);
    if constexpr (ACT == ACT_SWIGLU) r.p[1] = *reinterpret_cast<const u32x4*>(P + plane + at);
    return r;
  }
  __device__ __forceinline__ u32x4 operator()(int, int row, int col, const float (&d)[8], const Read& r) const {
    const int64_t at = (int64_t)row * F + col;
    if constexpr (ACT == ACT_IDENTITY) {
      *reinterpret_cast<u32x4*>(dP + at) = pack_bf16x8(d);
      return r.p[0];
    } else if constexpr (ACT == ACT_GELU_TANH) {
      float p[8], z[8], dp[8];
      unpack_bf16x8(r.p[0], p);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float slope;
        gelu_and_slope(p[i], z[i], slope);
        dp[i] = d[i] * slope;
      }
      *reinterpret_cast<u32x4*>(dP + at) = pack_bf16x8(dp);
      return pack_bf16x8(z);
    } else {
      float g[8], u[8], z[8], dg[8], du[8];
      unpack_bf16x8(r.p[0], g);
      unpack_bf16x8(r.p[1], u);
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
      return pack_bf16x8(z);
    }
  }
};

// X^T: [H, rows] from X [M, H], zeros for the rows past M.
struct Transpose {
  const uint16_t* X;
  uint16_t* Xt;
  int64_t H;
  int M, rows;
  __host__ __device__ int blocks() const { return Xt ? (int)(H / 64) * (rows / 64) : 0; }
  // Blocks of an item: one, but for the largest X, since a launch holds fewer than 2^32 work-items (1048576 rows of 32768).
  __host__ __device__ int each() const { return blocks() / kMostItems + 1; }
  __host__ __device__ int items() const { return (blocks() + each() - 1) / each(); }
  static constexpr int kMostItems = 1 << 21;
  template <int THREADS>
  __device__ __forceinline__ void run(int item, char* lds) const {
    const int n = each(), end = min((item + 1) * n, blocks());
    for (int block = item * n; block < end; ++block) {
      if (block > item * n) __syncthreads();  // the block ahead has left the LDS
      move<THREADS>(block, lds);
    }
  }
  // One 64 x 64 block, through LDS.
  template <int THREADS>
  __device__ __forceinline__ void move(int block, char* lds) const {
    constexpr int PITCH = 64 + 8;  // elements
    uint16_t* t = reinterpret_cast<uint16_t*>(lds);
    const int across = (int)(H / 64), h0 = block % across * 64, m0 = block / across * 64;
    static_assert(512 % THREADS == 0, "whole rounds");
#pragma unroll
    for (int j = 0; j < 512 / THREADS; ++j) {
      const int i = thread_here() + j * THREADS, m = i / 8, h = i % 8 * 8;
      u32x4 q = {0, 0, 0, 0};
      if (m0 + m < M) q = *reinterpret_cast<const u32x4*>(X + (int64_t)(m0 + m) * H + h0 + h);
#pragma unroll
      for (int e = 0; e < 8; ++e) t[(h + e) * PITCH + m] = (uint16_t)(q[e / 2] >> (16 * (e & 1)));
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 512 / THREADS; ++j) {
      const int i = thread_here() + j * THREADS, h = i / 8, m = i % 8 * 8;
      *reinterpret_cast<u32x4*>(Xt + (int64_t)(h0 + h) * rows + m0 + m) = *reinterpret_cast<const u32x4*>(t + h * PITCH + m);
    }
  }
};

// The first launch of the backward pass: the items of dZ, then the blocks of X^T.
template <class T, class P>
__global__ __launch_bounds__(T::THREADS) __attribute__((amdgpu_waves_per_eu(2))) void k_backward_first(const P a, const Transpose x) {
  __shared__ __align__(1024) char lds[lds_of<T, P>()];
  const int n = a.items(), item = blockIdx.x;
  if (item < n) run_product<T, Bf16>(a, item, 0, lds);
  else x.template run<T::THREADS>(item - n, lds);
}

// A bf16 result [M, N], or the two halves of its columns as matrices of their own (dW1 of a gated MLP).
struct StorePlain {
  using Read = Nothing;
  static constexpr bool kGated = false, kSymmetric = false, kMirror = false;
  uint16_t* C;
  int64_t ld;
  int64_t second;  // elements from the first matrix to the second
  int split;       // first column of the second matrix (INT_MAX: none)
  __device__ __forceinline__ Nothing read(int, int, int) const { return {}; }
  __device__ __forceinline__ void operator()(int, int row, int col, const float (&v)[8], Nothing) const {
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
  uint16_t* Z = nullptr;   // forward: [rows, F]; backward: its transpose, rows padded to 64
  uint16_t* dP = nullptr;  // [rows, nb F]
  uint16_t* Xt = nullptr;  // X^T, rows padded
  SplitSpace split{};
};

namespace {

template <int ACT>
hipError_t forward_first(const mlp2_train_s* p, int64_t M, const void* X, const void* W1, void* P, hipStream_t s) {
  const int64_t H = p->H, F = p->F;
  StoreForward<ACT> epi{(uint16_t*)P, p->Z, M * F, F};
  const Side r = make_side(X, H, M * H * 2);
  Side c = make_side(W1, F, p->nb * H * F * 2);
  if (p->nb == 2) c.panel = H * F;
  return product<Bf16, true>(r, c, M, F, H, 1, epi, p->split, p->num_cus, s);
}

template <int ACT>
hipError_t backward_first(const mlp2_train_s* p, int64_t M, const void* dY, const void* W2, const void* P, const Transpose& x, hipStream_t s) {
  const int64_t H = p->H, F = p->F;
  StoreBackward<ACT> epi{(const uint16_t*)P, p->dP, p->Z, M * F, F, (int)round_up(M, 64)};
  const Choice ch = choose({M, F, H, 1, false, false}, p->split, p->num_cus);
  return with_tile<StoreBackward<ACT>>(ch.tile, [&](auto tile) {
    using T = decltype(tile);
    using Dz = Problem<false, StoreBackward<ACT>>;
    const Dz a = make_problem<T, Dz>(make_side(dY, H, M * H * 2), make_side(W2, H, F * H * 2), M, F, H, 1, epi, ch.split,
                                 p->split);
    k_backward_first<T, Dz><<<a.items() + x.items(), T::THREADS, 0, s>>>(a, x);
    return hipGetLastError();
  });
}

// dX = sum dP_i W1_i^T, dW1 = X^T dP and dW2 = Z^T dY in one launch.
hipError_t backward_second(const mlp2_train_s* p, int64_t M, const void* dY, const void* W1, void* dX, void* dW1, void* dW2, hipStream_t s) {
  using Dx = Problem<false, StorePlain, true>;
  using Dw = Problem<true, StorePlain>;
  const int64_t H = p->H, F = p->F, nb = p->nb, rows = round_up(M, 64);
  // A gradient that is not asked for has no rows, and so no items.
  const int64_t mx = dX ? M : 0, m1 = dW1 ? H : 0, m2 = dW2 ? F : 0;
  int split[3];
  const Shape shapes[3] = {{mx, H, nb * F, 1, false, false}, {m1, nb * F, M, 1, false, false}, {m2, H, M, 1, false, false}};
  const int tile = choose_shared(shapes, p->split, p->num_cus, split);
  Side w1 = make_side(W1, F, H * F * 2);
  w1.jump_at = (int)(F / 64);  // without a gate K ends there
  w1.jump = H * F - F;
  return with_tile<StorePlain>(tile, [&](auto t) {
    using T = decltype(t);
    const Dx x = make_problem<T, Dx>(make_side(p->dP, nb * F, M * nb * F * 2), w1, mx, H, nb * F, 1, StorePlain{(uint16_t*)dX, H, 0, INT_MAX},
                                     split[0], p->split);
    SplitSpace ws = behind<T>(p->split, x);
    const Dw a = make_problem<T, Dw>(make_side(p->Xt, rows, H * rows * 2), make_side(p->dP, nb * F, M * nb * F * 2), m1, nb * F, M, 1,
                                     StorePlain{(uint16_t*)dW1, F, H * F, nb == 2 ? (int)F : INT_MAX}, split[1], ws);
    ws = behind<T>(ws, a);
    const Dw b = make_problem<T, Dw>(make_side(p->Z, rows, F * rows * 2), make_side(dY, H, M * H * 2), m2, H, M, 1,
                                     StorePlain{(uint16_t*)dW2, H, 0, INT_MAX}, split[2], ws);
    const int first = a.per > x.per ? x.items() : 0;
    k_products<T, Bf16, Dx, Dw, Dw><<<x.items() + a.items() + b.items(), T::THREADS, 0, s>>>(x, a, b, first);
    return hipGetLastError();
  });
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
  const int64_t padded = round_up(max_rows, 64), z = padded * F * 2, dp = z * p->nb, xt = padded * H * 2;
  const int64_t wide = H > p->nb * F ? H : p->nb * F;  // of any result
  const int64_t tall = padded > H ? (padded > F ? padded : F) : (H > F ? H : F);
  const int64_t floats = split_floats(tall, wide, 1), parts = floats * 4, counters = kSplitCounters * kLine * 4;
  if (hipMalloc((void**)&p->ws, (size_t)(z + dp + xt + parts + counters)) != hipSuccess ||
      hipMemset(p->ws + z + dp + xt + parts, 0, (size_t)counters) != hipSuccess ||
      hipStreamSynchronize(nullptr) != hipSuccess) {  // calls may come on any stream
    (void)hipGetLastError();
    (void)hipFree(p->ws);
    delete p;
    record_error(MLP2_ERR_HIP);
    return nullptr;
  }
  p->Z = (uint16_t*)p->ws;
  p->dP = (uint16_t*)(p->ws + z);
  p->Xt = (uint16_t*)(p->ws + z + dp);
  p->split = SplitSpace{(float*)(p->ws + z + dp + xt), floats, (uint32_t*)(p->ws + z + dp + xt + parts), kSplitCounters};
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
  if (p->act == MLP2_ACT_SWIGLU) e = forward_first<ACT_SWIGLU>(p, M, X, W1, P, s);
  else if (p->act == MLP2_ACT_GELU_TANH) e = forward_first<ACT_GELU_TANH>(p, M, X, W1, P, s);
  else e = forward_first<ACT_IDENTITY>(p, M, X, W1, P, s);
  if (e != hipSuccess) return status(e);
  const void* Z = p->act == MLP2_ACT_IDENTITY ? P : p->Z;
  return status(product<Bf16, true>(make_side(Z, F, M * F * 2), make_side(W2, H, F * H * 2), M, H, F, 1,
                                           StorePlain{(uint16_t*)Y, H, 0, INT_MAX}, p->split, p->num_cus, s));
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
  if (M > 0) {
    const Transpose x{(const uint16_t*)X, dW1 ? p->Xt : nullptr, H, (int)M, (int)round_up(M, 64)};
    hipError_t e;
    if (p->act == MLP2_ACT_SWIGLU) e = backward_first<ACT_SWIGLU>(p, M, dY, W2, P, x, s);
    else if (p->act == MLP2_ACT_GELU_TANH) e = backward_first<ACT_GELU_TANH>(p, M, dY, W2, P, x, s);
    else e = backward_first<ACT_IDENTITY>(p, M, dY, W2, P, x, s);
    if (e != hipSuccess) return status(e);
  } else if (!dW1 && !dW2) {
    return MLP2_OK;
  }
  // With no rows the weight gradients are sums over nothing: the products run no stage and store zeros.
  return status(backward_second(p, M, dY, W1, dX, dW1, dW2, s));
}

void mlp2_train_destroy(mlp2_train_t p) {
  if (!p) return;
  release_on(p->device, p->ws);
  delete p;
}

}  // extern "C"
