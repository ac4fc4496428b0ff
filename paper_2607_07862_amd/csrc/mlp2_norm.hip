// Layer norm over the rows of a matrix, forward and backward.
//
//   y  = (x - mean) rstd w + b,   rstd = (var + eps)^(-1/2)
//   dx = rstd (g - mean(g) - xhat mean(g xhat)),   g = dy w,  xhat = (x - mean) rstd
//   dw = sum over rows of dy xhat,   db = sum over rows of dy
//
// Both directions are bound by memory traffic: bf16 8192 x 4096 takes 26 to 29 us
// forward (4.7 to 5.1 TB/s; a large copy reaches 4.9) and 45 backward (4.5 TB/s, 5
// us of it in the second kernel), fp32 to bf16 16384 x 8192 146 (5.5 TB/s) and 260
// us (5.2), fp32 to fp32 194 and 312 (5.5 and 5.2).  Calls of a few rows are bound by their launch, 4 us.  A row is held in
// registers by a group of 16 to 1024 threads (up to 16 elements a thread), so
// each input is read once; the variance is taken around the mean in a second
// pass over the registers.  The groups of a persistent grid walk the rows with
// the weights (forward) or the running dw and db of their columns (backward) in
// registers.  The backward pass leaves one partial dw and db per work-group.  Few
// and short ones are added by the work-group that finishes last, others by a
// second small kernel; either adds in a fixed order and gives the same bits each
// run.
#include <new>

#include "mlp2_host.h"
#include "mlp2_vector.hpp"

namespace mlp2 {

constexpr int kNormMaxWidth = 16384;
constexpr int kNormBlock = 1024;  // backward: threads of a work-group

// Sums of N values over a group of NT threads, in every thread of it.  The
// groups of a work-group call it together; `buf` alternates between two
// regions, so one barrier a call is enough.
template <int NT, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float (*buf)[N]) {
#pragma unroll
  for (int d = (NT < 64 ? NT : 64) / 2; d > 0; d >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], d);
  if constexpr (NT > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) buf[wave][i] = v[i];
    __syncthreads();
    constexpr int W = NT / 64;
    const int first = wave / W * W;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += buf[first + w][i];
      v[i] = s;
    }
  }
}

struct NormArgs {
  const void* X;
  const void* dY;
  void* Y;          // forward: Y; backward: dX
  const float* w;   // null: ones
  const float* b;   // null: zeros
  float* mean;      // forward: written (may be null); backward: read
  float* rstd;
  float* part;      // backward: [work-groups][2][H], or null
  int64_t ldx, ldd, ldy;
  int M, H;
  float eps;
  float *dw, *db;     // backward: written by a work-group alone, or by the last one to arrive
  uint32_t* arrived;  // null: another kernel adds the parts
};

// Floats of a part's dw (and of its db, which follows).
__host__ __device__ __forceinline__ int part_pitch(int H) { return (H + 7) / 8 * 8; }

// NT threads a row, C pieces of 8 elements a thread: NT * 8 * C >= H.
template <class XT, class YT, int NT, int C>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void k_norm_forward(const NormArgs a) {
  constexpr int BLOCK = NT < 256 ? 256 : NT, GROUPS = BLOCK / NT;
  __shared__ float buf[2][BLOCK / 64][1];
  const int t = threadIdx.x % NT, group = threadIdx.x / NT;
  const float inv = 1.0f / (float)a.H;
  float w[C][8], b[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = 8 * (t + NT * c), n = a.H - col;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[c][i] = 1.f;
      b[c][i] = 0.f;
    }
    if (a.w && n > 0) load8(a.w + col, n, w[c]);
    if (a.b && n > 0) load8(a.b + col, n, b[c]);
  }
  Piece<XT> now[C], next[C];
  auto request = [&](Piece<XT> (&p)[C], int row) {
    const XT* x = (const XT*)a.X + (int64_t)(row < a.M ? row : a.M - 1) * a.ldx;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = 8 * (t + NT * c), n = a.H - col;
      if (n > 0) p[c].load(x + col, n);
    }
  };
  const int step = gridDim.x * GROUPS;
  request(next, blockIdx.x * GROUPS + group);
  for (int row0 = blockIdx.x * GROUPS; row0 < a.M; row0 += step) {
    const int row = row0 + group;
    const bool live = row < a.M;
#pragma unroll
    for (int c = 0; c < C; ++c) now[c] = next[c];
    if (row0 + step < a.M) request(next, row + step);
    float v[C][8], s[1] = {0.f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      now[c].values(v[c]);  // zeros past the row
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += v[c][i];
    }
    group_sum<NT>(s, buf[0]);
    const float mean = s[0] * inv;
    s[0] = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int n = a.H - 8 * (t + NT * c);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] -= mean;
      if (n < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] = i < n ? v[c][i] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += v[c][i] * v[c][i];
    }
    group_sum<NT>(s, buf[1]);
    const float rstd = 1.0f / sqrtf(s[0] * inv + a.eps);
    if (live && t == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    YT* y = (YT*)a.Y + (int64_t)row * a.ldy;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = 8 * (t + NT * c), n = a.H - col;
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = v[c][i] * rstd * w[c][i] + b[c][i];
      if (live && n > 0) store8(y + col, n, o);
    }
  }
}

// Every group requests its next row before it works on the present one, so a
// row's latency passes during the sums and stores of the row ahead of it (with
// 16 elements a thread the registers do not reach for that).
template <class XT, class YT, int NT, int C>
__global__ __launch_bounds__(kNormBlock) void k_norm_backward(const NormArgs a) {
  constexpr int GROUPS = kNormBlock / NT;
  __shared__ float buf[2][kNormBlock / 64][2];
  const int t = threadIdx.x % NT, group = threadIdx.x / NT;
  const float inv = 1.0f / (float)a.H;
  // dw and db of this thread's columns: in registers, with 16 elements a thread in LDS (its own words, no other thread's)
  constexpr bool IN_LDS = C > 1;
  static_assert(!IN_LDS || GROUPS == 1, "one row at a time");
  float dw[C][8], db[C][8];
  __shared__ f32x4 kept[IN_LDS ? 4 * C : 1][IN_LDS ? kNormBlock : 1];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[c][i] = db[c][i] = 0.f;
  if constexpr (IN_LDS)
#pragma unroll
    for (int i = 0; i < 4 * C; ++i) kept[i][threadIdx.x] = f32x4{0.f, 0.f, 0.f, 0.f};
  struct Row {
    Piece<XT> x[C];
    Piece<YT> d[C];
    float mean = 0.f, rstd = 0.f;  // (0 in threads without columns)
  };
  constexpr bool AHEAD = C == 1;
  auto request = [&](Row& r, int row) {
    const int64_t at = row < a.M ? row : a.M - 1;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = 8 * (t + NT * c), n = a.H - col;
      if (n > 0) {
        r.x[c].load((const XT*)a.X + at * a.ldx + col, n);
        r.d[c].load((const YT*)a.dY + at * a.ldd + col, n);
      }
    }
    if (!AHEAD || 8 * t < a.H) {
      r.mean = a.mean[at];
      r.rstd = a.rstd[at];
    }
  };
  auto weights = [&](int c, float (&w)[8]) {
    const int col = 8 * (t + NT * c), n = a.H - col;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.f;
    if (a.w && n > 0) load8(a.w + col, n, w);
  };
  float mine[8];  // the weights, kept where the registers reach, else read again for every row
  if constexpr (AHEAD) weights(0, mine);
  const int step = gridDim.x * GROUPS;
  Row now, next;
  if constexpr (AHEAD) request(next, blockIdx.x * GROUPS + group);
  int turn = 0;
  for (int row0 = blockIdx.x * GROUPS; row0 < a.M; row0 += step, turn ^= 1) {
    const int row = row0 + group;
    const bool live = row < a.M;
    if constexpr (AHEAD) {
      now = next;
      if (row0 + step < a.M) request(next, row + step);
    } else {
      request(now, row);
    }
    const float mean = live ? now.mean : 0.f, rstd = live ? now.rstd : 0.f;
    float xh[C][8], g[C][8], s[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float w[8];
      if constexpr (!AHEAD) weights(c, w);
      now.x[c].values(xh[c]);
      now.d[c].values(g[c]);
      // Where there is no element xhat is 0, not (0 - mean) rstd: that may be infinite, and its product with a dy of 0 a NaN.
      if (!live) {  // the last row again
#pragma unroll
        for (int i = 0; i < 8; ++i) xh[c][i] = g[c][i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) xh[c][i] = (xh[c][i] - mean) * rstd;
      const int n = a.H - 8 * (t + NT * c);
      if (n < 8 && (C > 1 || n > 0)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) xh[c][i] = i < n ? xh[c][i] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (!IN_LDS) {
          dw[c][i] += g[c][i] * xh[c][i];
          db[c][i] += g[c][i];
        }
      }
      if constexpr (IN_LDS) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f32x4 p = kept[4 * c + h][threadIdx.x], q = kept[4 * c + 2 + h][threadIdx.x];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[i] += g[c][4 * h + i] * xh[c][4 * h + i];
            q[i] += g[c][4 * h + i];
          }
          kept[4 * c + h][threadIdx.x] = p;
          kept[4 * c + 2 + h][threadIdx.x] = q;
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        g[c][i] *= AHEAD ? mine[i] : w[i];
        s[0] += g[c][i];
        s[1] += g[c][i] * xh[c][i];
      }
    }
    group_sum<NT>(s, buf[turn]);
    const float m0 = -rstd * (s[0] * inv), m1 = -rstd * (s[1] * inv);
    XT* dx = (XT*)a.Y + (int64_t)row * a.ldy;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = 8 * (t + NT * c), n = a.H - col;
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = rstd * g[c][i] + (m0 + xh[c][i] * m1);
      if (live && n > 0) store8(dx + col, n, o);
    }
  }
  if (!a.part) return;
  if constexpr (IN_LDS)
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        dw[c][i] = kept[4 * c + i / 4][threadIdx.x][i % 4];
        db[c][i] = kept[4 * c + 2 + i / 4][threadIdx.x][i % 4];
      }
  // The groups' sums of the same columns meet in LDS: eight groups a thread, then what is left.
  if constexpr (GROUPS > 1) {
    constexpr int COLS = NT * 8, LEFT = GROUPS > 8 ? GROUPS / 8 : 1, EACH = GROUPS / LEFT;
    __shared__ float sums[2][GROUPS][COLS];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sums[0][group][i * NT + t] = dw[0][i];
      sums[1][group][i * NT + t] = db[0][i];
    }
    __syncthreads();
    if constexpr (LEFT > 1) {
      const int col = threadIdx.x % COLS, first = threadIdx.x / COLS * EACH;
      float some[2] = {0.f, 0.f};
#pragma unroll
      for (int g = 0; g < EACH; ++g)
#pragma unroll
        for (int k = 0; k < 2; ++k) some[k] += sums[k][first + g][col];
      // (nobody else reads these columns of these groups)
      sums[0][first][col] = some[0];
      sums[1][first][col] = some[1];
      __syncthreads();
    }
    if (group == 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) dw[0][i] = db[0][i] = 0.f;
      constexpr int STEP = LEFT > 1 ? EACH : 1;
#pragma unroll
      for (int g = 0; g < GROUPS; g += STEP)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          dw[0][i] += sums[0][g][i * NT + t];
          db[0][i] += sums[1][g][i * NT + t];
        }
    }
  }
  constexpr int kSc1 = 16;  // device scope: stores written through, loads past this XCD's L2
  const int pitch = part_pitch(a.H);
  const auto parts = __builtin_amdgcn_make_buffer_rsrc(a.part, 0, (int)(gridDim.x * 8u * pitch), 0x00027000);
  if (group == 0) {
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = 8 * (t + NT * c), n = a.H - col;
        if (n <= 0) continue;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = which ? db[c][i] : dw[c][i];
        if (gridDim.x == 1) {
          float* to = which ? a.db : a.dw;
          if (to) store8(to + col, n, v);
        } else {
          const int at = 4 * ((blockIdx.x * 2 + which) * pitch + col);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]}), parts, at, 0, kSc1);
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{v[4], v[5], v[6], v[7]}), parts, at + 16, 0, kSc1);
        }
      }
  }
  if (!a.arrived || gridDim.x == 1) return;
  __shared__ uint32_t seen;
  wait_all_mem();
  __syncthreads();
  if (threadIdx.x == 0) seen = __hip_atomic_fetch_add(a.arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (uniform(seen) != gridDim.x - 1) return;
  if (threadIdx.x == 0) __hip_atomic_store(a.arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // as the next call expects it
  for (int col = 4 * threadIdx.x; col < 2 * pitch; col += 4 * kNormBlock) {
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int first = 0; first < (int)gridDim.x; first += 8) {
      u32x4 v[8] = {};  // in flight together
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (first + i < (int)gridDim.x) v[i] = __builtin_amdgcn_raw_buffer_load_b128(parts, 4 * ((first + i) * 2 * pitch + col), 0, kSc1);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += __builtin_bit_cast(f32x4, v[i]);
    }
    const int c = col >= pitch ? col - pitch : col;
    float* to = col >= pitch ? a.db : a.dw;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (to && c + i < a.H) to[c + i] = sum[i];
  }
}

// dw and db from the work-groups' partials: 32 columns of [parts][2 pitch] a work-group, 32 threads a column.
__global__ __launch_bounds__(1024) void k_norm_reduce(const float* part, int parts, int H, float* dw, float* db) {
  __shared__ float sums[32][33];
  const int lane = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int64_t pitch = part_pitch(H), width = 2 * pitch, col = (int64_t)blockIdx.x * 32 + lane;
  float s = 0.f;
  if (col < width) {
#pragma unroll 8
    for (int p = y; p < parts; p += 32) s += part[p * width + col];
  }
  sums[y][lane] = s;
  __syncthreads();
  if (y == 0 && col < width) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sums[i][lane];
    float* to = col < pitch ? dw : db;
    const int64_t c = col < pitch ? col : col - pitch;
    if (to && c < H) to[c] = s;
  }
}

}  // namespace mlp2

using namespace mlp2;

struct mlp2_norm_s {
  int64_t rows = 0, H = 0;
  int x = 0, y = 0, device = -1, num_cus = 0;
  float* part = nullptr;
  uint32_t* arrived = nullptr;  // work-groups of a backward pass whose part is written
  int max_parts = 0;
};

// The last work-group adds the parts of at most 32 work-groups and 128 KB: one
// CU reads these past its L2 in about 3 us, where another launch takes 3.4 us of
// the host and 4 of the GPU.  bf16, us a call one after the other, by the last
// work-group and by another kernel: 64 x 1024 (64 KB) 6.5 and 7.6, 8 x 4096 (128
// KB) 8.5 and 7.8 (10.4 where Python issues them), 256 x 1024 (256 KB) 8.2 and
// 7.6, 64 x 4096 (1 MB) 16.8 and 7.7.
constexpr int kJoinParts = 32, kJoinBytes = 128 << 10;

namespace {

// Threads of a row: the fewest of 16, 32, ... 1024 whose `each` elements cover
// it.  Forward 16 elements a thread; backward, where a thread also keeps its
// columns' dw and db and the next row, 8 as far as 1024 threads reach.
int row_threads(int64_t H, int each) {
  int nt = 16;
  while (nt < 1024 && nt * each < H) nt *= 2;
  return nt;
}
int backward_threads(int64_t H) { return row_threads(H, 8); }

// (C = 1 forward: only where a second piece would lie past every row)
template <class XT, class YT, int NT>
void launch_norm(bool forward, const NormArgs& a, int grid, hipStream_t s) {
  if (forward) {
    if (NT == 16 && a.H <= 128) k_norm_forward<XT, YT, NT, 1><<<grid, NT < 256 ? 256 : NT, 0, s>>>(a);
    else k_norm_forward<XT, YT, NT, 2><<<grid, NT < 256 ? 256 : NT, 0, s>>>(a);
  } else {
    if (NT == 1024 && a.H > 8192) k_norm_backward<XT, YT, 1024, 2><<<grid, kNormBlock, 0, s>>>(a);
    else k_norm_backward<XT, YT, NT, 1><<<grid, kNormBlock, 0, s>>>(a);
  }
}

template <class XT, class YT>
hipError_t launch_norm(bool forward, const NormArgs& a, int nt, int grid, hipStream_t s) {
  if (nt == 16) launch_norm<XT, YT, 16>(forward, a, grid, s);
  else if (nt == 32) launch_norm<XT, YT, 32>(forward, a, grid, s);
  else if (nt == 64) launch_norm<XT, YT, 64>(forward, a, grid, s);
  else if (nt == 128) launch_norm<XT, YT, 128>(forward, a, grid, s);
  else if (nt == 256) launch_norm<XT, YT, 256>(forward, a, grid, s);
  else if (nt == 512) launch_norm<XT, YT, 512>(forward, a, grid, s);
  else launch_norm<XT, YT, 1024>(forward, a, grid, s);
  return hipGetLastError();
}

hipError_t launch_norm(const mlp2_norm_s* p, bool forward, const NormArgs& a, int grid, hipStream_t s) {
  const int nt = forward ? row_threads(p->H, 16) : backward_threads(p->H);
  if (p->x == MLP2_DTYPE_BF16) return launch_norm<uint16_t, uint16_t>(forward, a, nt, grid, s);
  if (p->y == MLP2_DTYPE_BF16) return launch_norm<float, uint16_t>(forward, a, nt, grid, s);
  return launch_norm<float, float>(forward, a, nt, grid, s);
}

int64_t size_of(int dtype) { return dtype == MLP2_DTYPE_BF16 ? 2 : 4; }

Span matrix(const void* p, int64_t M, int64_t H, int64_t ld, int dtype) { return {p, H * size_of(dtype), M, ld * size_of(dtype)}; }

bool aligned(const void* p, int64_t a) { return (uintptr_t)p % (uint64_t)a == 0; }

}  // namespace

extern "C" {

mlp2_norm_t mlp2_norm_plan(int64_t max_rows, int64_t H, int x_dtype, int y_dtype) {
  clear_error();
  const bool known = (x_dtype == MLP2_DTYPE_BF16 || x_dtype == MLP2_DTYPE_F32) && (y_dtype == MLP2_DTYPE_BF16 || y_dtype == MLP2_DTYPE_F32);
  if (max_rows < 1 || H < 1 || !known) {
    record_error(MLP2_ERR_INVALID_ARG);
    return nullptr;
  }
  if (max_rows > (1 << 24) || H > kNormMaxWidth || (x_dtype == MLP2_DTYPE_BF16 && y_dtype == MLP2_DTYPE_F32)) {
    record_error(MLP2_ERR_UNSUPPORTED);
    return nullptr;
  }
  int device = -1, cus = 0;
  if (const int rc = current_device(&device, &cus)) {
    record_error(rc);
    return nullptr;
  }
  auto* p = new (std::nothrow) mlp2_norm_s();
  if (!p) {
    record_error(MLP2_ERR_HIP);
    return nullptr;
  }
  p->rows = max_rows;
  p->H = H;
  p->x = x_dtype;
  p->y = y_dtype;
  p->device = device;
  p->num_cus = cus;
  p->max_parts = cus;  // one backward work-group per CU
  const size_t bytes = (size_t)p->max_parts * 2 * part_pitch((int)H) * sizeof(float);
  if (hipMalloc((void**)&p->part, bytes + sizeof(uint32_t)) != hipSuccess ||
      hipMemset((char*)p->part + bytes, 0, sizeof(uint32_t)) != hipSuccess ||
      hipStreamSynchronize(nullptr) != hipSuccess) {  // calls may come on any stream
    (void)hipGetLastError();
    (void)hipFree(p->part);
    delete p;
    record_error(MLP2_ERR_HIP);
    return nullptr;
  }
  p->arrived = (uint32_t*)((char*)p->part + bytes);
  return p;
}

int mlp2_norm_forward(mlp2_norm_t p, int64_t M, const void* X, int64_t ldx, const float* weight, const float* bias, float eps,
                      void* Y, int64_t ldy, float* mean, float* rstd, void* stream) {
  if (!p || M < 0 || M > p->rows || !(eps >= 0.f)) return record_error(MLP2_ERR_INVALID_ARG);
  if (M == 0) return MLP2_OK;
  if (!X || !Y || ldx < p->H || ldy < p->H) return record_error(MLP2_ERR_INVALID_ARG);
  if (!aligned(X, size_of(p->x)) || !aligned(Y, size_of(p->y)) || !aligned(weight, 4) || !aligned(bias, 4) || !aligned(mean, 4) ||
      !aligned(rstd, 4))
    return record_error(MLP2_ERR_ALIGNMENT);
  const Span in[] = {matrix(X, M, p->H, ldx, p->x), {weight, p->H * 4}, {bias, p->H * 4}};
  const Span out[] = {matrix(Y, M, p->H, ldy, p->y), {mean, M * 4}, {rstd, M * 4}};
  if (outputs_overlap(in, out)) return record_error(MLP2_ERR_INVALID_ARG);
  if (!on_device(p->device)) return record_error(MLP2_ERR_DEVICE);
  NormArgs a{};
  a.X = X;
  a.Y = Y;
  a.w = weight;
  a.b = bias;
  a.mean = mean;
  a.rstd = rstd;
  a.ldx = ldx;
  a.ldy = ldy;
  a.M = (int)M;
  a.H = (int)p->H;
  a.eps = eps;
  const int nt = row_threads(p->H, 16), groups = nt < 256 ? 256 / nt : 1, block = nt < 256 ? 256 : nt;
  const int64_t blocks = (M + groups - 1) / groups, most = (int64_t)p->num_cus * (2048 / block);
  const hipError_t e = launch_norm(p, true, a, (int)(blocks < most ? blocks : most), (hipStream_t)stream);
  return e == hipSuccess ? MLP2_OK : record_error(MLP2_ERR_HIP);
}

int mlp2_norm_backward(mlp2_norm_t p, int64_t M, const void* dY, int64_t lddy, const void* X, int64_t ldx, const float* weight,
                       const float* mean, const float* rstd, void* dX, int64_t lddx, float* dweight, float* dbias, void* stream) {
  if (!p || M < 0 || M > p->rows) return record_error(MLP2_ERR_INVALID_ARG);
  if (M > 0 && (!dY || !X || !mean || !rstd || !dX || lddy < p->H || ldx < p->H || lddx < p->H)) return record_error(MLP2_ERR_INVALID_ARG);
  if (!aligned(dY, size_of(p->y)) || !aligned(X, size_of(p->x)) || !aligned(dX, size_of(p->x)) || !aligned(weight, 4) ||
      !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dweight, 4) || !aligned(dbias, 4))
    return record_error(MLP2_ERR_ALIGNMENT);
  const Span in[] = {matrix(dY, M, p->H, lddy, p->y), matrix(X, M, p->H, ldx, p->x), {weight, p->H * 4}, {mean, M * 4}, {rstd, M * 4}};
  const Span out[] = {matrix(dX, M, p->H, lddx, p->x), {dweight, p->H * 4}, {dbias, p->H * 4}};
  if (outputs_overlap(in, out)) return record_error(MLP2_ERR_INVALID_ARG);
  if (!on_device(p->device)) return record_error(MLP2_ERR_DEVICE);
  hipStream_t s = (hipStream_t)stream;
  const bool grads = dweight || dbias;
  int parts = 0;
  bool joined = false;
  if (M > 0) {
    NormArgs a{};
    a.X = X;
    a.dY = dY;
    a.Y = dX;
    a.w = weight;
    a.mean = const_cast<float*>(mean);
    a.rstd = const_cast<float*>(rstd);
    a.part = grads ? p->part : nullptr;
    a.ldx = ldx;
    a.ldd = lddy;
    a.ldy = lddx;
    a.M = (int)M;
    a.H = (int)p->H;
    const int groups = kNormBlock / backward_threads(p->H);
    const int64_t blocks = (M + groups - 1) / groups;
    parts = (int)(blocks < p->max_parts ? blocks : p->max_parts);
    joined = parts == 1 || (parts <= kJoinParts && parts * 8 * part_pitch(a.H) <= kJoinBytes);
    a.dw = dweight;
    a.db = dbias;
    a.arrived = joined ? p->arrived : nullptr;
    const hipError_t e = launch_norm(p, false, a, parts, s);
    if (e != hipSuccess) return record_error(MLP2_ERR_HIP);
  }
  if (grads && !joined) {
    k_norm_reduce<<<(unsigned)((2 * part_pitch((int)p->H) + 31) / 32), 1024, 0, s>>>(p->part, parts, (int)p->H, dweight, dbias);
    if (hipGetLastError() != hipSuccess) return record_error(MLP2_ERR_HIP);
  }
  return MLP2_OK;
}

void mlp2_norm_destroy(mlp2_norm_t p) {
  if (!p) return;
  release_on(p->device, p->part);
  delete p;
}

}  // extern "C"
