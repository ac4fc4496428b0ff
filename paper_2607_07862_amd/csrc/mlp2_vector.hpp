// 8-element accesses to rows that may start at any element.
#pragma once

#include "mlp2_device.hpp"

namespace mlp2 {

// 16-byte accesses with the alignment of one element (global memory takes them at any element's address).
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ void unpack_bf16x8(u32x4 q, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __builtin_bit_cast(float, q[i] << 16);
    v[2 * i + 1] = __builtin_bit_cast(float, q[i] & 0xFFFF0000u);
  }
}

// 8 elements from p, of which the first n exist (the others are 0); bf16 or fp32.
__device__ __forceinline__ void load8(const uint16_t* p, int n, float (&v)[8]) {
  if (n >= 8) {
    unpack_bf16x8(*reinterpret_cast<const u32x4_any*>(p), v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? __builtin_bit_cast(float, (uint32_t)p[i] << 16) : 0.f;
  }
}
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
  if (n >= 8) {
    const f32x4 a = *reinterpret_cast<const f32x4_any*>(p), b = *reinterpret_cast<const f32x4_any*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = a[i];
      v[4 + i] = b[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
  }
}

// The same 8 elements as they are stored, for loads that run ahead of their use; zeros until the first load.
template <class T>
struct Piece;
template <>
struct Piece<uint16_t> {
  u32x4 q = {0, 0, 0, 0};
  __device__ __forceinline__ void load(const uint16_t* p, int n) {
    if (n >= 8) {
      q = *reinterpret_cast<const u32x4_any*>(p);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = (2 * i < n ? (uint32_t)p[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)p[2 * i + 1] << 16 : 0u);
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const { unpack_bf16x8(q, v); }
};
template <>
struct Piece<float> {
  float f[8] = {};
  __device__ __forceinline__ void load(const float* p, int n) { load8(p, n, f); }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = f[i];
  }
};

// The first n of 8 packed 16-bit values (or fp32 values) to p.
__device__ __forceinline__ void store8_packed(uint16_t* p, int n, u32x4 q) {
  if (n >= 8) {
    *reinterpret_cast<u32x4_any*>(p) = q;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (uint16_t)(q[i / 2] >> (16 * (i & 1)));
  }
}
__device__ __forceinline__ void store8(uint16_t* p, int n, const float (&v)[8]) { store8_packed(p, n, pack_bf16x8(v)); }
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    *reinterpret_cast<f32x4_any*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_any*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = v[i];
  }
}

}  // namespace mlp2
