// What the C entry points of the training operators share on the host.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstring>

#include "../../include/mlp2.h"

namespace mlp2 {

int record_error(int code);   // sets mlp2_last_error() and returns the code (mlp2_api.cpp)
inline void clear_error() { (void)record_error(MLP2_OK); }

// The current device, if it is one the kernels are built for: MLP2_OK, MLP2_ERR_DEVICE or MLP2_ERR_HIP.
inline int current_device(int* device, int* num_cus) {
  hipDeviceProp_t prop;
  if (hipGetDevice(device) != hipSuccess) return MLP2_ERR_DEVICE;
  if (hipGetDeviceProperties(&prop, *device) != hipSuccess) return MLP2_ERR_HIP;
  if (std::strncmp(prop.gcnArchName, "gfx950", 6) != 0) return MLP2_ERR_DEVICE;
  *num_cus = prop.multiProcessorCount;
  return MLP2_OK;
}

inline bool on_device(int device) {
  int dev = -1;
  return hipGetDevice(&dev) == hipSuccess && dev == device;
}

// An operand's bytes: `rows` rows of `width` at a distance of `pitch`; one row is a plain range.
struct Span {
  const void* p;
  int64_t width;
  int64_t rows = 1, pitch = 0;
  int64_t bytes() const { return rows > 0 && width > 0 ? (rows - 1) * pitch + width : 0; }
};

// Whether two operands share a byte.  Rows of the same pitch may lie beside each other (columns of one buffer, rows in turn);
// of other shapes the whole ranges are compared, gaps between rows included.
inline bool overlap(const Span& a, const Span& b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  if (!a.p || !b.p || !a.bytes() || !b.bytes() || x >= y + (uint64_t)b.bytes() || y >= x + (uint64_t)a.bytes()) return false;
  if (a.rows == 1 || b.rows == 1 || a.pitch != b.pitch) return true;
  if (x > y) return overlap(b, a);
  // Row j of b starts `in` bytes into the pitch of row j + k of a.
  const int64_t k = (int64_t)((y - x) / (uint64_t)a.pitch), in = (int64_t)((y - x) % (uint64_t)a.pitch);
  return (in < a.width && k < a.rows) || (in + b.width > a.pitch && k + 1 < a.rows);
}

// Whether any of the outputs overlaps an input or another output.
template <int NI, int NO>
inline bool outputs_overlap(const Span (&in)[NI], const Span (&out)[NO]) {
  for (int o = 0; o < NO; ++o) {
    for (int i = 0; i < NI; ++i)
      if (overlap(out[o], in[i])) return true;
    for (int q = 0; q < o; ++q)
      if (overlap(out[o], out[q])) return true;
  }
  return false;
}

// Frees a plan's workspace once its device is idle: a plan does not record the streams it ran on.
inline void release_on(int device, void* ws) {
  int cur = -1;
  (void)hipGetDevice(&cur);
  if (cur != device) (void)hipSetDevice(device);
  (void)hipDeviceSynchronize();
  (void)hipFree(ws);
  if (cur != device && cur >= 0) (void)hipSetDevice(cur);
}

inline int64_t round_up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }

}  // namespace mlp2
