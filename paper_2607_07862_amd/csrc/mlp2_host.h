// What the C entry points of the training operators share on the host.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstring>

#include "../../include/mlp2.h"

namespace mlp2 {

int record_error(int code);   // sets mlp2_last_error() and returns the code (mlp2_api.cpp)
void clear_error();

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

struct Span {
  const void* p;
  int64_t bytes;
};

inline bool overlap(const Span& a, const Span& b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  return a.p && b.p && a.bytes > 0 && b.bytes > 0 && x < y + (uint64_t)b.bytes && y < x + (uint64_t)a.bytes;
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
