// Prints what the training operators launch, without a GPU: their sources on a runtime of stubs that writes launches down.
//
//   train <max_rows> <H> <F> <act> <M> <gradients: any of X 1 2, - for the forward pass>
//   norm <max_rows> <H> <x dtype> <y dtype> <M> <f or b>
//   ortho <count> <rows> <cols> <dtype> <steps>
//
// One line a command: its status, then kernel name (mangled), grid and block of each launch.
#include "mlp2_train.hip"
#include "mlp2_norm.hip"
#include "mlp2_ortho.hip"

#include <cstdio>
#include <iostream>
#include <map>
#include <string>
#include <vector>

namespace {
std::map<const void*, std::string> names;
struct Launch {
  std::string name;
  dim3 grid, block;
};
std::vector<Launch> launches;
dim3 next_grid, next_block;
char* const kMemory = (char*)(1ull << 40);  // addresses that nothing reads
}  // namespace

namespace mlp2 {
int record_error(int code) { return code; }
}  // namespace mlp2

extern "C" {
const char __hip_fatbin[64] = {};
void** __hipRegisterFatBinary(const void*) { return nullptr; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, uint3*, uint3*, dim3*, dim3*, int*) { names[host] = name; }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  next_grid = grid;
  next_block = block;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* s) {
  *grid = next_grid;
  *block = next_block;
  *lds = 0;
  *s = nullptr;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
  launches.push_back({names[f], grid, block});
  return hipSuccess;
}
hipError_t hipGetDevice(int* d) { return *d = 0, hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600* p, int) {
  std::memset(p, 0, sizeof *p);
  std::strcpy(p->gcnArchName, "gfx950");
  p->multiProcessorCount = 256;
  return hipSuccess;
}
hipError_t hipMalloc(void** p, size_t) { return *p = kMemory, hipSuccess; }
hipError_t hipFree(void*) { return hipSuccess; }
hipError_t hipMemset(void*, int, size_t) { return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
}

int main() {
  std::string op;
  while (std::cin >> op) {
    launches.clear();
    int rc = -1;
    char* at = kMemory + (1ull << 40);
    auto buffer = [&]() { return at += 1ull << 42; };
    if (op == "train") {
      int64_t rows, H, F, M;
      int act;
      std::string grads;
      std::cin >> rows >> H >> F >> act >> M >> grads;
      mlp2_train_t p = mlp2_train_plan(rows, H, F, act, MLP2_DTYPE_BF16);
      char *X = buffer(), *W1 = buffer(), *W2 = buffer(), *P = buffer(), *Y = buffer(), *dX = buffer(), *d1 = buffer(), *d2 = buffer();
      auto asked = [&](char c, char* to) { return grads.find(c) != std::string::npos ? to : nullptr; };
      if (p) rc = grads == "-" ? mlp2_train_forward(p, M, X, W1, W2, P, Y, nullptr)
                               : mlp2_train_backward(p, M, Y, X, W1, W2, P, asked('X', dX), asked('1', d1), asked('2', d2), nullptr);
      mlp2_train_destroy(p);
    } else if (op == "norm") {
      int64_t rows, H, M;
      int x, y;
      std::string dir;
      std::cin >> rows >> H >> x >> y >> M >> dir;
      mlp2_norm_t p = mlp2_norm_plan(rows, H, x, y);
      char *X = buffer(), *Y = buffer(), *dX = buffer();
      float *w = (float*)buffer(), *b = (float*)buffer(), *mean = (float*)buffer(), *rstd = (float*)buffer();
      if (p) rc = dir == "f" ? mlp2_norm_forward(p, M, X, H, w, b, 1e-5f, Y, H, mean, rstd, nullptr)
                             : mlp2_norm_backward(p, M, Y, H, X, H, nullptr, mean, rstd, dX, H, w, b, nullptr);
      mlp2_norm_destroy(p);
    } else {
      int64_t count, rows, cols;
      int dtype, steps;
      std::cin >> count >> rows >> cols >> dtype >> steps;
      mlp2_ortho_t p = mlp2_ortho_plan(count, rows, cols, dtype);
      const std::vector<float> coeffs(3 * steps, 1.f);
      if (p) rc = mlp2_ortho_run(p, buffer(), buffer(), steps, coeffs.data(), 1e-7f, nullptr);
      mlp2_ortho_destroy(p);
    }
    std::printf("%d", rc);
    for (const Launch& l : launches)
      std::printf(" %s %u,%u,%u %u", l.name.c_str(), l.grid.x, l.grid.y, l.grid.z, l.block.x);
    std::printf("\n");
  }
}
