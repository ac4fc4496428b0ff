// Prints what the 4-bit products and the experts launch, without a GPU: their sources on a runtime of stubs that writes launches down.
//
//   product <CUs> <max_rows> <N> <K> <act> <y dtype> <M>
//   experts <CUs> <max_tokens> <H> <F> <E> <k> <act> <w dtype> <T>
//
// One line a command: its status; for a product the tile (0: 64, 1: 128, 2: 256) and the parts of K that were chosen; then of each launch
// the kernel's name (mangled), grid and block, and for the experts' products their blocks of columns, steps of K, most parts, and the costs
// of an item and of a part that the device compares.
#define status mx_status
#include "mlp2_mx.hip"
#undef status
#define status moe_status
#include "mlp2_moe.hip"
#undef status

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
  Experts experts{};
};
std::vector<Launch> launches;
dim3 next_grid, next_block;
int cus = 256;
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
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
  Launch l{names[f], grid, block};
  if (l.name.find("k_moe_bf16") != std::string::npos || l.name.find("k_moe_mx") != std::string::npos) l.experts = *(const Experts*)args[0];
  launches.push_back(l);
  return hipSuccess;
}
hipError_t hipGetDevice(int* d) { return *d = 0, hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600* p, int) {
  std::memset(p, 0, sizeof *p);
  std::strcpy(p->gcnArchName, "gfx950");
  p->multiProcessorCount = cus;
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
  while (std::cin >> op >> cus) {
    launches.clear();
    int rc = -1;
    char* at = kMemory + (1ull << 40);
    auto buffer = [&]() { return at += 1ull << 42; };
    if (op == "product") {
      int64_t rows, N, K, M;
      int act, dtype;
      std::cin >> rows >> N >> K >> act >> dtype >> M;
      mlp2_mx_t p = mlp2_mx_plan(rows, N, K, act, dtype);
      char *A = buffer(), *As = buffer(), *W = buffer(), *Ws = buffer(), *Y = buffer();
      if (p) rc = mlp2_mx_product(p, M, A, As, W, Ws, Y, nullptr);
      const Choice ch = p ? choose({M, N, mx_padded(K) / 4, 1, act == MLP2_ACT_SWIGLU, false}, p->split, p->num_cus) : Choice{};
      mlp2_mx_destroy(p);
      std::printf("%d %d %d", rc, ch.tile, ch.split);
    } else {
      int64_t tokens, H, F, E, k, T;
      int act, dtype;
      std::cin >> tokens >> H >> F >> E >> k >> act >> dtype >> T;
      mlp2_moe_t p = mlp2_moe_plan(tokens, H, F, E, k, act, dtype);
      char *X = buffer(), *ids = buffer(), *gates = buffer(), *W1 = buffer(), *s1 = buffer(), *W2 = buffer(), *s2 = buffer(), *Y = buffer();
      if (dtype == MLP2_DTYPE_BF16) s1 = s2 = nullptr;
      if (p) rc = mlp2_moe_experts(p, T, X, ids, gates, W1, s1, W2, s2, Y, nullptr);
      mlp2_moe_destroy(p);
      std::printf("%d", rc);
    }
    for (const Launch& l : launches) {
      std::printf(" %s %u,%u,%u %u", l.name.c_str(), l.grid.x, l.grid.y, l.grid.z, l.block.x);
      if (op == "experts") std::printf(" %d,%d,%d,%.9g,%.9g", l.experts.blocks, l.experts.steps, l.experts.most, l.experts.item, l.experts.join);
    }
    std::printf("\n");
  }
}
