// Host threads that launch the token statistics at once, over stand-ins for the CUDA runtime that keep no state: built
// with ThreadSanitizer, so that whatever the launches share without order is reported.
#include <cuda_runtime.h>

#include <atomic>
#include <thread>
#include <vector>

#include "../paper_2309_00754_gb300/csrc/kernels.h"

namespace hydra {
int sm_count() { return 152; }
}  // namespace hydra

static thread_local int t_device;
static std::atomic<int> g_launches;

extern "C" {
cudaError_t cudaGetDevice(int* d) { return *d = t_device, cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveClusters(int* n, const void*, const cudaLaunchConfig_t*) { return *n = 36, cudaSuccess; }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void*, void**) { return ++g_launches, cudaSuccess; }
cudaError_t __cudaLaunchKernel(cudaKernel_t, dim3, dim3, void**, size_t, cudaStream_t) { return ++g_launches, cudaSuccess; }
cudaError_t __cudaGetKernel(cudaKernel_t*, const void*) { return cudaSuccess; }
char __cudaInitModule(void**) { return 0; }
void** __cudaRegisterFatBinary(void*) { static void* handle; return &handle; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
void __cudaRegisterVar(void**, char*, char*, const char*, int, size_t, int, int) {}
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, void*) { return 0; }
cudaError_t __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaSuccess; }
}

int main() {
  std::vector<std::thread> threads;
  for (int i = 0; i < 4; ++i)
    threads.emplace_back([i] {
      t_device = i / 2;
      for (int n = 0; n < 16; ++n) {
        hydra::TokenStatsArgs a = {};
        a.bf16 = n & 1;
        a.top_k = n & 2 ? 5 : 0;
        a.S = n & 4 ? 1000 : 3;  // rows by single CTAs, by clusters
        a.L = 1;
        a.V = a.ld = n & 8 ? 128000 : 32000;
        if (hydra::launch_token_stats(a, nullptr) != 0) g_launches = -1000;
      }
    });
  for (auto& t : threads) t.join();
  return g_launches == 64 ? 0 : 1;
}
