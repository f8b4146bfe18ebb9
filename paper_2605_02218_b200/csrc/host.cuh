// What the host parts of the library share: the text of the last CUDA error and the launches with attributes.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <string>

#include "covspec.h"

namespace covspec {

inline thread_local std::string g_cuda_error;

#define CUDA_TRY(expr)                                                                  \
  do {                                                                                  \
    cudaError_t e_ = (expr);                                                            \
    if (e_ != cudaSuccess) {                                                            \
      ::covspec::g_cuda_error = std::string(#expr) + ": " + cudaGetErrorString(e_);     \
      return COVSPEC_ERR_CUDA;                                                          \
    }                                                                                   \
  } while (0)

// A step that may have said itself, in g_cuda_error, what failed; else the text is made of its status.
template <typename F>
int status_of(const char* what, F step) {
  std::string before;
  before.swap(g_cuda_error);
  const cudaError_t e = step();
  if (e == cudaSuccess) {
    g_cuda_error.swap(before);
    return COVSPEC_OK;
  }
  if (g_cuda_error.empty()) g_cuda_error = std::string(what) + ": " + cudaGetErrorString(e);
  return COVSPEC_ERR_CUDA;
}

// Launch that may overlap the end of the kernel before it on the stream; the kernel calls
// wait_for_previous_kernel (common.cuh) before it uses anything of that kernel's.  About 2 us less between two
// short kernels.  cluster > 1: CTAs per cluster (kernels without a size of their own).
template <typename... P, typename... A>
cudaError_t launch_clusters(int cluster, bool dependent, void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s,
                            A... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2]{};
  cfg.attrs = attr;
  if (dependent) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = (unsigned)cluster;
    attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
    ++cfg.numAttrs;
  }
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
template <typename... P, typename... A>
cudaError_t launch_dependent(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, A... args) {
  return launch_clusters(1, true, kernel, grid, threads, smem, s, args...);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                  const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_tiled_fn() {
  static EncodeTiledFn fn = [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      ptr = nullptr;
    return reinterpret_cast<EncodeTiledFn>(ptr);
  }();
  return fn;
}

// Once for each device: the kernel's limit of dynamic shared memory.
template <auto Kernel>
cudaError_t allow_shared(int bytes) {
  static std::atomic<unsigned long long> configured{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !(configured.load(std::memory_order_acquire) >> dev & 1ull)) {
    e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    if (dev < 64) configured.fetch_or(1ull << dev, std::memory_order_release);
  }
  return cudaSuccess;
}

}  // namespace covspec
