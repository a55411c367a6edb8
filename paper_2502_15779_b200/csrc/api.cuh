// What the library's entry points share: the last CUDA error, launches, sizes of the device.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>
#include <mutex>
#include <utility>

#include "../../include/rcp.h"

namespace rcp {

inline thread_local int g_last_cuda_error = 0;

namespace api {

constexpr int kMaxDevices = 64;

inline int cuda_fail(cudaError_t e) {
  g_last_cuda_error = (int)e;
  return RCP_ERR_CUDA;
}

#define RCP_CUDA(call)                            \
  do {                                            \
    cudaError_t e__ = (call);                     \
    if (e__ != cudaSuccess) return ::rcp::api::cuda_fail(e__); \
  } while (0)

// Launches with programmatic stream serialization: the kernel may start while the preceding
// kernel on the stream is still running and must execute griddepcontrol.wait before it touches
// anything that kernel may read or write.
template <typename... KArgs, typename... Args>
cudaError_t launch_overlapped(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st,
                              Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, std::forward<Args>(args)...);
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// SMs of the current device (remembered per device; 148 if the query fails)
inline int sm_count() {
  static std::mutex mu;
  static int n[kMaxDevices] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 148;
  std::lock_guard<std::mutex> lock(mu);
  if (!n[dev] && cudaDeviceGetAttribute(&n[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) n[dev] = 148;
  return n[dev];
}

// cudaFuncAttributeMaxDynamicSharedMemorySize belongs to the (kernel, device) pair: set once per device (mu and done
// belong to the kernel)
template <typename Kern>
cudaError_t set_max_smem(Kern kern, int bytes, std::mutex& mu, bool (&done)[kMaxDevices]) {
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (!done[dev]) {
    const cudaError_t r = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (r != cudaSuccess) return r;
    done[dev] = true;
  }
  return cudaSuccess;
}

}  // namespace api
}  // namespace rcp
