// Checks of arguments that the operators around the mask (head.cu, logprobs.cu) share.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>
#include <initializer_list>

#include "../../include/fmt.h"
#include "kernels.h"

namespace fmt {

inline fmt_status refuse(const char* msg) {
  set_last_error(msg);
  return FMT_ERR_INVALID_ARG;
}

inline fmt_status launch_result(cudaError_t e) {
  if (e == cudaSuccess) return FMT_OK;
  cudaGetLastError();
  set_last_error(cudaGetErrorString(e));
  return FMT_ERR_CUDA;
}

inline bool misaligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// Every pointer (NULL: not given) is memory that kernels of the current device can reach: its own, managed or page-locked.
// A pointer that is not would fault the kernel, and with it every other user of the context.
inline fmt_status reachable(std::initializer_list<const void*> ptrs) {
  int dev = -1;
  if (cudaError_t e = cudaGetDevice(&dev)) return launch_result(e);
  for (const void* p : ptrs) {
    if (!p) continue;
    cudaPointerAttributes a;
    if (cudaError_t e = cudaPointerGetAttributes(&a, p)) return launch_result(e);
    if (a.type == cudaMemoryTypeDevice ? a.device == dev : a.type == cudaMemoryTypeManaged || (a.type == cudaMemoryTypeHost && a.devicePointer == p))
      continue;
    return refuse(a.type == cudaMemoryTypeDevice ? "a pointer belongs to another device than the current one"
                                                 : "a device pointer is host memory that the device cannot reach");
  }
  return FMT_OK;
}

inline fmt_status count_sms(uint32_t* sms) {  // of the current device
  int dev = -1, n = 0;
  if (cudaError_t e = cudaGetDevice(&dev)) return launch_result(e);
  if (cudaError_t e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev)) return launch_result(e);
  *sms = (uint32_t)n;
  return FMT_OK;
}

}  // namespace fmt
