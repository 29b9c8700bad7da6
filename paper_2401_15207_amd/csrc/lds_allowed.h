// LDS beyond 64 KB has to be allowed for a kernel, once on each device that runs it: one of these a kernel, static where it is launched.  Threads may
// launch at the same time; two that come first both ask, which is harmless.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include <atomic>

namespace hift {

class LdsAllowed {
  std::atomic<uint64_t> devices_{0};  // those of the first 64 where it was asked for

 public:
  hipError_t operator()(const void* kernel, int bytes) {
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
    if (devices_.load(std::memory_order_acquire) & bit) return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) devices_.fetch_or(bit, std::memory_order_release);
    return e;
  }
};

}  // namespace hift
