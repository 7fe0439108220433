// Host side: kernels that need more than 64 KiB of LDS.
#pragma once
#include <hip/hip_runtime.h>
#include <mutex>

namespace gecc {
namespace {

// the LDS limit of a kernel, raised once per device, whichever host thread comes first
struct LdsLimit {
  static constexpr int MAX_DEVICES = 64;
  std::mutex mu;
  bool done[MAX_DEVICES] = {};
  hipError_t raise(const void* kernel, int bytes) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) return hipErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(mu);
    if (done[dev]) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    done[dev] = e == hipSuccess;
    return e;
  }
};

}  // namespace
}  // namespace gecc
