// Host helper of kernels that want more LDS than a launch has by default.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

namespace slp {
namespace {

// Lets a kernel have that much LDS, once on each device (bit of `done`); host threads that launch first together both do.
inline hipError_t allow_lds(const void* kernel, int bytes, std::atomic<uint64_t>& done) {
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  const uint64_t bit = (uint64_t)1 << (device & 63);
  if (device < 64 && (done.load(std::memory_order_acquire) & bit)) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess && device < 64) done.fetch_or(bit, std::memory_order_release);
  return e;
}

}  // namespace
}  // namespace slp
