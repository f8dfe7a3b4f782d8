// Launches with more LDS than 64 KB (host side).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

namespace per {

// Lets a kernel take `lds` bytes: asked for once per kernel and device.
inline hipError_t grant_lds(const void* kernel, std::atomic<uint64_t>* granted, uint32_t lds) {
  if (lds <= 64 * 1024) return hipSuccess;
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  const uint64_t bit = device < 64 ? 1ull << device : 0;
  if (granted->load(std::memory_order_relaxed) & bit) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e == hipSuccess) granted->fetch_or(bit, std::memory_order_relaxed);
  return e;
}

}  // namespace per
