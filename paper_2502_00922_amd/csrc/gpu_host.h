// Host-side helpers shared by the launchers of the gfx950 kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>

#include "hufflm.h"

namespace hl {

constexpr int kMaxDevices = 64;

// The current GPU's compute units; asked of the runtime once per GPU (a
// launch's plan needs them several times).
inline int device_cus() {
  static std::atomic<int> known[kMaxDevices];
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 256;
  const bool keep = dev >= 0 && dev < kMaxDevices;
  if (keep && (cus = known[dev].load(std::memory_order_relaxed)) > 0) return cus;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    return 256;
  if (keep) known[dev].store(cus, std::memory_order_relaxed);
  return cus;
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Whether a launch of this many blocks along x can be: its threads along x must
// be fewer than 2^32.
inline bool grid_fits(uint64_t blocks, uint64_t threads) { return blocks < (1ull << 32) / threads; }

// Enqueues a kernel that uses only static LDS.
template <class K, class... A>
hl_status enqueue(K kernel, dim3 grid, dim3 block, hipStream_t s, A... args) {
  hipLaunchKernelGGL(kernel, grid, block, 0, s, args...);
  return hipGetLastError() == hipSuccess ? HL_OK : HL_EHIP;
}

}  // namespace hl
