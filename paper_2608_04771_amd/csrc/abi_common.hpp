// What the C entry points share.  Not part of the public ABI.
#pragma once

#include "reco.h"

#include <hip/hip_runtime.h>

#include <atomic>

namespace reco {

inline reco_status_t hip_status(hipError_t e) { return e == hipSuccess ? RECO_OK : RECO_ERR_HIP; }

// Compute units of the current device, read once per device (256 on a whole
// MI355X; a partitioned GPU shows fewer).  Falls back to 256 if the query
// fails, which only changes the split count, never correctness.
inline int current_compute_units() {
  constexpr int kMaxDevices = 64;
  static std::atomic<int> cached[kMaxDevices];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return 256;
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n > 0) return n;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) n = 256;
  cached[dev].store(n, std::memory_order_relaxed);
  return n;
}

}  // namespace reco
