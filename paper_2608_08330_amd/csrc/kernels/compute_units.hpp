// Compute units of the current HIP device, asked once per device.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>

namespace rtcc {
namespace kern {
namespace {

inline int compute_units() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    n = known[dev].load(std::memory_order_relaxed);
    if (n > 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    known[dev].store(n, std::memory_order_relaxed);
    return n;
}

}  // namespace
}  // namespace kern
}  // namespace rtcc
