// What the planners ask of the current device (host only).
#pragma once
#include <hip/hip_runtime_api.h>

#include <atomic>

namespace dlm {

// CUs of the current device, asked for once: threads that plan at the same time may both ask, and store the same number.
inline int device_cus() {
    static std::atomic<int> cus[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    int n = cus[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
        cus[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

}  // namespace dlm
