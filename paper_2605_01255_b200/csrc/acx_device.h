// What the library keeps per device: found by the device that is current.
#pragma once
#include <cuda_runtime.h>
#include <atomic>

namespace acx {

// One-time set-up that holds per device (a kernel's function attributes are set for the device that is current):
// `static DeviceOnce once; if (once.needed()) { ...; once.done(); }`.  Safe to race: the set-up is idempotent.
class DeviceOnce {
  std::atomic<unsigned long long> mask_{0};
  static unsigned long long bit() {
    int dev = 0;
    cudaGetDevice(&dev);
    return 1ull << (unsigned(dev) & 63u);
  }

 public:
  bool needed() const { return (mask_.load(std::memory_order_acquire) & bit()) == 0; }
  void done() { mask_.fetch_or(bit(), std::memory_order_release); }
};

// COUNT numbers per device, each 0 until it is set.  The current device's, or nullptr where there is none to be had (the
// number is then asked for again every time).
template <int COUNT>
class DeviceNumbers {
  static constexpr int kDevices = 64;
  std::atomic<int> n_[kDevices][COUNT] = {};

 public:
  std::atomic<int>* here() {
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && dev >= 0 && dev < kDevices ? n_[dev] : nullptr;
  }
};

}  // namespace acx
