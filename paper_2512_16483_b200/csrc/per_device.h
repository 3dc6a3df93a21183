// What a kernel's host side finds out or sets once for each device.  Calls come without the interpreter lock, from any thread.
#pragma once
#include <cuda_runtime.h>

#include <mutex>

namespace fvar {

constexpr int kMaxDevices = 64;                // devices that are remembered; others are set up for every call

class PerDevice {
 public:
  // Runs f, which returns a cudaError_t, unless it has succeeded for this device before.  Who comes meanwhile waits, and what f has
  // stored is visible to every caller that gets cudaSuccess.
  template <typename F>
  cudaError_t once(int dev, F f) {
    std::lock_guard<std::mutex> lock(mu_);
    if (dev < kMaxDevices && (done_ >> dev & 1)) return cudaSuccess;
    const cudaError_t e = f();
    if (e == cudaSuccess && dev < kMaxDevices) done_ |= 1ull << dev;
    return e;
  }

 private:
  std::mutex mu_;
  unsigned long long done_ = 0;                // a bit a device
};

}  // namespace fvar
