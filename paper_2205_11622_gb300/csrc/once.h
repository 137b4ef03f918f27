// Something that a launcher does once a device.  Host code; also compiled without
// nvcc.
#pragma once

#include <atomic>
#include <cuda_runtime.h>

namespace slnr {

// Runs something until it has succeeded once on a device: the attributes of a
// kernel.  What failed is run again by the next call: a kernel that could not be
// loaded for want of memory can be later.
class OncePerDevice {
 public:
  template <typename F>
  cudaError_t operator()(F f) {
    int d = 0;
    const cudaError_t e = cudaGetDevice(&d);
    if (e != cudaSuccess) return e;
    if (d < 0 || d >= kDevices) return f();
    if (done_[d].load(std::memory_order_acquire)) return cudaSuccess;
    const cudaError_t r = f();  // by two threads at once: the same attributes twice
    if (r == cudaSuccess) done_[d].store(true, std::memory_order_release);
    return r;
  }

 private:
  static constexpr int kDevices = 64;
  std::atomic<bool> done_[kDevices] = {};
};

}  // namespace slnr
