// The stream of a call and how its kernels are launched on it. Internal.
#pragma once
#include <cuda_runtime.h>

#include <atomic>

namespace ecmoe {

// SMs of a GB300, for caps on grids and for splits whose summands lie in the workspace: its size
// is asked for before any call, also where there is no device, so it cannot come from one.
constexpr int kSms = 152;

// overlap: launch each kernel with programmatic stream serialisation, so that its CTAs start
// while the kernel before it finishes (see pdl_begin in common.cuh). Converts to and from a plain
// stream (no overlap).
struct LaunchStream {
  cudaStream_t s;
  bool overlap;
  LaunchStream(cudaStream_t st, bool o = false) : s(st), overlap(o) {}
  operator cudaStream_t() const { return s; }
};

// What a launch sets or finds out once: a kernel's attributes belong to the device that is current when
// they are set, and a process may use several. `make` leaves a value other than 0; two threads may both
// come to it, with the same outcome.
class PerDevice {
 public:
  template <typename F>
  cudaError_t get(int* value, F&& make) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    std::atomic<int>* slot = dev < kDevices ? &v_[dev] : nullptr;
    *value = slot ? slot->load(std::memory_order_acquire) : 0;
    if (*value != 0) return cudaSuccess;
    e = make(value);
    if (e == cudaSuccess && slot) slot->store(*value, std::memory_order_release);
    return e;
  }

 private:
  static constexpr int kDevices = 64;   // past them every launch asks anew
  std::atomic<int> v_[kDevices] = {};
};

}  // namespace ecmoe
