// The calling thread's current device inside an entry point.
#pragma once
#include <cuda_runtime_api.h>

namespace muloco {

// Makes `device` the calling thread's current device until the end of the scope.  Launches, allocations, copies and
// events of a context belong on its device whatever device the caller has current: with contexts on two devices, both on
// their default stream, the stream's handle is 0 for either, so a launch would go to the wrong one without complaint.
class DeviceScope {
 public:
  explicit DeviceScope(int device) {
    error_ = cudaGetDevice(&before_);
    if (error_ != cudaSuccess || before_ == device) return;
    error_ = cudaSetDevice(device);
    changed_ = error_ == cudaSuccess;
  }
  ~DeviceScope() {
    if (changed_) cudaSetDevice(before_);
  }
  DeviceScope(const DeviceScope&) = delete;
  DeviceScope& operator=(const DeviceScope&) = delete;
  cudaError_t error() const { return error_; }

 private:
  int before_ = 0;
  bool changed_ = false;
  cudaError_t error_ = cudaSuccess;
};

}  // namespace muloco
