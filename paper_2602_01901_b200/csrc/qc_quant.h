// What the calls on a 4-bit cache share on the host.  Not part of the public ABI.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace qc {

// The calling thread's current device is `device` while this lives, and the one before afterwards.
class DeviceGuard {
 public:
  explicit DeviceGuard(int32_t device) {
    if (cudaGetDevice(&before_) != cudaSuccess) return;
    ok_ = before_ == device || cudaSetDevice(device) == cudaSuccess;
    changed_ = ok_ && before_ != device;
  }
  ~DeviceGuard() {
    if (changed_) cudaSetDevice(before_);
  }
  DeviceGuard(const DeviceGuard&) = delete;
  DeviceGuard& operator=(const DeviceGuard&) = delete;
  bool ok() const { return ok_; }

 private:
  int before_ = 0;
  bool ok_ = false, changed_ = false;
};

}  // namespace qc
