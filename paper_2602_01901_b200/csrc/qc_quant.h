// What the calls on a 4-bit cache share on the host.  Not part of the public ABI.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/qc.h"

namespace qc {

// The status of a CUDA call.  What failed is told here and not again by whatever asks CUDA for its last error next.
inline int32_t status_of(cudaError_t e) {
  if (e == cudaSuccess) return QC_OK;
  cudaGetLastError();
  return QC_ERR_CUDA;
}

// The calling thread's current device is `device` while this lives, and the one before afterwards.
class DeviceGuard {
 public:
  explicit DeviceGuard(int32_t device) {
    if (status_of(cudaGetDevice(&before_)) != QC_OK) return;
    ok_ = before_ == device || status_of(cudaSetDevice(device)) == QC_OK;
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
