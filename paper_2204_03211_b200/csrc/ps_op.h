// Shared by the operators that work without a service (ps_clip.cu, ps_mx.cu):
// the error text of the calling thread and the device they run on.
#pragma once

#include <cuda_runtime.h>

#include "../../include/ps_b200.h"

namespace psb {

// Remembers the text of a failed CUDA call for ps_op_last_error (per host thread) and returns PS_ERR_CUDA.
int op_cuda_error(const char* what, cudaError_t e);

// What a launch needs to know of the current device; looked up once per device.
struct OpDevice {
  int id = -1;
  int num_sms = 0;
};
int op_device(OpDevice* out);

// Makes `device` current for a scope, and then what the calling thread had before: other calls launch on the current
// device, and a handle on another one may be destroyed at any time (a garbage collector's).
class DeviceScope {
 public:
  explicit DeviceScope(int device) {
    int now = -1;
    error = cudaGetDevice(&now);
    if (error != cudaSuccess || now == device) return;
    error = cudaSetDevice(device);
    if (error == cudaSuccess) before_ = now;
  }
  ~DeviceScope() {
    if (before_ >= 0) cudaSetDevice(before_);
  }
  DeviceScope(const DeviceScope&) = delete;
  DeviceScope& operator=(const DeviceScope&) = delete;
  cudaError_t error;

 private:
  int before_ = -1;
};

}  // namespace psb
