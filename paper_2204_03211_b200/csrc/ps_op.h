// Shared by the operators that work without a service (ps_clip.cu, ps_mx.cu, ps_ortho.cu, ps_xent.cu):
// the error text of the calling thread, the device they run on, launches and tensor maps.
#pragma once

#include <cuda.h>
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

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
int op_encoder(EncodeTiled* out);

// A launch that may overlap its prologue with the tail of the stream's previous one (it waits for that launch to
// complete before it touches memory), optionally in clusters.
template <typename... KArgs, typename... Args>
int op_launch(const char* what, void (*kernel)(KArgs...), unsigned int grid, int block, size_t smem, int cluster,
           cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
  return e == cudaSuccess ? PS_OK : op_cuda_error(what, e);
}

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
