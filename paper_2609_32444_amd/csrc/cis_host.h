// What the host side of the entry points shares: the current device, launches, and checks of
// arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include <mutex>

#include "../../include/cis.h"

namespace cis::host {

constexpr int kMaxDevices = 64;

// Compute units of the current device, or CIS_ERR_DEVICE.
inline int device_cus() {
  static std::mutex mu;
  static int cus[kMaxDevices] = {};   // 0: not looked at yet
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return CIS_ERR_DEVICE;
  std::lock_guard<std::mutex> lk(mu);
  if (cus[dev] == 0) {
    hipDeviceProp_t prop;
    if (hipGetDeviceProperties(&prop, dev) != hipSuccess) return CIS_ERR_DEVICE;
    cus[dev] = strncmp(prop.gcnArchName, "gfx950", 6) == 0 ? prop.multiProcessorCount
                                                           : CIS_ERR_DEVICE;
  }
  return cus[dev];
}

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline bool known(int dtype) { return dtype == CIS_BF16 || dtype == CIS_F32; }
inline int elem_bytes(int dtype) { return dtype == CIS_BF16 ? 2 : 4; }

inline int launch(const void* fn, int64_t grid, int block, void* arg, hipStream_t stream) {
  void* args[] = {arg};
  return hipLaunchKernel(fn, dim3((unsigned)grid), dim3(block), args, 0, stream) == hipSuccess
             ? CIS_OK
             : CIS_ERR_LAUNCH;
}

inline int check_workspace(const void* workspace, size_t have, size_t need) {
  if (!aligned(workspace, 256)) return CIS_ERR_ALIGN;
  return have < need ? CIS_ERR_WORKSPACE : CIS_OK;
}


}  // namespace cis::host
