// What the host sources of the operators of language models share.
#pragma once
#include <hip/hip_runtime.h>

namespace st {

// Makes a plan's device the current one for a call, and puts back the caller's.
struct OnDevice {
  hipError_t error = hipSuccess;
  int before = -1;
  explicit OnDevice(int device) {
    int now = -1;
    error = hipGetDevice(&now);
    if (error == hipSuccess && now != device) {
      error = hipSetDevice(device);
      if (error == hipSuccess) before = now;
    }
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;
};

}  // namespace st
