// Errors and the current device at the C boundary.
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "../../include/flashvla.h"

namespace fv {

struct FvError {
  fv_status st;
  std::string msg;
};

[[noreturn]] inline void fail(fv_status st, const std::string& m) { throw FvError{st, m}; }

#define FV_HIP(x)                                                                       \
  do {                                                                                  \
    hipError_t e_ = (x);                                                                \
    if (e_ != hipSuccess) fail(FV_ERR_HIP, std::string(#x) + ": " + hipGetErrorString(e_)); \
  } while (0)

// Restores the caller's current device on scope exit.
struct DeviceScope {
  int prev = -1;
  explicit DeviceScope(int dev) {
    if (hipGetDevice(&prev) != hipSuccess) prev = -1;
    if (prev != dev) FV_HIP(hipSetDevice(dev));
  }
  ~DeviceScope() {
    int cur = -1;
    if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
  }
};

inline void need(const void* p, const char* what) {
  if (!p) fail(FV_ERR_INVALID_ARG, std::string("NULL pointer: ") + what);
}

}  // namespace fv
