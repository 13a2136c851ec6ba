// What the C entries of the operators share.
#pragma once

#include <hip/hip_runtime.h>

#include <exception>
#include <string>

#include "recycle_stage.h"

rc_status rc_set_error(rc_status s, const std::string& msg);

namespace {

rc_status fail(rc_status s, const std::string& msg) { return rc_set_error(s, msg); }

// No exception leaves a C entry.
template <class F>
rc_status guarded(F f) {
  try {
    return f();
  } catch (const std::exception& e) {
    return fail(RC_ERR_HIP, std::string("host: ") + e.what());
  }
}

// The stream's device as the current one, while in scope (kernels start on the current one).
struct OnDevice {
  int back = -1;
  hipError_t err = hipSuccess;
  explicit OnDevice(hipStream_t s) {
    if (!s) return;
    int cur = 0;
    err = hipGetDevice(&cur);
    const int dev = hipGetStreamDeviceId(s);
    if (err != hipSuccess || dev < 0 || dev == cur) return;
    err = hipSetDevice(dev);
    if (err == hipSuccess) back = cur;
  }
  ~OnDevice() {
    if (back >= 0) (void)hipSetDevice(back);
  }
};

rc_status hip_result(hipError_t e, const char* what) {
  if (e == hipSuccess) return RC_OK;
  return fail(RC_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

int elt_of(int dtype) { return dtype == RC_BF16 ? 2 : 4; }

#define TRY(expr)                  \
  do {                             \
    const rc_status r_ = (expr);   \
    if (r_ != RC_OK) return r_;    \
  } while (0)

}  // namespace
