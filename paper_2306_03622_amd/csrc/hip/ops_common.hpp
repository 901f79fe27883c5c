// What the operators' C entry points share: the device of the stream, statuses, scratch, limits.
#pragma once
#include <hip/hip_runtime_api.h>

#include <string>

#include "../core/errors.hpp"
#include "../kernels/kernels.hpp"

namespace tp {

// Makes the stream's device current for a call, and the caller's again behind it.
class OnDeviceOf {
 public:
  explicit OnDeviceOf(hipStream_t s) {
    if (!s) return;
    int dev = 0;
    if ((error = hipGetDevice(&back_)) != hipSuccess || (error = hipStreamGetDevice(s, &dev)) != hipSuccess) return;
    if (dev == back_) return;
    error = hipSetDevice(dev);
    moved_ = error == hipSuccess;
  }
  ~OnDeviceOf() {
    if (moved_) (void)hipSetDevice(back_);
  }
  OnDeviceOf(const OnDeviceOf&) = delete;
  OnDeviceOf& operator=(const OnDeviceOf&) = delete;
  hipError_t error = hipSuccess;

 private:
  int back_ = 0;
  bool moved_ = false;
};

inline tp_status inval(const char* who, const char* what) { return fail(TP_E_INVAL, std::string(who) + ": " + what); }

inline tp_status done(const char* who, hipError_t e) {
  if (e == hipSuccess) return ok();
  return fail(e == hipErrorInvalidValue ? TP_E_INVAL : TP_E_HIP, std::string(who) + ": " + hipGetErrorString(e));
}

inline k::Split scratch(void* work, uint64_t bytes) {
  k::Split sp;
  sp.partials = static_cast<float*>(work);
  sp.partial_bytes = work ? bytes : 0;
  return sp;
}

// Lengths and positions stay below this, so that sums of two of them fit 32 bits.
constexpr int32_t kMostTokens = (1 << 30) - 1;
constexpr int64_t kMostStride = 1ll << 40;

}  // namespace tp
