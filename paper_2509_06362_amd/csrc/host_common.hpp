// What the host sides of the library's two parts share.
#pragma once

#include <hip/hip_runtime.h>

namespace maaso {

// The device a call works on, for as long as the guard lives.
struct DeviceGuard {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuard(int dev) {
    if (hipGetDevice(&prev) != hipSuccess) { ok = false; (void)hipGetLastError(); return; }
    if (prev != dev && hipSetDevice(dev) != hipSuccess) { ok = false; (void)hipGetLastError(); }
  }
  ~DeviceGuard() {
    int cur = -1;
    if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
  }
};

inline bool hip_ok(hipError_t e) {
  if (e == hipSuccess) return true;
  (void)hipGetLastError();
  return false;
}

inline bool is_captured(hipStream_t s) {
  if (s == nullptr) return false;  // (the null stream cannot be)
  hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
  return hip_ok(hipStreamIsCapturing(s, &status)) && status != hipStreamCaptureStatusNone;
}

}  // namespace maaso
