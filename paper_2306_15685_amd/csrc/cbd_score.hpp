// What the code on either side of the score rows shares: element types.
#ifndef CBD_SCORE_HPP_
#define CBD_SCORE_HPP_

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <cstdint>

namespace cbd {

typedef _Float16 f16;
typedef __bf16 bf16;

inline size_t dtype_size(int32_t dtype) { return dtype == 0 ? 4 : 2; }

// Makes `device` current for the scope and the caller's device afterwards.
struct DeviceScope {
  int before = -1;
  hipError_t error = hipSuccess;
  explicit DeviceScope(int device) {
    int now = -1;
    error = hipGetDevice(&now);
    if (error == hipSuccess && now != device) {
      error = hipSetDevice(device);
      if (error == hipSuccess) before = now;
    }
  }
  ~DeviceScope() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

// Is the stream one of `device`?  (The null stream is every device's.)
inline bool stream_is_of(hipStream_t stream, int device) {
  hipDevice_t d = -1;
  return !stream || (hipStreamGetDevice(stream, &d) == hipSuccess && (int)d == device);
}

inline bool is_capturing(hipStream_t stream) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  return stream && hipStreamIsCapturing(stream, &st) == hipSuccess && st != hipStreamCaptureStatusNone;
}

}  // namespace cbd

#endif  // CBD_SCORE_HPP_
