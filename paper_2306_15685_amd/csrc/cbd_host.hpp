// Host helpers shared by the library's translation units: error text, device memory, pinned upload slots.
#ifndef CBD_HOST_HPP_
#define CBD_HOST_HPP_

#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "../../include/cbd.h"

#define HIPCHK(expr)                                                                              \
  do {                                                                                            \
    hipError_t e_ = (expr);                                                                       \
    if (e_ != hipSuccess)                                                                         \
      return fail(CBD_E_HIP, std::string(#expr) + ": " + hipGetErrorString(e_));                  \
  } while (0)

namespace cbd {

// Notes the text cbd_last_error() returns on this thread; returns `code`.
__attribute__((visibility("hidden"))) int32_t fail(int32_t code, const std::string &msg);

template <typename T> hipError_t dmalloc(T **p, size_t n, size_t *total) {
  size_t bytes = std::max<size_t>(n, 1) * sizeof(T);
  hipError_t e = hipMalloc((void **)p, bytes);
  if (e == hipSuccess && total) *total += bytes;
  return e;
}

// A small ring of pinned host buffers with matching device buffers, so that
// argument lists can be uploaded asynchronously without racing their reuse.
struct StageRing {
  static constexpr int kSlots = 8;
  void *host[kSlots] = {};
  void *dev[kSlots] = {};
  hipEvent_t ev[kSlots] = {};
  bool busy[kSlots] = {};
  size_t cap = 0;
  int next = 0;

  hipError_t init(size_t bytes) {
    cap = bytes;
    for (int i = 0; i < kSlots; ++i) {
      hipError_t e = hipHostMalloc(&host[i], bytes, hipHostMallocDefault);
      if (e != hipSuccess) return e;
      e = hipMalloc(&dev[i], bytes);
      if (e != hipSuccess) return e;
      e = hipEventCreateWithFlags(&ev[i], hipEventDisableTiming);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  void destroy() {
    for (int i = 0; i < kSlots; ++i) {
      if (host[i]) (void)hipHostFree(host[i]);
      if (dev[i]) (void)hipFree(dev[i]);
      if (ev[i]) (void)hipEventDestroy(ev[i]);
    }
  }
  // Returns a slot whose previous upload has been consumed.
  hipError_t acquire(int *slot) {
    int s = next;
    next = (next + 1) % kSlots;
    if (busy[s]) {
      hipError_t e = hipEventSynchronize(ev[s]);
      if (e != hipSuccess) return e;
      busy[s] = false;
    }
    *slot = s;
    return hipSuccess;
  }
  // Upload `bytes` of the slot's host buffer; call release() after the consumer is enqueued.
  hipError_t upload(int s, size_t bytes, hipStream_t st) {
    return hipMemcpyAsync(dev[s], host[s], bytes, hipMemcpyHostToDevice, st);
  }
  hipError_t release(int s, hipStream_t st) {
    if (s < 0) return hipSuccess;   // (nothing was uploaded: the list was already on the device)
    busy[s] = true;
    return hipEventRecord(ev[s], st);
  }
};

}  // namespace cbd

#endif  // CBD_HOST_HPP_
