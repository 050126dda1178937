// device_setup.h -- host code shared by the C ABIs of the GPU libraries (ts_attn.cpp, ts_cache.cpp): once-per-device set-up
// and stream capture.
#pragma once
#include <hip/hip_runtime_api.h>

#include <atomic>
#include <mutex>

#include "ts_attn.h"

namespace tshost {

constexpr int kMaxDevices = 64;

// What a library keeps of a device, as a base.
struct DeviceSetup {
  std::once_flag once;
  std::atomic<bool> set_up{false};  // the set-up has run (whatever its outcome)
  int status = TS_ERR_UNSUPPORTED;  // TS_OK once the device is known to be usable
};

// Whether stream s is recording a HIP graph.  A failed query (which leaves an error behind that
// a later launch check would report) is cleared and read as "not capturing".
inline bool capturing(hipStream_t s) {
  hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(s, &cs) != hipSuccess) {
    (void)hipGetLastError();
    return false;
  }
  return cs != hipStreamCaptureStatusNone;
}

// The calling thread's current device, or -1.
inline int current_index() {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) {
    (void)hipGetLastError();
    return -1;
  }
  return dev;
}

// The state of the calling thread's current device, set up once by init(dev, state) -- never under stream
// capture, where set-up has no place (TS_ERR_CAPTURE).
template <typename State, typename Init>
State* current_device(State (&all)[kMaxDevices], Init&& init, int* status, hipStream_t s) {
  const int dev = current_index();
  if (dev < 0) {
    *status = TS_ERR_UNSUPPORTED;
    return nullptr;
  }
  State* st = &all[dev];
  if (!st->set_up.load(std::memory_order_acquire) && capturing(s)) {
    *status = TS_ERR_CAPTURE;
    return nullptr;
  }
  std::call_once(st->once, [&] {
    init(dev, st);
    st->set_up.store(true, std::memory_order_release);
  });
  *status = st->status;
  return st->status == TS_OK ? st : nullptr;
}

}  // namespace tshost
