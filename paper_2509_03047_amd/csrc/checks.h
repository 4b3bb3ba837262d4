// Argument checks shared by the C-ABI entry points.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "flashrestore.h"

namespace fr {

extern thread_local int g_last_hip_error;

struct Region {
  const void* p;
  uint64_t bytes;
};

inline int device_error(hipError_t e) {
  g_last_hip_error = int(e);
  return FR_E_DEVICE;
}

inline int check_device_and_stream(int device, hipStream_t stream) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return device_error(e);
  if (dev != device) return FR_E_DEVICE_MISMATCH;
  if (stream) {
    hipDevice_t sd = -1;
    e = hipStreamGetDevice(hipStream_t(stream), &sd);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      return FR_E_INVAL;
    }
    if (int(sd) != device) return FR_E_DEVICE_MISMATCH;
  }
  return FR_OK;
}

// A buffer the kernels will touch: it must be device memory of the plan's
// device, aligned, and lie inside one allocation.  An empty buffer is never
// touched, so any pointer (NULL included) is accepted for it.
inline int check_buffer(int device, const void* p, uint64_t bytes, uint64_t align) {
  if (bytes == 0) return FR_OK;
  if (p == nullptr) return FR_E_INVAL;
  if (reinterpret_cast<uintptr_t>(p) % align) return FR_E_ALIGN;
  hipPointerAttribute_t attr{};
  hipError_t e = hipPointerGetAttributes(&attr, p);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return FR_E_INVAL;  // not memory HIP knows about
  }
  if (attr.type != hipMemoryTypeDevice && attr.type != hipMemoryTypeManaged) return FR_E_INVAL;
  if (attr.device != device) return FR_E_DEVICE_MISMATCH;
  hipDeviceptr_t base = nullptr;
  size_t size = 0;
  e = hipMemGetAddressRange(&base, &size, hipDeviceptr_t(const_cast<void*>(p)));
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return FR_E_INVAL;
  }
  const uintptr_t b = reinterpret_cast<uintptr_t>(base), q = reinterpret_cast<uintptr_t>(p);
  if (q < b || bytes > size || q - b > size - bytes) return FR_E_RANGE;
  return FR_OK;
}

inline bool overlap(const Region& x, const Region& y) {
  if (!x.p || !y.p || x.bytes == 0 || y.bytes == 0) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(x.p), b = reinterpret_cast<uintptr_t>(y.p);
  return a < b + y.bytes && b < a + x.bytes;
}

// Outputs must not overlap each other or any input.
inline int check_disjoint(const Region* outs, int n_out, const Region* ins, int n_in) {
  for (int i = 0; i < n_out; i++) {
    for (int j = i + 1; j < n_out; j++)
      if (overlap(outs[i], outs[j])) return FR_E_OVERLAP;
    for (int j = 0; j < n_in; j++)
      if (overlap(outs[i], ins[j])) return FR_E_OVERLAP;
  }
  return FR_OK;
}

inline int launch_result(int hip_rc) {
  if (hip_rc == 0) return FR_OK;
  return device_error(hipError_t(hip_rc));
}

#define FR_TRY(expr)            \
  do {                          \
    const int rc_ = (expr);     \
    if (rc_ != FR_OK) return rc_; \
  } while (0)

}  // namespace fr
