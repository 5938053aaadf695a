// Host helpers shared by the entry points: pointer alignment, the gfx950
// device check and the status of a launch.
#pragma once
#include <hip/hip_runtime.h>

#include <cstring>
#include <mutex>

#include "adaserve.h"
#include "host_plan.h"

namespace adaserve {

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

// gfx950 check, once per device ordinal.
inline int32_t check_device() {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail(ADASERVE_ERR_DEVICE, "hipGetDevice failed: %s", hipGetErrorString(e));
  static std::mutex mu;
  static signed char arch_ok[256];  // 0 unknown, 1 gfx950, -1 other
  if (dev < 0 || dev >= 256) return fail(ADASERVE_ERR_DEVICE, "device ordinal %d out of range", dev);
  std::lock_guard<std::mutex> lock(mu);
  if (arch_ok[dev] == 0) {
    hipDeviceProp_t prop;
    e = hipGetDeviceProperties(&prop, dev);
    if (e != hipSuccess)
      return fail(ADASERVE_ERR_DEVICE, "hipGetDeviceProperties failed: %s", hipGetErrorString(e));
    arch_ok[dev] = std::strncmp(prop.gcnArchName, "gfx950", 6) == 0 ? 1 : -1;
  }
  if (arch_ok[dev] < 0) return fail(ADASERVE_ERR_UNSUPPORTED, "device %d is not gfx950", dev);
  return ADASERVE_OK;
}

inline int32_t launch_status(hipError_t e, const char *what) {
  if (e == hipSuccess) return ADASERVE_OK;
  return fail(ADASERVE_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace adaserve
