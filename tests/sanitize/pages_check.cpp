// The pages' entry points with arguments at the ends of their types, under the
// sanitizers: HIP and the launches are stood in for, so nothing reaches a device.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "adaserve.h"
#include "pages.h"

static adaserve::CopyPagesArgs launched;
static int launches;

extern "C" {
hipError_t hipGetDevice(int *device) {
  *device = 0;
  return hipSuccess;
}
hipError_t hipGetDeviceProperties(hipDeviceProp_t *prop, int) {
  std::strcpy(prop->gcnArchName, "gfx950");
  return hipSuccess;
}
const char *hipGetErrorString(hipError_t) { return ""; }
}

namespace adaserve {
hipError_t launch_update_pages(const PagesArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_fork_pages(const PagesArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_compact_pages(const PagesArgs &, hipStream_t) {
  ++launches;   // (the counts of an empty pool are written, too)
  return hipSuccess;
}
hipError_t launch_copy_pages(const CopyPagesArgs &a, hipStream_t) {
  launched = a;
  ++launches;
  return hipSuccess;
}
}  // namespace adaserve

#define CHECK(x)                                                  \
  do {                                                            \
    if (!(x)) {                                                   \
      std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x);         \
      std::exit(1);                                               \
    }                                                             \
  } while (0)

static char *at(int i) { return (char *)(uintptr_t)(0x10000 + i * 0x100000); }

static int32_t copy(int32_t layers, int64_t stride, int32_t dtype) {
  return adaserve_copy_pages(3, (int32_t *)at(1), (int32_t *)at(2), nullptr, at(3), at(4), layers, stride, 10, 2, 16, 64,
                             dtype, nullptr);
}

int main() {
  for (int32_t dtype : {ADASERVE_BF16, ADASERVE_F32}) {
    const int64_t esz = dtype == ADASERVE_BF16 ? 2 : 4;
    for (int64_t stride : {INT64_MAX, INT64_MAX - 15, (int64_t)1 << 62, (int64_t)1 << 61, ((int64_t)1 << 47) + 16})
      CHECK(copy(2, stride, dtype) == ADASERVE_ERR_UNSUPPORTED);
    for (int64_t stride : {INT64_MIN, (int64_t)-1, (int64_t)0, ((int64_t)1 << 47) - 1})
      CHECK(copy(2, stride, dtype) == ADASERVE_ERR_INVALID_ARGUMENT);
    CHECK(launches == 0);
    CHECK(copy(2, (int64_t)1 << 47, dtype) == ADASERVE_OK && launched.layer_bytes == esz << 47);
    // one layer: any stride, which nothing is multiplied by
    for (int64_t stride : {INT64_MAX, INT64_MIN, (int64_t)-1, (int64_t)0, (int64_t)7})
      CHECK(copy(1, stride, dtype) == ADASERVE_OK && launched.layer_bytes == 0);
    CHECK(launches == 6);
    launches = 0;
  }
  // nothing at all: no bytes of workspace are needed, and none are asked for
  CHECK(adaserve_pages_workspace_bytes(0, 0) == 0);
  int32_t *const counts = (int32_t *)at(1);
  for (void *workspace : {(void *)nullptr, (void *)at(2)}) {
    CHECK(adaserve_update_pages(0, nullptr, nullptr, 0, 0, 16, nullptr, 4, nullptr, 0, nullptr, nullptr, nullptr, workspace, 0,
                                nullptr) == ADASERVE_OK);
    CHECK(adaserve_fork_pages(0, 0, nullptr, nullptr, 16, nullptr, 4, nullptr, 0, nullptr, nullptr, nullptr, nullptr, nullptr,
                              workspace, 0, nullptr) == ADASERVE_OK);
    CHECK(launches == 0);
    CHECK(adaserve_compact_pages(0, nullptr, 4, nullptr, 0, nullptr, nullptr, nullptr, nullptr, nullptr, counts, workspace, 0,
                                 nullptr) == ADASERVE_OK);
    CHECK(launches == 1);
    launches = 0;
  }
  CHECK(adaserve_compact_pages(1, counts, 1, nullptr, 0, counts, nullptr, nullptr, nullptr, nullptr, (int32_t *)at(3), nullptr, 0,
                               nullptr) == ADASERVE_ERR_WORKSPACE);
  std::printf("pages checks passed\n");
}
