// The little state the library keeps: per device, whether the kernel attributes have been set;
// per thread, the text of the last HIP error.
#include <cstdio>

#include "common.h"
#include "device_once.h"

namespace adwin {

static thread_local char g_hip_error[256] = "";

const char* last_hip_error_text() { return g_hip_error; }

void set_last_hip_error(hipError_t e, const char* where) {
  snprintf(g_hip_error, sizeof(g_hip_error), "HIP error %d (%s) at %s", (int)e,
           hipGetErrorString(e), where);
}

hipError_t once_on_device(Once what, hipError_t (*prepare)()) {
  static DeviceOnce once[kOnce];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) dev = -1;
  return once[what].run(dev, prepare);
}

}  // namespace adwin
