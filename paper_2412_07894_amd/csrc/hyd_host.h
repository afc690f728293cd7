// What the host sides of the library's translation units share (defined in hyd_api.hip).
#pragma once
#include "../../include/hyd_attn.h"

#include <hip/hip_runtime.h>

namespace hyd {

// The current device: its number and its compute units.  HYD_ERR_ARCH unless it is a gfx950.
hyd_status current_device(int* device, int* cus);

struct TimedKernel { const char* name; hipEvent_t e0, e1; };
struct KernelTimer {       // brackets one launch with events when timing is on (hyd_enable_kernel_timing)
    hipStream_t st; bool on; TimedKernel tk;
    KernelTimer(const char* name, hipStream_t s);
    ~KernelTimer();
};

}  // namespace hyd
