// How the library's translation units report a launch.
#ifndef NMS_LAUNCH_H
#define NMS_LAUNCH_H

#include <hip/hip_runtime.h>

#include "../../include/nms.h"

// The calling thread's most recent failed launch (nms_last_launch_error); lives in nms_kernels.hip.
extern thread_local hipError_t nms_last_hip_error_of_thread __attribute__((visibility("hidden")));

// The runtime's "last error" is per thread and sticky across libraries: an unrelated
// earlier failure (for example a probe made by the host framework) would otherwise be
// reported as ours.  begin_launch() discards it, launch_status() reads ours.
static inline void begin_launch() { (void)hipGetLastError(); }

static inline int launch_status()
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return NMS_OK;
    nms_last_hip_error_of_thread = e;
    return NMS_ERR_LAUNCH;
}

#endif
