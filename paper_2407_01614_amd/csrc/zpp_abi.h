// Host helpers shared by the files of the C ABI: argument checks, events and
// the thread's last HIP error.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "zpp.h"

namespace zpp {

inline thread_local int g_last_hip_error = 0;

inline zpp_status hip_fail(hipError_t e) {
    g_last_hip_error = (int)e;
    return ZPP_EHIP;
}

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

inline zpp_status wait_on(hipStream_t stream, hipEvent_t ev) {
    if (!ev)
        return ZPP_OK;
    const hipError_t e = hipStreamWaitEvent(stream, ev, 0);
    return e == hipSuccess ? ZPP_OK : hip_fail(e);
}

inline zpp_status record(hipStream_t stream, hipEvent_t ev) {
    if (!ev)
        return ZPP_OK;
    const hipError_t e = hipEventRecord(ev, stream);
    return e == hipSuccess ? ZPP_OK : hip_fail(e);
}

}  // namespace zpp
