// What the entry points of quant_rows.hip, i8_gemm.hip and experts.hip do around a launch.
#pragma once
#include <hip/hip_runtime.h>

#include "ft_internal.h"

namespace ftk {

// A kernel runs where its stream belongs: a stream of another device than the current one is refused.  The default streams, by any of their handles, are the
// current device's, and the latter two are no objects that could be asked.
inline ft_status op_stream_check(void *stream) {
    if (!stream || stream == static_cast<void *>(hipStreamLegacy) || stream == static_cast<void *>(hipStreamPerThread)) return FT_OK;
    int dev = -1;
    hipDevice_t of = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e == hipSuccess) e = hipStreamGetDevice(static_cast<hipStream_t>(stream), &of);
    if (e != hipSuccess) { ftd_set_hip_error((int)e); return FT_ERR_HIP; }
    return (int)of == dev ? FT_OK : FT_ERR_INVALID_ARG;
}
inline ft_status op_launched() {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return FT_OK;
    ftd_set_hip_error((int)e);
    return FT_ERR_HIP;
}

}  // namespace ftk
