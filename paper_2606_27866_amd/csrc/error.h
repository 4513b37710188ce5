// Error reporting of the C ABI: one message per thread, read by
// flexmoe_last_error.
#pragma once

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdio.h>

#include "flexmoe.h"

namespace flexmoe {

inline thread_local char g_err[512] = "";

inline int fail(int code, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
    return code;
}

inline int hip_fail(hipError_t e, const char* what) {
    return fail(FLEXMOE_EHIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace flexmoe
