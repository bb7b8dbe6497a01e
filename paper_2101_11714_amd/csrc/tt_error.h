// The text behind tt_last_error() and the way every entry point fails: one buffer per thread, shared by the library's
// translation units.
#pragma once

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/tt_emb.h"

namespace tt {

inline thread_local char g_err[512] = "";

inline int fail(int code, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return code;
}

inline int hip_fail(hipError_t e, const char *what) { return fail(TT_ERR_HIP, "%s: %s", what, hipGetErrorString(e)); }

}  // namespace tt
