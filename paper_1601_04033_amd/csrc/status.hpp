// The calling thread's error text and the status returns of the C entry
// points, shared by the files that implement them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/fasgd.h"

namespace fasgd {

inline thread_local char g_err[512];

inline fasgd_status fail(fasgd_status s, const char* fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
    return s;
}

inline fasgd_status ok()
{
    g_err[0] = '\0';
    return FASGD_OK;
}

inline fasgd_status hip_fail(hipError_t e, const char* what)
{
    return fail(FASGD_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace fasgd
