// Shared by the C entry points: the calling thread's last error and the checks of arguments (host code,
// before any HIP call).
#pragma once

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include <string>

#include "../../include/mtgr_hstu.h"

namespace mtgr_api {

inline thread_local std::string g_last_error;

inline mtgr_status_t fail(mtgr_status_t st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
inline mtgr_status_t fail(mtgr_status_t st, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    g_last_error = buf;
    return st;
}

inline mtgr_status_t ok() {
    g_last_error.clear();
    return MTGR_SUCCESS;
}

inline mtgr_status_t device_fail(hipError_t e, const char* where) {
    return fail(MTGR_ERROR_DEVICE, "%s: %s", where, hipGetErrorString(e));
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace mtgr_api
