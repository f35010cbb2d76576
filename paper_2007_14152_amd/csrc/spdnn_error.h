// The calling thread's last error, shared by the library's translation units.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <string>

#include "../../include/spdnn.h"

namespace spdnn {

inline std::string& last_error() {
    static thread_local std::string text;
    return text;
}

inline int fail(int code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try {
        last_error() = buf;
    } catch (...) {  // no memory for the message: the code alone has to do
    }
    return code;
}

}  // namespace spdnn

#define HIP_TRY(expr)                                                                                \
    do {                                                                                             \
        hipError_t e_ = (expr);                                                                      \
        if (e_ != hipSuccess)                                                                        \
            return spdnn::fail(SPDNN_EHIP, "%s failed: %s (%s:%d)", #expr, hipGetErrorString(e_),    \
                               __FILE__, __LINE__);                                                  \
    } while (0)
