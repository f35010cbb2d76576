// Checks of arguments that the entry points of the row operators and the dense products share, before any HIP call.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/spdnn.h"
#include "spdnn_error.h"

#define CHECK(expr)                        \
    do {                                   \
        const int rc_ = (expr);            \
        if (rc_ != SPDNN_OK) return rc_;   \
    } while (0)

namespace spdnn {

constexpr size_t kAlign = 256;
constexpr int32_t kMostWidth = 1 << 30;  // columns: a vector beyond a row's end must not pass 32 bits

inline int size_of(int32_t type) { return type == SPDNN_F32 ? 4 : type == SPDNN_BF16 || type == SPDNN_F16 ? 2 : 0; }

// A matrix of rows: not NULL where there is a row, aligned to its elements; rows that are written are apart from each other.
enum Access { kRead, kWritten };
inline int check_rows(const char* what, const void* p, int32_t type, int64_t rows, int32_t width, int64_t stride, Access access) {
    const int size = size_of(type);
    if (!size) return fail(SPDNN_EINVAL, "%s: type must be SPDNN_F32, SPDNN_BF16 or SPDNN_F16", what);
    if (stride < (access == kWritten ? width : 0))
        return fail(SPDNN_EINVAL, "%s: a stride of %lld elements, width %d", what, (long long)stride, width);
    if (rows > 0 && stride > INT64_MAX / 8 / rows) return fail(SPDNN_EINVAL, "%s: stride %lld is too large", what, (long long)stride);
    if (rows > 0 && !p) return fail(SPDNN_EINVAL, "%s is NULL", what);
    if (reinterpret_cast<uintptr_t>(p) % size) return fail(SPDNN_EINVAL, "%s is not aligned to its elements", what);
    return SPDNN_OK;
}
inline int check_array(const char* what, const void* p, int64_t n, int size) {
    if (n > 0 && !p) return fail(SPDNN_EINVAL, "%s is NULL", what);
    if (reinterpret_cast<uintptr_t>(p) % size) return fail(SPDNN_EINVAL, "%s is not aligned to its elements", what);
    return SPDNN_OK;
}
inline int check_width(int32_t width) {
    if (width < 1 || width > kMostWidth) return fail(SPDNN_EINVAL, "need 1 <= width <= %d", kMostWidth);
    return SPDNN_OK;
}
inline int check_work(const void* work, size_t bytes, size_t need) {
    if (bytes < need) return fail(SPDNN_ESIZE, "work has %zu bytes, %zu needed", bytes, need);
    if (need && !work) return fail(SPDNN_EINVAL, "work is NULL");
    if (reinterpret_cast<uintptr_t>(work) % kAlign) return fail(SPDNN_EINVAL, "work must be 256-byte aligned");
    return SPDNN_OK;
}

// f(T{}) with the C++ type of an SPDNN_F32 ...
template <typename F>
inline void with_type(int32_t type, F f) {
    if (type == SPDNN_F32) f(float{});
    else if (type == SPDNN_BF16) f(__bf16{});
    else f(_Float16{});
}

// Outputs of this many bytes go past the caches, for whoever reads them next does not find them there (256 MB at the most) anyway,
// and so do inputs that are read once.  Rows of 4096 bf16 by id, alone and with a kernel behind that reads them, through -> past:
// 400 MB 128 -> 117 and 266 -> 256 us, 200 MB 70 -> 62 and 141 -> 137, 128 MB 42 -> 41 and 83 -> 87, 16 MB 10.4 -> 11.8 and
// 15.9 -> 17.5.  combine of 4 such rows each, its input through -> past: 512 MB 128 -> 112 us, 256 MB 64 -> 60, 128 MB 28.5 -> 35.6.
constexpr int64_t kPastBytes = 160 << 20;

inline int launched() {
    HIP_TRY(hipGetLastError());
    return SPDNN_OK;
}

}  // namespace spdnn
