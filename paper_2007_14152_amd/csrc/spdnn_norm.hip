// Host side of layer norm (spdnn_layer_norm, spdnn_layer_norm_grad of include/spdnn.h): argument checks and launches.
#include "../../include/spdnn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "spdnn_check.h"
#include "spdnn_error.h"
#include "spdnn_norm_kernels.h"

namespace {

using namespace spdnn;

constexpr int64_t kMostGroups = 1 << 20;

int check_param(int32_t param_type, int32_t type) {
    if (param_type != type && param_type != SPDNN_F32) return fail(SPDNN_EINVAL, "parameters are of the rows' type or SPDNN_F32");
    return SPDNN_OK;
}

// Threads that take rows in turn: as many as the chip's 256 CUs hold.
constexpr int64_t kNormThreads = 2048 * 256;
// Workgroups that add columns, each of which leaves a part: two a CU.  60000 x 1024 bf16: 256 107 us, 512 98, 768 102, 1024 111, 2048 113.
constexpr int64_t kParts = 512;
// And where registers do not hold a row (the workgroups have 256 columns each).
constexpr int64_t kLongParts = 16;
// The most parts for any type: rows of more columns than this no type's registers hold.
constexpr int32_t kHeldVecs = 4096, kHeldWidth = kHeldVecs * 8;
int64_t most_parts(int32_t rows, int32_t width) { return std::min(static_cast<int64_t>(rows), width > kHeldWidth ? kLongParts : kParts); }

// f(U, G, threads) for a row that registers hold: so many vectors a lane, lanes of a team and of a workgroup; false for longer ones.
template <int V, typename F>
bool with_row(int32_t width, F f) {
    const int vecs = (width - 1) / V + 1;
#define SPDNN_ROW(U, G, THREADS) f(std::integral_constant<int, U>{}, std::integral_constant<int, G>{}, std::integral_constant<int, THREADS>{})
    if (vecs <= 64) SPDNN_ROW(1, 64, 256);
    else if (vecs <= 128) SPDNN_ROW(2, 64, 256);
    else if (vecs <= 256) SPDNN_ROW(1, 256, 256);
    else if (vecs <= 512) SPDNN_ROW(2, 256, 256);
    else if (vecs <= 1024) SPDNN_ROW(4, 256, 256);
    else if (vecs <= 2048) SPDNN_ROW(2, 1024, 1024);
    else if (vecs <= kHeldVecs) SPDNN_ROW(4, 1024, 1024);
    else return false;
#undef SPDNN_ROW
    return true;
}
template <typename T, typename F>
bool with_row_of(int32_t width, F f) {
    constexpr int V = 16 / sizeof(T);
    if (width < V) return with_row<1>(width, [&](auto u, auto g, auto threads) { f(std::integral_constant<int, 1>{}, std::true_type{}, u, g, threads); });
    return with_row<V>(width, [&](auto u, auto g, auto threads) {
        if (width % V == 0) f(std::integral_constant<int, V>{}, std::true_type{}, u, g, threads);
        else f(std::integral_constant<int, V>{}, std::false_type{}, u, g, threads);
    });
}

}  // namespace

extern "C" {

int spdnn_layer_norm(const void* x, int32_t type, int32_t rows, int32_t width, int64_t x_stride, const void* weight, const void* bias,
                     int32_t param_type, float eps, void* out, int32_t out_type, int64_t out_stride, float* stats, void* hip_stream) {
    if (rows < 0) return fail(SPDNN_EINVAL, "rows < 0");
    CHECK(check_width(width));
    CHECK(check_rows("x", x, type, rows, width, x_stride, kRead));
    CHECK(check_rows("out", out, out_type, rows, width, out_stride, kWritten));
    if (out_type != type && out_type != SPDNN_F32) return fail(SPDNN_EINVAL, "out is of x's type or SPDNN_F32");
    CHECK(check_param(param_type, type));
    CHECK(check_array("weight", weight, 0, size_of(param_type)));
    CHECK(check_array("bias", bias, 0, size_of(param_type)));
    CHECK(check_array("stats", stats, 0, 8));
    if (!(eps >= 0.0f)) return fail(SPDNN_EINVAL, "need eps >= 0");
    if (rows == 0) return SPDNN_OK;
    const hipStream_t s = (hipStream_t)hip_stream;
    const Norm p{rows, width, weight, bias, param_type == SPDNN_F32, eps, (float2*)stats, (int64_t)rows * width * size_of(out_type) >= kPastBytes};
    with_type(type, [&](auto tt) {
        using T = decltype(tt);
        const auto run = [&](auto to) {
            using O = decltype(to);
            const bool held = with_row_of<T>(width, [&](auto v, auto whole, auto u, auto g, auto threads) {
                constexpr int G = decltype(g)::value, THREADS = decltype(threads)::value;
                const int64_t groups = std::min<int64_t>((rows - 1) / (THREADS / G) + 1, kNormThreads / THREADS);
                layer_norm_kernel<T, O, decltype(v)::value, decltype(whole)::value, decltype(u)::value, G, THREADS><<<dim3((unsigned)groups), THREADS, 0, s>>>(p, (const T*)x, x_stride, (O*)out, out_stride);
            });
            if (!held)
                layer_norm_long_kernel<T, O><<<dim3((unsigned)std::min<int64_t>(rows, kMostGroups)), 1024, 0, s>>>(p, (const T*)x, x_stride, (O*)out, out_stride);
        };
        if (out_type == type) run(T{});
        else run(float{});
    });
    return launched();
}

int spdnn_layer_norm_grad_bytes(int32_t rows, int32_t width, size_t* bytes) {
    if (!bytes) return fail(SPDNN_EINVAL, "bytes is NULL");
    if (rows < 0) return fail(SPDNN_EINVAL, "rows < 0");
    CHECK(check_width(width));
    *bytes = ((size_t)most_parts(rows, width) * 2 * (size_t)width * sizeof(float) + kAlign - 1) / kAlign * kAlign;
    return SPDNN_OK;
}

int spdnn_layer_norm_grad(const void* dout, int32_t type, int64_t dout_stride, const void* x, int32_t rows, int32_t width, int64_t x_stride,
                          const float* stats, const void* weight, int32_t param_type, const void* add, int64_t add_stride, void* dx,
                          int64_t dx_stride, void* dweight, void* dbias, int32_t grad_type, void* work, size_t work_bytes, void* hip_stream) {
    size_t need = 0;
    CHECK(spdnn_layer_norm_grad_bytes(rows, width, &need));
    CHECK(check_rows("dout", dout, type, rows, width, dout_stride, kRead));
    CHECK(check_rows("x", x, type, rows, width, x_stride, kRead));
    CHECK(check_rows("dx", dx, type, rows, width, dx_stride, kWritten));
    if (add) CHECK(check_rows("add", add, type, rows, width, add_stride, kRead));
    CHECK(check_array("stats", stats, rows, 8));
    CHECK(check_param(param_type, type));
    CHECK(check_array("weight", weight, 0, size_of(param_type)));
    const bool sums = dweight || dbias;
    if (sums) {
        if (grad_type != type && grad_type != SPDNN_F32) return fail(SPDNN_EINVAL, "dweight and dbias are of the rows' type or SPDNN_F32");
        CHECK(check_array("dweight", dweight, 0, size_of(grad_type)));
        CHECK(check_array("dbias", dbias, 0, size_of(grad_type)));
        CHECK(check_work(work, work_bytes, need));
    }
    const hipStream_t s = (hipStream_t)hip_stream;
    const int64_t most = most_parts(rows, width);
    const NormGrad p{rows, width, (const float2*)stats, weight, param_type == SPDNN_F32, sums ? (float*)work : nullptr, (int64_t)rows * width * size_of(type) >= kPastBytes};
    with_type(type, [&](auto tt) {
        using T = decltype(tt);
        int64_t parts = 0;
        if (rows > 0) {
            const bool held = with_row_of<T>(width, [&](auto v, auto whole, auto u, auto g, auto threads) {
                constexpr int G = decltype(g)::value, THREADS = decltype(threads)::value;
                parts = std::min<int64_t>((rows - 1) / (THREADS / G) + 1, most);
                layer_norm_grad_kernel<T, decltype(v)::value, decltype(whole)::value, decltype(u)::value, G, THREADS><<<dim3((unsigned)parts), THREADS, 0, s>>>(p, (const T*)dout, dout_stride, (const T*)x, x_stride, (const T*)add, add_stride, (T*)dx, dx_stride);
            });
            if (!held) {
                layer_norm_grad_long_kernel<T><<<dim3((unsigned)std::min<int64_t>(rows, kMostGroups)), 1024, 0, s>>>(p, (const T*)dout, dout_stride, (const T*)x, x_stride, (const T*)add, add_stride, (T*)dx, dx_stride);
                if (sums) {
                    parts = std::min<int64_t>(rows, kLongParts);
                    layer_norm_columns_kernel<T><<<dim3((unsigned)std::min((width - 1) / 256 + 1, 65536), (unsigned)parts), 256, 0, s>>>(p, (const T*)dout, dout_stride, (const T*)x, x_stride);
                }
            }
        }
        if (sums) {
            const int groups = (int)std::min<int64_t>((2 * (int64_t)width - 1) / 64 + 1, kMostGroups);
            if (grad_type == SPDNN_F32) layer_norm_join_kernel<float><<<groups, 1024, 0, s>>>(p.parts, (int32_t)parts, width, (float*)dweight, (float*)dbias);
            else layer_norm_join_kernel<T><<<groups, 1024, 0, s>>>(p.parts, (int32_t)parts, width, (T*)dweight, (T*)dbias);
        }
    });
    return launched();
}

}  // extern "C"
