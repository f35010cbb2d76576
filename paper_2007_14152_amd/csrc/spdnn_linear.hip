// Host side of the dense products (spdnn_linear, spdnn_linear_grad of include/spdnn.h): argument checks and launches.
#include "../../include/spdnn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "spdnn_check.h"
#include "spdnn_error.h"
#include "spdnn_linear_kernels.h"

namespace {

using namespace spdnn;

constexpr int64_t kMostGroups = 1 << 20;
constexpr int64_t kMostTiles = 1 << 30;

int step_of(int32_t type) { return type == SPDNN_F32 ? 32 : 64; }
size_t aligned(size_t bytes) { return (bytes + kAlign - 1) / kAlign * kAlign; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int check_sizes(int32_t rows, int32_t width, int32_t cols, int32_t experts, int32_t type) {
    if (rows < 0) return fail(SPDNN_EINVAL, "rows < 0");
    CHECK(check_width(width));
    if (cols < 1 || cols > kMostWidth) return fail(SPDNN_EINVAL, "need 1 <= cols <= %d", kMostWidth);
    if (experts < 1 || experts > SPDNN_MAX_EXPERTS) return fail(SPDNN_EINVAL, "need 1 <= experts <= %d", SPDNN_MAX_EXPERTS);
    if (!size_of(type)) return fail(SPDNN_EINVAL, "type must be SPDNN_F32, SPDNN_BF16 or SPDNN_F16");
    return SPDNN_OK;
}
int check_groups(const int32_t* offsets, int32_t experts) {
    if (!offsets && experts != 1) return fail(SPDNN_EINVAL, "offsets is NULL, with %d experts", experts);
    return check_array("offsets", offsets, 0, 4);
}
// W or dW: its stored rows (width of them with cols numbers each, or the other way round) and the experts' matrices.
int check_matrix(const char* what, const void* p, int32_t type, int32_t width, int32_t cols, int32_t transposed, int64_t stride, int32_t experts,
                 int64_t set, Access access) {
    const int32_t lines = transposed ? cols : width, along = transposed ? width : cols;
    CHECK(check_rows(what, p, type, lines, along, stride, access));
    if (experts > 1) {
        if (set < 0 || set > INT64_MAX / 16 / experts) return fail(SPDNN_EINVAL, "%s: a stride of %lld elements between experts", what, (long long)set);
        if (access == kWritten && set < stride * (lines - 1) + along)
            return fail(SPDNN_EINVAL, "%s: the experts' matrices overlap", what);
    }
    return SPDNN_OK;
}
int check_output(const char* what, const void* p, int32_t out_type, int32_t type) {
    if (out_type != type && out_type != SPDNN_F32) return fail(SPDNN_EINVAL, "%s is of x's type or SPDNN_F32", what);
    (void)p;
    return SPDNN_OK;
}

// How a product is cut.
constexpr int kTile = 128;
struct Cut {
    int64_t mtiles, ntiles;
    int64_t splits, per_split;  // of k
    size_t parts;               // bytes
};
// Splits: as many as give every CU a workgroup, of kLeastSteps steps of k at least.
constexpr int64_t kGroupsWanted = 256, kLeastSteps = 8;
int64_t splits_of(int64_t tiles, int64_t steps) { return std::max<int64_t>(1, std::min(kGroupsWanted / std::max<int64_t>(tiles, 1), steps / kLeastSteps)); }

Cut cut_product(int32_t rows, int32_t k, int32_t cols, bool grouped, int32_t experts, int32_t type) {
    Cut c;
    c.mtiles = grouped ? rows / kTile + experts + 1 : ceil_div(rows, kTile);
    c.ntiles = ceil_div(cols, kTile);
    const int64_t busy = grouped ? std::min<int64_t>(c.mtiles, rows) : c.mtiles;
    const int64_t steps = ceil_div(k, step_of(type));
    c.splits = splits_of(busy * c.ntiles, steps);
    c.per_split = ceil_div(steps, c.splits) * step_of(type);
    c.splits = ceil_div(k, c.per_split);
    c.parts = c.splits > 1 ? aligned((size_t)c.splits * rows * cols * sizeof(float)) : 0;
    return c;
}
Cut cut_grad(int32_t rows, int32_t m, int32_t n, bool grouped, int32_t experts, int32_t type) {
    Cut c;
    c.mtiles = ceil_div(m, kTile);
    c.ntiles = ceil_div(n, kTile);
    c.splits = splits_of(c.mtiles * c.ntiles * experts, ceil_div(ceil_div(rows, experts), step_of(type)));
    c.per_split = 0;
    c.parts = c.splits > 1 ? aligned((size_t)c.splits * experts * m * n * sizeof(float)) : 0;
    (void)grouped;
    return c;
}
int check_tiles(const Cut& c, int64_t sets) {
    if ((double)c.mtiles * (double)c.ntiles * (double)c.splits * (double)sets > (double)kMostTiles)
        return fail(SPDNN_EINVAL, "sizes too large: more than 2^30 tiles");
    return SPDNN_OK;
}

void run_product(int32_t type, Adjacent adj, const Cut& c, Product p, Ending e, hipStream_t s) {
    p.mtiles = (int32_t)c.mtiles;
    p.ntiles = (int32_t)c.ntiles;
    p.splits = (int32_t)c.splits;
    p.per_split = c.per_split;
    const dim3 grid((unsigned)(c.mtiles * c.ntiles * c.splits));
    with_type(type, [&](auto tt) {
        using T = decltype(tt);
        if (adj == Adjacent::K) linear_kernel<T, Adjacent::K, 4, 2, 2><<<grid, 256, 0, s>>>(p, e);
        else linear_kernel<T, Adjacent::L, 4, 2, 2><<<grid, 256, 0, s>>>(p, e);
        if (c.splits > 1) {
            const int64_t items = (int64_t)p.rows * ceil_div(p.cols, kEnd);
            linear_join_kernel<T><<<dim3((unsigned)std::min(ceil_div(items, 256), kMostGroups)), 256, 0, s>>>(p, e);
        }
    });
}

// Work memory of the gradients: d in the rows' type where dout is not that already, and parts, which the three steps use in turn.
struct GradWork {
    bool own_d;
    int64_t d_stride;  // elements
    size_t d, parts, bytes;
    Cut dx, dw;
    int64_t bias_splits;
    GradWork(int32_t rows, int32_t width, int32_t cols, bool grouped, int32_t experts, int32_t type, int32_t dout_type, int32_t act, int32_t transposed) {
        own_d = act != SPDNN_ACT_NONE || dout_type != type;
        d_stride = ceil_div(cols, 16) * 16;
        d = own_d ? aligned((size_t)rows * d_stride * size_of(type)) : 0;
        dx = cut_product(rows, cols, width, grouped, experts, type);
        dw = transposed ? cut_grad(rows, cols, width, grouped, experts, type) : cut_grad(rows, width, cols, grouped, experts, type);
        bias_splits = std::max<int64_t>(1, std::min(1024 / (ceil_div(cols, 64) * experts), ceil_div(rows, experts) / 32));
        parts = std::max({dx.parts, dw.parts, bias_splits > 1 ? aligned((size_t)bias_splits * experts * cols * sizeof(float)) : 0});
        bytes = d + parts;
    }
};

int check_act(int32_t act) {
    if (act < SPDNN_ACT_NONE || act > SPDNN_ACT_SILU) return fail(SPDNN_EINVAL, "act must be one of SPDNN_ACT_NONE ... SPDNN_ACT_SILU");
    return SPDNN_OK;
}

}  // namespace

extern "C" {

int spdnn_linear_bytes(int32_t rows, int32_t width, int32_t cols, int32_t grouped, int32_t experts, int32_t type, size_t* bytes) {
    if (!bytes) return fail(SPDNN_EINVAL, "bytes is NULL");
    CHECK(check_sizes(rows, width, cols, experts, type));
    const Cut c = cut_product(rows, width, cols, grouped != 0, experts, type);
    CHECK(check_tiles(c, 1));
    *bytes = c.parts;
    return SPDNN_OK;
}

int spdnn_linear(const void* x, int32_t type, int32_t rows, int32_t width, int64_t x_stride, const int32_t* offsets, int32_t experts,
                 const void* weight, int32_t transposed, int64_t weight_stride, int64_t expert_stride, int32_t cols, const void* bias,
                 int32_t bias_type, int32_t act, const void* add, int64_t add_stride, void* out, int32_t out_type, int64_t out_stride, void* pre,
                 int64_t pre_stride, void* work, size_t work_bytes, void* hip_stream) {
    size_t need = 0;
    CHECK(spdnn_linear_bytes(rows, width, cols, offsets != nullptr, experts, type, &need));
    CHECK(check_groups(offsets, experts));
    CHECK(check_act(act));
    CHECK(check_rows("x", x, type, rows, width, x_stride, kRead));
    CHECK(check_matrix("weight", weight, type, width, cols, transposed, weight_stride, experts, expert_stride, kRead));
    CHECK(check_output("out", out, out_type, type));
    CHECK(check_rows("out", out, out_type, rows, cols, out_stride, kWritten));
    if (pre) CHECK(check_rows("pre", pre, out_type, rows, cols, pre_stride, kWritten));
    if (add) CHECK(check_rows("add", add, out_type, rows, cols, add_stride, kRead));
    if (bias) {
        CHECK(check_output("bias", bias, bias_type, type));
        CHECK(check_array("bias", bias, 0, size_of(bias_type)));
    }
    CHECK(check_work(work, work_bytes, need));
    if (rows == 0) return SPDNN_OK;
    const int size = size_of(type), out_size = size_of(out_type);
    const Cut c = cut_product(rows, width, cols, offsets != nullptr, experts, type);
    Product p{};
    p.x = {(const char*)x, x_stride * size, 0};
    p.w = {(const char*)weight, weight_stride * size, expert_stride * size};
    p.offsets = offsets;
    p.rows = rows;
    p.width = width;
    p.cols = cols;
    p.experts = experts;
    p.parts = (float*)work;
    Ending e{};
    e.bias = bias;
    e.bias_f32 = bias_type == SPDNN_F32;
    e.add = (const char*)add;
    e.add_line = add_stride * out_size;
    e.pre = (char*)pre;
    e.pre_line = pre_stride * out_size;
    e.out = (char*)out;
    e.out_line = out_stride * out_size;
    e.cols = cols;
    e.act = act;
    e.out_f32 = out_type == SPDNN_F32;
    run_product(type, transposed ? Adjacent::K : Adjacent::L, c, p, e, (hipStream_t)hip_stream);
    return launched();
}

int spdnn_linear_grad_bytes(int32_t rows, int32_t width, int32_t cols, int32_t grouped, int32_t experts, int32_t type, int32_t dout_type, int32_t act,
                            int32_t transposed, size_t* bytes) {
    if (!bytes) return fail(SPDNN_EINVAL, "bytes is NULL");
    CHECK(check_sizes(rows, width, cols, experts, type));
    CHECK(check_output("dout", nullptr, dout_type, type));
    CHECK(check_act(act));
    const GradWork w(rows, width, cols, grouped != 0, experts, type, dout_type, act, transposed);
    CHECK(check_tiles(w.dx, 1));
    CHECK(check_tiles(w.dw, experts));
    *bytes = w.bytes;
    return SPDNN_OK;
}

int spdnn_linear_grad(const void* dout, int32_t dout_type, int64_t dout_stride, const void* pre, int64_t pre_stride, int32_t act, const void* x,
                      int32_t type, int32_t rows, int32_t width, int64_t x_stride, const int32_t* offsets, int32_t experts, const void* weight,
                      int32_t transposed, int64_t weight_stride, int64_t expert_stride, int32_t cols, void* dx, int64_t dx_stride, void* dweight,
                      int64_t dweight_stride, int64_t dexpert_stride, void* dbias, int32_t grad_type, void* work, size_t work_bytes, void* hip_stream) {
    size_t need = 0;
    CHECK(spdnn_linear_grad_bytes(rows, width, cols, offsets != nullptr, experts, type, dout_type, act, transposed, &need));
    CHECK(check_groups(offsets, experts));
    CHECK(check_rows("dout", dout, dout_type, rows, cols, dout_stride, kRead));
    if (act != SPDNN_ACT_NONE) CHECK(check_rows("pre", pre, dout_type, rows, cols, pre_stride, kRead));
    if (dx) {
        CHECK(check_matrix("weight", weight, type, width, cols, transposed, weight_stride, experts, expert_stride, kRead));
        CHECK(check_rows("dx", dx, type, rows, width, dx_stride, kWritten));
    }
    if (dweight) {
        CHECK(check_rows("x", x, type, rows, width, x_stride, kRead));
        CHECK(check_matrix("dweight", dweight, grad_type, width, cols, transposed, dweight_stride, experts, dexpert_stride, kWritten));
    }
    if (dweight || dbias) CHECK(check_output("dweight, dbias", nullptr, grad_type, type));
    if (dbias) CHECK(check_array("dbias", dbias, 0, size_of(grad_type)));
    CHECK(check_work(work, work_bytes, need));
    const hipStream_t s = (hipStream_t)hip_stream;
    const GradWork w(rows, width, cols, offsets != nullptr, experts, type, dout_type, act, transposed);
    const int size = size_of(type);
    float* const parts = (float*)((char*)work + w.d);
    const void* d = dout;
    int64_t d_stride = dout_stride;
    if (w.own_d && rows > 0) {
        d = work;
        d_stride = w.d_stride;
        const int64_t items = (int64_t)rows * ceil_div(cols, 8);
        const dim3 grid((unsigned)std::min(ceil_div(items, 256), kMostGroups));
        with_type(type, [&](auto tt) {
            using T = decltype(tt);
            const auto run = [&](auto td) {
                using D = decltype(td);
                slope_kernel<T, D><<<grid, 256, 0, s>>>((const D*)dout, dout_stride, act == SPDNN_ACT_NONE ? nullptr : (const D*)pre, pre_stride, act, rows, cols, offsets, experts, (T*)work, d_stride);
            };
            if (dout_type == type) run(T{});
            else run(float{});
        });
    }
    if (dx && rows > 0) {
        Product p{};
        p.x = {(const char*)d, d_stride * size, 0};
        p.w = {(const char*)weight, weight_stride * size, expert_stride * size};
        p.offsets = offsets;
        p.rows = rows;
        p.width = cols;
        p.cols = width;
        p.experts = experts;
        p.parts = parts;
        Ending e{};
        e.out = (char*)dx;
        e.out_line = dx_stride * size;
        e.cols = width;
        e.act = SPDNN_ACT_NONE;
        e.out_f32 = type == SPDNN_F32;
        run_product(type, transposed ? Adjacent::L : Adjacent::K, w.dx, p, e, s);
    }
    if (dweight) {
        const Side sx{(const char*)x, x_stride * size, 0}, sd{(const char*)d, d_stride * size, 0};
        WeightGrad p{};
        p.a = transposed ? sd : sx;
        p.b = transposed ? sx : sd;
        p.offsets = offsets;
        p.rows = rows;
        p.m = transposed ? cols : width;
        p.n = transposed ? width : cols;
        p.experts = experts;
        p.mtiles = (int32_t)w.dw.mtiles;
        p.ntiles = (int32_t)w.dw.ntiles;
        p.splits = (int32_t)w.dw.splits;
        p.parts = parts;
        Ending e{};
        e.out = (char*)dweight;
        e.out_line = dweight_stride * size_of(grad_type);
        e.out_set = dexpert_stride * size_of(grad_type);
        e.cols = p.n;
        e.act = SPDNN_ACT_NONE;
        e.out_f32 = grad_type == SPDNN_F32;
        with_type(type, [&](auto tt) {
            using T = decltype(tt);
            weight_grad_kernel<T, 4, 2, 2><<<dim3((unsigned)(w.dw.mtiles * w.dw.ntiles * experts * w.dw.splits)), 256, 0, s>>>(p, e);
            if (w.dw.splits > 1) {
                const int64_t items = (int64_t)experts * p.m * ceil_div(p.n, kEnd);
                weight_grad_join_kernel<T><<<dim3((unsigned)std::min(ceil_div(items, 256), kMostGroups)), 256, 0, s>>>(p, e);
            }
        });
    }
    if (dbias)
        with_type(type, [&](auto tt) {
            using T = decltype(tt);
            const dim3 grid((unsigned)ceil_div(cols, 64), (unsigned)experts, (unsigned)w.bias_splits);
            bias_grad_kernel<T><<<grid, 256, 0, s>>>((const T*)d, d_stride, offsets, rows, cols, (int32_t)w.bias_splits, parts, dbias, grad_type == SPDNN_F32);
            if (w.bias_splits > 1) {
                const int64_t n = (int64_t)experts * cols;
                bias_grad_join_kernel<T><<<dim3((unsigned)ceil_div(n, 256)), 256, 0, s>>>(parts, (int32_t)w.bias_splits, n, dbias, grad_type == SPDNN_F32);
            }
        });
    return launched();
}

}  // extern "C"
