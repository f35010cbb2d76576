// Host side of the dense products (spdnn_linear, spdnn_linear_grad of include/spdnn.h): argument checks and launches.
#include "../../include/spdnn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "spdnn_check.h"
#include "spdnn_error.h"
#include "spdnn_linear_launch.h"

namespace {

using namespace spdnn;

static_assert(kPartsAlign == kAlign);

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
int check_output(const char* what, int32_t out_type, int32_t type) {
    if (out_type != type && out_type != SPDNN_F32) return fail(SPDNN_EINVAL, "%s is of x's type or SPDNN_F32", what);
    return SPDNN_OK;
}

int check_tiles(const Plan& p, int32_t sets) {
    if ((double)p.mtiles * p.ntiles * p.splits * sets > (double)most_tiles(p.few ? 0 : p.bm)) return fail(SPDNN_EINVAL, "sizes too large: too many tiles");
    return SPDNN_OK;
}
// The most work memory that any alignment asks for.
int most_parts(int32_t rows, int32_t k, int32_t cols, bool grouped, int32_t experts, int32_t type, size_t* parts) {
    *parts = 0;
    for (const Adjacent adj : {Adjacent::K, Adjacent::L})
        for (const bool dma : {false, true}) {
            const Plan p = plan_product(rows, k, cols, grouped, experts, type, dma, adj);
            CHECK(check_tiles(p, 1));
            *parts = std::max(*parts, p.parts);
        }
    return SPDNN_OK;
}

// Whether an operand can go straight to LDS: tiles within reach of 32-bit offsets, rows of k that do not overlap.  And lines that are all one row
// in memory have to end with a word: the range check leaves out half a word for every one of them, and only the last line's is stored.
bool dma_side(const Side& s, Adjacent adj, int32_t along, int32_t type) {
    if (adj == Adjacent::K && s.line == 0 && (int64_t)along * size_of(type) % 4 != 0) return false;
    return s.line <= kDmaSpan / 256 - 256 && (adj == Adjacent::K || s.line >= (int64_t)along * size_of(type));
}

Plan plan_of(int32_t type, Adjacent adj, Product& p) {
    if (p.rows == 1) p.x.line = (int64_t)p.width * size_of(type);  // whatever the stride of one row is
    const bool dma = dma_side(p.x, Adjacent::K, p.width, type) && dma_side(p.w, adj, adj == Adjacent::K ? p.width : p.cols, type);
    const Plan c = plan_product(p.rows, p.width, p.cols, p.offsets != nullptr, p.experts, type, dma, adj);
    p.mtiles = (int32_t)c.mtiles;
    p.ntiles = (int32_t)c.ntiles;
    p.splits = (int32_t)c.splits;
    p.per_split = c.per_split;
    return c;
}

// Work memory of the gradients: d in the rows' type where dout is not that already, and parts, which the three steps use in turn.
struct GradWork {
    bool own_d;
    int64_t d_stride;  // elements
    size_t d, bytes;
    int64_t bias_splits;
    int64_t slope_rows;   // of a workgroup that adds up d's columns beside
    int32_t slope_lanes;  // that have a row's columns, eight each
};
int grad_work(int32_t rows, int32_t width, int32_t cols, bool grouped, int32_t experts, int32_t type, int32_t dout_type, int32_t act, bool transposed,
              GradWork* w) {
    w->own_d = act != SPDNN_ACT_NONE || dout_type != type;
    w->d_stride = ceil_div(cols, 16) * 16;
    w->d = w->own_d ? aligned((size_t)rows * w->d_stride * size_of(type)) : 0;
    w->bias_splits = std::max<int64_t>(1, std::min(1024 / (ceil_div(cols, 64) * experts), ceil_div(rows, experts) / 32));
    size_t parts = 0;
    CHECK(most_parts(rows, cols, width, grouped, experts, type, &parts));
    for (const bool dma : {false, true}) {
        const Plan p = plan_grad(rows, transposed ? cols : width, transposed ? width : cols, experts, type, dma);
        CHECK(check_tiles(p, experts));
        parts = std::max(parts, p.parts + (p.splits > 1 ? aligned((size_t)p.splits * experts * cols * sizeof(float)) : 0));
    }
    // Chunks of rows: up to four workgroups a CU and 512 chunks, whose parts are added up; a row to four for each team as long as CUs are idle, but
    // no more than an expert's on average, as a chunk takes experts one after the other.  Up to eight rows a team are one chunk, without parts.
    w->slope_lanes = 64;
    while (w->slope_lanes > 1 && w->slope_lanes / 2 * 8 >= cols) w->slope_lanes /= 2;
    const int64_t teams = 256 / w->slope_lanes, blocks = ceil_div(cols, w->slope_lanes * 8);
    int64_t least = std::max(teams, std::min(4 * teams, ceil_div(rows * blocks, 256)));
    if (grouped) least = std::min(least, std::max<int64_t>(1, ceil_div(rows, experts)));
    else if (rows <= 8 * teams) least = 8 * teams;
    w->slope_rows = std::max({least, ceil_div(rows * blocks, 1024), ceil_div(rows, 512)});
    w->slope_rows = std::min<int64_t>(w->slope_rows, INT32_MAX);
    if (w->own_d && type != SPDNN_F32) parts = std::max(parts, aligned((size_t)(ceil_div(rows, w->slope_rows) + experts) * cols * sizeof(float)));
    if (w->bias_splits > 1) parts = std::max(parts, aligned((size_t)w->bias_splits * experts * cols * sizeof(float)));
    w->bytes = w->d + parts;
    return SPDNN_OK;
}

int check_act(int32_t act) {
    if (act < SPDNN_ACT_NONE || act > SPDNN_ACT_SILU) return fail(SPDNN_EINVAL, "act must be one of SPDNN_ACT_NONE ... SPDNN_ACT_SILU");
    return SPDNN_OK;
}

}  // namespace

extern "C" {

int spdnn_linear_bytes(int32_t rows, int32_t width, int32_t cols, int32_t grouped, int32_t experts, int32_t type, size_t* bytes) {
    if (!bytes) return fail(SPDNN_EINVAL, "bytes is NULL");
    CHECK(check_sizes(rows, width, cols, experts, type));
    return most_parts(rows, width, cols, grouped != 0, experts, type, bytes);
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
    CHECK(check_output("out", out_type, type));
    CHECK(check_rows("out", out, out_type, rows, cols, out_stride, kWritten));
    if (pre) CHECK(check_rows("pre", pre, out_type, rows, cols, pre_stride, kWritten));
    if (add) CHECK(check_rows("add", add, out_type, rows, cols, add_stride, kRead));
    if (bias) {
        CHECK(check_output("bias", bias_type, type));
        CHECK(check_array("bias", bias, 0, size_of(bias_type)));
    }
    CHECK(check_work(work, work_bytes, need));
    if (rows == 0) return SPDNN_OK;
    const int size = size_of(type), out_size = size_of(out_type);
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
    const Adjacent adj = transposed ? Adjacent::K : Adjacent::L;
    const Plan c = plan_of(type, adj, p);
    with_type(type, [&](auto tt) { launch_product<decltype(tt)>(c, adj, p, e, (hipStream_t)hip_stream); });
    return launched();
}

int spdnn_linear_grad_bytes(int32_t rows, int32_t width, int32_t cols, int32_t grouped, int32_t experts, int32_t type, int32_t dout_type, int32_t act,
                            int32_t transposed, size_t* bytes) {
    if (!bytes) return fail(SPDNN_EINVAL, "bytes is NULL");
    CHECK(check_sizes(rows, width, cols, experts, type));
    CHECK(check_output("dout", dout_type, type));
    CHECK(check_act(act));
    GradWork w;
    CHECK(grad_work(rows, width, cols, grouped != 0, experts, type, dout_type, act, transposed != 0, &w));
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
    if (dweight || dbias) CHECK(check_output("dweight, dbias", grad_type, type));
    if (dbias) CHECK(check_array("dbias", dbias, 0, size_of(grad_type)));
    CHECK(check_work(work, work_bytes, need));
    const hipStream_t s = (hipStream_t)hip_stream;
    GradWork w;
    CHECK(grad_work(rows, width, cols, offsets != nullptr, experts, type, dout_type, act, transposed != 0, &w));
    const int size = size_of(type);
    float* const parts = (float*)((char*)work + w.d);
    const void* d = dout;
    int64_t d_stride = dout_stride;
    // dbias of 16-bit rows is the sum of d as it is in 32 bits.
    const bool sums = w.own_d && rows > 0 && dbias && type != SPDNN_F32;
    void* const bias_left = sums ? nullptr : dbias;
    if (sums) {
        with_type(type, [&](auto tt) {
            launch_slope_sums<decltype(tt)>(dout_type == SPDNN_F32, dout, dout_stride, act == SPDNN_ACT_NONE ? nullptr : pre, pre_stride, act, rows, cols, offsets, experts,
                                            dx || dweight ? work : nullptr, w.d_stride, (int32_t)w.slope_rows, w.slope_lanes, parts, dbias, grad_type == SPDNN_F32, s);
        });
    }
    if (w.own_d && rows > 0) {
        d = work;
        d_stride = w.d_stride;
        if (!sums) with_type(type, [&](auto tt) {
            launch_slope<decltype(tt)>(dout_type == SPDNN_F32, dout, dout_stride, act == SPDNN_ACT_NONE ? nullptr : pre, pre_stride, act, rows, cols, offsets, experts, work,
                                       d_stride, s);
        });
    }
    const bool has_x = dx && rows > 0;
    const Adjacent adj = transposed ? Adjacent::L : Adjacent::K;
    Product px{};
    Ending ex{};
    Plan cx{};
    if (has_x) {
        Product& p = px;
        p.x = {(const char*)d, d_stride * size, 0};
        p.w = {(const char*)weight, weight_stride * size, expert_stride * size};
        p.offsets = offsets;
        p.rows = rows;
        p.width = cols;
        p.cols = width;
        p.experts = experts;
        p.parts = parts;
        Ending& e = ex;
        e.out = (char*)dx;
        e.out_line = dx_stride * size;
        e.cols = width;
        e.act = SPDNN_ACT_NONE;
        e.out_f32 = type == SPDNN_F32;
        cx = plan_of(type, adj, p);
    }
    const auto run_x = [&] {
        if (has_x) with_type(type, [&](auto tt) { launch_product<decltype(tt)>(cx, adj, px, ex, s); });
    };
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
        p.parts = parts;
        const bool dma = dma_side(p.a, Adjacent::L, p.m, type) && dma_side(p.b, Adjacent::L, p.n, type);
        const Plan c = plan_grad(rows, p.m, p.n, experts, type, dma);
        p.mtiles = (int32_t)c.mtiles;
        p.ntiles = (int32_t)c.ntiles;
        p.splits = (int32_t)c.splits;
        p.bias_parts = (float*)((char*)parts + c.parts);
        p.dbias = bias_left;
        p.bias_f32 = grad_type == SPDNN_F32;
        p.d_is_a = transposed != 0;
        p.sorted = offsets && experts <= 64 && rows / experts >= 256;
        Ending e{};
        e.out = (char*)dweight;
        e.out_line = dweight_stride * size_of(grad_type);
        e.out_set = dexpert_stride * size_of(grad_type);
        e.cols = p.n;
        e.act = SPDNN_ACT_NONE;
        e.out_f32 = grad_type == SPDNN_F32;
        const auto small = [](const Plan& q) { return q.dma && !q.few && q.bm == 64 && q.splits == 1; };
        if (has_x && small(cx) && small(c) && cx.mtiles * cx.ntiles + c.mtiles * c.ntiles * experts + 8 <= most_tiles(64)) {
            with_type(type, [&](auto tt) { launch_grads<decltype(tt)>(cx, adj, px, ex, c, p, e, s); });
        } else {
            run_x();
            with_type(type, [&](auto tt) { launch_weight_grad<decltype(tt)>(c, p, e, s); });
        }
        return launched();
    }
    run_x();
    if (bias_left) {
        with_type(type, [&](auto tt) {
            launch_bias_grad<decltype(tt)>(d, d_stride, offsets, rows, cols, experts, (int32_t)w.bias_splits, parts, bias_left, grad_type == SPDNN_F32, s);
        });
    }
    return launched();
}

}  // extern "C"
