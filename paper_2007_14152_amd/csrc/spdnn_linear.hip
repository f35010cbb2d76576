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

constexpr int64_t kMostGroups = 1 << 20;
// Tiles of a launch: HIP takes less than 2^32 threads, of which tiles of 64 and 128 have 256, others up to 512.
int64_t most_tiles(int b) { return (b == 64 || b == 128 ? 1 << 24 : 1 << 23) - 1; }

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

constexpr int64_t kGroupsWanted = 256;     // workgroups that the CUs ask for at least
constexpr size_t kMostParts = 256 << 20;  // bytes that sums in parts may take

// How long n tiles of b x b take with `k` k each, us.  A CU holds four workgroups with tiles of 64, two of 128, one of 256; `us` is a
// round of one to four of them on every CU for 4096 k, `ends` what a round takes besides.  Measured with K = 64 to 4096; what is left over
// of full rounds takes what its own number of workgroups does.  longest: k of the longest tile, which no order of the others hides.
double cost(int b, int64_t n, double k, double longest, int32_t type) {
    struct Row {
        int per_cu;
        double us[4], ends;
    };
    static const Row k16[3] = {{4, {26, 35, 44, 52}, 3.5}, {2, {49, 73}, 7}, {1, {104}, 10}};
    static const Row k32[3] = {{4, {93, 149, 209, 269}, 4}, {2, {275, 491}, 9}, {1, {966}, 18}};
    const Row& r = (type == SPDNN_F32 ? k32 : k16)[b == 64 ? 0 : b == 128 ? 1 : 2];
    const int64_t full = 256 * r.per_cu, rest = n % full;
    const double rounds = n / full * r.us[r.per_cu - 1] + (rest ? r.us[(rest - 1) / 256] : 0.0);
    const int64_t beside = std::min<int64_t>(r.per_cu, ceil_div(std::max<int64_t>(n, 1), 256));
    return std::max(rounds * k, r.us[beside - 1] * longest) / 4096 + r.ends * ceil_div(n, full);
}
// The tile and the number of parts of k with which `tiles(b)` tiles take least.  Parts are written and read once more, out_bytes a part,
// which a join does in 9 us and at 4 TB/s.  uneven: how many times the k of all on average the longest tile may have.  (777 x 1500 x 1021 floats: 110 us
// with tiles of 128, 40 with tiles of 64.  dW of 12 experts of 10007 rows in all, 1500 x 777 floats: 532 us with tiles of 128.)
template <typename F>
void choose(F tiles, int64_t steps, double uneven, size_t out_bytes, int32_t type, bool dma, int* b, int64_t* splits) {
    const double k = (double)steps * step_of(type);
    double best = 1e300;
    for (const int tile : {256, 128, 64}) {
        if (!dma && tile != 128) continue;
        for (int64_t s = 1; s <= 64; s *= 2) {
            if (s > 1 && (steps / s < 4 || s * out_bytes > kMostParts)) break;
            if (best < 1e300 && tiles(tile) * s > most_tiles(tile)) break;
            const double us = cost(tile, tiles(tile) * s, k / s, uneven * k / s, type) + (s > 1 ? 9.0 + 2.0 * s * out_bytes / 4e6 : 0.0);
            if (us < best) {
                best = us;
                *b = tile;
                *splits = s;
            }
        }
    }
}

Plan plan_product(int32_t rows, int32_t k, int32_t cols, bool grouped, int32_t experts, int32_t type, bool dma, Adjacent adj) {
    Plan p{};
    p.dma = dma;
    const int64_t sets = grouped ? std::max<int64_t>(1, std::min(experts, rows)) : 1;
    const int64_t steps = ceil_div(k, step_of(type));
    const auto tiles = [&](int bm, int bn) { return (grouped ? rows / bm + sets : ceil_div(rows, bm)) * ceil_div(cols, bn); };  // that have rows
    const int64_t each = ceil_div(rows, sets);
    // (Few rows: W's bytes are what counts.  In 32 bits the matrix instructions do, from 32 rows on.)
    if (dma && each <= (type == SPDNN_F32 ? 32 : grouped ? 48 : 128) && tiles(16, 64) <= most_tiles(0)) {
        p.few = each <= (grouped ? 8 : 16) ? 1 : each <= (grouped ? 20 : 32) ? 2 : 4;
        p.bm = 16 * p.few;
        // Tiles of 16 columns where those of 64 leave CUs idle; but columns of adjacent k, or k that are not many: 32 bytes of a row of
        // W at a time come from memory at two thirds of the rate.  One row: 4096 x 1024 6.2 us with 16 columns, 9.0 with 64; 4096 x 4096
        // 9.8 and 10.5 (k adjacent 6.0 and 10.0); 16384 x 4096 33.2 and, with k in four splits, 29.3 (k adjacent 21.4).
        p.narrow = tiles(p.bm, 64) < kGroupsWanted && (adj == Adjacent::K || steps < 128 || grouped);
        p.bn = p.narrow ? 16 : 64;
        p.splits = std::max<int64_t>(1, std::min(kGroupsWanted / std::max<int64_t>(tiles(p.bm, p.bn), 1), steps / 32));
    } else {
        choose([&](int b) { return tiles(b, b); }, steps, 1.0, (size_t)rows * cols * sizeof(float), type, dma, &p.bm, &p.splits);
        p.bn = p.bm;
    }
    p.mtiles = grouped ? std::min<int64_t>(rows, rows / p.bm + experts + 1) : ceil_div(rows, p.bm);
    p.ntiles = ceil_div(cols, p.bn);
    p.per_split = ceil_div(steps, p.splits) * step_of(type);
    p.splits = ceil_div(k, p.per_split);
    p.parts = p.splits > 1 ? aligned((size_t)p.splits * rows * cols * sizeof(float)) : 0;
    p.alone = type != SPDNN_F32 && tiles(p.bm, p.bn) * p.splits <= kGroupsWanted;
    return p;
}
Plan plan_grad(int32_t rows, int32_t m, int32_t n, int32_t experts, int32_t type, bool dma) {
    Plan p{};
    p.dma = dma;
    const auto tiles = [&](int b) { return ceil_div(m, b) * ceil_div(n, b) * experts; };
    const int64_t steps = std::max<int64_t>(1, ceil_div(ceil_div(rows, experts), step_of(type)));
    choose(tiles, steps, experts > 1 ? 3.0 : 1.0, (size_t)experts * m * n * sizeof(float), type, dma, &p.bm, &p.splits);
    p.bn = p.bm;
    p.mtiles = ceil_div(m, p.bm);
    p.ntiles = ceil_div(n, p.bn);
    p.parts = p.splits > 1 ? aligned((size_t)p.splits * experts * m * n * sizeof(float)) : 0;
    p.alone = type != SPDNN_F32 && tiles(p.bm) * p.splits <= kGroupsWanted;
    return p;
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
    // Chunks of rows: up to four workgroups a CU and 256 chunks, whose parts are added up; a row to eight for each team as long as CUs are idle, but
    // no more than two experts' on average, which a chunk takes one after the other.
    w->slope_lanes = 64;
    while (w->slope_lanes > 1 && w->slope_lanes / 2 * 8 >= cols) w->slope_lanes /= 2;
    const int64_t teams = 256 / w->slope_lanes, blocks = ceil_div(cols, w->slope_lanes * 8);
    const int64_t least = std::min(std::max(teams, std::min(8 * teams, ceil_div(rows * blocks, 256))), std::max<int64_t>(1, 2 * ceil_div(rows, experts)));
    w->slope_rows = std::max({least, ceil_div(rows * blocks, 1024), ceil_div(rows, 256)});
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
    CHECK(check_output("dout", nullptr, dout_type, type));
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
    if (dweight || dbias) CHECK(check_output("dweight, dbias", nullptr, grad_type, type));
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
