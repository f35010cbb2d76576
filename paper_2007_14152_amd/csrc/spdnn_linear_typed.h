// The definitions of spdnn_linear_launch.h, for the translation units that instantiate them.
#pragma once
#include "spdnn_linear_launch.h"

namespace spdnn {

constexpr int64_t kMostLoopGroups = 1 << 20;  // workgroups of a launch whose workgroups take turns
inline unsigned loop_groups(int64_t items) { return (unsigned)std::max<int64_t>(1, std::min((items + 255) / 256, kMostLoopGroups)); }

template <typename T, Adjacent ADJ, int R>
void launch_few(const Plan& c, dim3 grid, const Product& p, const Ending& e, hipStream_t s) {
    constexpr int KW = R == 4 ? 2 : 4, NARROW_KW = R == 4 ? 4 : 8;
    if (c.narrow) linear_short_kernel<T, ADJ, R, 1, NARROW_KW, 2><<<grid, NARROW_KW * 64, 0, s>>>(p, e);
    else linear_short_kernel<T, ADJ, R, 4, KW, 2><<<grid, KW * 64, 0, s>>>(p, e);
}
template <typename T, Adjacent ADJ>
void launch_stored(const Plan& c, const Product& p, const Ending& e, hipStream_t s) {
    const dim3 grid((unsigned)(c.mtiles * c.ntiles * c.splits));
    if (c.few == 1) launch_few<T, ADJ, 1>(c, grid, p, e, s);
    else if (c.few == 2) launch_few<T, ADJ, 2>(c, grid, p, e, s);
    else if (c.few == 4) launch_few<T, ADJ, 4>(c, grid, p, e, s);
    else if (c.bm == 256) linear_kernel<T, ADJ, Large, true><<<grid, 512, 0, s>>>(p, e);
    else if (c.bm == 64 && c.alone) linear_kernel<T, ADJ, Small<3>, true><<<grid, 256, 0, s>>>(p, e);
    else if (c.bm == 64) linear_kernel<T, ADJ, Small<2>, true><<<grid, 256, 0, s>>>(p, e);
    else if (c.dma && c.alone) linear_kernel<T, ADJ, Middle<3>, true><<<grid, 256, 0, s>>>(p, e);
    else if (c.dma) linear_kernel<T, ADJ, Middle<2>, true><<<grid, 256, 0, s>>>(p, e);
    else linear_kernel<T, ADJ, Middle<2>, false><<<grid, 256, 0, s>>>(p, e);
}
template <typename T>
void launch_product(const Plan& c, Adjacent adj, const Product& p, const Ending& e, hipStream_t s) {
    if (adj == Adjacent::K) launch_stored<T, Adjacent::K>(c, p, e, s);
    else launch_stored<T, Adjacent::L>(c, p, e, s);
    if (c.splits > 1) linear_join_kernel<T><<<loop_groups((int64_t)p.rows * p.cols), 256, 0, s>>>(p, e);
}

template <typename T>
void launch_slope(bool dout_f32, const void* dout, int64_t dout_stride, const void* pre, int64_t pre_stride, int act, int32_t rows, int32_t cols,
                  const int32_t* offsets, int32_t experts, void* d, int64_t d_stride, hipStream_t s) {
    const unsigned groups = loop_groups((int64_t)rows * ((cols - 1) / 8 + 1));
    if (dout_f32)
        slope_kernel<T, float><<<groups, 256, 0, s>>>((const float*)dout, dout_stride, (const float*)pre, pre_stride, act, rows, cols, offsets, experts, (T*)d, d_stride);
    else
        slope_kernel<T, T><<<groups, 256, 0, s>>>((const T*)dout, dout_stride, (const T*)pre, pre_stride, act, rows, cols, offsets, experts, (T*)d, d_stride);
}

template <typename T>
void launch_slope_sums(bool dout_f32, const void* dout, int64_t dout_stride, const void* pre, int64_t pre_stride, int act, int32_t rows, int32_t cols,
                       const int32_t* offsets, int32_t experts, void* d, int64_t d_stride, int32_t each, int32_t lanes, float* parts, void* dbias, bool f32, hipStream_t s) {
    const dim3 grid((unsigned)((cols - 1) / (lanes * 8) + 1), (unsigned)((rows - 1) / each + 1));
    if (!offsets && grid.y == 1) parts = nullptr;
    if (dout_f32)
        slope_sums_kernel<T, float><<<grid, 256, 0, s>>>((const float*)dout, dout_stride, (const float*)pre, pre_stride, act, rows, cols, offsets, experts, (T*)d, d_stride, each, lanes, parts, dbias, f32);
    else
        slope_sums_kernel<T, T><<<grid, 256, 0, s>>>((const T*)dout, dout_stride, (const T*)pre, pre_stride, act, rows, cols, offsets, experts, (T*)d, d_stride, each, lanes, parts, dbias, f32);
    if (!parts) return;
    slope_join_kernel<T><<<dim3((unsigned)std::min((cols - 1) / 64 + 1, 1 << 16), (unsigned)experts), 1024, 0, s>>>(parts, rows, cols, offsets, experts, each, dbias, f32);
}

template <typename T>
void launch_weight_grad(const Plan& c, const WeightGrad& p, const Ending& e, hipStream_t s) {
    const dim3 grid((unsigned)(c.mtiles * c.ntiles * p.experts * c.splits));
    if (c.bm == 256) weight_grad_kernel<T, Large, true><<<grid, 512, 0, s>>>(p, e);
    else if (c.bm == 64 && c.alone) weight_grad_kernel<T, Small<3>, true><<<grid, 256, 0, s>>>(p, e);
    else if (c.bm == 64) weight_grad_kernel<T, Small<2>, true><<<grid, 256, 0, s>>>(p, e);
    else if (c.dma && c.alone) weight_grad_kernel<T, Middle<3>, true><<<grid, 256, 0, s>>>(p, e);
    else if (c.dma) weight_grad_kernel<T, Middle<2>, true><<<grid, 256, 0, s>>>(p, e);
    else weight_grad_kernel<T, Middle<2>, false><<<grid, 256, 0, s>>>(p, e);
    if (c.splits > 1) {
        weight_grad_join_kernel<T><<<loop_groups((int64_t)p.experts * p.m * p.n), 256, 0, s>>>(p, e);
        const int64_t n = (int64_t)p.experts * (p.d_is_a ? p.m : p.n);
        if (p.dbias) bias_grad_join_kernel<T><<<(unsigned)((n + 255) / 256), 256, 0, s>>>(p.bias_parts, c.splits, n, p.dbias, p.bias_f32);
    }
}

template <typename T>
void launch_grads(const Plan& cx, Adjacent adj, const Product& x, const Ending& ex, const Plan& cw, const WeightGrad& w, const Ending& ew, hipStream_t s) {
    const int64_t first = (cx.mtiles * cx.ntiles + 7) / 8 * 8;
    const dim3 grid((unsigned)(first + cw.mtiles * cw.ntiles * w.experts));
    if (adj == Adjacent::K) grads_kernel<T, Adjacent::K, Small<2>><<<grid, 256, 0, s>>>(x, ex, w, ew, (int)first);
    else grads_kernel<T, Adjacent::L, Small<2>><<<grid, 256, 0, s>>>(x, ex, w, ew, (int)first);
}

template <typename T>
void launch_bias_grad(const void* d, int64_t d_stride, const int32_t* offsets, int32_t rows, int32_t cols, int32_t experts, int32_t splits, float* parts,
                      void* dbias, bool f32, hipStream_t s) {
    const dim3 grid((unsigned)std::min((cols - 1) / 64 + 1, 1 << 22), (unsigned)experts, (unsigned)splits);
    bias_grad_kernel<T><<<grid, 256, 0, s>>>((const T*)d, d_stride, offsets, rows, cols, splits, parts, dbias, f32);
    const int64_t n = (int64_t)experts * cols;
    if (splits > 1) bias_grad_join_kernel<T><<<(unsigned)((n + 255) / 256), 256, 0, s>>>(parts, splits, n, dbias, f32);
}

}  // namespace spdnn

#define SPDNN_LINEAR_LAUNCHES(T)                                                                                                                       \
    template void spdnn::launch_product<T>(const Plan&, Adjacent, const Product&, const Ending&, hipStream_t);                                         \
    template void spdnn::launch_slope<T>(bool, const void*, int64_t, const void*, int64_t, int, int32_t, int32_t, const int32_t*, int32_t, void*,      \
                                         int64_t, hipStream_t);                                                                                        \
    template void spdnn::launch_slope_sums<T>(bool, const void*, int64_t, const void*, int64_t, int, int32_t, int32_t, const int32_t*, int32_t, void*, \
                                              int64_t, int32_t, int32_t, float*, void*, bool, hipStream_t);                                            \
    template void spdnn::launch_weight_grad<T>(const Plan&, const WeightGrad&, const Ending&, hipStream_t);                                            \
    template void spdnn::launch_grads<T>(const Plan&, Adjacent, const Product&, const Ending&, const Plan&, const WeightGrad&, const Ending&, hipStream_t); \
    template void spdnn::launch_bias_grad<T>(const void*, int64_t, const int32_t*, int32_t, int32_t, int32_t, int32_t, float*, void*, bool, hipStream_t);
