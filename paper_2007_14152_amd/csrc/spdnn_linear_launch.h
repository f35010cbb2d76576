// Launches of the dense products' kernels for one type of rows; a translation unit for each (spdnn_linear_f32.hip ...).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "spdnn_linear_kernels.h"
#include "spdnn_linear_plan.h"

namespace spdnn {

template <typename T>
void launch_product(const Plan& c, Adjacent adj, const Product& p, const Ending& e, hipStream_t s);
// dout is of T or of float.
template <typename T>
void launch_slope(bool dout_f32, const void* dout, int64_t dout_stride, const void* pre, int64_t pre_stride, int act, int32_t rows, int32_t cols,
                  const int32_t* offsets, int32_t experts, void* d, int64_t d_stride, hipStream_t s);
// With dbias of d before it is rounded: chunks of `each` rows, teams of `lanes` lanes.  d may be null.
template <typename T>
void launch_slope_sums(bool dout_f32, const void* dout, int64_t dout_stride, const void* pre, int64_t pre_stride, int act, int32_t rows, int32_t cols,
                       const int32_t* offsets, int32_t experts, void* d, int64_t d_stride, int32_t each, int32_t lanes, float* parts, void* dbias, bool f32, hipStream_t s);
template <typename T>
void launch_weight_grad(const Plan& c, const WeightGrad& p, const Ending& e, hipStream_t s);
// Both at once: tiles of 64 x 64 that go straight to LDS, without splits.
template <typename T>
void launch_grads(const Plan& cx, Adjacent adj, const Product& x, const Ending& ex, const Plan& cw, const WeightGrad& w, const Ending& ew, hipStream_t s);
template <typename T>
void launch_bias_grad(const void* d, int64_t d_stride, const int32_t* offsets, int32_t rows, int32_t cols, int32_t experts, int32_t splits, float* parts,
                      void* dbias, bool f32, hipStream_t s);

}  // namespace spdnn
