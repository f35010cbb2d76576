// Kernels of layer norm (spdnn_layer_norm, spdnn_layer_norm_grad of include/spdnn.h).  T: type of rows, O: of the output.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "spdnn_vec.h"

#pragma clang fp contract(off)

namespace spdnn {

// Vector `vec` of a row begins at column min(vec * V, width - V), so that none is short; the first `again` of its numbers belong to
// the one before it and take no part in sums.
template <int V>
struct NormAt {
    int col, again;
    __device__ NormAt(int vec, int width) : col(min(vec * V, width - V)), again(vec * V - col) {}
};
template <int V>
__device__ inline void load_param(const void* p, bool f32, const float*, int col, float (&to)[V]) {
    const auto v = load_vec<V>((const float*)p + col);
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = v[i];
}
template <int V, typename T>
__device__ inline void load_param(const void* p, bool f32, const T*, int col, float (&to)[V]) {
    if (f32) {
        load_param<V>(p, true, (const float*)nullptr, col, to);
    } else {
        const auto v = load_vec<V>((const T*)p + col);
#pragma unroll
        for (int i = 0; i < V; ++i) to[i] = (float)v[i];
    }
}

// Sums over the G lanes of a team, the same in all of them: a wave's, or a whole workgroup's by way of LDS.  The order is fixed.
template <int G, int N>
__device__ inline void team_sums(float (&x)[N], float* lds) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = team_sum<64>(x[i]);
    if constexpr (G > 64) {
        constexpr int W = G / 64;
        const int wave = threadIdx.x / 64;
        __syncthreads();  // what the last call left has been read
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) lds[i * W + wave] = x[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = lds[i * W];
#pragma unroll
            for (int w = 1; w < W; ++w) x[i] += lds[i * W + w];
        }
    }
}

struct Norm {
    int64_t rows;
    int32_t width;
    const void* weight;
    const void* bias;
    bool param_f32;
    float eps;
    float2* stats;
    bool past;  // stores that leave nothing in the caches
};

// out[t] = (x[t] - mean) * rstd * weight + bias.  A team of G lanes (a wave, or the workgroup) has a row, U vectors a lane, in
// registers: it is read once, and the variance is that of the differences from the mean, which does not cancel.  (WHOLE: V divides the
// width, and no vector has numbers of the one before it.)  A team takes rows in turn, with the next row under way and the parameters in
// registers.  Bound by memory: 24000 x 4096 bf16 73 us (5.4 TB/s; stores that stay in the caches 78; a wave for every row, which reads the
// parameters for it, 116).
template <typename T, typename O, int V, bool WHOLE, int U, int G, int THREADS>
__global__ __launch_bounds__(THREADS) void layer_norm_kernel(Norm p, const T* __restrict__ x, int64_t x_stride, O* __restrict__ out, int64_t out_stride) {
    __shared__ float lds[G > 64 ? 2 * (G / 64) : 1];
    constexpr int TEAMS = THREADS / G;
    const int lane = threadIdx.x % G;
    const int vecs = (p.width - 1) / V + 1;
    const float inv = 1.0f / (float)p.width;
    int64_t row = (int64_t)blockIdx.x * TEAMS + threadIdx.x / G;
    if (row >= p.rows) return;  // of a whole team
    const auto load = [&](int64_t r, Pack<T, V>(&v)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u * G + lane < vecs) v[u] = load_vec<V>(x + r * x_stride + NormAt<V>(u * G + lane, p.width).col);
    };
    Pack<T, V> v[U], next[U];
    load(row, v);
    float w[U][V], b[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[u][i] = 1.0f;
            b[u][i] = 0.0f;
        }
        if (u * G + lane < vecs) {
            const int col = NormAt<V>(u * G + lane, p.width).col;
            if (p.weight) load_param<V>(p.weight, p.param_f32, (const T*)nullptr, col, w[u]);
            if (p.bias) load_param<V>(p.bias, p.param_f32, (const T*)nullptr, col, b[u]);
        }
    }
    while (true) {
        const int64_t then = row + (int64_t)gridDim.x * TEAMS;
        if (then < p.rows) load(then, next);
        float sum[1] = {0};
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u * G + lane < vecs) {
                const int again = NormAt<V>(u * G + lane, p.width).again;
#pragma unroll
                for (int i = 0; i < V; ++i) sum[0] += !WHOLE && i < again ? 0.0f : (float)v[u][i];
            }
        team_sums<G>(sum, lds);
        const float mean = sum[0] * inv;
        float square[1] = {0};
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u * G + lane < vecs) {
                const int again = NormAt<V>(u * G + lane, p.width).again;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = (float)v[u][i] - mean;
                    square[0] += !WHOLE && i < again ? 0.0f : d * d;
                }
            }
        team_sums<G>(square, lds);
        const float rstd = 1.0f / sqrtf(square[0] * inv + p.eps);
        if (p.stats && lane == 0) p.stats[row] = make_float2(mean, rstd);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u * G + lane < vecs) {
                float y[V];
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = ((float)v[u][i] - mean) * rstd * w[u][i] + b[u][i];
                store_vec<V, O>(out + row * out_stride + NormAt<V>(u * G + lane, p.width).col, rounded_vec<O, V>(y), p.past);
            }
        if (then >= p.rows) break;
        row = then;
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = next[u];
    }
}

// The same for rows that registers do not hold: three passes over the row, the last two from the caches.
template <typename T, typename O>
__global__ __launch_bounds__(1024) void layer_norm_long_kernel(Norm p, const T* __restrict__ x, int64_t x_stride, O* __restrict__ out, int64_t out_stride) {
    __shared__ float lds[32];
    const float inv = 1.0f / (float)p.width;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T* const from = x + row * x_stride;
        float sum[1] = {0};
        for (int c = threadIdx.x; c < p.width; c += 1024) sum[0] += (float)from[c];
        team_sums<1024>(sum, lds);
        const float mean = sum[0] * inv;
        float square[1] = {0};
        for (int c = threadIdx.x; c < p.width; c += 1024) {
            const float d = (float)from[c] - mean;
            square[0] += d * d;
        }
        team_sums<1024>(square, lds);
        const float rstd = 1.0f / sqrtf(square[0] * inv + p.eps);
        if (p.stats && threadIdx.x == 0) p.stats[row] = make_float2(mean, rstd);
        for (int c = threadIdx.x; c < p.width; c += 1024) {
            float y = ((float)from[c] - mean) * rstd;
            if (p.weight) y *= p.param_f32 ? ((const float*)p.weight)[c] : (float)((const T*)p.weight)[c];
            if (p.bias) y += p.param_f32 ? ((const float*)p.bias)[c] : (float)((const T*)p.bias)[c];
            out[row * out_stride + c] = rounded<O>(y);
        }
    }
}

struct NormGrad {
    int64_t rows;
    int32_t width;
    const float2* stats;
    const void* weight;
    bool param_f32;
    float* parts;  // [workgroup][dweight, dbias][width], or null
    bool past;     // stores that leave nothing in the caches
};

// With h = (x - mean) * rstd and g = dout * weight: dx = rstd * (g - mean(g) - h * mean(g * h)) + add, and for a part of the rows
// the sums of dout * h and of dout, column by column.  A team takes rows in turn and keeps its columns' sums in registers; the teams
// of a workgroup are added in order through LDS.  60000 x 1024 bf16 with add 98 us (5.0 TB/s) with the join, 78 of which what is read and
// written asks for.
template <typename T, int V, bool WHOLE, int U, int G, int THREADS>
__global__ __launch_bounds__(THREADS) void layer_norm_grad_kernel(NormGrad p, const T* __restrict__ dout, int64_t dout_stride, const T* __restrict__ x,
                                                                  int64_t x_stride, const T* __restrict__ add, int64_t add_stride, T* __restrict__ dx,
                                                                  int64_t dx_stride) {
    constexpr int TEAMS = THREADS / G;
    __shared__ float lds[G > 64 ? 2 * (G / 64) : 1];
    __shared__ float team_parts[TEAMS > 1 ? (TEAMS - 1) * G * V : 1];
    const int lane = threadIdx.x % G, team = threadIdx.x / G;
    const int vecs = (p.width - 1) / V + 1;
    const float inv = 1.0f / (float)p.width;
    float w[U][V], dw[U][V], db[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[u][i] = 1.0f;
            dw[u][i] = db[u][i] = 0.0f;
        }
        if (p.weight && u * G + lane < vecs) load_param<V>(p.weight, p.param_f32, (const T*)nullptr, NormAt<V>(u * G + lane, p.width).col, w[u]);
    }
    struct Row {
        Pack<T, V> x[U], d[U], add[U];
        float2 st;
    };
    const auto load = [&](int64_t r, Row& to) {
        to.st = p.stats[r];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u * G + lane < vecs) {
                const int col = NormAt<V>(u * G + lane, p.width).col;
                to.x[u] = load_vec<V>(x + r * x_stride + col);
                to.d[u] = load_vec<V>(dout + r * dout_stride + col);
                if (add) to.add[u] = load_vec<V>(add + r * add_stride + col);
            }
    };
    int64_t row = (int64_t)blockIdx.x * TEAMS + team;
    Row now, next;
    if (row < p.rows) load(row, now);
    while (row < p.rows) {
        const int64_t then = row + (int64_t)gridDim.x * TEAMS;
        if (then < p.rows) load(then, next);
        float sums[2] = {0, 0};
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u * G + lane < vecs) {
                const int again = NormAt<V>(u * G + lane, p.width).again;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float h = ((float)now.x[u][i] - now.st.x) * now.st.y, d = (float)now.d[u][i];
                    const float g = d * w[u][i];
                    sums[0] += !WHOLE && i < again ? 0.0f : g;
                    sums[1] += !WHOLE && i < again ? 0.0f : g * h;
                    dw[u][i] += d * h;
                    db[u][i] += d;
                }
            }
        team_sums<G>(sums, lds);
        const float a = sums[0] * inv, b = sums[1] * inv;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u * G + lane < vecs) {
                float y[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float h = ((float)now.x[u][i] - now.st.x) * now.st.y;
                    y[i] = now.st.y * ((float)now.d[u][i] * w[u][i] - a - h * b);
                    if (add) y[i] += (float)now.add[u][i];
                }
                store_vec<V, T>(dx + row * dx_stride + NormAt<V>(u * G + lane, p.width).col, rounded_vec<T, V>(y), p.past);
            }
        row = then;
        now = next;
    }
    if (!p.parts) return;
    float* const own = p.parts + (int64_t)blockIdx.x * 2 * p.width;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float s[V];
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] = which ? db[u][i] : dw[u][i];
            if constexpr (TEAMS > 1) {
                __syncthreads();
                if (team)
#pragma unroll
                    for (int i = 0; i < V; ++i) team_parts[(team - 1) * (G * V) + i * G + lane] = s[i];
                __syncthreads();
                if (team) continue;
                for (int t = 0; t < TEAMS - 1; ++t)
#pragma unroll
                    for (int i = 0; i < V; ++i) s[i] += team_parts[t * (G * V) + i * G + lane];
            }
            if (u * G + lane < vecs) {
                Pack<float, V> to;
#pragma unroll
                for (int i = 0; i < V; ++i) to[i] = s[i];
                store_vec<V, float>(own + (int64_t)which * p.width + NormAt<V>(u * G + lane, p.width).col, to, false);
            }
        }
}

// The same for rows that registers do not hold: dx with two passes over the row; the columns' sums by workgroups of their own.
template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_grad_long_kernel(NormGrad p, const T* __restrict__ dout, int64_t dout_stride, const T* __restrict__ x,
                                                                    int64_t x_stride, const T* __restrict__ add, int64_t add_stride, T* __restrict__ dx,
                                                                    int64_t dx_stride) {
    __shared__ float lds[32];
    const float inv = 1.0f / (float)p.width;
    const auto weight = [&](int c) { return !p.weight ? 1.0f : p.param_f32 ? ((const float*)p.weight)[c] : (float)((const T*)p.weight)[c]; };
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T* const xr = x + row * x_stride;
        const T* const dr = dout + row * dout_stride;
        const float2 st = p.stats[row];
        float sums[2] = {0, 0};
        for (int c = threadIdx.x; c < p.width; c += 1024) {
            const float g = (float)dr[c] * weight(c);
            sums[0] += g;
            sums[1] += g * (((float)xr[c] - st.x) * st.y);
        }
        team_sums<1024>(sums, lds);
        const float a = sums[0] * inv, b = sums[1] * inv;
        for (int c = threadIdx.x; c < p.width; c += 1024) {
            const float h = ((float)xr[c] - st.x) * st.y;
            float y = st.y * ((float)dr[c] * weight(c) - a - h * b);
            if (add) y += (float)add[row * add_stride + c];
            dx[row * dx_stride + c] = rounded<T>(y);
        }
    }
}
template <typename T>
__global__ __launch_bounds__(256) void layer_norm_columns_kernel(NormGrad p, const T* __restrict__ dout, int64_t dout_stride, const T* __restrict__ x,
                                                                 int64_t x_stride) {
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < p.width; c += (int64_t)gridDim.x * 256) {
        float dw = 0, db = 0;
        for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
            const float2 st = p.stats[row];
            const float d = (float)dout[row * dout_stride + c];
            dw += d * (((float)x[row * x_stride + c] - st.x) * st.y);
            db += d;
        }
        float* const own = p.parts + (int64_t)blockIdx.y * 2 * p.width;
        own[c] = dw;
        own[p.width + c] = db;
    }
}

// The parts added up: a workgroup has 64 columns of dweight and dbias side by side, its 16 waves every 16th part, added in order.
template <typename D>
__global__ __launch_bounds__(1024) void layer_norm_join_kernel(const float* __restrict__ parts, int32_t count, int32_t width, D* dweight, D* dbias) {
    __shared__ float sums[16][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t all = 2 * (int64_t)width;
    for (int64_t c0 = (int64_t)blockIdx.x * 64; c0 < all; c0 += (int64_t)gridDim.x * 64) {
        const int64_t c = c0 + lane;
        float sum = 0;
        if (c < all)
#pragma unroll 4
            for (int i = wave; i < count; i += 16) sum += parts[i * all + c];
        sums[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && c < all) {
            for (int w = 1; w < 16; ++w) sum += sums[w][lane];
            D* const to = c < width ? dweight : dbias;
            if (to) to[c < width ? c : c - width] = rounded<D>(sum);
        }
        __syncthreads();
    }
}

}  // namespace spdnn
