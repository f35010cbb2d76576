// Kernels of the row operators (spdnn_embed ... spdnn_combine_grad of include/spdnn.h): rows by token id, the choice of
// experts, rows sorted by expert and back, and the gradients.  T, S: types of rows (float, __bf16, _Float16).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "spdnn_vec.h"

#pragma clang fp contract(off)

namespace spdnn {

constexpr int kRowThreads = 256;

// --- tiles of rows ----------------------------------------------------------
//
// Kernels that only move rows take them as vectors of V elements, 16 bytes of the wider type, or of one element where a row
// has less than V.  The last vector of a row ends with the row, so that none is short: where V does not divide the width it
// covers elements of the one before it again.  A workgroup's tile is `per` whole rows next to each other, so that rows of any
// length keep all lanes busy (vectors are numbered through the tile), or `slab` vectors of one row where rows are long; lanes
// beyond its end take its last vector once more.  What is covered twice is computed and stored twice, alike: there is no
// branch around a load or a store, and none waits for another.
struct Tiles {
    int64_t rows;
    int32_t width;
    int32_t vecs;    // vectors of a row
    int32_t per;     // rows of a tile
    int32_t slab;    // vectors of a row in a tile
    uint32_t magic;  // ceil(2^32 / slab): quotients by slab > 1 for what is less than 2^16
    bool past;       // stores that leave nothing in the caches
    bool past_in;    // and loads (of the input that is as large as all that)
};
constexpr int kTileVecs = 4096;  // at most, of a tile

// f(places of U vectors of the tile) until the tile is done; f has the loads of all of them to overlap.
struct At {
    int64_t row;
    int32_t col;
};
template <int V, int U, typename F>
__device__ inline void each_vec(const Tiles& g, F f) {
    for (int64_t r0 = (int64_t)blockIdx.x * g.per; r0 < g.rows; r0 += (int64_t)gridDim.x * g.per)
        for (int vec0 = blockIdx.y * g.slab; vec0 < g.vecs; vec0 += gridDim.y * g.slab) {
            const int rows = (int)min((int64_t)g.per, g.rows - r0);
            const int items = rows * g.slab;
            for (int i0 = threadIdx.x; i0 < items; i0 += U * kRowThreads) {
                At at[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const uint32_t i = min(i0 + u * kRowThreads, items - 1);
                    const uint32_t r = g.per == 1 ? 0 : g.slab == 1 ? i : __umulhi(i, g.magic);
                    const int vec = min(vec0 + (int)(i - r * g.slab), g.vecs - 1);
                    at[u].row = r0 + r;
                    at[u].col = min(vec * V, g.width - V);
                }
                f(at);
            }
        }
}

constexpr int kEmbedVecs = 4;  // vectors that a lane has under way

// out[t] = scale * table[ids[t]].  Bound by memory: 24000 rows of 4096 bf16 (264 MB) 47 us, 5.6 TB/s.  The loads of a lane's four
// ids and then of its four vectors are under way together; one row takes 2 us, most of it the two loads that wait for each other.
template <typename T, typename S, typename I, int V>
__global__ __launch_bounds__(kRowThreads) void embed_kernel(Tiles g, const T* __restrict__ table, int64_t table_stride, uint32_t vocab,
                                                            const I* __restrict__ ids, float scale, S* __restrict__ out, int64_t out_stride) {
    each_vec<V, kEmbedVecs>(g, [&](const At (&at)[kEmbedVecs]) {
        I id[kEmbedVecs];
        Pack<T, V> x[kEmbedVecs];
#pragma unroll
        for (int u = 0; u < kEmbedVecs; ++u) id[u] = ids[at[u].row];
#pragma unroll
        for (int u = 0; u < kEmbedVecs; ++u) {
            const bool in = id[u] >= 0 && id[u] < (I)vocab;
            x[u] = load_vec<V>(table + (in ? (int64_t)id[u] : 0) * table_stride + at[u].col);
        }
        Pack<S, V> y[kEmbedVecs];
#pragma unroll
        for (int u = 0; u < kEmbedVecs; ++u) {
            const bool in = id[u] >= 0 && id[u] < (I)vocab;
            float to[V];
#pragma unroll
            for (int i = 0; i < V; ++i) to[i] = in ? scale * (float)x[u][i] : 0.0f;
            y[u] = rounded_vec<S, V>(to);
        }
        store_all<V, S>(y, g.past, [&](int u) { return out + at[u].row * out_stride + at[u].col; });
    });
}

// --- choice of experts ------------------------------------------------------

// A logit (with bias) and its column as one number whose order is that of the choice: the larger logit first, then the lower
// column.  It is the logit in 64 bits, of which a 32-bit float leaves the last 29 free: the column goes there, turned round
// where a larger last part makes a larger number.  +inf becomes a finite number beyond all floats, -0 becomes 0, and what is
// not open (-inf, a NaN) the smallest number of all, whose last bits are set already.
constexpr uint32_t kColumnBits = 0x3ff;
static_assert(SPDNN_MAX_EXPERTS <= kColumnBits + 1);
__device__ inline double closed() { return -1.7976931348623157e308; }
__device__ inline double rank_of(float r, int col) {
    const double d = fmin(fmax((double)(r + 0.0f), closed()), 0x1p1000);
    const int hi = __double2hiint(d);
    return __hiloint2double(hi, __double2loint(d) | (int)((uint32_t)col ^ kColumnBits ^ ((uint32_t)(hi >> 31) & kColumnBits)));
}
__device__ inline int column_of(double d) {  // -1: none
    if (d == closed()) return -1;
    return (int)(((uint32_t)__double2loint(d) & kColumnBits) ^ (__double2hiint(d) >= 0 ? kColumnBits : 0u));
}

// Networks of compare-exchanges: K numbers in descending order, K a power of two.
__device__ inline void order_two(double& a, double& b) {
    const double x = fmax(a, b), y = fmin(a, b);
    a = x;
    b = y;
}
template <int K>
__device__ inline void order_bitonic(double (&a)[K]) {  // a rises, then falls, or the other way round
#pragma unroll
    for (int m = K / 2; m; m /= 2)
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (!(i & m)) order_two(a[i], a[i | m]);
}
template <int K>
__device__ inline void order_all(double (&a)[K]) {  // odd-even merges: 19 exchanges for 8 numbers, where bitonic ones take 24
#pragma unroll
    for (int n = 1; n < K; n *= 2)
#pragma unroll
        for (int m = n; m; m /= 2)
#pragma unroll
            for (int i = m % n; i + m < K; i += 2 * m)
#pragma unroll
                for (int j = 0; j < m; ++j)
                    if (i + j + m < K && (i + j) / (2 * n) == (i + j + m) / (2 * n)) order_two(a[i + j], a[i + j + m]);
}
// The first K of a and b, both in order.
template <int K>
__device__ inline void keep_first(double (&a)[K], const double (&b)[K]) {
#pragma unroll
    for (int i = 0; i < K; ++i) a[i] = fmax(a[i], b[K - 1 - i]);
    order_bitonic(a);
}
template <int G, int K, int STEP = 1>
__device__ inline void keep_first_of_team(double (&a)[K]) {
    if constexpr (STEP < G) {
        double b[K];
#pragma unroll
        for (int i = 0; i < K; ++i) b[i] = other<STEP>(a[i]);
        keep_first(a, b);
        keep_first_of_team<G, K, 2 * STEP>(a);
    }
}

__device__ inline float log_sigmoid(float x) { return fminf(x, 0.0f) - log1pf(expf(-fabsf(x))); }
__device__ inline float sigmoid(float x) {  // no overflow on the way: small values stay apart from zero
    const float e = expf(-fabsf(x)), r = 1.0f / (1.0f + e);
    return x >= 0.0f ? r : e * r;
}

// Weights of the chosen experts before the scale: lane j < k of a team has the logit of slot j, valid says whether the slot has
// an expert.  Softmax over the open experts: top and total are the largest of their logits and the sum of exp(logit - top).
template <int G>
__device__ inline float slot_weight(float l, bool valid, int score, int normalise, float top, float total) {
    if (normalise) {
        const float x = score == SPDNN_SIGMOID ? log_sigmoid(l) : l;
        const float m = team_max<G>(valid ? x : -INFINITY);
        const float e = valid ? expf(x - m) : 0.0f;
        const float sum = team_sum<G>(e);
        return valid ? e / sum : 0.0f;
    }
    if (!valid) return 0.0f;
    return score == SPDNN_SIGMOID ? sigmoid(l) : expf(l - top) / total;
}

// V logits of a row from column col on, minus infinity beyond its end.
template <int V, typename T>
__device__ inline void load_logits(const T* __restrict__ row, int col, int experts, float (&l)[V]) {
    if (col + V <= experts) {
        const Pack<T, V> x = load_vec<V>(row + col);
#pragma unroll
        for (int i = 0; i < V; ++i) l[i] = (float)x[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) l[i] = col + i < experts ? (float)row[col + i] : -INFINITY;
    }
}
// What the choice goes by: logits l of columns from col on, with their bias.
template <int V>
__device__ inline void add_bias(const float* __restrict__ bias, int col, int experts, const float (&l)[V], float (&r)[V]) {
    if (bias) {
        float b[V];
        load_logits<V>(bias, col, experts, b);
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = l[i] + b[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = l[i];
    }
}

// The largest open logit of a team's row, and the sum of exp(logit - the largest) over the open ones.
// (The two-instruction exp rounds x log2(e) at the size of x and makes zero of what is below 2^-126: weights that a float holds would
// be lost.  expf instead, 60000 rows, a call in a graph: 256 floats, 8 experts 24.4 -> 27.3 us, its gradient 25.3 -> 25.4; 64 bf16, 2
// experts 7.4 -> 8.3, its gradient 6.8 -> 7.7.)
template <int V, int G, typename T>
__device__ inline void softmax_sums(const T* __restrict__ row, const float* __restrict__ bias, int lane, int columns, float& top, float& total) {
    top = -INFINITY;
    total = 0.0f;
    for (int col = lane * V; col < columns; col += G * V) {
        float l[V], r[V];
        load_logits<V>(row, col, columns, l);
        add_bias<V>(bias, col, columns, l, r);
#pragma unroll
        for (int i = 0; i < V; ++i) top = r[i] > -INFINITY ? fmaxf(top, l[i]) : top;
    }
    top = team_max<G>(top);
    for (int col = lane * V; col < columns; col += G * V) {
        float l[V], r[V];
        load_logits<V>(row, col, columns, l);
        add_bias<V>(bias, col, columns, l, r);
#pragma unroll
        for (int i = 0; i < V; ++i) total += r[i] > -INFINITY ? expf(l[i] - top) : 0.0f;
    }
    total = team_sum<G>(total);
}

// A team of G lanes takes a row, kLogits columns a lane at a time.  Every lane keeps the first K of its columns in order (K: k
// rounded up), the lanes' lists are merged pairwise, and lane j weighs slot j.  No round per expert, no branch on values.
// 60000 rows of 256 floats, 8 experts: 16.9 us (3.9 TB/s), 13 us of vector instructions: 1104 for the eight rows of a wave, of
// which 150 order the lanes' columns, 170 merge lists of a lane, 170 those of lanes (a round per expert: 149 us in all).
constexpr int kLogits = 8;
template <typename T, int K, int G>
__global__ __launch_bounds__(kRowThreads) void route_kernel(const T* __restrict__ logits, int64_t stride, int rows, int experts, int k,
                                                            const float* __restrict__ bias, const uint8_t* __restrict__ keep, int score, int normalise,
                                                            float scale, int32_t* __restrict__ chosen, float* __restrict__ weight) {
    static_assert(K <= G);
    constexpr int V = K > kLogits ? K : kLogits, kTeams = kRowThreads / G;
    const int lane = threadIdx.x % G, team = threadIdx.x / G;
    const bool all = score == SPDNN_SOFTMAX && !normalise;  // the weights need all open experts
    for (int64_t t0 = (int64_t)blockIdx.x * kTeams; t0 < rows; t0 += (int64_t)gridDim.x * kTeams) {
        const int64_t t = min(t0 + team, (int64_t)rows - 1);  // teams beyond the rows repeat the last one
        const T* row = logits + t * stride;
        const int columns = !keep || keep[t] ? experts : 0;
        double first[K];
        for (int col = lane * V, turn = 0; turn == 0 || col < columns; col += G * V, ++turn) {
            float l[V], r[V];
            load_logits<V>(row, col, columns, l);
            add_bias<V>(bias, col, columns, l, r);
#pragma unroll
            for (int c = 0; c < V; c += K) {
                double some[K];
#pragma unroll
                for (int i = 0; i < K; ++i) some[i] = rank_of(r[c + i], col + c + i);
                order_all(some);
                if (turn == 0 && c == 0) {
#pragma unroll
                    for (int i = 0; i < K; ++i) first[i] = some[i];
                } else {
                    keep_first(first, some);
                }
            }
        }
        keep_first_of_team<G>(first);
        float top = 0.0f, total = 0.0f;
        if (all) softmax_sums<V, G>(row, bias, lane, columns, top, total);
        double mine = closed();
#pragma unroll
        for (int i = 0; i < K; ++i) mine = lane == i && i < k ? first[i] : mine;
        const int e = column_of(mine);
        const float l = e >= 0 ? (float)row[e] : 0.0f;
        const float w = slot_weight<G>(l, e >= 0, score, normalise, top, total);
        if (lane < k) {
            chosen[t * k + lane] = e;
            weight[t * k + lane] = scale * w;
        }
    }
}

// A team of G lanes takes a row: the slots' weights and their gradient, then all of the row but for the chosen experts, then
// those.  Softmax over the open experts needs all of the row; a row of at most G * kLogits logits is read once and stays in
// registers as exp(logit - top).  60000 rows of 64 bf16, 2 experts: 7.7 us, its 15.6 MB would take 2.5; launch, two loads that wait
// for each other, exp and five sums over the team are the rest.
template <typename T, int G>
__global__ __launch_bounds__(kRowThreads) void route_grad_kernel(const float* __restrict__ dweight, const T* __restrict__ logits, int64_t stride,
                                                                 const int32_t* __restrict__ chosen, int rows, int experts, int k,
                                                                 const float* __restrict__ bias, int score, int normalise, float scale,
                                                                 T* __restrict__ dlogits, int64_t dstride) {
    constexpr int V = kLogits, kTeams = kRowThreads / G;
    const int lane = threadIdx.x % G, team = threadIdx.x / G;
    const bool all = score == SPDNN_SOFTMAX && !normalise, one = experts <= G * V;
    for (int64_t t0 = (int64_t)blockIdx.x * kTeams; t0 < rows; t0 += (int64_t)gridDim.x * kTeams) {
        const int64_t t = min(t0 + team, (int64_t)rows - 1);
        const T* row = logits + t * stride;
        T* to = dlogits + t * dstride;
        float x[V];
        if (all && one) load_logits<V>(row, lane * V, experts, x);
        const int e = lane < k ? chosen[t * k + lane] : -1;
        const bool valid = e >= 0 && e < experts;
        const float g = valid ? scale * dweight[t * k + lane] : 0.0f;
        const float l = valid ? (float)row[e] : 0.0f;
        const bool any = team_max<G>(valid ? 1.0f : 0.0f) > 0.0f;
        float top = 0.0f, total = 0.0f;
        if (all && one) {
            float r[V];
            add_bias<V>(bias, lane * V, experts, x, r);
            top = -INFINITY;
#pragma unroll
            for (int i = 0; i < V; ++i) top = r[i] > -INFINITY ? fmaxf(top, x[i]) : top;
            top = team_max<G>(top);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[i] = r[i] > -INFINITY ? expf(x[i] - top) : 0.0f;
                total += x[i];
            }
            total = team_sum<G>(total);
        } else if (all) {
            softmax_sums<V, G>(row, bias, lane, experts, top, total);
        }
        const float w = slot_weight<G>(l, valid, score, normalise, top, total);
        const float mean = team_sum<G>(g * w), back = any ? -mean / total : 0.0f;
        float d;  // of the slot's logit
        if (normalise) d = w * (g - mean) * (score == SPDNN_SIGMOID ? sigmoid(-l) : 1.0f);
        else d = score == SPDNN_SIGMOID ? g * w * sigmoid(-l) : w * (g - mean);
        for (int col = lane * V; col < experts; col += G * V) {
            float y[V] = {};
            if (all && one) {
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = any ? x[i] * back : 0.0f;
            } else if (all) {
                float r[V];
                load_logits<V>(row, col, experts, x);
                add_bias<V>(bias, col, experts, x, r);
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = any && r[i] > -INFINITY ? expf(x[i] - top) * back : 0.0f;
            }
            if (col + V <= experts) {
                store_vec<V, T>(to + col, rounded_vec<T, V>(y), false);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (col + i < experts) to[col + i] = rounded<T>(y[i]);
            }
        }
        // The wave's stores to one address keep their order, whichever lanes they come from.
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (valid) to[e] = rounded<T>(d);
    }
}

// --- rows by expert ---------------------------------------------------------

// A stable counting sort of pairs (or of ids, a digit of their bits at a time) by a number d < bins, in two launches: the pairs
// are cut into chunks, a workgroup per chunk counts (count_kernel), then every workgroup adds up the counts of all chunks for
// itself, which is cheaper than a launch for it, and places its chunk's pairs (place_kernel).  A chunk is cut into a segment per
// wave; a wave takes 64 pairs at a time, whose rank among equals comes from ballots, a bit of d at a time: no pair's position
// depends on which wave was first.  One chunk needs no count.  Few workgroups and one thing waiting for another: 48000 pairs of 64
// experts 4.6 + 6.4 us, 60000 ids 512 bins at a time 3 to 4 + 9.3.  (Counts of the next digit by atomics from the launch before it
// saved a launch and cost 20 us: frequent ids meet in them.)
constexpr int kSortAhead = 4;  // pairs that a lane has under way
constexpr int kSortWaves = 8, kSortThreads = 64 * kSortWaves;
constexpr int kLeastChunk = kSortAhead * kSortThreads;
constexpr int kMostChunks = 128;  // more pairs than these hold make the chunks longer
constexpr int kMostBins = 1024;

// What is sorted: `at` loads a pair, `digit` is its number d (-1: it has no place).
struct PairItems {
    using Item = int32_t;
    const int32_t* chosen;
    int experts;
    __device__ Item at(int64_t p) const { return chosen[p]; }
    __device__ int digit(Item e) const { return e >= 0 && e < experts ? e : -1; }
};

template <int WAVES, int BINS = kMostBins>
struct SortLds {
    int32_t start[WAVES][BINS];
    int32_t total[BINS];
    int32_t wave_sum[WAVES];
    int32_t end;  // behind the last position
};

// Rows first .. last - 1 of a matrix whose elements become zero, by workgroups that a launch has to spare.
struct Clear {
    char* base;
    int64_t stride;  // bytes
    int32_t bytes;   // of a row, 16 at least
    int64_t first, last;
    bool past;
};
__device__ inline void clear(const Clear& c, int group, int groups) {
    constexpr int kRows = 16;
    const int vecs = (c.bytes - 1) / 16 + 1;
    for (int64_t r0 = c.first + (int64_t)group * kRows; r0 < c.last; r0 += (int64_t)groups * kRows) {
        const int rows = (int)min((int64_t)kRows, c.last - r0);
        for (int64_t i = threadIdx.x; i < (int64_t)rows * vecs; i += blockDim.x) {
            const int64_t r = i / vecs;
            const int at = min((int)(i - r * vecs) * 16, c.bytes - 16);
            store_vec<8, uint16_t>(reinterpret_cast<uint16_t*>(c.base + (r0 + r) * c.stride + at), Pack<uint16_t, 8>{}, c.past);
        }
    }
}

// Workgroups beyond the chunks clear.
template <typename D>
__global__ __launch_bounds__(kSortThreads) void count_kernel(D in, int64_t n, int log_chunk, int chunks, int bins, int32_t* __restrict__ table, Clear c) {
    __shared__ int32_t count[kMostBins];
    if ((int)blockIdx.x >= chunks) {
        clear(c, blockIdx.x - chunks, gridDim.x - chunks);
        return;
    }
    for (int e = threadIdx.x; e < bins; e += kSortThreads) count[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x << log_chunk, last = min(first + (1ll << log_chunk), n);
    for (int64_t p0 = first + threadIdx.x; p0 < last; p0 += kSortAhead * kSortThreads) {
        typename D::Item x[kSortAhead];
#pragma unroll
        for (int a = 0; a < kSortAhead; ++a) x[a] = in.at(min(p0 + a * kSortThreads, last - 1));
#pragma unroll
        for (int a = 0; a < kSortAhead; ++a) {
            const int d = in.digit(x[a]);
            if (d >= 0 && p0 + a * kSortThreads < last) atomicAdd(&count[d], 1);
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < bins; e += kSortThreads) table[(int64_t)blockIdx.x * bins + e] = count[e];
}

// to(pair, item, position) for every pair of chunk `me`, position -1 without a digit; offsets (may be NULL): first positions of
// the bins, and the end.  table: the counts of `chunks` chunks, or NULL if there is only this one.
template <int WAVES, int BINS, typename D, typename F>
__device__ inline void place_chunk(D in, int64_t first, int64_t last, int bins, const int32_t* __restrict__ table, int chunks, int me,
                                   SortLds<WAVES, BINS>& lds, int32_t* __restrict__ offsets, F to) {
    constexpr int A = kSortAhead, kThreads = 64 * WAVES;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t part = ((last - first + kThreads - 1) / kThreads) * 64;
    const int64_t mine = min(first + wave * part, last), end = min(mine + part, last);
    typename D::Item x[A];  // the wave's pairs, A * 64 at a time; where there are no more, they are loaded once
    const auto load = [&](int64_t p0) {
#pragma unroll
        for (int a = 0; a < A; ++a) x[a] = in.at(min(p0 + a * 64 + lane, end - 1));
    };
    if (mine < end) load(mine);
    for (int e = threadIdx.x; e < bins; e += kThreads)
        for (int w = 0; w < WAVES; ++w) lds.start[w][e] = 0;
    __syncthreads();
    for (int64_t p0 = mine; p0 < end; p0 += A * 64) {
        if (p0 != mine) load(p0);
#pragma unroll
        for (int a = 0; a < A; ++a) {
            const int d = in.digit(x[a]);
            if (d >= 0 && p0 + a * 64 + lane < end) atomicAdd(&lds.start[wave][d], 1);
        }
    }
    __syncthreads();
    // bin e's pairs in all chunks, and in start[w][e] where wave w's first one goes, within the bin
    for (int e = threadIdx.x; e < bins; e += kThreads) {
        int before = 0, total = 0;
        if (table) {
            constexpr int B = 16;
            for (int c0 = 0; c0 < chunks; c0 += B) {
                int y[B];
#pragma unroll
                for (int c = 0; c < B; ++c) y[c] = table[(int64_t)min(c0 + c, chunks - 1) * bins + e];
#pragma unroll
                for (int c = 0; c < B; ++c) {
                    total += c0 + c < chunks ? y[c] : 0;
                    before += c0 + c < me ? y[c] : 0;
                }
            }
        }
        for (int w = 0; w < WAVES; ++w) {
            const int y = lds.start[w][e];
            lds.start[w][e] = before;
            before += y;
        }
        lds.total[e] = table ? total : before;
    }
    __syncthreads();
    // a thread's bins next to each other: their sum, the sums before it, then each bin's first position
    constexpr int kEach = BINS / kThreads;
    static_assert(BINS % kThreads == 0);
    int many[kEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int e = threadIdx.x * kEach + i;
        many[i] = e < bins ? lds.total[e] : 0;
        sum += many[i];
    }
    int upto = sum;
    for (int m = 1; m < 64; m <<= 1) {
        const int o = __shfl_up(upto, m);
        if (lane >= m) upto += o;
    }
    if (lane == 63) lds.wave_sum[wave] = upto;
    __syncthreads();
    int base = upto - sum;
    for (int w = 0; w < wave; ++w) base += lds.wave_sum[w];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int e = threadIdx.x * kEach + i;
        if (e < bins) {
            if (offsets) offsets[e] = base;
            for (int w = 0; w < WAVES; ++w) lds.start[w][e] += base;
            base += many[i];
            if (e == bins - 1) {
                lds.end = base;
                if (offsets) offsets[bins] = base;
            }
        }
    }
    __syncthreads();
    const int bits = 32 - __clz(bins - 1 | 1);
    volatile int32_t* start = lds.start[wave];  // read and written by this wave alone, in the order written here
    for (int64_t p0 = mine; p0 < end; p0 += A * 64) {
        if (end - mine > A * 64) load(p0);
#pragma unroll
        for (int a = 0; a < A; ++a) {
            if (p0 + a * 64 >= end) break;
            const int64_t p = p0 + a * 64 + lane;
            const int d = p < end ? in.digit(x[a]) : -1;
            uint64_t same = __ballot(d >= 0);
            for (int b = 0; b < bits; ++b) {
                const uint64_t set = __ballot(d >> b & 1);
                same &= d >> b & 1 ? set : ~set;
            }
            int at = -1;
            if (d >= 0) {
                at = start[d] + __popcll(same & ((1ull << lane) - 1));
                if (lane == 63 - __clzll(same)) start[d] = at + 1;  // the last of its kind leaves where the next one goes
            }
            if (p < end) to(p, x[a], at);
        }
    }
}

__global__ __launch_bounds__(kSortThreads) void expert_place_kernel(PairItems in, int64_t n, int log_chunk, const int32_t* __restrict__ table,
                                                                    int chunks, int32_t* __restrict__ offsets, int32_t* __restrict__ place) {
    __shared__ SortLds<kSortWaves> lds;
    const int64_t first = (int64_t)blockIdx.x << log_chunk;
    place_chunk(in, first, min(first + (1ll << log_chunk), n), in.experts, table, chunks, blockIdx.x, lds, blockIdx.x == 0 ? offsets : nullptr,
                [&](int64_t p, int32_t, int at) { place[p] = at; });
}

// --- gradient of a table ----------------------------------------------------

// Ids of tokens with the tokens they belong to, `vocab` for those outside the table, sorted by a digit of their bits at a time: from
// the caller's ids, or from what an earlier digit has sorted.
struct Token {
    uint32_t key;
    int32_t token;
};
template <typename I>
struct IdItems {
    using Item = Token;
    const I* ids;
    uint32_t vocab;
    int shift, mask;
    __device__ Item at(int64_t p) const {
        const I id = ids[p];
        return {id >= 0 && id < (I)vocab ? (uint32_t)id : vocab, (int32_t)p};
    }
    __device__ int digit(Item x) const { return (int)(x.key >> shift) & mask; }
};
struct KeyItems {
    using Item = Token;
    const uint32_t* keys;
    const int32_t* tokens;
    int shift, mask;
    __device__ Item at(int64_t p) const { return {keys[p], tokens[p]}; }
    __device__ int digit(Item x) const { return (int)(x.key >> shift) & mask; }
};

// Sorted by one more digit; workgroups beyond the chunks clear.
template <typename D>
__global__ __launch_bounds__(kSortThreads) void key_place_kernel(D in, int64_t n, int log_chunk, int chunks, const int32_t* __restrict__ table,
                                                                 uint32_t* __restrict__ keys, int32_t* __restrict__ tokens, Clear c) {
    __shared__ SortLds<kSortWaves> lds;
    if ((int)blockIdx.x >= chunks) {
        clear(c, blockIdx.x - chunks, gridDim.x - chunks);
        return;
    }
    const int64_t first = (int64_t)blockIdx.x << log_chunk;
    place_chunk(in, first, min(first + (1ll << log_chunk), n), in.mask + 1, table, chunks, blockIdx.x, lds, nullptr, [&](int64_t, Token x, int at) {
        keys[at] = x.key;
        tokens[at] = x.token;
    });
}

// V elements of a row of the gradient from the sums of dout; the first `again` of them are left to the vector before this one.
template <typename S, int V>
__device__ inline void put_grad(S* __restrict__ to, int again, const float (&sum)[V], float scale, bool accumulate, bool past) {
    float x[V];
    Pack<S, V> old = {};
    if (accumulate) old = load_vec<V>(to);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = fmaf(scale, sum[i], (float)old[i]);
    const Pack<S, V> y = rounded_vec<S, V>(x);
    if (again == 0) {
        store_vec<V, S>(to, y, past);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i >= again) to[i] = y[i];
    }
}

// The sum of dout's rows tokens[first] .. tokens[last - 1], columns from col on, in that order, kAhead of them under way.
constexpr int kAhead = 8;
template <int V, typename T, typename F>
__device__ inline void add_rows(const T* __restrict__ dout, int64_t dout_stride, int col, int first, int last, F token, float (&sum)[V]) {
    for (int i0 = first; i0 < last; i0 += kAhead) {
        Pack<T, V> x[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) x[a] = load_vec<V>(dout + (int64_t)token(min(i0 + a, last - 1)) * dout_stride + col);
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] = i0 + a < last ? sum[i] + (float)x[a][i] : sum[i];
    }
}

// dtable[v] = [dtable[v] +] scale * sum of the dout[t] with ids[t] == v.
//
// Few ids, one launch and no sort.  n * slabs workgroups have a token each: the one that is the first with its id finds the others
// in order and adds their rows, a quarter of them per wave, 64 vectors of columns at a time (shared out over the slabs).  Those
// before them (none if accumulate) clear `per` rows each, but for rows that an id has.  777 rows of 1500 floats into 10007 rows:
// 17.0 us, of which clearing 60 MB takes 11.5 (a fill 9.3); with those that clear behind or in turn 20.  A workgroup's work grows
// with the ids: 1000 of them into 1000 rows of 1024 12 us, where the sort takes 19, but 4096 49 us, where it takes 26.  Those are ids by
// Zipf's law.  Where a few ids have most of the tokens, few workgroups add: 1024 tokens, rows of 4096 (bf16 to floats), one id 103 us
// (sorted 15), two ids 58 (15); 256 tokens of one id into 10007 rows 32 (40).  The rule does not see that, the host has no ids.
constexpr int kFewIds = 1024, kMostRowsToClear = 1024;
template <typename T, typename S, typename I, int V>
__global__ __launch_bounds__(kRowThreads) void embed_grad_short_kernel(const T* __restrict__ dout, int64_t dout_stride, const I* __restrict__ ids, int n,
                                                                     int vocab, int width, int slabs, int per, float scale, bool accumulate,
                                                                     S* __restrict__ dtable, int64_t dtable_stride, bool past) {
    constexpr int kWaves = kRowThreads / 64, kRounds = kFewIds / kRowThreads;
    __shared__ uint64_t with_id[kRounds * kWaves];
    __shared__ int32_t tokens[kFewIds];
    __shared__ float sums[kWaves][64][V];
    __shared__ bool there[kMostRowsToClear];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, adders = n * slabs;
    const int vecs = (width - 1) / V + 1;
    I id[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) id[r] = n > 0 ? ids[min(r * kRowThreads + (int)threadIdx.x, n - 1)] : (I)-1;
    const int clearers = (int)gridDim.x - adders, number = (int)blockIdx.x - clearers;
    if (number < 0) {
        for (int64_t v0 = (int64_t)blockIdx.x * per; v0 < vocab; v0 += (int64_t)clearers * per) {
            const int rows = (int)min((int64_t)per, vocab - v0);
            __syncthreads();
            for (int r = threadIdx.x; r < rows; r += kRowThreads) there[r] = false;
            __syncthreads();
#pragma unroll
            for (int r = 0; r < kRounds; ++r)
                if (id[r] >= (I)v0 && id[r] < (I)(v0 + rows)) there[(int)(id[r] - (I)v0)] = true;
            __syncthreads();
            for (int64_t i = threadIdx.x; i < (int64_t)rows * vecs; i += kRowThreads) {
                const int r = (int)(i / vecs), vec = (int)(i - (int64_t)r * vecs);
                if (!there[r]) store_vec<V, S>(dtable + (v0 + r) * dtable_stride + min(vec * V, width - V), Pack<S, V>{}, past);
            }
        }
        return;
    }
    const int t = number % n, slab = number / n;
    const I v = ids[t];
    if (v < 0 || v >= (I)vocab) return;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const uint64_t mine = __ballot(id[r] == v && r * kRowThreads + (int)threadIdx.x < n);
        if (lane == 0) with_id[r * kWaves + wave] = mine;
    }
    __syncthreads();
    int many = 0, first = -1;
#pragma unroll
    for (int i = 0; i < kRounds * kWaves; ++i) {
        const uint64_t some = with_id[i];
        if (first < 0 && some) first = i * 64 + __ffsll((unsigned long long)some) - 1;
        if (i % kWaves == wave && (some >> lane & 1)) tokens[many + __popcll(some & ((1ull << lane) - 1))] = i * 64 + lane;
        many += __popcll(some);
    }
    if (first != t) return;
    __syncthreads();
    const int each = (many + kWaves - 1) / kWaves, from = min(wave * each, many), to = min(from + each, many);
    for (int v0 = slab * 64; v0 < vecs; v0 += slabs * 64) {
        const int vec = min(v0 + lane, vecs - 1), col = min(vec * V, width - V);
        float sum[V] = {};
        add_rows<V>(dout, dout_stride, col, from, to, [&](int a) { return tokens[a]; }, sum);
        if (many > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) sums[wave][lane][i] = sum[i];
            __syncthreads();
        }
        if (wave == 0 && v0 + lane < vecs) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (many > 1) sum[i] = (sum[i] + sums[1][lane][i]) + (sums[2][lane][i] + sums[3][lane][i]);
            put_grad<S, V>(dtable + (int64_t)v * dtable_stride + col, vec * V - col, sum, scale, accumulate, past);
        }
    }
}

// Many ids, sorted: the order is cut into pieces of kPiece places, and a team of L lanes adds up a piece, L * V columns of it.
// Where an id's places lie in one piece, its row is done.  Otherwise the piece's part of the sum goes to the work memory, and
// embed_grad_join_kernel adds the parts up: long runs of a frequent id are shared out, and no atomics decide an order.
// parts: two rows of `width` floats per piece: for the id that comes in from the piece before, and for the one that goes on.
// 60000 rows of 1024 bf16 into 65536 rows of floats: 104 us for 389 MB (a copy of as much: 62), of which the sort takes 36 and
// clears 128 MB beside, this kernel 54 (6 TB/s with what it writes twice) and the join 10.  Pieces of 16, 32 and 64 places: 53 + 19,
// 55 + 11 and 60 + 7 us.
constexpr int kPiece = 32;
struct GradOrder {
    const uint32_t* keys;
    const int32_t* tokens;
    int32_t n;
    uint32_t vocab;
    // the first place whose key is not less than v
    __device__ int lower(uint32_t v) const {
        int lo = 0, hi = n;
        while (lo < hi) {
            const int mid = lo + (hi - lo) / 2;
            if (keys[mid] < v) lo = mid + 1;
            else hi = mid;
        }
        return lo;
    }
};

template <typename T, typename S, int V, int L>
__device__ inline void add_pieces(const GradOrder& o, const T* __restrict__ dout, int64_t dout_stride, int width, float scale, bool accumulate,
                                  S* __restrict__ dtable, int64_t dtable_stride, float* __restrict__ parts, int group, int groups, int slab, int slabs) {
    constexpr int kTeams = kRowThreads / L;
    __shared__ uint32_t keys[kTeams][kPiece + 2];  // from the place before the piece to the one behind it; vocab where there is none
    __shared__ int32_t tokens[kTeams][kPiece];
    const int lane = threadIdx.x % L, team = threadIdx.x / L;
    const int vecs = (width - 1) / V + 1;
    const int pieces = (o.n - 1) / kPiece + 1;
    for (int64_t piece0 = (int64_t)group * kTeams; piece0 < pieces; piece0 += (int64_t)groups * kTeams) {
        __syncthreads();
        for (int i = threadIdx.x; i < kTeams * (kPiece + 2); i += kRowThreads) {
            const int in = i % (kPiece + 2);
            const int64_t at = (piece0 + i / (kPiece + 2)) * kPiece + in - 1;
            keys[i / (kPiece + 2)][in] = at >= 0 && at < o.n ? o.keys[at] : o.vocab;
            if (in >= 1 && in <= kPiece) tokens[i / (kPiece + 2)][in - 1] = at < o.n ? o.tokens[at] : 0;
        }
        __syncthreads();
        const uint32_t* key = keys[team] + 1;
        int many = 0;  // of the piece's places have an id: the others are the last of all
        for (int a = 0; a < kPiece; ++a) many += key[a] < o.vocab;
        const int64_t piece = piece0 + team;
        for (int vec = slab * L + lane; vec < vecs && many > 0; vec += slabs * L) {
            const int col = min(vec * V, width - V), again = vec * V - col;
            float sum[V] = {};
            bool in = key[-1] == key[0];  // the run at hand began in the piece before
            for (int a0 = 0; a0 < many; a0 += kAhead) {
                Pack<T, V> x[kAhead];
#pragma unroll
                for (int a = 0; a < kAhead; ++a) x[a] = load_vec<V>(dout + (int64_t)tokens[team][min(a0 + a, many - 1)] * dout_stride + col);
#pragma unroll
                for (int a = 0; a < kAhead; ++a) {
                    if (a0 + a >= many) break;
#pragma unroll
                    for (int i = 0; i < V; ++i) sum[i] += (float)x[a][i];
                    const uint32_t v = key[a0 + a];
                    const bool on = v == key[a0 + a + 1];
                    if (on && a0 + a + 1 < kPiece) continue;
                    if (!in && !on) {
                        put_grad<S, V>(dtable + (int64_t)v * dtable_stride + col, again, sum, scale, accumulate, false);
                    } else {
                        float* to = parts + (piece * 2 + (in ? 0 : 1)) * width + col;
                        store_vec<V, float>(to, rounded_vec<float, V>(sum), false);
                    }
                    in = false;
#pragma unroll
                    for (int i = 0; i < V; ++i) sum[i] = 0.0f;
                }
            }
        }
    }
}

// Zeros in the first `end` rows, in those of ids that do not occur.
template <typename S, int V>
__device__ inline void clear_rows(const GradOrder& o, uint32_t end, int width, int per, S* __restrict__ dtable, int64_t dtable_stride, bool past, int group, int groups) {
    __shared__ bool there[kRowThreads];
    const int vecs = (width - 1) / V + 1;
    for (int64_t v0 = (int64_t)group * per; v0 < end; v0 += (int64_t)groups * per) {
        const int rows = (int)min((int64_t)per, (int64_t)end - v0);
        __syncthreads();
        if ((int)threadIdx.x < rows) {
            const int at = o.lower((uint32_t)v0 + threadIdx.x);
            there[threadIdx.x] = at < o.n && o.keys[at] == (uint32_t)v0 + threadIdx.x;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < rows * vecs; i += kRowThreads) {
            const int r = i / vecs, vec = i - r * vecs;
            if (!there[r]) store_vec<V, S>(dtable + (v0 + r) * dtable_stride + min(vec * V, width - V), Pack<S, V>{}, past);
        }
    }
}

// adders * slabs workgroups add pieces, a slab of columns each, the others (none if accumulate) clear those of the first `end` rows
// that have no id, `per` at a time; in turn as long as there are both, for one sort waits for loads and the other stores.  (3000 ids,
// 60000 rows of 4096 bf16: 106 us a call, with those that clear first 113.)
template <typename T, typename S, int V, int L>
__global__ __launch_bounds__(kRowThreads) void embed_grad_kernel(GradOrder o, const T* __restrict__ dout, int64_t dout_stride, int width, float scale,
                                                                 bool accumulate, S* __restrict__ dtable, int64_t dtable_stride,
                                                                 float* __restrict__ parts, int adders, int slabs, uint32_t end, int per, bool past) {
    const int b = blockIdx.x, all = adders * slabs, both = min(all, (int)gridDim.x - all);
    const int number = b < 2 * both ? b >> 1 : b - both;
    if (b < 2 * both ? !(b & 1) : all > both)
        add_pieces<T, S, V, L>(o, dout, dout_stride, width, scale, accumulate, dtable, dtable_stride, parts, number / slabs, adders, number % slabs, slabs);
    else
        clear_rows<S, V>(o, end, width, per, dtable, dtable_stride, past, number, gridDim.x - all);
}

// The rows of ids whose places lie in more than one piece: workgroups per piece, which have work if such a run begins there.  A run
// of at most kAhead parts is added by the first of them, every lane for its columns.  Of a longer one each workgroup has 64
// vectors of columns at a time, each wave adds a quarter of the parts, and the quarters are added in order.
constexpr int kJoinVec = 4;
template <int V>
__device__ inline void add_parts(const float* __restrict__ parts, int64_t piece, int width, int col, int from, int to, float (&sum)[V]) {
    for (int i0 = from; i0 < to; i0 += kAhead) {
        Pack<float, V> x[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const int i = min(i0 + a, to - 1);
            x[a] = load_vec<V>(parts + ((piece + i) * 2 + (i == 0 ? 1 : 0)) * width + col);
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] = i0 + a < to ? sum[i] + x[a][i] : sum[i];
    }
}
template <typename S, int V>
__global__ __launch_bounds__(kRowThreads) void embed_grad_join_kernel(GradOrder o, int width, float scale, bool accumulate, S* __restrict__ dtable,
                                                                      int64_t dtable_stride, const float* __restrict__ parts) {
    constexpr int kWaves = kRowThreads / 64;
    __shared__ float sums[kWaves][64][V];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int vecs = (width - 1) / V + 1;
    const int pieces = (o.n - 1) / kPiece + 1;
    for (int64_t piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
        const int64_t first = piece * kPiece, end = min(first + kPiece, (int64_t)o.n), far = first + kAhead * kPiece;
        const uint32_t v = o.keys[end - 1], next = o.keys[min(end, (int64_t)o.n - 1)], head = o.keys[first], before = o.keys[max(first - 1, (int64_t)0)];
        const bool long_run = far < o.n && o.keys[far] == v;  // more than kAhead parts
        if (end == o.n || next != v || v >= o.vocab || (head == v && first > 0 && before == v) || (!long_run && blockIdx.y)) continue;
        int64_t last = piece + 1;  // the run's last piece: the first one that does not end with v and go on so
        for (;; last += 64) {
            const int64_t e = min((last + lane + 1) * kPiece, (int64_t)o.n);
            const uint64_t stops = __ballot(e == o.n || o.keys[e - 1] != v || o.keys[e] != v);
            if (stops) {
                last += __ffsll((unsigned long long)stops) - 1;
                break;
            }
        }
        const int many = (int)(last - piece) + 1, each = (many + kWaves - 1) / kWaves;
        S* const row = dtable + (int64_t)v * dtable_stride;
        if (!long_run) {
            for (int vec = threadIdx.x; vec < vecs; vec += kRowThreads) {
                const int col = min(vec * V, width - V);
                float sum[V] = {};
                add_parts<V>(parts, piece, width, col, 0, many, sum);
                put_grad<S, V>(row + col, vec * V - col, sum, scale, accumulate, false);
            }
            continue;
        }
        for (int v0 = blockIdx.y * 64; v0 < vecs; v0 += gridDim.y * 64) {
            const int vec = min(v0 + lane, vecs - 1), col = min(vec * V, width - V);
            float sum[V] = {};
            const int from = min(wave * each, many);
            add_parts<V>(parts, piece, width, col, from, min(from + each, many), sum);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) sums[wave][lane][i] = sum[i];
            __syncthreads();
            if (wave == 0 && v0 + lane < vecs) {
#pragma unroll
                for (int i = 0; i < V; ++i) sum[i] = (sum[i] + sums[1][lane][i]) + (sums[2][lane][i] + sums[3][lane][i]);
                put_grad<S, V>(row + col, vec * V - col, sum, scale, accumulate, false);
            }
        }
    }
}

// J of a row's places at a time, -1 where there is none: all of them before the first load or store that needs one, for a wait
// for a load is a wait for every load and store before it.
template <int J, int U>
__device__ inline void load_places(const int32_t* __restrict__ place, const At (&at)[U], int j0, int k, int64_t n, int (&to)[U][J]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < J; ++j) to[u][j] = place[at[u].row * k + min(j0 + j, k - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (j0 + j >= k || to[u][j] >= n) to[u][j] = -1;
}

// xs[place[t][j]] = x[t], and zeros in those of the positions t * k .. t * k + k - 1 that no pair has.  A row is read once and
// written k times.  24000 rows of 4096 bf16 to 2 experts (590 MB): 110 us, 5.4 TB/s.
constexpr int kDispatchVecs = 2, kDispatchPlaces = 4;
template <typename T, int V>
__device__ inline void dispatch_rows(const Tiles& g, const T* __restrict__ x, int64_t x_stride, int k, const int32_t* __restrict__ place, int used,
                                     T* __restrict__ xs, int64_t xs_stride) {
    constexpr int U = kDispatchVecs, J = kDispatchPlaces;
    each_vec<V, U>(g, [&](const At (&at)[U]) {
        Pack<T, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = load_vec<V, T>(x + at[u].row * x_stride + at[u].col, g.past_in);
        for (int j0 = 0; j0 < k; j0 += J) {
            int to[U][J];
            load_places<J, U>(place, at, j0, k, g.rows * k, to);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < J; ++j)
                    if (to[u][j] >= 0) store_vec<V, T>(xs + (int64_t)to[u][j] * xs_stride + at[u].col, v[u], g.past);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            for (int64_t p = max(at[u].row * k, (int64_t)used); p < (at[u].row + 1) * k; ++p)
                store_vec<V, T>(xs + p * xs_stride + at[u].col, Pack<T, V>{}, g.past);
    });
}

template <typename T, int V>
__global__ __launch_bounds__(kRowThreads) void dispatch_rows_kernel(Tiles g, const T* __restrict__ x, int64_t x_stride, int k,
                                                                    const int32_t* __restrict__ place, const int32_t* __restrict__ count,
                                                                    T* __restrict__ xs, int64_t xs_stride) {
    dispatch_rows<T, V>(g, x, x_stride, k, place, *count, xs, xs_stride);
}

// Few pairs: every workgroup sorts all of them for itself and moves its tile of rows, one launch in all.  4096 bf16, 8 of 256
// experts, beside two launches (place, move): 32 rows 5.8 and 7.7 us, 128 rows 8.2 and 9.0; 1000 rows, 2 of 8: 10.6 and 8.1.
constexpr int kFewPairs = 1024;
template <typename T, int V>
__global__ __launch_bounds__(kRowThreads) void dispatch_short_kernel(Tiles g, const T* __restrict__ x, int64_t x_stride, int k, PairItems in,
                                                                   int32_t* __restrict__ offsets, int32_t* __restrict__ place, T* __restrict__ xs,
                                                                   int64_t xs_stride) {
    __shared__ SortLds<kRowThreads / 64> lds;
    __shared__ int32_t places[kFewPairs];
    const bool first = blockIdx.x == 0 && blockIdx.y == 0;
    place_chunk(in, 0, g.rows * k, in.experts, nullptr, 1, 0, lds, first ? offsets : nullptr, [&](int64_t p, int32_t, int at) {
        places[p] = at;
        if (first) place[p] = at;
    });
    __syncthreads();
    dispatch_rows<T, V>(g, x, x_stride, k, places, lds.end, xs, xs_stride);
}

// out[t] = add[t] + sum of weight[t][j] * ys[place[t][j]], j ascending, one fused multiply-add each.  J slots at a time, whose loads
// are under way together.  10007 rows of 1500 floats, 4 experts and a residual (337 MB): 59 us, 5.7 TB/s; one row of 4096 bf16, 8
// experts: 4 us, place, row and store one behind the other.
constexpr int kCombineVecs = 2;
template <typename T, int V, int J, bool WEIGHTED>
__global__ __launch_bounds__(kRowThreads) void combine_kernel(Tiles g, const T* __restrict__ ys, int64_t ys_stride, const int32_t* __restrict__ place,
                                                              const float* __restrict__ weight, int k, const T* __restrict__ add,
                                                              int64_t add_stride, T* __restrict__ out, int64_t out_stride) {
    constexpr int U = kCombineVecs;
    each_vec<V, U>(g, [&](const At (&at)[U]) {
        float sum[U][V] = {};
        Pack<T, V> r[U] = {};
        for (int j0 = 0; j0 < k; j0 += J) {
            int from[U][J];
            float w[U][J];
            Pack<T, V> y[U][J];
            if (WEIGHTED) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int j = 0; j < J; ++j) w[u][j] = weight[at[u].row * k + min(j0 + j, k - 1)];
            }
            load_places<J, U>(place, at, j0, k, g.rows * k, from);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < J; ++j)
                    if (from[u][j] >= 0) y[u][j] = load_vec<V, T>(ys + (int64_t)from[u][j] * ys_stride + at[u].col, g.past_in);
            if (add && j0 == 0) {
#pragma unroll
                for (int u = 0; u < U; ++u) r[u] = load_vec<V>(add + at[u].row * add_stride + at[u].col);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float x = WEIGHTED ? fmaf(w[u][j], (float)y[u][j][i], sum[u][i]) : sum[u][i] + (float)y[u][j][i];
                        sum[u][i] = from[u][j] >= 0 ? x : sum[u][i];
                    }
        }
        Pack<T, V> y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (add) {
#pragma unroll
                for (int i = 0; i < V; ++i) sum[u][i] += (float)r[u][i];
            }
            y[u] = rounded_vec<T, V>(sum[u]);
        }
        store_all<V, T>(y, g.past, [&](int u) { return out + at[u].row * out_stride + at[u].col; });
    });
}

// dys[place[t][j]] = weight[t][j] * dout[t], dweight[t][j] = <dout[t], ys[place[t][j]]>, zeros in those of the positions
// t * k .. t * k + k - 1 that no pair has.  L lanes take a row, J of its slots at a time: dout is read once for all of them, and
// a slot's row of ys comes in while its row of dys goes out.  A lane adds up its vectors in order, then the lanes' sums are
// added pairwise.  8000 rows of 4096 bf16, 4 experts (590 MB): 104 us, 5.7 TB/s.
constexpr int kCombineGradVecs = 2;
template <typename T, int V, int J, int L>
__global__ __launch_bounds__(kRowThreads) void combine_grad_kernel(const T* __restrict__ dout, int64_t dout_stride, const T* __restrict__ ys, int64_t ys_stride,
                                                                   const int32_t* __restrict__ place, const float* __restrict__ weight,
                                                                   const int32_t* __restrict__ count, int rows, int k, int width, T* __restrict__ dys,
                                                                   int64_t dys_stride, float* __restrict__ dweight, bool past) {
    constexpr int U = kCombineGradVecs, kTeams = kRowThreads / L;
    __shared__ float sums[kRowThreads / 64][J];
    const int lane = threadIdx.x % L, team = threadIdx.x / L;
    const int vecs = (width - 1) / V + 1;
    const int64_t n = (int64_t)rows * k;
    const int used = *count;
    for (int64_t t0 = (int64_t)blockIdx.x * kTeams; t0 < rows; t0 += (int64_t)gridDim.x * kTeams) {
        const int64_t t = min(t0 + team, (int64_t)rows - 1);  // teams beyond the rows repeat the last one
        for (int j0 = 0; j0 < k; j0 += J) {
            int at[J];
            float w[J], dot[J];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int64_t p = t * k + min(j0 + j, k - 1);
                at[j] = place[p];
                w[j] = weight[p];
                dot[j] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (j0 + j >= k || at[j] >= n) at[j] = -1;
            for (int v0 = lane; v0 < vecs; v0 += U * L) {
                int col[U], again[U];  // the vector's elements that count start at `again`: the others were in one before
                Pack<T, V> g[U], y[U][J];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int vec = v0 + u * L;
                    col[u] = min(vec * V, width - V);
                    again[u] = vec < vecs ? vec * V - col[u] : V;
                    g[u] = load_vec<V>(dout + t * dout_stride + col[u]);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int j = 0; j < J; ++j)
                        if (at[j] >= 0) y[u][j] = load_vec<V, T>(ys + (int64_t)at[j] * ys_stride + col[u], past);
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        float d[V];
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            d[i] = w[j] * (float)g[u][i];
                            const float x = fmaf((float)g[u][i], (float)y[u][j][i], dot[j]);
                            dot[j] = i >= again[u] && at[j] >= 0 ? x : dot[j];
                        }
                        if (at[j] >= 0) store_vec<V, T>(dys + (int64_t)at[j] * dys_stride + col[u], rounded_vec<T, V>(d), past);
                    }
            }
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int m = min(L, 64) / 2; m; m >>= 1) dot[j] += __shfl_xor(dot[j], m);
            if constexpr (L > 64) {
                static_assert(L == kRowThreads);
                __syncthreads();
                if (threadIdx.x % 64 == 0)
                    for (int j = 0; j < J; ++j) sums[threadIdx.x / 64][j] = dot[j];
                __syncthreads();
#pragma unroll
                for (int j = 0; j < J; ++j) dot[j] = (sums[0][j] + sums[1][j]) + (sums[2][j] + sums[3][j]);
            }
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (lane == 0 && j0 + j < k) dweight[t * k + j0 + j] = dot[j];
        }
        for (int64_t p = max(t * k, (int64_t)used); p < (t + 1) * k; ++p)
            for (int v = lane; v < vecs; v += L) store_vec<V, T>(dys + p * dys_stride + min(v * V, width - V), Pack<T, V>{}, past);
    }
}

}  // namespace spdnn
