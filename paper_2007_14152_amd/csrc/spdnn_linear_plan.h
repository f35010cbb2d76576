// How the dense products are cut into tiles and parts of k.  Host code only, also built without HIP for tests.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "../../include/spdnn.h"

namespace spdnn {

// Which dimension of an operand is adjacent in memory: k, or its lines (rows of x, columns of W).
enum class Adjacent { K, L };

constexpr size_t kPartsAlign = 256;

// How a product is cut: into tiles of bm x bn, and of k (a multiple of a step each).
struct Plan {
    bool dma;      // operands go straight to LDS
    int few;       // linear_short_kernel: fragments of rows in a tile (1, 2 or 4); 0: linear_kernel
    bool narrow;   // and whether its tiles have 16 columns instead of 64
    int bm, bn;
    bool alone;    // no CU has two workgroups
    int64_t mtiles, ntiles, splits, per_split;
    size_t parts;  // bytes
};

// Tiles of a launch: HIP takes less than 2^32 threads, of which tiles of 64 and 128 have 256, others up to 512.
inline int64_t most_tiles(int b) { return (b == 64 || b == 128 ? 1 << 24 : 1 << 23) - 1; }

inline int step_of(int32_t type) { return type == SPDNN_F32 ? 32 : 64; }
inline size_t aligned(size_t bytes) { return (bytes + kPartsAlign - 1) / kPartsAlign * kPartsAlign; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int64_t kGroupsWanted = 256;     // workgroups that the CUs ask for at least
constexpr size_t kMostParts = 256 << 20;  // bytes that sums in parts may take

// How long n tiles of b x b take with `k` k each, us.  A CU holds four workgroups with tiles of 64, two of 128, one of 256; `us` is a
// round of one to four of them on every CU for 4096 k, `ends` what a round takes besides.  Measured with K = 64 to 4096; what is left over
// of full rounds takes what its own number of workgroups does.  longest: k of the longest tile, which no order of the others hides.
inline double cost(int b, int64_t n, double k, double longest, int32_t type) {
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
// launched: workgroups of a part, which are no fewer (all of them take part in the limit of a launch).
template <typename F, typename G>
inline void choose(F tiles, G launched, int64_t steps, double uneven, size_t out_bytes, int32_t type, bool dma, int* b, int64_t* splits) {
    const double k = (double)steps * step_of(type);
    double best = 1e300;
    *b = 128;  // (too many for every tile: refused)
    *splits = 1;
    for (const int tile : {256, 128, 64}) {
        if (!dma && tile != 128) continue;
        for (int64_t s = 1; s <= 64; s *= 2) {
            if (s > 1 && (steps / s < 4 || s * out_bytes > kMostParts)) break;
            if (launched(tile) * s > most_tiles(tile)) break;
            const double us = cost(tile, tiles(tile) * s, k / s, uneven * k / s, type) + (s > 1 ? 9.0 + 2.0 * s * out_bytes / 4e6 : 0.0);
            if (us < best) {
                best = us;
                *b = tile;
                *splits = s;
            }
        }
    }
}

inline Plan plan_product(int32_t rows, int32_t k, int32_t cols, bool grouped, int32_t experts, int32_t type, bool dma, Adjacent adj) {
    Plan p{};
    p.dma = dma;
    const int64_t sets = grouped ? std::max<int64_t>(1, std::min(experts, rows)) : 1;
    const int64_t steps = ceil_div(k, step_of(type));
    const auto tiles = [&](int bm, int bn) { return (grouped ? rows / bm + sets : ceil_div(rows, bm)) * ceil_div(cols, bn); };  // that have rows
    const auto mtiles = [&](int bm) { return grouped ? std::min<int64_t>(rows, rows / bm + experts + 1) : ceil_div(rows, bm); };
    const int64_t each = ceil_div(rows, sets);
    // (Few rows: W's bytes are what counts.  In 32 bits the matrix instructions do, from 32 rows on.)
    if (dma && each <= (type == SPDNN_F32 ? 32 : grouped ? 48 : 128) && mtiles(16) * ceil_div(cols, 64) <= most_tiles(0)) {
        p.few = each <= (grouped ? 8 : 16) ? 1 : each <= (grouped ? 20 : 32) ? 2 : 4;
        p.bm = 16 * p.few;
        // Tiles of 16 columns where those of 64 leave CUs idle; but columns of adjacent k, or k that are not many: 32 bytes of a row of
        // W at a time come from memory at two thirds of the rate.  One row: 4096 x 1024 6.2 us with 16 columns, 9.0 with 64; 4096 x 4096
        // 9.8 and 10.5 (k adjacent 6.0 and 10.0); 16384 x 4096 33.2 and, with k in four splits, 29.3 (k adjacent 21.4).
        p.narrow = tiles(p.bm, 64) < kGroupsWanted && (adj == Adjacent::K || steps < 128 || grouped);
        p.bn = p.narrow ? 16 : 64;
        p.splits = std::max<int64_t>(1, std::min(kGroupsWanted / std::max<int64_t>(tiles(p.bm, p.bn), 1), steps / 32));
    } else {
        choose([&](int b) { return tiles(b, b); }, [&](int b) { return mtiles(b) * ceil_div(cols, b); }, steps, 1.0, (size_t)rows * cols * sizeof(float), type, dma, &p.bm, &p.splits);
        p.bn = p.bm;
    }
    p.mtiles = mtiles(p.bm);
    p.ntiles = ceil_div(cols, p.bn);
    p.per_split = ceil_div(steps, p.splits) * step_of(type);
    p.splits = ceil_div(k, p.per_split);
    p.parts = p.splits > 1 ? aligned((size_t)p.splits * rows * cols * sizeof(float)) : 0;
    p.alone = type != SPDNN_F32 && tiles(p.bm, p.bn) * p.splits <= kGroupsWanted;
    return p;
}
inline Plan plan_grad(int32_t rows, int32_t m, int32_t n, int32_t experts, int32_t type, bool dma) {
    Plan p{};
    p.dma = dma;
    const auto tiles = [&](int b) { return ceil_div(m, b) * ceil_div(n, b) * experts; };
    const int64_t steps = std::max<int64_t>(1, ceil_div(ceil_div(rows, experts), step_of(type)));
    choose(tiles, tiles, steps, experts > 1 ? 3.0 : 1.0, (size_t)experts * m * n * sizeof(float), type, dma, &p.bm, &p.splits);
    p.bn = p.bm;
    p.mtiles = ceil_div(m, p.bm);
    p.ntiles = ceil_div(n, p.bn);
    p.parts = p.splits > 1 ? aligned((size_t)p.splits * experts * m * n * sizeof(float)) : 0;
    p.alone = type != SPDNN_F32 && tiles(p.bm) * p.splits <= kGroupsWanted;
    return p;
}

}  // namespace spdnn
