// Host side of the row operators (the second half of include/spdnn.h): argument checks and launches.
#include "../../include/spdnn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "spdnn_error.h"
#include "spdnn_rows_kernels.h"

namespace {

using spdnn::fail;

constexpr size_t kAlign = 256;
constexpr int64_t kMostPairs = 1 << 30;   // rows * k
constexpr int32_t kMostWidth = 1 << 30;   // columns: a vector beyond a row's end must not pass 32 bits
constexpr int64_t kMostGroups = 1 << 20;  // workgroups of a launch; more rows take turns

int size_of(int32_t type) { return type == SPDNN_F32 ? 4 : type == SPDNN_BF16 || type == SPDNN_F16 ? 2 : 0; }

// A matrix of rows: not NULL where there is a row, aligned to its elements; rows that are written are apart from each other.
enum Access { kRead, kWritten };
int check_rows(const char* what, const void* p, int32_t type, int64_t rows, int32_t width, int64_t stride, Access access) {
    const int size = size_of(type);
    if (!size) return fail(SPDNN_EINVAL, "%s: type must be SPDNN_F32, SPDNN_BF16 or SPDNN_F16", what);
    if (stride < (access == kWritten ? width : 0))
        return fail(SPDNN_EINVAL, "%s: a stride of %lld elements, width %d", what, (long long)stride, width);
    if (rows > 0 && stride > INT64_MAX / 8 / rows) return fail(SPDNN_EINVAL, "%s: stride %lld is too large", what, (long long)stride);
    if (rows > 0 && !p) return fail(SPDNN_EINVAL, "%s is NULL", what);
    if (reinterpret_cast<uintptr_t>(p) % size) return fail(SPDNN_EINVAL, "%s is not aligned to its elements", what);
    return SPDNN_OK;
}
int check_array(const char* what, const void* p, int64_t n, int size) {
    if (n > 0 && !p) return fail(SPDNN_EINVAL, "%s is NULL", what);
    if (reinterpret_cast<uintptr_t>(p) % size) return fail(SPDNN_EINVAL, "%s is not aligned to its elements", what);
    return SPDNN_OK;
}
#define CHECK(expr)                        \
    do {                                   \
        const int rc_ = (expr);            \
        if (rc_ != SPDNN_OK) return rc_;   \
    } while (0)

int check_width(int32_t width) {
    if (width < 1 || width > kMostWidth) return fail(SPDNN_EINVAL, "need 1 <= width <= %d", kMostWidth);
    return SPDNN_OK;
}
int check_pairs(int32_t rows, int32_t k, int32_t experts) {
    if (rows < 0) return fail(SPDNN_EINVAL, "rows < 0");
    if (k < 1 || k > SPDNN_MAX_CHOSEN) return fail(SPDNN_EINVAL, "need 1 <= k <= %d", SPDNN_MAX_CHOSEN);
    if (experts < 1 || experts > SPDNN_MAX_EXPERTS) return fail(SPDNN_EINVAL, "need 1 <= experts <= %d", SPDNN_MAX_EXPERTS);
    if ((int64_t)rows * k > kMostPairs) return fail(SPDNN_EINVAL, "rows * k exceeds 2^30");
    return SPDNN_OK;
}
int check_route(int32_t rows, int32_t experts, int32_t k, const float* bias, int32_t score) {
    CHECK(check_pairs(rows, k, experts));
    if (k > experts) return fail(SPDNN_EINVAL, "k = %d of %d experts", k, experts);
    if (score != SPDNN_SOFTMAX && score != SPDNN_SIGMOID) return fail(SPDNN_EINVAL, "score must be SPDNN_SOFTMAX or SPDNN_SIGMOID");
    return check_array("bias", bias, 0, 4);
}
int check_work(const void* work, size_t bytes, size_t need) {
    if (bytes < need) return fail(SPDNN_ESIZE, "work has %zu bytes, %zu needed", bytes, need);
    if (need && !work) return fail(SPDNN_EINVAL, "work is NULL");
    if (reinterpret_cast<uintptr_t>(work) % kAlign) return fail(SPDNN_EINVAL, "work must be 256-byte aligned");
    return SPDNN_OK;
}

dim3 groups(int64_t n) { return dim3((unsigned)std::max<int64_t>(1, std::min(n, kMostGroups))); }

// Outputs of this many bytes go past the caches, for whoever reads them next does not find them there (256 MB at the most) anyway,
// and so do inputs that are read once.  Rows of 4096 bf16 by id, alone and with a kernel behind that reads them, through -> past:
// 400 MB 128 -> 117 and 266 -> 256 us, 200 MB 70 -> 62 and 141 -> 137, 128 MB 42 -> 41 and 83 -> 87, 16 MB 10.4 -> 11.8 and
// 15.9 -> 17.5.  combine of 4 such rows each, its input through -> past: 512 MB 128 -> 112 us, 256 MB 64 -> 60, 128 MB 28.5 -> 35.6.
constexpr int64_t kPastBytes = 160 << 20;

// Tiles of rows x width elements in vectors of v, `unroll` a lane at a time, out_bytes of output in all: as many rows to a tile as
// fill its workgroup's turns best, but not so many that less than two workgroups per CU are left.
constexpr int64_t kTilesAtLeast = 512;
spdnn::Tiles tiles(int64_t rows, int32_t width, int v, int unroll, int64_t out_bytes) {
    spdnn::Tiles g;
    g.rows = rows;
    g.width = width;
    g.vecs = (width - 1) / v + 1;
    g.slab = std::min(g.vecs, spdnn::kTileVecs);
    g.past = out_bytes >= kPastBytes;
    g.past_in = false;
    g.per = 1;
    const int64_t turn = unroll * spdnn::kRowThreads;  // vectors that a workgroup takes at a time
    double best = 0;
    const auto consider = [&](int64_t per) {
        const double full = (double)(per * g.slab) / (double)((per * g.slab + turn - 1) / turn * turn);
        if (full > best + 0.02) {
            best = full;
            g.per = (int32_t)per;
        }
    };
    consider(1);
    for (int64_t vecs = turn; vecs <= spdnn::kTileVecs; vecs += turn) consider(std::max<int64_t>(1, std::min(vecs / g.slab, rows / kTilesAtLeast)));
    g.magic = (uint32_t)(((1ull << 32) + g.slab - 1) / g.slab);
    return g;
}
dim3 groups(const spdnn::Tiles& g) {
    const int64_t x = std::min((g.rows + g.per - 1) / g.per, kMostGroups);
    return dim3((unsigned)x, (unsigned)std::min((g.vecs + g.slab - 1) / g.slab, 1024));
}

// f(T{}) with the C++ type of an SPDNN_F32 ...
template <typename F>
void with_type(int32_t type, F f) {
    if (type == SPDNN_F32) f(float{});
    else if (type == SPDNN_BF16) f(__bf16{});
    else f(_Float16{});
}
template <typename F>
void with_ids(int32_t type, F f) {
    if (type == SPDNN_I32) f(int32_t{});
    else f(int64_t{});
}

// How n pairs are cut for the sort.
struct Chunks {
    int log_size;
    int32_t count;  // 1 at least
};
Chunks chunks_of(int64_t n) {
    int log = 0;
    while ((int64_t)1 << log < spdnn::kLeastChunk || (int64_t)spdnn::kMostChunks << log < n) ++log;
    return {log, (int32_t)std::max<int64_t>(1, ((n - 1) >> log) + 1)};
}

// Work memory of the gradient of a table, and how many bits of the ids are sorted at a time.
struct GradWork {
    size_t keys[2], tokens[2], table, parts, bytes;
    int passes, bits;
    GradWork(int32_t vocab, int32_t width, int32_t n) : keys{}, tokens{}, table(0), parts(0), bytes(0), passes(0), bits(0) {
        if (n <= spdnn::kFewIds) return;
        int all = 0;  // bits of 0 .. vocab: ids outside the table are sorted as `vocab`, behind all others
        while ((int64_t)vocab >> all) ++all;
        passes = (all + 9) / 10;
        bits = (all + passes - 1) / passes;
        const auto take = [&](size_t size) {
            const size_t at = bytes;
            bytes += (size + kAlign - 1) / kAlign * kAlign;
            return at;
        };
        for (int i = 0; i < 2; ++i) {
            keys[i] = take(sizeof(uint32_t) * (size_t)n);
            tokens[i] = take(sizeof(int32_t) * (size_t)n);
        }
        table = take(sizeof(int32_t) * ((size_t)1 << bits) * chunks_of(n).count);
        parts = take(sizeof(float) * 2 * (size_t)width * ((size_t)(n - 1) / spdnn::kPiece + 1));
    }
};
static_assert(spdnn::kMostBins >= 1 << 10);
constexpr int64_t kClearBytes = 128 << 10;  // of a table that a workgroup clears at a time
// What a launch of the sort clears beside: as much as is stored while the sort waits.  Nothing, this, twice this: 60000 ids, 65536 rows
// of 1024 floats 87.6, 83.7 and 97.4 us; 3000 ids, 60000 rows of 4096 bf16 118, 105 and 104; 20000 ids, 30000 rows of 1024 floats 57.3,
// 56.0 and 58.4.
constexpr int64_t kCountClears = 24 << 20, kPlaceClears = 40 << 20;
// Workgroups for that, three per CU.  256, 768 and 2048 of them, the same tables: 82.7, 83.7 and 83.7 us; 107, 105 and 105; 57.5, 56.0
// and 55.9.
constexpr int kSpareGroups = 768;
// Workgroups that add with few ids: most end at once, for a frequent id's they have to be enough.  1024, 4096 and 16384 of them: 777
// ids, 10007 rows of 1500 floats 17.3, 18.0 and 19.3 us; 1000 ids, 1000 rows of 8192 (bf16 to floats) 75, 33 and 45; 1024 times one id,
// rows of 4096 333, 103 and 64.
constexpr int64_t kFewGroups = 4096;

// f(V) with the elements of a vector: V, or 1 where a row has less.
template <int V, typename F>
void with_vec(int32_t width, F f) {
    if (width >= V) f(std::integral_constant<int, V>{});
    else f(std::integral_constant<int, 1>{});
}

// f(J) with the slots of a row that are taken at a time.
template <typename F>
void with_places(int32_t k, F f) {
    if (k == 1) f(std::integral_constant<int, 1>{});
    else if (k == 2) f(std::integral_constant<int, 2>{});
    else f(std::integral_constant<int, 4>{});
}

// f(K), k rounded up to a power of two.
template <typename F>
void with_chosen(int32_t k, F f) {
    if (k == 1) f(std::integral_constant<int, 1>{});
    else if (k == 2) f(std::integral_constant<int, 2>{});
    else if (k <= 4) f(std::integral_constant<int, 4>{});
    else if (k <= 8) f(std::integral_constant<int, 8>{});
    else f(std::integral_constant<int, 16>{});
}

// f(G) with the lanes that take a row of logits, at least G0: so many that a lane has kLogits of them, but a wave at most.  (The
// gradient through a softmax over 256 logits, which then reads its row once: 16384 rows of floats 13.3 us with 8 lanes, 10.0 with 32.)
template <int G0, typename F>
void with_team(int32_t experts, F f) {
    if constexpr (G0 <= 8) {
        if (experts <= 8 * spdnn::kLogits) return f(std::integral_constant<int, 8>{});
    }
    if (experts <= 16 * spdnn::kLogits) f(std::integral_constant<int, 16>{});
    else if (experts <= 32 * spdnn::kLogits) f(std::integral_constant<int, 32>{});
    else f(std::integral_constant<int, 64>{});
}

// Up to so many rows the lanes of a route_kernel team are as many as the logits ask for; above, as few as the slots allow, for what
// the lanes do together (merge lists) costs a wave the same whether it has one row or eight.  256 logits, 8 experts, 8 lanes and 32:
// 64 rows 4.4 and 3.6 us, 2048 rows 4.6 and 3.8, 4096 rows 4.6 and 4.5, 16384 rows 6.0 and 9.5.  Where they meet depends on the lists:
// 512 logits, 4 experts, 8 lanes and 64: 4096 rows 5.8 and 5.0, 8192 rows 6.6 and 7.3; 1024 logits, 16 experts, 16 lanes and 64: 2048
// rows 7.5 both, 4096 rows 8.2 and 11.4; 1024 logits, 2 experts, 8 and 64: 8192 rows 9.4 and 8.0, 16384 rows 13.9 and 14.7.
constexpr int32_t kFewRows = 4096;

int launched() {
    HIP_TRY(hipGetLastError());
    return SPDNN_OK;
}

}  // namespace

extern "C" {

int spdnn_embed(const void* table, int32_t table_type, int32_t vocab, int32_t width, int64_t table_stride, const void* ids,
                int32_t ids_type, int32_t n, float scale, void* out, int32_t out_type, int64_t out_stride, void* hip_stream) {
    if (vocab < 1 || n < 0) return fail(SPDNN_EINVAL, "need vocab >= 1, n >= 0");
    CHECK(check_width(width));
    if (ids_type != SPDNN_I32 && ids_type != SPDNN_I64) return fail(SPDNN_EINVAL, "ids_type must be SPDNN_I32 or SPDNN_I64");
    CHECK(check_rows("table", table, table_type, vocab, width, table_stride, kRead));
    CHECK(check_rows("out", out, out_type, n, width, out_stride, kWritten));
    CHECK(check_array("ids", ids, n, ids_type == SPDNN_I32 ? 4 : 8));
    if (n == 0) return SPDNN_OK;
    const hipStream_t s = (hipStream_t)hip_stream;
    with_type(table_type, [&](auto tt) {
        with_type(out_type, [&](auto to) {
            with_ids(ids_type, [&](auto ti) {
                using T = decltype(tt);
                using S = decltype(to);
                using I = decltype(ti);
                with_vec<16 / std::max(sizeof(T), sizeof(S))>(width, [&](auto v) {
                    constexpr int V = decltype(v)::value;
                    const spdnn::Tiles g = tiles(n, width, V, spdnn::kEmbedVecs, (int64_t)n * width * sizeof(S));
                    spdnn::embed_kernel<T, S, I, V><<<groups(g), spdnn::kRowThreads, 0, s>>>(g, (const T*)table, table_stride, (uint32_t)vocab, (const I*)ids, scale, (S*)out, out_stride);
                });
            });
        });
    });
    return launched();
}

int spdnn_embed_grad_bytes(int32_t vocab, int32_t width, int32_t n, size_t* bytes) {
    if (!bytes) return fail(SPDNN_EINVAL, "bytes is NULL");
    if (vocab < 1 || n < 0) return fail(SPDNN_EINVAL, "need vocab >= 1, n >= 0");
    CHECK(check_width(width));
    *bytes = GradWork(vocab, width, n).bytes;
    return SPDNN_OK;
}

int spdnn_embed_grad(const void* dout, int32_t dout_type, int64_t dout_stride, const void* ids, int32_t ids_type, int32_t n,
                     int32_t vocab, int32_t width, float scale, int32_t accumulate, void* dtable, int32_t dtable_type,
                     int64_t dtable_stride, void* work, size_t work_bytes, void* hip_stream) {
    size_t need = 0;
    CHECK(spdnn_embed_grad_bytes(vocab, width, n, &need));
    if (ids_type != SPDNN_I32 && ids_type != SPDNN_I64) return fail(SPDNN_EINVAL, "ids_type must be SPDNN_I32 or SPDNN_I64");
    CHECK(check_rows("dout", dout, dout_type, n, width, dout_stride, kRead));
    CHECK(check_rows("dtable", dtable, dtable_type, vocab, width, dtable_stride, kWritten));
    CHECK(check_array("ids", ids, n, ids_type == SPDNN_I32 ? 4 : 8));
    CHECK(check_work(work, work_bytes, need));
    const hipStream_t s = (hipStream_t)hip_stream;
    if (n == 0 && accumulate) return SPDNN_OK;
    const bool past = !accumulate && (int64_t)vocab * width * size_of(dtable_type) >= kPastBytes;
    const int64_t row_bytes = (int64_t)width * size_of(dtable_type);
    if (n <= spdnn::kFewIds) {
        with_type(dout_type, [&](auto tt) {
            with_type(dtable_type, [&](auto to) {
                with_ids(ids_type, [&](auto ti) {
                    using T = decltype(tt);
                    using S = decltype(to);
                    using I = decltype(ti);
                    with_vec<16 / std::max(sizeof(T), sizeof(S))>(width, [&](auto v) {
                        constexpr int V = decltype(v)::value;
                        const int vecs = (width - 1) / V + 1;
                        const int per = (int)std::min<int64_t>(std::max<int64_t>(kClearBytes / row_bytes, 1), spdnn::kMostRowsToClear);
                        const int64_t clear = accumulate ? 0 : std::min<int64_t>((vocab - 1) / per + 1, kMostGroups);
                        // as many workgroups for a token's columns as make kFewGroups in all
                        const int slabs = (int)std::max<int64_t>(1, std::min<int64_t>((vecs - 1) / 64 + 1, kFewGroups / std::max(n, 1)));
                        spdnn::embed_grad_short_kernel<T, S, I, V><<<dim3((unsigned)(n * slabs + clear)), spdnn::kRowThreads, 0, s>>>((const T*)dout, dout_stride, (const I*)ids, n, vocab, width, slabs, per, scale, accumulate != 0, (S*)dtable, dtable_stride, past);
                    });
                });
            });
        });
        return launched();
    }
    // the ids sorted, a few of their bits at a time
    const GradWork w(vocab, width, n);
    char* const base = (char*)work;
    const Chunks c = chunks_of(n);
    const int bins = 1 << w.bits;
    int32_t* const table = c.count > 1 ? (int32_t*)(base + w.table) : nullptr;
    const uint32_t* keys = nullptr;
    const int32_t* tokens = nullptr;
    // The sort's launches leave most of the chip idle: meanwhile the last rows of the table are cleared, whether their ids occur
    // or not.  (The last ones because ids are mostly numbered by frequency: rows that are written again cost twice.)
    spdnn::Clear rows{(char*)dtable, dtable_stride * size_of(dtable_type), (int32_t)std::min<int64_t>(row_bytes, INT32_MAX), vocab, vocab, past};
    const auto spare = [&](int64_t bytes) -> int {  // workgroups that clear so much, and the rows for it
        rows.last = rows.first;
        if (accumulate || row_bytes < 16 || row_bytes > INT32_MAX) return 0;
        rows.first = std::max<int64_t>(0, rows.last - bytes / row_bytes);
        return rows.first < rows.last ? kSpareGroups : 0;
    };
    for (int pass = 0; pass < w.passes; ++pass) {
        uint32_t* const to_keys = (uint32_t*)(base + w.keys[pass & 1]);
        int32_t* const to_tokens = (int32_t*)(base + w.tokens[pass & 1]);
        const int shift = pass * w.bits;
        const auto sort = [&](auto in) {
            if (table) {
                const int more = spare(kCountClears);
                spdnn::count_kernel<<<c.count + more, spdnn::kSortThreads, 0, s>>>(in, n, c.log_size, c.count, bins, table, rows);
            }
            const int more = spare(kPlaceClears);
            spdnn::key_place_kernel<<<c.count + more, spdnn::kSortThreads, 0, s>>>(in, n, c.log_size, c.count, table, to_keys, to_tokens, rows);
        };
        if (pass == 0)
            with_ids(ids_type, [&](auto ti) {
                using I = decltype(ti);
                sort(spdnn::IdItems<I>{(const I*)ids, (uint32_t)vocab, shift, bins - 1});
            });
        else
            sort(spdnn::KeyItems{keys, tokens, shift, bins - 1});
        keys = to_keys;
        tokens = to_tokens;
    }
    const spdnn::GradOrder order{keys, tokens, n, (uint32_t)vocab};
    float* const parts = (float*)(base + w.parts);
    const int64_t pieces = (n - 1) / spdnn::kPiece + 1;
    with_type(dout_type, [&](auto tt) {
        with_type(dtable_type, [&](auto to) {
            using T = decltype(tt);
            using S = decltype(to);
            with_vec<16 / std::max(sizeof(T), sizeof(S))>(width, [&](auto v) {
                constexpr int V = decltype(v)::value;
                const int vecs = (width - 1) / V + 1;
                const auto run = [&](auto l) {
                    constexpr int L = decltype(l)::value;
                    const int adders = (int)std::min<int64_t>((pieces - 1) / (spdnn::kRowThreads / L) + 1, kMostGroups);
                    const int per = (int)std::min<int64_t>(std::max<int64_t>(kClearBytes / row_bytes, 1), spdnn::kRowThreads);
                    const int clear = accumulate ? 0 : (int)std::min<int64_t>((rows.first + per - 1) / per, kMostGroups);
                    const int slabs = (int)std::min<int64_t>((vecs - 1) / L + 1, std::max<int64_t>(1, kMostGroups / adders));
                    const dim3 grid((unsigned)(adders * slabs + clear));
                    spdnn::embed_grad_kernel<T, S, V, L><<<grid, spdnn::kRowThreads, 0, s>>>(order, (const T*)dout, dout_stride, width, scale, accumulate != 0, (S*)dtable, dtable_stride, parts, adders, slabs, (uint32_t)rows.first, per, past);
                };
                if (vecs <= 16) run(std::integral_constant<int, 16>{});
                else if (vecs <= 64) run(std::integral_constant<int, 64>{});
                else run(std::integral_constant<int, 256>{});
            });
            with_vec<spdnn::kJoinVec>(width, [&](auto v) {
                constexpr int V = decltype(v)::value;
                const dim3 grid((unsigned)std::min(pieces, kMostGroups), (unsigned)std::min((width - 1) / (64 * V) + 1, 64));
                spdnn::embed_grad_join_kernel<S, V><<<grid, spdnn::kRowThreads, 0, s>>>(order, width, scale, accumulate != 0, (S*)dtable, dtable_stride, parts);
            });
        });
    });
    return launched();
}

int spdnn_route(const void* logits, int32_t type, int64_t stride, int32_t rows, int32_t experts, int32_t k, const float* bias,
                const uint8_t* keep, int32_t score, int32_t normalise, float scale, int32_t* chosen, float* weight,
                void* hip_stream) {
    CHECK(check_route(rows, experts, k, bias, score));
    CHECK(check_rows("logits", logits, type, rows, experts, stride, kRead));
    CHECK(check_array("chosen", chosen, rows, 4));
    CHECK(check_array("weight", weight, rows, 4));
    if (rows == 0) return SPDNN_OK;
    with_type(type, [&](auto tt) {
        using T = decltype(tt);
        with_chosen(k, [&](auto kk) {
            constexpr int K = decltype(kk)::value;
            constexpr int G0 = K > 8 ? K : 8;
            const auto run = [&](auto gg) {
                constexpr int G = decltype(gg)::value;
                spdnn::route_kernel<T, K, G><<<groups((rows - 1) / (spdnn::kRowThreads / G) + 1), spdnn::kRowThreads, 0, (hipStream_t)hip_stream>>>((const T*)logits, stride, rows, experts, k, bias, keep, score, normalise, scale, chosen, weight);
            };
            if (rows > kFewRows) run(std::integral_constant<int, G0>{});
            else with_team<G0>(experts, run);
        });
    });
    return launched();
}

int spdnn_route_grad(const float* dweight, const void* logits, int32_t type, int64_t stride, const int32_t* chosen, int32_t rows,
                     int32_t experts, int32_t k, const float* bias, int32_t score, int32_t normalise, float scale, void* dlogits,
                     int64_t dstride, void* hip_stream) {
    CHECK(check_route(rows, experts, k, bias, score));
    CHECK(check_rows("logits", logits, type, rows, experts, stride, kRead));
    CHECK(check_rows("dlogits", dlogits, type, rows, experts, dstride, kWritten));
    CHECK(check_array("chosen", chosen, rows, 4));
    CHECK(check_array("dweight", dweight, rows, 4));
    if (rows == 0) return SPDNN_OK;
    with_type(type, [&](auto tt) {
        using T = decltype(tt);
        const auto run = [&](auto gg) {
            constexpr int G = decltype(gg)::value;
            spdnn::route_grad_kernel<T, G><<<groups((rows - 1) / (spdnn::kRowThreads / G) + 1), spdnn::kRowThreads, 0, (hipStream_t)hip_stream>>>(dweight, (const T*)logits, stride, chosen, rows, experts, k, bias, score, normalise, scale, (T*)dlogits, dstride);
        };
        if (k <= 8) with_team<8>(experts, run);  // a lane per slot
        else with_team<16>(experts, run);
    });
    return launched();
}

int spdnn_dispatch_bytes(int32_t rows, int32_t k, int32_t experts, size_t* bytes) {
    if (!bytes) return fail(SPDNN_EINVAL, "bytes is NULL");
    CHECK(check_pairs(rows, k, experts));
    const Chunks c = chunks_of((int64_t)rows * k);
    *bytes = c.count > 1 ? sizeof(int32_t) * experts * c.count : 0;
    return SPDNN_OK;
}

int spdnn_dispatch(const int32_t* chosen, int32_t rows, int32_t k, int32_t experts, const void* x, int32_t type, int32_t width,
                   int64_t x_stride, void* xs, int64_t xs_stride, int32_t* offsets, int32_t* place, void* work,
                   size_t work_bytes, void* hip_stream) {
    size_t need = 0;
    CHECK(spdnn_dispatch_bytes(rows, k, experts, &need));
    CHECK(check_width(width));
    const int n = rows * k;
    CHECK(check_rows("x", x, type, rows, width, x_stride, kRead));
    CHECK(check_rows("xs", xs, type, n, width, xs_stride, kWritten));
    CHECK(check_array("chosen", chosen, rows, 4));
    CHECK(check_array("place", place, rows, 4));
    CHECK(check_array("offsets", offsets, 1, 4));
    CHECK(check_work(work, work_bytes, need));
    const hipStream_t s = (hipStream_t)hip_stream;
    const spdnn::PairItems in{chosen, experts};
    const bool few = n > 0 && n <= spdnn::kFewPairs;
    if (!few) {
        const Chunks c = chunks_of(n);
        int32_t* const table = c.count > 1 ? (int32_t*)work : nullptr;
        if (table) spdnn::count_kernel<<<c.count, spdnn::kSortThreads, 0, s>>>(in, n, c.log_size, c.count, experts, table, spdnn::Clear{});
        spdnn::expert_place_kernel<<<c.count, spdnn::kSortThreads, 0, s>>>(in, n, c.log_size, table, c.count, offsets, place);
    }
    if (n > 0)
        with_type(type, [&](auto tt) {
            using T = decltype(tt);
            with_vec<16 / sizeof(T)>(width, [&](auto v) {
                constexpr int V = decltype(v)::value;
                spdnn::Tiles g = tiles(rows, width, V, spdnn::kDispatchVecs, (int64_t)n * width * sizeof(T));
                g.past_in = (int64_t)rows * width * (int64_t)sizeof(T) >= kPastBytes;
                if (few)
                    spdnn::dispatch_short_kernel<T, V><<<groups(g), spdnn::kRowThreads, 0, s>>>(g, (const T*)x, x_stride, k, in, offsets, place, (T*)xs, xs_stride);
                else
                    spdnn::dispatch_rows_kernel<T, V><<<groups(g), spdnn::kRowThreads, 0, s>>>(g, (const T*)x, x_stride, k, place, offsets + experts, (T*)xs, xs_stride);
            });
        });
    return launched();
}

int spdnn_combine(const void* ys, int32_t type, int32_t width, int64_t ys_stride, const int32_t* place, const float* weight,
                  int32_t rows, int32_t k, const void* add, int64_t add_stride, void* out, int64_t out_stride, void* hip_stream) {
    CHECK(check_pairs(rows, k, 1));
    CHECK(check_width(width));
    const int n = rows * k;
    CHECK(check_rows("ys", ys, type, n, width, ys_stride, kRead));
    CHECK(check_rows("out", out, type, rows, width, out_stride, kWritten));
    if (add) CHECK(check_rows("add", add, type, rows, width, add_stride, kRead));
    CHECK(check_array("place", place, rows, 4));
    CHECK(check_array("weight", weight, 0, 4));
    if (rows == 0) return SPDNN_OK;
    with_type(type, [&](auto tt) {
        using T = decltype(tt);
        with_vec<16 / sizeof(T)>(width, [&](auto v) {
            constexpr int V = decltype(v)::value;
            spdnn::Tiles g = tiles(rows, width, V, spdnn::kCombineVecs, (int64_t)rows * width * sizeof(T));
            g.past_in = (int64_t)n * width * (int64_t)sizeof(T) >= kPastBytes;
            const auto run = [&](auto j, auto weighted) {
                spdnn::combine_kernel<T, V, decltype(j)::value, decltype(weighted)::value><<<groups(g), spdnn::kRowThreads, 0, (hipStream_t)hip_stream>>>(g, (const T*)ys, ys_stride, place, weight, k, (const T*)add, add_stride, (T*)out, out_stride);
            };
            with_places(k, [&](auto j) {
                if (weight) run(j, std::true_type{});
                else run(j, std::false_type{});
            });
        });
    });
    return launched();
}

int spdnn_combine_grad(const void* dout, int32_t type, int32_t width, int64_t dout_stride, const void* ys, int64_t ys_stride,
                       const int32_t* place, const float* weight, const int32_t* count, int32_t rows, int32_t k, void* dys,
                       int64_t dys_stride, float* dweight, void* hip_stream) {
    CHECK(check_pairs(rows, k, 1));
    CHECK(check_width(width));
    const int n = rows * k;
    CHECK(check_rows("dout", dout, type, rows, width, dout_stride, kRead));
    CHECK(check_rows("ys", ys, type, n, width, ys_stride, kRead));
    CHECK(check_rows("dys", dys, type, n, width, dys_stride, kWritten));
    CHECK(check_array("place", place, rows, 4));
    CHECK(check_array("weight", weight, rows, 4));
    CHECK(check_array("count", count, rows, 4));
    CHECK(check_array("dweight", dweight, rows, 4));
    if (rows == 0) return SPDNN_OK;
    with_type(type, [&](auto tt) {
        using T = decltype(tt);
        const bool past = (int64_t)n * width * (int64_t)sizeof(T) >= kPastBytes;
        with_vec<16 / sizeof(T)>(width, [&](auto v) {
            constexpr int V = decltype(v)::value;
            const int vecs = (width - 1) / V + 1;
            const auto run = [&](auto j, auto l) {
                constexpr int L = decltype(l)::value;
                spdnn::combine_grad_kernel<T, V, decltype(j)::value, L><<<groups((rows - 1) / (spdnn::kRowThreads / L) + 1), spdnn::kRowThreads, 0, (hipStream_t)hip_stream>>>((const T*)dout, dout_stride, (const T*)ys, ys_stride, place, weight, count, rows, k, width, (T*)dys, dys_stride, dweight, past);
            };
            with_places(k, [&](auto j) {
                // bf16, 4 experts, with 16, 64 and 256 lanes: 20000 rows of 512 30.1, 32.9 and 72 us; 4000 of 1024 15.4, 13.4 and
                // 21.3; 4000 of 2048 28.0, 24.6 and 28.3; 8000 of 4096 115, 117 and 103; 512 of 4096 31.5, 11.2 and 8.3
                if (vecs <= 64) run(j, std::integral_constant<int, 16>{});
                else if (vecs <= 256) run(j, std::integral_constant<int, 64>{});
                else run(j, std::integral_constant<int, 256>{});
            });
        });
    });
    return launched();
}

}  // extern "C"
