// Kernels of the dense products (spdnn_linear, spdnn_linear_grad of include/spdnn.h): act(x W + b) + add for one matrix W or for
// every expert's own on rows sorted by expert, and the gradients.  T: type of rows and weights (float, __bf16, _Float16).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "spdnn_vec.h"

#pragma clang fp contract(off)

namespace spdnn {

// --- matrix instructions ----------------------------------------------------
//
// A fragment is 16 lines (rows of x, or columns of W) by 64 bytes of k: lane l has 16 bytes of line l % 16.  acc[q] of lane l is the
// sum for line 4 (l / 16) + q of the first fragment and line l % 16 of the second: with W's first and x's second a lane has four
// adjacent columns of one row.  Products of 16-bit numbers are exact in the 32 bits in which they are added.
template <typename T>
using Frag __attribute__((ext_vector_type(16 / sizeof(T)))) = T;
using Acc __attribute__((ext_vector_type(4))) = float;

__device__ inline Acc mma(Frag<__bf16> a, Frag<__bf16> b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline Acc mma(Frag<_Float16> a, Frag<_Float16> b, Acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ inline Acc mma(Frag<float> a, Frag<float> b, Acc c) {  // 4 instructions of 4 k each: the order of the k is the same for both sides
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

// --- activations ------------------------------------------------------------

constexpr float kClip = 32.0f;  // that of the sparse networks

// A NaN stays one.
__device__ inline float activated(float x, int act) {
    switch (act) {
        case SPDNN_ACT_RELU: return x < 0.0f ? 0.0f : x;
        case SPDNN_ACT_CLIP: return x < 0.0f ? 0.0f : x > kClip ? kClip : x;
        case SPDNN_ACT_GELU: return 0.5f * x * (1.0f + erff(x * 0.70710678f));
        case SPDNN_ACT_SILU: return x / (1.0f + expf(-x));
    }
    return x;
}
__device__ inline float act_slope(float x, int act) {
    switch (act) {
        case SPDNN_ACT_RELU: return x <= 0.0f ? 0.0f : 1.0f;
        case SPDNN_ACT_CLIP: return x <= 0.0f || x >= kClip ? 0.0f : 1.0f;
        case SPDNN_ACT_GELU: return 0.5f * (1.0f + erff(x * 0.70710678f)) + x * (0.39894228f * expf(-0.5f * x * x));
        case SPDNN_ACT_SILU: {
            const float s = 1.0f / (1.0f + expf(-x));
            return s + x * s * (1.0f - s);
        }
    }
    return 1.0f;
}

// --- operands in LDS --------------------------------------------------------
//
// A step of k is 128 bytes of it: 64 numbers of 16 bits or 32 floats.  An operand's tile is LINES lines by one step, LINES * 128
// bytes, in chunks of 16 bytes as they lie in memory:
//   Adjacent::K  (x's rows; W if its k are adjacent)       line r has 8 chunks; chunk c stands at place c ^ (r / 2) % 8
//   Adjacent::L  (W if its columns are adjacent, and both   k row has LINES numbers; blocks of 16 numbers stand at place
//                 operands of a gradient of W)              block ^ f(k)
// so that the lanes that read a fragment together meet all banks.  The second form is turned round on the way to registers: for 16
// bits by the transposing LDS read (16 lanes give 4 rows of 16 numbers, lane i gets column i), floats are read one by one.
enum class Adjacent { K, L };

struct Side {
    const char* p;
    int64_t line;  // bytes between neighbours in the dimension that is not adjacent
    int64_t set;   // bytes between experts' matrices
};

template <typename T, Adjacent ADJ, int LINES, int THREADS>
struct Tile {
    static constexpr int kChunk = 16 / sizeof(T);      // numbers of a chunk
    static constexpr int kStep = 128 / sizeof(T);      // numbers of a step of k
    static constexpr int kBytes = LINES * 128;
    static constexpr int kChunks = LINES * 8 / THREADS;  // chunks of a thread
    static_assert(LINES * 8 % THREADS == 0 && LINES % 16 == 0);
    static constexpr int kPerRow = ADJ == Adjacent::K ? 8 : LINES / kChunk;  // chunks of a memory row of the tile
    static constexpr int kBlock = sizeof(T) == 2 ? 2 : 4;                    // chunks of 16 numbers
    static constexpr int kBlocks = LINES / 16;

    __device__ static int turn(int k) {  // f(k)
        const int f = sizeof(T) == 2 ? (k & 3) | (k >> 3 & 1) << 2 : k >> 2 & 3;
        return f & (kBlocks >= 8 ? 7 : kBlocks >= 4 ? 3 : kBlocks >= 2 ? 1 : 0);
    }
    // Which memory row and chunk of it stand at chunk q of the tile.
    struct At {
        int row, chunk;
    };
    __device__ static At at(int q) {
        const int row = q / kPerRow, place = q % kPerRow;
        if constexpr (ADJ == Adjacent::K) return {row, place ^ (row >> 1 & 7)};
        else return {row, place ^ turn(row) * kBlock};
    }
    // Fragment of lines line0 .. line0 + 15, half `half` of the step.
    __device__ static Frag<T> read(const char* tile, int line0, int half, int lane) {
        const int i = lane % 16, g = lane / 16;
        if constexpr (ADJ == Adjacent::K) {
            const int r = line0 + i;
            return *reinterpret_cast<const Frag<T>*>(tile + r * 128 + ((half * 4 + g) ^ (i >> 1)) * 16);
        } else if constexpr (sizeof(T) == 2) {
            const int k = half * 32 + g * 8 + i / 4;
            const char* const from = tile + k * (LINES * 2) + ((line0 / 16) ^ turn(k)) * 32 + i % 4 * 8;
            typedef short Four __attribute__((ext_vector_type(4)));
            using Lds = __attribute__((address_space(3))) Four;
            const Four a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)from);
            const Four b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(from + 4 * LINES * 2));
            return __builtin_bit_cast(Frag<T>, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            Frag<T> x;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = half * 16 + g * 4 + j;
                x[j] = *reinterpret_cast<const float*>(tile + k * (LINES * 4) + ((line0 / 16) ^ turn(k)) * 64 + i * 4);
            }
            return x;
        }
    }
};

// Loads of a tile through registers: any alignment, zeros for lines from `lines` on and k from `ks` on (counted from the tile's
// first), so that nothing that lies there reaches a sum.
template <typename T, Adjacent ADJ, int LINES, int THREADS>
struct ByRegisters {
    using G = Tile<T, ADJ, LINES, THREADS>;
    Frag<T> x[G::kChunks];
    __device__ void load(const char* p, int64_t line_bytes, int lines, int64_t ks, int thread) {
#pragma unroll
        for (int c = 0; c < G::kChunks; ++c) {
            const auto at = G::at(c * THREADS + thread);
            const int first = at.chunk * G::kChunk;
            const int64_t here = ADJ == Adjacent::K ? ks - first : lines - first;  // numbers there are
            const bool row = ADJ == Adjacent::K ? at.row < lines : at.row < ks;
            const T* const from = reinterpret_cast<const T*>(p + at.row * line_bytes) + first;
            Frag<T> v = {};
            if (row && here >= G::kChunk) {
                v = load_vec<G::kChunk>(from);
            } else if (row) {
#pragma unroll
                for (int i = 0; i < G::kChunk; ++i)
                    if (i < here) v[i] = from[i];
            }
            x[c] = v;
        }
    }
    __device__ void store(char* tile, int thread) const {
#pragma unroll
        for (int c = 0; c < G::kChunks; ++c) *reinterpret_cast<Frag<T>*>(tile + (c * THREADS + thread) * 16) = x[c];
    }
};

// Loads of a tile straight into LDS, 16 bytes a lane.  What is not there comes as zeros, from the range check of the buffer: lines
// beyond the last, and what lies behind the last k (Adjacent::K: a lane whose chunk does has kOutside added to its offset).  Lines and
// the first chunk are aligned to 16 bytes and have whole chunks, a tile's lines lie within kDmaSpan bytes, and the k rows of
// Adjacent::L do not overlap.
//
// They are written as instructions: the compiler would let the transposing LDS reads wait for all loads of this kind that are under way,
// for it cannot tell that they go to the other stage.  Whoever reads what they have stored waits with loads_done() and a barrier first.
constexpr uint32_t kOutside = 1u << 31;
using Memory __attribute__((ext_vector_type(4))) = int;  // address, bytes, format: the same for all lanes
__device__ inline void load_to_lds(Memory memory, uint32_t offset, char* lds, const int more) {
    const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 4\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane((int)to)), "i"(more), "v"(offset), "s"(memory)
                 : "memory", "scc", "m0");
}
__device__ inline void loads_done() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
constexpr int64_t kDmaSpan = 1 << 30;
template <typename T, Adjacent ADJ, int LINES, int THREADS>
struct ByDma {
    using G = Tile<T, ADJ, LINES, THREADS>;
    static constexpr int kRows = THREADS / G::kPerRow;  // memory rows that all lanes take at a time
    // The swizzle repeats after so many of them (16 rows): a lane's offsets are that many and multiples of a number that all share.
    static constexpr int kBases = kRows % 16 == 0 ? 1 : 16 / kRows;
    static_assert(kRows % 16 == 0 || 16 % kRows == 0);
    static_assert(G::kChunks % kBases == 0);
    uint32_t from[kBases];
    uint32_t line, step;
    __device__ void begin(int64_t line_bytes, int thread) {
        line = (uint32_t)line_bytes;
        step = kRows * kBases * line;
#pragma unroll
        for (int c = 0; c < kBases; ++c) {
            const auto at = G::at(c * THREADS + thread);
            from[c] = (uint32_t)at.row * line + at.chunk * 16;
        }
    }
    // lines, ks: what there is of both from p on.
    __device__ void load(const char* p, char* tile, int lines, int64_t ks, int thread, int wave) const {
        const int k = (int)min(ks, (int64_t)G::kStep);  // nothing is loaded if there is none
        const uint32_t bytes = k <= 0 ? 0 : ADJ == Adjacent::K ? (lines - 1) * line + k * (uint32_t)sizeof(T) : (k - 1) * line + lines * (uint32_t)sizeof(T);
        const uint64_t base = (uint64_t)p;
        const Memory memory = {__builtin_amdgcn_readfirstlane((int)base), __builtin_amdgcn_readfirstlane((int)(base >> 32) & 0xffff),
                               __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000};
        uint32_t at[kBases];
#pragma unroll
        for (int c = 0; c < kBases; ++c) at[c] = from[c];
        if (ADJ == Adjacent::K && k < G::kStep)
#pragma unroll
            for (int c = 0; c < kBases; ++c)
                if (G::at(c * THREADS + thread).chunk * G::kChunk >= k) at[c] += kOutside;
#pragma unroll
        for (int c = 0; c < G::kChunks; ++c) load_to_lds(memory, at[c % kBases] + c / kBases * step, tile + wave * 1024, c * (THREADS * 16));
    }
};

// --- what is done with the sums ---------------------------------------------

struct Ending {
    const void* bias;  // cols numbers per set, or null
    const char* add;
    int64_t add_line;
    char* pre;
    int64_t pre_line;
    char* out;
    int64_t out_line;
    int64_t out_set;
    int32_t cols;
    int32_t act;
    bool bias_f32;
    bool out_f32;  // type of out, add and pre: float or T
};

constexpr int kEnd = 8;  // columns that a lane ends at a time

template <typename T, typename O>
__device__ inline void end_sums(const Ending& e, int set, int64_t row, int col, const float (&sum)[kEnd]) {
    const int here = min(kEnd, e.cols - col);
    float y[kEnd];
#pragma unroll
    for (int i = 0; i < kEnd; ++i) y[i] = sum[i];
    if (e.bias) {
        const int64_t at = (int64_t)set * e.cols + col;
        const auto take = [&](auto* b) {
            if (here == kEnd) {
                const auto v = load_vec<kEnd>(b + at);
#pragma unroll
                for (int i = 0; i < kEnd; ++i) y[i] += (float)v[i];
            } else {
#pragma unroll
                for (int i = 0; i < kEnd; ++i)
                    if (i < here) y[i] += (float)b[at + i];
            }
        };
        if (e.bias_f32) take((const float*)e.bias);
        else take((const T*)e.bias);
    }
    const auto put = [&](char* to, int64_t line) {
        O* const o = reinterpret_cast<O*>(to + row * line) + col;
        if (here == kEnd) {
            store_vec<kEnd, O>(o, rounded_vec<O, kEnd>(y), false);
        } else {
#pragma unroll
            for (int i = 0; i < kEnd; ++i)
                if (i < here) o[i] = rounded<O>(y[i]);
        }
    };
    if (e.pre) put(e.pre, e.pre_line);
    if (e.act != SPDNN_ACT_NONE)
#pragma unroll
        for (int i = 0; i < kEnd; ++i) y[i] = activated(y[i], e.act);
    if (e.add) {
        const O* const a = reinterpret_cast<const O*>(e.add + row * e.add_line) + col;
        if (here == kEnd) {
            const auto v = load_vec<kEnd>(a);
#pragma unroll
            for (int i = 0; i < kEnd; ++i) y[i] += (float)v[i];
        } else {
#pragma unroll
            for (int i = 0; i < kEnd; ++i)
                if (i < here) y[i] += (float)a[i];
        }
    }
    put(e.out + set * e.out_set, e.out_line);
}
template <typename T>
__device__ inline void end_sums(const Ending& e, int set, int64_t row, int col, const float (&sum)[kEnd]) {
    if (sizeof(T) == 2 && e.out_f32) end_sums<T, float>(e, set, row, col, sum);
    else end_sums<T, T>(e, set, row, col, sum);
}
// Zeros, for rows of no expert.
template <typename T>
__device__ inline void end_zeros(const Ending& e, int64_t row, int col) {
    const int size = e.out_f32 ? 4 : (int)sizeof(T);
    const int bytes = min(kEnd, e.cols - col) * size;
    for (char* to : {e.out, e.pre})
        if (to) {
            char* const at = to + row * (to == e.out ? e.out_line : e.pre_line) + (int64_t)col * size;
            for (int i = 0; i < bytes; i += 2) *reinterpret_cast<uint16_t*>(at + i) = 0;
        }
}

// --- which tile -------------------------------------------------------------

// Workgroups go to the 8 XCDs in turn: neighbours in t are made neighbours on one of them, whose L2 they share.
__device__ inline int xcd_order(int bid, int total) {
    const int q = total / 8, r = total % 8, xcd = bid % 8;
    return xcd * q + min(xcd, r) + bid / 8;
}
// Tile t of mtiles x ntiles in bands of `band` m-tiles, column by column.
struct TileAt {
    int m, n;
};
__device__ inline TileAt banded(int t, int mtiles, int ntiles, int band) {
    const int b = t / (band * ntiles), in = t - b * (band * ntiles);
    const int high = min(band, mtiles - b * band);
    return {b * band + in % high, in / high};
}

// Rows of x by expert, in tiles of BM rows that begin with an expert's first: tile t is the (t - start(e))th of the last expert e
// whose start(e) = offsets[e] / BM + e is not beyond t.  (An expert of n rows at offset o needs at most (o + n) / BM + 1 - o / BM
// tiles, so that starts leave room; what is left over has no rows.)  What stands behind the last expert's rows is counted as one more,
// `experts`.  Every lane of a wave gets the same.  Offsets that do not ascend within 0 .. rows give wrong rows, but none outside.
struct RowTile {
    int set;
    int64_t first, last;  // rows; none if first >= last
};
template <int BM>
__device__ inline RowTile row_tile(const int32_t* offsets, int experts, int32_t rows, int t) {
    if (!offsets) return {0, (int64_t)t * BM, rows};
    const int lane = threadIdx.x % 64;
    int before = 0;
    for (int e0 = 0; e0 <= experts; e0 += 64) {
        const int e = e0 + lane;
        const bool in = e <= experts && min(max(offsets[min(e, experts)], 0), rows) / BM + e <= t;
        before += __popcll(__ballot(in));
    }
    const int set = max(before - 1, 0);
    const int first = min(max(offsets[set], 0), rows);
    const int last = set == experts ? rows : min(max(offsets[set + 1], first), rows);
    const int tile = t - (first / BM + set);
    if (tile < 0) return {set, last, last};
    return {set, first + (int64_t)tile * BM, last};
}

// --- the product of a tile --------------------------------------------------
//
// A workgroup of WM x WN waves, each with MF x 4 fragments: WM * MF * 16 lines of a, WN * 64 lines of b.
template <typename T, int MF, int WM, int WN>
struct Shape {
    static constexpr int kThreads = WM * WN * 64;
    static constexpr int kM = WM * MF * 16;
    static constexpr int kN = WN * 64;
};

template <typename T, Adjacent AA, Adjacent AB, int MF, int WM, int WN, bool DMA>
struct TileProduct {
    using S = Shape<T, MF, WM, WN>;
    using A = Tile<T, AA, S::kM, S::kThreads>;
    using B = Tile<T, AB, S::kN, S::kThreads>;
    static constexpr int kStage = A::kBytes + B::kBytes;
    static constexpr int kEndBytes = WM * WN * (MF < 4 ? MF : 4) * 16 * 64 * 4;
    static constexpr int kLds = 2 * kStage > kEndBytes ? 2 * kStage : kEndBytes;

    Acc acc[MF][4];

    __device__ void step(const char* stage, int lane, int wm, int wn) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            Frag<T> a[MF], b[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) b[n] = B::read(stage + A::kBytes, wn * 64 + n * 16, half, lane);
#pragma unroll
            for (int m = 0; m < MF; ++m) a[m] = A::read(stage, (wm * MF + m) * 16, half, lane);
#pragma unroll
            for (int m = 0; m < MF; ++m)
#pragma unroll
                for (int n = 0; n < 4; ++n) acc[m][n] = mma(b[n], a[m], acc[m][n]);
        }
    }
    static constexpr int kPart = MF / 2 > 0 ? MF / 2 : 1;
    static constexpr int kReadsA = kPart * (AA == Adjacent::K ? 1 : sizeof(T) == 2 ? 2 : 4);
    static constexpr int kReadsB = 4 * (AB == Adjacent::K ? 1 : sizeof(T) == 2 ? 2 : 4);
    __device__ static void read_b(const char* stage, int half, int lane, int wn, Frag<T> (&b)[4]) {
#pragma unroll
        for (int n = 0; n < 4; ++n) b[n] = B::read(stage + A::kBytes, wn * 64 + n * 16, half, lane);
    }
    __device__ static void read_a(const char* stage, int half, int part, int lane, int wm, Frag<T> (&a)[kPart]) {
#pragma unroll
        for (int m = 0; m < kPart; ++m) a[m] = A::read(stage, (wm * MF + part * kPart + m) * 16, half, lane);
    }
    template <int PART>
    __device__ void multiply(const Frag<T> (&a)[kPart], const Frag<T> (&b)[4]) {
#pragma unroll
        for (int m = 0; m < kPart; ++m)
#pragma unroll
            for (int n = 0; n < 4; ++n) acc[PART * kPart + m][n] = mma(b[n], a[m], acc[PART * kPart + m][n]);
    }
    // READS reads of what comes next between the products of now.
    template <int READS>
    __device__ static void interleave() {
        constexpr int kProducts = kPart * 4 * (sizeof(T) == 2 ? 1 : 4);
        constexpr int kBetween = kProducts / READS > 0 ? kProducts / READS : 1;
        constexpr int kTogether = (READS + kProducts - 1) / kProducts;
#pragma unroll
        for (int i = 0; i < READS / kTogether; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, kTogether, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, kBetween, 0);
        }
    }
    // a, b: the first number of the tile's lines at the first k; alines, blines: lines there are; ks: k there are.
    __device__ void run(char* lds, const char* a, int64_t aline, int alines, const char* b, int64_t bline, int blines, int64_t ks) {
        const int thread = threadIdx.x, lane = thread % 64, wave = thread / 64, wm = wave / WN, wn = wave % WN;
#pragma unroll
        for (int m = 0; m < MF; ++m)
#pragma unroll
            for (int n = 0; n < 4; ++n) acc[m][n] = Acc{0, 0, 0, 0};
        const int64_t astep = AA == Adjacent::K ? 128 : aline * A::kStep;
        const int64_t bstep = AB == Adjacent::K ? 128 : bline * B::kStep;
        if constexpr (DMA) {
            const int w = __builtin_amdgcn_readfirstlane(wave);
            ByDma<T, AA, S::kM, S::kThreads> da;
            ByDma<T, AB, S::kN, S::kThreads> db;
            da.begin(aline, thread);
            db.begin(bline, thread);
            const auto load = [&](char* to) {
                da.load(a, to, alines, ks, thread, w);
                db.load(b, to + A::kBytes, blines, ks, thread, w);
                ks -= A::kStep;
                a += astep;
                b += bstep;
            };
            if (ks <= 0) return;
            // Four parts a step: while the products of one run, what the next needs is read.  The reads of the last part are those of the next
            // step's first (behind the last step, of what stands there, which nothing uses).
            Frag<T> fa[2][kPart], fb[2][4];
            int64_t steps = (ks + A::kStep - 1) / A::kStep;
            load(lds);
            loads_done();
            __builtin_amdgcn_s_barrier();
            if (ks > 0) load(lds + kStage);
            int at = 0;
            read_b(lds, 0, lane, wn, fb[0]);
            read_a(lds, 0, 0, lane, wm, fa[0]);
            do {
                const char* now = lds + at;
                read_a(now, 0, 1, lane, wm, fa[1]);
                multiply<0>(fa[0], fb[0]);
                interleave<kReadsA>();
                read_b(now, 1, lane, wn, fb[1]);
                read_a(now, 1, 0, lane, wm, fa[0]);
                multiply<1>(fa[1], fb[0]);
                interleave<kReadsA + kReadsB>();
                read_a(now, 1, 1, lane, wm, fa[1]);
                multiply<0>(fa[0], fb[1]);
                interleave<kReadsA>();
                __builtin_amdgcn_sched_barrier(0);
                loads_done();
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_sched_barrier(0);
                if (ks > 0) load(lds + at);
                at = kStage - at;
                now = lds + at;
                read_b(now, 0, lane, wn, fb[0]);
                read_a(now, 0, 0, lane, wm, fa[0]);
                multiply<1>(fa[1], fb[1]);
                interleave<kReadsA + kReadsB>();
                __builtin_amdgcn_sched_barrier(0);
            } while (--steps > 0);
            __syncthreads();
            return;
        }
        ByRegisters<T, AA, S::kM, S::kThreads> ra;
        ByRegisters<T, AB, S::kN, S::kThreads> rb;
        char* now = lds;
        char* next = lds + kStage;
        if (ks > 0) {
            ra.load(a, aline, alines, ks, thread);
            rb.load(b, bline, blines, ks, thread);
            ra.store(now, thread);
            rb.store(now + A::kBytes, thread);
        }
        __syncthreads();
        while (ks > 0) {
            ks -= A::kStep;
            a += astep;
            b += bstep;
            if (ks > 0) {
                ra.load(a, aline, alines, ks, thread);
                rb.load(b, bline, blines, ks, thread);
            }
            step(now, lane, wm, wn);
            if (ks > 0) {
                ra.store(next, thread);
                rb.store(next + A::kBytes, thread);
            }
            __syncthreads();
            char* const t = now;
            now = next;
            next = t;
        }
    }
    // f(line of a, first of 8 lines of b, sums) for all of the tile, by way of LDS: rows of 64 sums of a wave's own, chunk c of row r at
    // place c ^ r % 16.
    template <typename F>
    __device__ void each(char* lds, F f) {
        constexpr int kTurn = MF < 4 ? MF : 4;
        const int thread = threadIdx.x, lane = thread % 64, wave = thread / 64, wm = wave / WN, wn = wave % WN;
        char* const own = lds + wave * (kTurn * 16 * 256);
#pragma unroll
        for (int m0 = 0; m0 < MF; m0 += kTurn) {
#pragma unroll
            for (int m = 0; m < kTurn; ++m)
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    *reinterpret_cast<Acc*>(own + (m * 16 + lane % 16) * 256 + ((n * 4 + lane / 16) ^ (lane % 16)) * 16) = acc[m0 + m][n];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
            for (int r0 = 0; r0 < kTurn * 16; r0 += 8) {
                const int r = r0 + lane / 8, c = lane % 8 * 2;
                const Acc lo = *reinterpret_cast<const Acc*>(own + r * 256 + (c ^ (r % 16)) * 16);
                const Acc hi = *reinterpret_cast<const Acc*>(own + r * 256 + ((c + 1) ^ (r % 16)) * 16);
                const float sum[kEnd] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                f((wm * MF + m0) * 16 + r, wn * 64 + c * 4, sum);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
};

// out[r] = act(x[r] W + b) + add[r].  Tiles of rows by expert, of columns, and of k (splits: the sums go to parts [split][row][col]).
struct Product {
    Side x, w;
    const int32_t* offsets;
    int32_t rows, width, cols, experts;
    int32_t mtiles, ntiles, splits;
    int64_t per_split;  // k of a split, a multiple of a step
    float* parts;
};

template <typename T, Adjacent AB, int MF, int WM, int WN, bool DMA>
__global__ __launch_bounds__(WM* WN * 64) void linear_kernel(Product p, Ending e) {
    using P = TileProduct<T, Adjacent::K, AB, MF, WM, WN, DMA>;
    __shared__ __align__(16) char lds[P::kLds];
    constexpr int BM = P::S::kM, BN = P::S::kN;
    const int per = p.mtiles * p.ntiles;
    const int t = xcd_order(blockIdx.x, gridDim.x);
    const int split = t / per;
    const TileAt tile = banded(t - split * per, p.mtiles, p.ntiles, 8);
    const RowTile r = row_tile<BM>(p.offsets, p.experts, p.rows, tile.m);
    if (r.first >= r.last) return;
    const int n0 = tile.n * BN;
    if (r.set == p.experts) {  // rows of no expert
        if (split == 0 && p.splits == 1)
            for (int64_t row = r.first + threadIdx.x / (BN / kEnd); row < min(r.last, r.first + BM); row += blockDim.x / (BN / kEnd)) {
                const int col = n0 + threadIdx.x % (BN / kEnd) * kEnd;
                if (col < p.cols) end_zeros<T>(e, row, col);
            }
        return;
    }
    const int64_t k0 = split * p.per_split;
    const int64_t ks = min(p.per_split, p.width - k0);
    const char* const a = p.x.p + r.first * p.x.line + k0 * sizeof(T);
    const char* const b = p.w.p + r.set * p.w.set + (AB == Adjacent::K ? n0 * p.w.line + k0 * sizeof(T) : k0 * p.w.line + n0 * sizeof(T));
    P product;
    product.run(lds, a, p.x.line, (int)min((int64_t)BM, r.last - r.first), b, p.w.line, min(BN, p.cols - n0), ks);
    product.each(lds, [&](int line, int col, const float(&sum)[kEnd]) {
        const int64_t row = r.first + line;
        col += n0;
        if (row >= r.last || col >= p.cols) return;
        if (p.splits == 1) {
            end_sums<T>(e, r.set, row, col, sum);
        } else {
            float* const to = p.parts + ((int64_t)split * p.rows + row) * p.cols + col;
#pragma unroll
            for (int i = 0; i < kEnd; ++i)
                if (col + i < p.cols) to[i] = sum[i];
        }
    });
}

// The same for few rows (R * 16 of a tile), where the weights' bytes are what counts.  Every wave has all of the tile (NF * 16 columns) and
// every KW-th step of k, for which it keeps D stages of its own in LDS under way, without a barrier; the waves' sums are added in order.
template <typename T, Adjacent AB, int R, int NF, int KW, int D>
__global__ __launch_bounds__(KW * 64) void linear_short_kernel(Product p, Ending e) {
    using A = Tile<T, Adjacent::K, R * 16, 64>;
    using B = Tile<T, AB, NF * 16, 64>;
    constexpr int kStage = A::kBytes + B::kBytes, kOwn = D * kStage, kSums = R * 16 * NF * 64;
    static_assert(kSums <= kOwn);
    constexpr int BM = R * 16, BN = NF * 16;
    __shared__ __align__(16) char lds[KW * kOwn];
    const int per = p.mtiles * p.ntiles;
    const int t = xcd_order(blockIdx.x, gridDim.x);
    const int split = t / per;
    const TileAt tile = banded(t - split * per, p.mtiles, p.ntiles, 8);
    const RowTile r = row_tile<BM>(p.offsets, p.experts, p.rows, tile.m);
    if (r.first >= r.last) return;
    const int n0 = tile.n * BN;
    if (r.set == p.experts) {  // rows of no expert
        if (split == 0 && p.splits == 1)
            for (int64_t row = r.first + threadIdx.x / (BN / kEnd); row < min(r.last, r.first + BM); row += KW * 64 / (BN / kEnd)) {
                const int col = n0 + threadIdx.x % (BN / kEnd) * kEnd;
                if (col < p.cols) end_zeros<T>(e, row, col);
            }
        return;
    }
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t k0 = split * p.per_split + wave * A::kStep;
    int64_t ks = min(p.per_split - wave * A::kStep, p.width - k0);  // from this wave's first step on
    const int alines = (int)min((int64_t)BM, r.last - r.first), blines = min(BN, p.cols - n0);
    const char* a = p.x.p + r.first * p.x.line + k0 * (int64_t)sizeof(T);
    const char* b = p.w.p + r.set * p.w.set + (AB == Adjacent::K ? n0 * p.w.line + k0 * (int64_t)sizeof(T) : k0 * p.w.line + n0 * (int64_t)sizeof(T));
    const int64_t astep = KW * 128, bstep = AB == Adjacent::K ? KW * 128 : p.w.line * A::kStep * KW;
    ByDma<T, Adjacent::K, R * 16, 64> da;
    ByDma<T, AB, BN, 64> db;
    da.begin(p.x.line, lane);
    db.begin(p.w.line, lane);
    char* const own = lds + wave * kOwn;
    const auto load = [&](int stage) {
        da.load(a, own + stage * kStage, alines, ks, lane, 0);
        db.load(b, own + stage * kStage + A::kBytes, blines, ks, lane, 0);
        ks -= KW * A::kStep;
        a += astep;
        b += bstep;
    };
    Acc acc[R][NF];
#pragma unroll
    for (int m = 0; m < R; ++m)
#pragma unroll
        for (int n = 0; n < NF; ++n) acc[m][n] = Acc{0, 0, 0, 0};
    int64_t steps = ks > 0 ? (ks - 1) / (KW * A::kStep) + 1 : 0;
#pragma unroll
    for (int i = 0; i < D; ++i) load(i);
    int stage = 0;
    for (; steps > 0; --steps) {
        constexpr int kLater = (D - 1) * (A::kChunks + B::kChunks);  // loads that were asked for behind this stage's
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLater) : "memory");
        Frag<T> fa[2][R], fb[2][NF];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int n = 0; n < NF; ++n) fb[half][n] = B::read(own + stage * kStage + A::kBytes, n * 16, half, lane);
#pragma unroll
            for (int m = 0; m < R; ++m) fa[half][m] = A::read(own + stage * kStage, m * 16, half, lane);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        load(stage);
        stage = stage == D - 1 ? 0 : stage + 1;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int m = 0; m < R; ++m)
#pragma unroll
                for (int n = 0; n < NF; ++n) acc[m][n] = mma(fb[half][n], fa[half][m], acc[m][n]);
    }
    loads_done();  // (those behind the last step too: they store zeros)
#pragma unroll
    for (int m = 0; m < R; ++m)
#pragma unroll
        for (int n = 0; n < NF; ++n)
            *reinterpret_cast<Acc*>(own + (m * 16 + lane % 16) * (NF * 64) + ((n * 4 + lane / 16) ^ (lane % (NF * 4))) * 16) = acc[m][n];
    __syncthreads();
    for (int i = threadIdx.x; i < BM * (BN / kEnd); i += KW * 64) {
        const int line = i / (BN / kEnd), c = i % (BN / kEnd) * 2;
        const int64_t row = r.first + line;
        const int col = n0 + c * 4;
        if (row >= r.last || col >= p.cols) continue;
        float sum[kEnd] = {};
#pragma unroll
        for (int w = 0; w < KW; ++w) {
            const Acc lo = *reinterpret_cast<const Acc*>(lds + w * kOwn + line * (NF * 64) + (c ^ (line % (NF * 4))) * 16);
            const Acc hi = *reinterpret_cast<const Acc*>(lds + w * kOwn + line * (NF * 64) + ((c + 1) ^ (line % (NF * 4))) * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sum[j] += lo[j];
                sum[j + 4] += hi[j];
            }
        }
        if (p.splits == 1) {
            end_sums<T>(e, r.set, row, col, sum);
        } else {
            float* const to = p.parts + ((int64_t)split * p.rows + row) * p.cols + col;
#pragma unroll
            for (int j = 0; j < kEnd; ++j)
                if (col + j < p.cols) to[j] = sum[j];
        }
    }
}

// Parts of sums added up, split by split.
template <typename T>
__global__ __launch_bounds__(256) void linear_join_kernel(Product p, Ending e) {
    const int vecs = (p.cols - 1) / kEnd + 1;
    const int64_t items = (int64_t)p.rows * vecs;
    for (int64_t i0 = (int64_t)blockIdx.x * 256; i0 < items; i0 += (int64_t)gridDim.x * 256) {
        const int64_t i = i0 + threadIdx.x;
        if (i >= items) continue;
        const int64_t row = i / vecs;
        const int col = (int)(i - row * vecs) * kEnd;
        int set = 0;
        if (p.offsets) {  // the last expert that begins at the row or before
            int lo = 0, hi = p.experts + 1;
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (p.offsets[mid] <= row) lo = mid;
                else hi = mid;
            }
            set = lo;
        }
        if (set == p.experts) {
            end_zeros<T>(e, row, col);
            continue;
        }
        float sum[kEnd] = {};
        for (int s = 0; s < p.splits; ++s) {
            const float* const from = p.parts + ((int64_t)s * p.rows + row) * p.cols + col;
#pragma unroll
            for (int j = 0; j < kEnd; ++j)
                if (col + j < p.cols) sum[j] += from[j];
        }
        end_sums<T>(e, set, row, col, sum);
    }
}

// --- gradients --------------------------------------------------------------

// d[r] = dout[r] * act'(pre[r]) in the rows' type, rows of no expert left out: what both products of the gradient take.  The matrix
// instructions take 16 bits a number: this is where the slope's product is rounded to them.
template <typename T, typename D>
__global__ __launch_bounds__(256) void slope_kernel(const D* dout, int64_t dout_stride, const D* pre, int64_t pre_stride, int act, int32_t rows,
                                                    int32_t cols, const int32_t* offsets, int32_t experts, T* d, int64_t d_stride) {
    constexpr int V = 8;
    const int vecs = (cols - 1) / V + 1;
    const int64_t used = offsets ? min(max(offsets[experts], 0), rows) : rows;
    const int64_t items = used * vecs;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / vecs;
        const int col = (int)(i - row * vecs) * V;
        const D* const from = dout + row * dout_stride + col;
        const D* const at = pre ? pre + row * pre_stride + col : nullptr;
        T* const to = d + row * d_stride + col;
        if (col + V <= cols) {
            const auto x = load_vec<V>(from);
            float y[V];
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] = (float)x[j];
            if (at) {
                const auto z = load_vec<V>(at);
#pragma unroll
                for (int j = 0; j < V; ++j) y[j] *= act_slope((float)z[j], act);
            }
            store_vec<V, T>(to, rounded_vec<T, V>(y), false);
        } else {
            for (int j = 0; col + j < cols; ++j) to[j] = rounded<T>((float)from[j] * (at ? act_slope((float)at[j], act) : 1.0f));
        }
    }
}

// dW[e] = sum over the rows of expert e of a[r] b[r]^T, a and b being x and d, or d and x where W is stored the other way round.  Sums
// of long batches are split: parts [split][expert][line of a][line of b].
struct WeightGrad {
    Side a, b;
    const int32_t* offsets;
    int32_t rows, m, n, experts;
    int32_t mtiles, ntiles, splits;
    float* parts;
};

// Rows of expert `set` that split `split` adds.
struct RowRange {
    int64_t first, last;
};
template <int STEP>
__device__ inline RowRange grad_rows(const int32_t* offsets, int32_t rows, int set, int split, int splits) {
    int64_t first = 0, last = rows;
    if (offsets) {
        first = min(max(offsets[set], 0), rows);
        last = min(max((int64_t)offsets[set + 1], first), (int64_t)rows);
    }
    const int64_t steps = (last - first + STEP - 1) / STEP;
    const int64_t per = (steps + splits - 1) / splits * STEP;
    first = min(first + per * split, last);
    return {first, min(first + per, last)};
}

template <typename T, int MF, int WM, int WN, bool DMA>
__global__ __launch_bounds__(WM* WN * 64) void weight_grad_kernel(WeightGrad p, Ending e) {
    using P = TileProduct<T, Adjacent::L, Adjacent::L, MF, WM, WN, DMA>;
    __shared__ __align__(16) char lds[P::kLds];
    constexpr int BM = P::S::kM, BN = P::S::kN;
    const int per = p.mtiles * p.ntiles;
    const int t = xcd_order(blockIdx.x, gridDim.x);
    const int set = t / per % p.experts, split = t / per / p.experts;
    const TileAt tile = banded(t % per, p.mtiles, p.ntiles, 8);
    const RowRange r = grad_rows<P::A::kStep>(p.offsets, p.rows, set, split, p.splits);
    const int m0 = tile.m * BM, n0 = tile.n * BN;
    const char* const a = p.a.p + r.first * p.a.line + m0 * sizeof(T);
    const char* const b = p.b.p + r.first * p.b.line + n0 * sizeof(T);
    P product;
    product.run(lds, a, p.a.line, min(BM, p.m - m0), b, p.b.line, min(BN, p.n - n0), r.last - r.first);
    product.each(lds, [&](int line, int col, const float(&sum)[kEnd]) {
        line += m0;
        col += n0;
        if (line >= p.m || col >= p.n) return;
        if (p.splits == 1) {
            end_sums<T>(e, set, line, col, sum);
        } else {
            float* const to = p.parts + (((int64_t)split * p.experts + set) * p.m + line) * p.n + col;
#pragma unroll
            for (int i = 0; i < kEnd; ++i)
                if (col + i < p.n) to[i] = sum[i];
        }
    });
}

template <typename T>
__global__ __launch_bounds__(256) void weight_grad_join_kernel(WeightGrad p, Ending e) {
    const int vecs = (p.n - 1) / kEnd + 1;
    const int64_t lines = (int64_t)p.experts * p.m, items = lines * vecs;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
        const int64_t line = i / vecs;
        const int col = (int)(i - line * vecs) * kEnd;
        float sum[kEnd] = {};
        for (int s = 0; s < p.splits; ++s) {
            const float* const from = p.parts + (s * lines + line) * p.n + col;
#pragma unroll
            for (int j = 0; j < kEnd; ++j)
                if (col + j < p.n) sum[j] += from[j];
        }
        end_sums<T>(e, (int)(line / p.m), line % p.m, col, sum);
    }
}

// dbias[e][c] = sum over the rows of expert e of d[r][c]: a workgroup has 64 columns; its four waves add every fourth row, and
// their sums are added in order.
template <typename T>
__global__ __launch_bounds__(256) void bias_grad_kernel(const T* d, int64_t d_stride, const int32_t* offsets, int32_t rows, int32_t cols, int32_t splits,
                                                        float* parts, void* dbias, bool f32) {
    __shared__ float sums[4][64];
    const int set = blockIdx.y, split = blockIdx.z, col = blockIdx.x * 64 + threadIdx.x % 64, wave = threadIdx.x / 64;
    const RowRange r = grad_rows<1>(offsets, rows, set, split, splits);
    float sum = 0;
    if (col < cols)
        for (int64_t row = r.first + wave; row < r.last; row += 4) sum += (float)d[row * d_stride + col];
    sums[wave][threadIdx.x % 64] = sum;
    __syncthreads();
    if (wave || col >= cols) return;
    for (int w = 1; w < 4; ++w) sum += sums[w][threadIdx.x];
    const int64_t at = (int64_t)set * cols + col;
    if (splits > 1) parts[split * ((int64_t)gridDim.y * cols) + at] = sum;
    else if (f32) ((float*)dbias)[at] = sum;
    else ((T*)dbias)[at] = rounded<T>(sum);
}
template <typename T>
__global__ __launch_bounds__(256) void bias_grad_join_kernel(const float* parts, int32_t splits, int64_t n, void* dbias, bool f32) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float sum = 0;
    for (int s = 0; s < splits; ++s) sum += parts[s * n + i];
    if (f32) ((float*)dbias)[i] = sum;
    else ((T*)dbias)[i] = rounded<T>(sum);
}

}  // namespace spdnn
