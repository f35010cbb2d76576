// Kernels of the dense products (spdnn_linear, spdnn_linear_grad of include/spdnn.h): act(x W + b) + add for one matrix W or for
// every expert's own on rows sorted by expert, and the gradients.  T: type of rows and weights (float, __bf16, _Float16).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "../../include/spdnn.h"
#include "spdnn_linear_plan.h"
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

// exp for results of 16 bits (EXACT: of 32): exp2 of the hardware, off by an ulp and by 2 U |x| of its argument.  (Slopes of 8000 x
// 16384 numbers by the library's expf and erff: 183 us, where memory asks for 125.)
template <bool EXACT>
__device__ inline float act_exp(float x) {
    if constexpr (EXACT) return expf(x);
    else return __builtin_amdgcn_exp2f(x * 1.44269504f);
}
// What the normal distribution has above a >= 0: erfc(a / sqrt 2) / 2, from bell = exp(-a^2 / 2).  gelu(x) is max(x, 0) - a tail(a) with a =
// |x|: in 1 + erf a negative x loses its digits.  For 16 bits bell times a polynomial of t = 1 / (1 + 0.42 a / sqrt 2) without constant
// term, whose six coefficients were fitted here: off by less than 1.5e-7, and by less than 6e-5 of itself down to where floats end (half a
// unit of fp16 is 4.9e-4).  24000 x 4096 x 4096 bf16: 740 us with 1 + erf, 745 so; floats, by erfcf, 4096 x 128 x 8192: 118
// and 133.
template <bool EXACT>
__device__ inline float act_tail(float a, float bell) {
    if constexpr (EXACT) return 0.5f * erfcf(a * 0.70710678f);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.29698485f, a, 1.0f));
    const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, -0.081158183f, 0.23612749f), -0.036497519f), 0.15147993f), 0.1110982f), 0.11894995f);
    return poly * bell;
}
// |x|, but 64 at the most, where bell and the tail are 0: an infinity has the limits, gelu 0 and x, slopes 0 and 1.  A NaN stays one.
__device__ inline float act_size(float x) { return fabsf(x) > 64.0f ? 64.0f : fabsf(x); }
// What a sigmoid is multiplied with: within the range where it is neither 0 nor 1 in 32 bits, so that infinities have their limits here too.
__device__ inline float act_within(float x) { return x < -128.0f ? -128.0f : x > 128.0f ? 128.0f : x; }
// A NaN stays one.
template <bool EXACT>
__device__ __forceinline__ float activated(float x, int act) {
    switch (act) {
        case SPDNN_ACT_RELU: return x < 0.0f ? 0.0f : x;
        case SPDNN_ACT_CLIP: return x < 0.0f ? 0.0f : x > kClip ? kClip : x;
        case SPDNN_ACT_GELU: {
            const float a = act_size(x);
            return (x < 0.0f ? 0.0f : x) - a * act_tail<EXACT>(a, EXACT ? 0.0f : act_exp<EXACT>(-0.5f * a * a));
        }
        case SPDNN_ACT_SILU: {
            const float y = x < -128.0f ? -128.0f : x;
            return EXACT ? y / (1.0f + expf(-y)) : y * __builtin_amdgcn_rcpf(1.0f + act_exp<EXACT>(-y));
        }
    }
    return x;
}
template <bool EXACT>
__device__ inline float act_slope(float x, int act) {
    switch (act) {
        case SPDNN_ACT_RELU: return x <= 0.0f ? 0.0f : 1.0f;
        case SPDNN_ACT_CLIP: return x <= 0.0f || x >= kClip ? 0.0f : 1.0f;
        case SPDNN_ACT_GELU: {
            const float a = act_size(x), bell = act_exp<EXACT>(-0.5f * a * a);
            const float below = fmaf(-a, 0.39894228f * bell, act_tail<EXACT>(a, bell));  // the slope at -a
            return x < 0.0f ? below : 1.0f - below;
        }
        case SPDNN_ACT_SILU: {
            const float s = EXACT ? 1.0f / (1.0f + expf(-x)) : __builtin_amdgcn_rcpf(1.0f + act_exp<EXACT>(-x));
            return s + act_within(x) * s * (1.0f - s);
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

    __device__ static int turn(int k) {  // f(k) of Adjacent::L
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
// beyond the last, and what lies behind the last k (Adjacent::K: a lane whose chunk does has kOutside added to its offset; of a chunk
// that is there in part, clear() clears the rest).  Addresses may have any alignment; a tile's lines lie within kDmaSpan bytes, and the k
// rows of Adjacent::L do not overlap.  The range check goes by words of 4 bytes.  Where the last memory row of a tile ends within one, the
// range takes in the two bytes behind it if the matrix goes on there (`follows`), and otherwise patch() stores the number that is missing.
//
// They are written as instructions: the compiler would let the transposing LDS reads wait for all loads of this kind that are under way,
// for it cannot tell that they go to the other stage.  Whoever reads what they have stored waits for its count (or all, loads_done()) and at a barrier first.
constexpr uint32_t kOutside = 1u << 31;
using Memory __attribute__((ext_vector_type(4))) = int;  // address, bytes, format: the same for all lanes
// past: leaves nothing in the caches.
template <bool PAST>
__device__ inline void load_to_lds(Memory memory, uint32_t offset, char* lds, const int more) {
    const int to = __builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds);
    if constexpr (PAST)
        asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 4\n\tbuffer_load_dwordx4 %2, %3, 0 offen nt lds"
                     :
                     : "s"(to), "i"(more), "v"(offset), "s"(memory)
                     : "memory", "scc", "m0");
    else
        asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 4\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds"
                     :
                     : "s"(to), "i"(more), "v"(offset), "s"(memory)
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
    bool follows;
    __device__ void begin(int64_t line_bytes, bool goes_on, int thread) {
        follows = goes_on;
        line = (uint32_t)line_bytes;
        step = kRows * kBases * line;
#pragma unroll
        for (int c = 0; c < kBases; ++c) {
            const auto at = G::at(c * THREADS + thread);
            from[c] = (uint32_t)at.row * line + at.chunk * 16;
        }
    }
    // Clears what the last chunk of k has behind the last k: ks of a step that is not whole.  To be called between barriers.
    __device__ static void clear(char* tile, int ks, int thread) {
        if constexpr (ADJ == Adjacent::K)
#pragma unroll 1
            for (int line = thread; line < LINES; line += THREADS)
#pragma unroll 1
                for (int i = ks % G::kChunk; i < G::kChunk; ++i)
                    reinterpret_cast<T*>(tile + line * 128 + (ks / G::kChunk ^ (line >> 1 & 7)) * 16)[i] = (T)0.0f;
    }
    // Whether the last number of the last memory row is missing in a last step of k, and the store of it.  p: as for begin_step.
    __device__ __forceinline__ bool misses(int lines, int k) const { return sizeof(T) == 2 && !follows && ((ADJ == Adjacent::K ? k : lines) & 1); }
    __device__ void patch(const char* p, char* tile, int lines, int k, int thread) const {
        if (!misses(lines, k) || thread != 0) return;
        const int row = ADJ == Adjacent::K ? lines - 1 : k - 1, col = ADJ == Adjacent::K ? k - 1 : lines - 1;  // of memory
        constexpr int kRow = G::kPerRow * 16;
        const int place = ADJ == Adjacent::K ? col / G::kChunk ^ (row >> 1 & 7) : col / G::kChunk ^ G::turn(row) * G::kBlock;
        reinterpret_cast<T*>(tile + row * kRow + place * 16)[col % G::kChunk] = reinterpret_cast<const T*>(p + (int64_t)row * line)[col];
    }
    // Loads of one step, to be asked for one chunk of every lane after the other.  lines, ks: what there is of both from p on.
    struct Step {
        Memory memory;
        uint32_t at[kBases], step;
        char* tile;
        template <bool PAST = false>
        __device__ __forceinline__ void load(int c) const {
            load_to_lds<PAST>(memory, at[c % kBases] + c / kBases * step, tile, c * (THREADS * 16));
        }
    };
    __device__ __forceinline__ Step begin_step(const char* p, char* tile, int lines, int64_t ks, int thread, int wave) const {
        const int k = (int)min(ks, (int64_t)G::kStep);  // nothing is loaded if there is none
        uint32_t bytes = k <= 0 ? 0 : ADJ == Adjacent::K ? (lines - 1) * line + k * (uint32_t)sizeof(T) : (k - 1) * line + lines * (uint32_t)sizeof(T);
        if constexpr (sizeof(T) == 2)
            if (k > 0 && (follows || (ADJ == Adjacent::L && ks > G::kStep))) bytes += (ADJ == Adjacent::K ? k & 1 : lines & 1) * 2;
        const uint64_t base = (uint64_t)p;
        Step s;
        s.memory = {__builtin_amdgcn_readfirstlane((int)base), __builtin_amdgcn_readfirstlane((int)(base >> 32) & 0xffff),
                    __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000};
        s.step = step;
        s.tile = tile + wave * 1024;
#pragma unroll
        for (int c = 0; c < kBases; ++c) s.at[c] = from[c];
        if (ADJ == Adjacent::K && k < G::kStep)
#pragma unroll
            for (int c = 0; c < kBases; ++c)
                if (G::at(c * THREADS + thread).chunk * G::kChunk >= k) s.at[c] += kOutside;
        return s;
    }
    template <bool PAST = false>
    __device__ __forceinline__ void load(const char* p, char* tile, int lines, int64_t ks, int thread, int wave) const {
        const Step s = begin_step(p, tile, lines, ks, thread, wave);
#pragma unroll
        for (int c = 0; c < G::kChunks; ++c) s.template load<PAST>(c);
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

// What the eight columns of a lane need besides their sums, asked for before these are there: b is the same for all rows of a tile.
using Words __attribute__((ext_vector_type(4))) = float;
template <typename T>
struct Biases {
    float b[kEnd];
    __device__ __forceinline__ void load(const Ending& e, int set, int col) {
        const int64_t at = (int64_t)set * e.cols + col;
#pragma unroll
        for (int i = 0; i < kEnd; ++i) b[i] = 0.0f;
        if (!e.bias || col + kEnd > e.cols) return;
        if (e.bias_f32) {
            const auto v = load_vec<kEnd>((const float*)e.bias + at);
#pragma unroll
            for (int i = 0; i < kEnd; ++i) b[i] = v[i];
        } else {
            const auto v = load_vec<kEnd>((const T*)e.bias + at);
#pragma unroll
            for (int i = 0; i < kEnd; ++i) b[i] = (float)v[i];
        }
    }
};
template <typename T>
struct Added {
    Words raw[2];
    __device__ __forceinline__ void load(const Ending& e, int64_t row, int col) {
        if (!e.add || col + kEnd > e.cols) return;
        if constexpr (sizeof(T) == 2)
            if (!e.out_f32) {
                raw[0] = __builtin_bit_cast(Words, load_vec<kEnd>(reinterpret_cast<const T*>(e.add + row * e.add_line) + col));
                return;
            }
        const float* const from = reinterpret_cast<const float*>(e.add + row * e.add_line) + col;
        raw[0] = load_vec<4>(from);
        raw[1] = load_vec<4>(from + 4);
    }
    template <typename O>
    __device__ __forceinline__ void add_to(float (&y)[kEnd]) const {
        if constexpr (sizeof(O) == 4) {
#pragma unroll
            for (int i = 0; i < kEnd; ++i) y[i] += raw[i / 4][i % 4];
        } else {
            typedef O Eight __attribute__((ext_vector_type(8)));
            const Eight v = __builtin_bit_cast(Eight, raw[0]);
#pragma unroll
            for (int i = 0; i < kEnd; ++i) y[i] += (float)v[i];
        }
    }
};

// One number, where a row has less than eight left.
template <typename T, typename O>
__device__ inline void end_one(const Ending& e, int set, int64_t row, int col, float y) {
    if (e.bias) {
        const int64_t at = (int64_t)set * e.cols + col;
        y += e.bias_f32 ? ((const float*)e.bias)[at] : (float)((const T*)e.bias)[at];
    }
    if (e.pre) reinterpret_cast<O*>(e.pre + row * e.pre_line)[col] = rounded<O>(y);
    y = activated<sizeof(O) == 4>(y, e.act);
    if (e.add) y += (float)reinterpret_cast<const O*>(e.add + row * e.add_line)[col];
    reinterpret_cast<O*>(e.out + set * e.out_set + row * e.out_line)[col] = rounded<O>(y);
}
// out, pre: where the eight go.
template <typename T, typename O>
__device__ __forceinline__ void end_eight(const Ending& e, char* out, char* pre, float (&y)[kEnd], const Biases<T>& bias, const Added<T>& added) {
    if (e.bias)
#pragma unroll
        for (int i = 0; i < kEnd; ++i) y[i] += bias.b[i];
    if (e.pre) store_vec<kEnd, O>(reinterpret_cast<O*>(pre), rounded_vec<O, kEnd>(y), false);
    if (e.act != SPDNN_ACT_NONE)
#pragma unroll
        for (int i = 0; i < kEnd; ++i) y[i] = activated<sizeof(O) == 4>(y[i], e.act);
    if (e.add) added.template add_to<O>(y);
    store_vec<kEnd, O>(reinterpret_cast<O*>(out), rounded_vec<O, kEnd>(y), false);
}
// Where column `col` of row `row` is in out and in pre.
template <typename T>
struct Places {
    char *out, *pre;
    __device__ __forceinline__ Places(const Ending& e, int set, int64_t row, int col) {
        const int size = sizeof(T) == 4 || e.out_f32 ? 4 : 2;
        out = e.out + set * e.out_set + row * e.out_line + (int64_t)col * size;
        pre = e.pre + row * e.pre_line + (int64_t)col * size;
    }
    __device__ __forceinline__ void down(const Ending& e, int rows) {
        out += rows * e.out_line;
        pre += rows * e.pre_line;
    }
};
template <typename T>
__device__ __forceinline__ void end_sums(const Ending& e, const Places<T>& at, float (&sum)[kEnd], const Biases<T>& bias, const Added<T>& added) {
    if (sizeof(T) == 2 && e.out_f32) end_eight<T, float>(e, at.out, at.pre, sum, bias, added);
    else end_eight<T, T>(e, at.out, at.pre, sum, bias, added);
}
// The columns from `col` to the row's end, where they are less than eight; one(i): the sum of column col + i.
template <typename T, typename F>
__device__ __forceinline__ void end_rest(const Ending& e, int set, int64_t row, int col, F one) {
#pragma unroll 1
    for (int i = 0; col + i < e.cols; ++i) {
        if (sizeof(T) == 2 && e.out_f32) end_one<T, float>(e, set, row, col + i, one(i));
        else end_one<T, T>(e, set, row, col + i, one(i));
    }
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

// Rows of x by expert, in tiles of BM rows that begin with an expert's first; what stands behind the last expert's rows is one more,
// `experts`.  Only tiles with rows are counted: others would make the XCDs' shares uneven (48000 rows of 64 experts, 4096 x 4096 bf16: 1796 us
// with them, 1734 without; 256 rows of 256 experts, 4096 x 1024: 291 and 238).  Every wave counts for itself, a lane experts / 64 + 1 experts side by
// side.  Offsets that do not ascend within 0 .. rows give wrong rows, but none outside.
struct RowTile {
    int set;
    int64_t first, last;  // rows; none if first >= last
};
template <int BM>
struct RowTiles {
    const int32_t* offsets;
    int experts, rows, each;
    int first, own;  // this lane's tiles
    int all;

    __device__ __forceinline__ int expert_first(int e) const { return min(max(offsets[min(e, experts)], 0), rows); }
    __device__ __forceinline__ int expert_last(int e, int from) const { return e >= experts ? rows : min(max(offsets[e + 1], from), rows); }
    __device__ __forceinline__ int expert_tiles(int e) const {
        const int from = expert_first(e), to = expert_last(e, from);
        return e > experts || to <= from ? 0 : (to - from - 1) / BM + 1;
    }
    // Sums over this lane and those before it.
    __device__ __forceinline__ static int upto(int x) {
        const int lane = threadIdx.x % 64;
#pragma unroll
        for (int step = 1; step < 64; step *= 2) {
            const int other = __shfl_up(x, step);
            if (lane >= step) x += other;
        }
        return x;
    }
    // others: tiles of the launch, which are all where there are no offsets.
    __device__ __forceinline__ RowTiles(const int32_t* o, int e, int32_t r, int others) : offsets(o), experts(e), rows(r), each(e / 64 + 1), first(0), own(0), all(others) {
        if (!offsets) return;
        const int lane = threadIdx.x % 64;
#pragma unroll 4
        for (int i = 0; i < each; ++i) own += expert_tiles(lane * each + i);
        own = min(own, others);  // (of wrong offsets more, whose sums would pass 32 bits)
        const int until = upto(own);
        first = until - own;
        all = min(__builtin_amdgcn_readlane(until, 63), others);
    }
    // Tile t of all * ntiles, and its columns'.  Bands of eight tiles of rows, so that an XCD's workgroups share W's columns and x's
    // rows in its L2; EACH: bands that end with an expert's rows, so that they share one W (48000 rows of 64 experts, 4096 x 4096 bf16: 1684
    // us, so 1580 to 1610).  For few rows, where no W is shared, bands over experts are better by up to 15 %.
    template <bool EACH>
    __device__ __forceinline__ RowTile tile(int t, int ntiles, int* n) const {
        TileAt at = banded(t, all, ntiles, 8);
        int set = 0, begin = 0, count = all, from = 0, to = rows;
        if (offsets) {
            const int m = EACH ? t / ntiles : at.m;
            const uint64_t found = __ballot(m >= first && m < first + own);
            if (!found) return {0, rows, rows};
            const int lane = __ffsll((unsigned long long)found) - 1;
            set = lane * each;
            begin = __builtin_amdgcn_readlane(first, lane);
            count = __builtin_amdgcn_readlane(own, lane);
            if (each > 1) {
                const int mine = (int)(threadIdx.x % 64) < each ? expert_tiles(set + (int)(threadIdx.x % 64)) : 0;
                const int until = begin + upto(mine);
                const uint64_t which = __ballot(m >= until - mine && m < until);
                if (!which) return {0, rows, rows};
                const int next = __ffsll((unsigned long long)which) - 1;
                set += next;
                count = __builtin_amdgcn_readlane(mine, next);
                begin = __builtin_amdgcn_readlane(until, next) - count;
            }
            from = expert_first(set);
            to = expert_last(set, from);
            if (EACH) at = banded(t - begin * ntiles, count, ntiles, 8);
            else at.m -= begin;
        }
        *n = at.n;
        return {set, from + (int64_t)at.m * BM, to};
    }
};

// --- the product of a tile --------------------------------------------------
//
// Bound by the matrix instructions and, for tiles of 256, by the power that they may take: 8192 x 8192 x 8192 bf16 1330 TFLOP/s with k
// adjacent in both operands, 1400 else (products alone, on what registers hold, 2000; the library's best 1530, 1220 and 1080 for the
// three layouts), floats 146 to 149 (154).  Neither 160 KB of stages with half the step, nor four waves of 128 x 128, nor one barrier for
// fewer products gave more.  A wave of a tile of 256 x 256 reads 12 KB of LDS for 32 instructions: three quarters of what LDS gives in that
// time; smaller tiles read more for each product, and are taken where there are few tiles or little k (choose() of spdnn_linear.hip).
//
// A workgroup of WM x WN waves, each with MF x NF fragments: WM * MF * 16 lines of a, WN * NF * 16 lines of b.
// With operands that go straight to LDS, STAGES steps of k are there or under way.
template <int MF, int NF, int WM, int WN, int STAGES>
struct Shape {
    static constexpr int kMF = MF, kNF = NF, kWM = WM, kWN = WN, kStages = STAGES;
    static constexpr int kThreads = WM * WN * 64;
    static constexpr int kM = WM * MF * 16;
    static constexpr int kN = WN * NF * 16;
};
using Large = Shape<8, 4, 2, 4, 2>;  // 256 x 256
// 128 x 128 and 64 x 64; where a CU has no second workgroup, with a stage more, as nothing else covers the loads' way (4096 k of
// bf16, 256 tiles: 60.7 and 54.1 us, 39.6 and 29.8; with 512 tiles 80 and 115, 40 and 37, and with 1024 57 and 68).
template <int STAGES>
using Middle = Shape<4, 4, 2, 2, STAGES>;
template <int STAGES>
using Small = Shape<2, 2, 2, 2, STAGES>;

template <typename T, Adjacent AA, Adjacent AB, typename SHAPE, bool DMA>
struct TileProduct {
    using S = SHAPE;
    static constexpr int MF = S::kMF, NF = S::kNF, WM = S::kWM, WN = S::kWN;
    using A = Tile<T, AA, S::kM, S::kThreads>;
    using B = Tile<T, AB, S::kN, S::kThreads>;
    static constexpr int kStage = A::kBytes + B::kBytes;
    static constexpr int kEndBytes = WM * WN * (MF < 4 ? MF : 4) * 16 * NF * 64;
    static constexpr int kStages = DMA ? S::kStages : 2;
    static constexpr int kLds = kStages * kStage > kEndBytes ? kStages * kStage : kEndBytes;

    Acc acc[MF][NF];
    // Sums over k of the lines of b (OF_B) or of a (OF_A), products with ones beside the others: one accumulator a fragment, for lines that
    // are not there may hold anything, which must not meet another line's sum, not even times zero.  a's fragments are shared out to the
    // WN waves that have the same, one of a part each.
    Acc sums[NF > 2 ? NF : 2];

    enum { NO_SUMS = 0, OF_A = 1, OF_B = 2 };
    template <int OF>
    __device__ __forceinline__ void step(const char* stage, int lane, int wm, int wn) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            Frag<T> a[2][kPart], b[NF];
            read_b(stage, half, lane, wn, b);
            read_a(stage, half, 0, lane, wm, a[0]);
            read_a(stage, half, 1, lane, wm, a[1]);
            multiply<0, OF>(a[0], b);
            multiply<1, OF>(a[1], b);
        }
    }
    static_assert(MF % 2 == 0);
    static constexpr int kPart = MF / 2;
    static constexpr int kReadsA = kPart * (AA == Adjacent::K ? 1 : sizeof(T) == 2 ? 2 : 4);
    static constexpr int kReadsB = NF * (AB == Adjacent::K ? 1 : sizeof(T) == 2 ? 2 : 4);
    __device__ static void read_b(const char* stage, int half, int lane, int wn, Frag<T> (&b)[NF]) {
#pragma unroll
        for (int n = 0; n < NF; ++n) b[n] = B::read(stage + A::kBytes, (wn * NF + n) * 16, half, lane);
    }
    __device__ static void read_a(const char* stage, int half, int part, int lane, int wm, Frag<T> (&a)[kPart]) {
#pragma unroll
        for (int m = 0; m < kPart; ++m) a[m] = A::read(stage, (wm * MF + part * kPart + m) * 16, half, lane);
    }
    static constexpr int kLoads = A::kChunks + B::kChunks;  // of a step
    static_assert(kPart <= WN);
    template <int PART>
    __device__ __forceinline__ void sum_a(const Frag<T> (&a)[kPart]) {
        const int wn = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) % WN;
        typedef int Bits __attribute__((ext_vector_type(4)));
        Frag<T> ones;
        for (int i = 0; i < A::kChunk; ++i) ones[i] = (T)1.0f;
        Bits own = __builtin_bit_cast(Bits, a[0]) & (wn == 0 ? -1 : 0);  // (a choice between fragments would put them into memory)
#pragma unroll
        for (int m = 1; m < kPart; ++m) own |= __builtin_bit_cast(Bits, a[m]) & (wn == m ? -1 : 0);
        sums[PART] = mma(ones, __builtin_bit_cast(Frag<T>, own), sums[PART]);
    }
    template <int PART>
    __device__ __forceinline__ void multiply_line(int m, const Frag<T>& a, const Frag<T> (&b)[NF]) {
#pragma unroll
        for (int n = 0; n < NF; ++n) acc[PART * kPart + m][n] = mma(b[n], a, acc[PART * kPart + m][n]);
    }
    template <int PART, int OF>
    __device__ __forceinline__ void multiply(const Frag<T> (&a)[kPart], const Frag<T> (&b)[NF]) {
        Frag<T> ones;
        for (int i = 0; i < A::kChunk; ++i) ones[i] = (T)1.0f;
        if constexpr (OF == OF_B && PART == 0)
#pragma unroll
            for (int n = 0; n < NF; ++n) sums[n] = mma(b[n], ones, sums[n]);
        if constexpr (OF == OF_A) sum_a<PART>(a);
#pragma unroll
        for (int m = 0; m < kPart; ++m)
#pragma unroll
            for (int n = 0; n < NF; ++n) acc[PART * kPart + m][n] = mma(b[n], a[m], acc[PART * kPart + m][n]);
    }
    // READS reads of what comes next between the products of now.
    template <int READS>
    __device__ static void interleave() {
        constexpr int kProducts = kPart * NF * (sizeof(T) == 2 ? 1 : 4);
        constexpr int kBetween = kProducts / READS > 0 ? kProducts / READS : 1;
        constexpr int kTogether = (READS + kProducts - 1) / kProducts;
#pragma unroll
        for (int i = 0; i < READS / kTogether; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, kTogether, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, kBetween, 0);
        }
    }
    // a, b: the first number of the tile's lines at the first k; alines, blines: lines there are; ks: k there are.
    // HALF: only the first half of a's lines is there, and the waves of the other half only load.
    // afollows, bfollows: see ByDma.
    template <int OF, bool HALF = false>
    __device__ __forceinline__ void run(char* lds, const char* a, int64_t aline, int alines, bool afollows, const char* b, int64_t bline, int blines, bool bfollows,
                                        int64_t ks) {
        const int thread = threadIdx.x, lane = thread % 64, wave = thread / 64, wm = wave / WN, wn = wave % WN;
#pragma unroll
        for (int m = 0; m < MF; ++m)
#pragma unroll
            for (int n = 0; n < NF; ++n) acc[m][n] = Acc{0, 0, 0, 0};
        if constexpr (OF != NO_SUMS)
#pragma unroll
            for (int i = 0; i < (OF == OF_A ? 2 : NF); ++i) sums[i] = Acc{0, 0, 0, 0};
        const int64_t astep = AA == Adjacent::K ? 128 : aline * A::kStep;
        const int64_t bstep = AB == Adjacent::K ? 128 : bline * B::kStep;
        if constexpr (DMA) {
            const int w = __builtin_amdgcn_readfirstlane(wave);
            ByDma<T, AA, S::kM, S::kThreads> da;
            ByDma<T, AB, S::kN, S::kThreads> db;
            da.begin(aline, afollows, thread);
            db.begin(bline, bfollows, thread);
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
            Frag<T> fa[2][kPart], fb[2][NF];
            int steps = (int)((ks + A::kStep - 1) / A::kStep);
            // What the range check leaves to be done in the last step's stage.  a and b stand kStages steps behind it then.
            const auto mend = [&](char* stage) __attribute__((always_inline)) {
                const int rest = (int)ks & (A::kStep - 1), tail = rest ? rest : A::kStep;  // k of the last step
                const bool partial = (AA == Adjacent::K || AB == Adjacent::K) && rest % A::kChunk;
                if (!partial && !da.misses(alines, tail) && !db.misses(blines, tail)) return;
                if (partial) {
                    ByDma<T, AA, S::kM, S::kThreads>::clear(stage, rest, threadIdx.x);
                    ByDma<T, AB, S::kN, S::kThreads>::clear(stage + A::kBytes, rest, threadIdx.x);
                }
                da.patch(a - kStages * astep, stage, alines, tail, threadIdx.x);
                db.patch(b - kStages * bstep, stage + A::kBytes, blines, tail, threadIdx.x);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();
            };
#pragma unroll
            for (int i = 0; i < kStages; ++i) load(lds + i * kStage);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kStages - 1) * kLoads) : "memory");
            __builtin_amdgcn_s_barrier();
            if (steps == 1) mend(lds);
            int at = 0;
            read_b(lds, 0, lane, wn, fb[0]);
            read_a(lds, 0, 0, lane, wm, fa[0]);
            const bool idle = HALF && w / WN >= WM / 2;
            do {
                const char* now = lds + at;
                const int then = at == (kStages - 1) * kStage ? 0 : at + kStage;
                // What the next loads need, worked out beside products.  (Behind the last step too, of nothing.)  They are asked for one by
                // one between products: eight at a time hold up a wave for longer than its products take (24000 x 4096 x 4096 bf16 627
                // us, so 609).
                const auto sa = da.begin_step(a, lds + at, alines, ks, thread, w);
                const auto sb = db.begin_step(b, lds + at + A::kBytes, blines, ks, thread, w);
                ks -= A::kStep;
                a += astep;
                b += bstep;
                if (!idle) {
                    read_a(now, 0, 1, lane, wm, fa[1]);
                    multiply<0, OF>(fa[0], fb[0]);
                    interleave<kReadsA>();
                    read_b(now, 1, lane, wn, fb[1]);
                    read_a(now, 1, 0, lane, wm, fa[0]);
                    multiply<1, OF>(fa[1], fb[0]);
                    interleave<kReadsA + kReadsB>();
                    read_a(now, 1, 1, lane, wm, fa[1]);
                    multiply<0, OF>(fa[0], fb[1]);
                    interleave<kReadsA>();
                }
                __builtin_amdgcn_sched_barrier(0);
                // the next stage is there, for all waves; this one is free, all of it being in registers
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((kStages - 2) * kLoads) : "memory");
                __builtin_amdgcn_s_barrier();
                __builtin_amdgcn_sched_barrier(0);
                if (steps == 2) mend(lds + then);
                at = then;
                now = lds + at;
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (OF == OF_A) sum_a<1>(fa[1]);
#pragma unroll
                for (int m = 0; m < kPart; ++m) {
                    if (!idle) {
#pragma unroll
                        for (int n = m * NF / kPart; n < (m + 1) * NF / kPart; ++n) fb[0][n] = B::read(now + A::kBytes, (wn * NF + n) * 16, 0, lane);
                        fa[0][m] = A::read(now, (wm * MF + m) * 16, 0, lane);
                        multiply_line<1>(m, fa[1][m], fb[1]);
                    }
#pragma unroll
                    for (int c = m * kLoads / kPart; c < (m + 1) * kLoads / kPart; ++c) {
                        if (c < A::kChunks) sa.load(c);
                        else sb.load(c - A::kChunks);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            } while (--steps > 0);
            loads_done();  // the loads of nothing store zeros
            __builtin_amdgcn_s_barrier();
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
            step<OF>(now, lane, wm, wn);
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
    // Ends the tile by way of LDS: rows of NF * 16 sums of a wave's own, chunk c of row r at place c ^ r (its last bits).  first, last:
    // out's rows; n0: the first column; parts: where sums go that are not all there yet (rows of out's), or null.  What add has is asked
    // for kAhead rows a lane at a time, before the rows ahead of them are ended: with one workgroup on a CU nothing else hides it.
    __device__ __forceinline__ void end(char* lds, const Ending& e, int set, int64_t first, int64_t last, int n0, float* parts) {
        constexpr int kTurn = MF < 4 ? MF : 4, kLanes = NF * 2, kRows = 64 / kLanes, kAhead = kTurn * 16 / kRows < 4 ? kTurn * 16 / kRows : 4;
        constexpr int kLine = NF * 64, kMask = NF * 4 - 1;
        const int thread = threadIdx.x, lane = thread % 64, wave = thread / 64, wm = wave / WN, wn = wave % WN;
        char* const own = lds + wave * (kTurn * 16 * kLine);
        const int c = lane % kLanes * 2, col = n0 + wn * (NF * 16) + c * 4;
        Biases<T> bias;
        if (!parts) bias.load(e, set, col);
        Places<T> places(e, set, first + wm * MF * 16 + lane / kLanes, col);
        Added<T> added[kAhead], then[kAhead];
        const auto fetch = [&](int line, Added<T>(&to)[kAhead]) __attribute__((always_inline)) {
            const int64_t row0 = first + wm * MF * 16 + line + lane / kLanes;
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (!parts && row0 + i * kRows < last) to[i].load(e, row0 + i * kRows, col);
        };
        fetch(0, added);
#pragma unroll
        for (int m0 = 0; m0 < MF; m0 += kTurn) {
#pragma unroll
            for (int m = 0; m < kTurn; ++m)
#pragma unroll
                for (int n = 0; n < NF; ++n)
                    *reinterpret_cast<Acc*>(own + (m * 16 + lane % 16) * kLine + ((n * 4 + lane / 16) ^ (lane & kMask)) * 16) = acc[m0 + m][n];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
            for (int r0 = 0; r0 < kTurn * 16; r0 += kRows * kAhead) {
                const int64_t row0 = first + (wm * MF + m0) * 16 + r0 + lane / kLanes;
                if (m0 * 16 + r0 + kRows * kAhead < MF * 16) fetch(m0 * 16 + r0 + kRows * kAhead, then);
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int r = r0 + i * kRows + lane / kLanes;
                    const int64_t row = row0 + i * kRows;
                    const Places<T> here = places;
                    places.down(e, kRows);
                    if (row >= last || col >= e.cols) continue;
                    const char* const at = own + r * kLine;
                    const Acc lo = *reinterpret_cast<const Acc*>(at + (c ^ (r & kMask)) * 16);
                    const Acc hi = *reinterpret_cast<const Acc*>(at + ((c + 1) ^ (r & kMask)) * 16);
                    float sum[kEnd] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                    if (parts) {
                        float* const to = parts + row * e.cols + col;
#pragma unroll
                        for (int j = 0; j < kEnd; ++j)
                            if (col + j < e.cols) to[j] = sum[j];
                    } else if (col + kEnd <= e.cols) {
                        end_sums<T>(e, here, sum, bias, added[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < kAhead; ++i) added[i] = then[i];
            }
            // A row's last columns, less than eight, by a lane for each row (by the lane that has them above 64 experts' 4764 x 79 took 173 us,
            // where 80 columns take 66).
            const int base = n0 + wn * (NF * 16), rest = base + (e.cols - base) / kEnd * kEnd;
            if (!parts && base < e.cols && rest < e.cols && rest < base + NF * 16) {
                const int64_t row = first + (wm * MF + m0) * 16 + lane;
                if (lane < kTurn * 16 && row < last)
                    end_rest<T>(e, set, row, rest, [&](int j) {
                        return *reinterpret_cast<const float*>(own + lane * kLine + (((rest - base + j) / 4) ^ (lane & kMask)) * 16 + (rest - base + j) % 4 * 4);
                    });
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

// Whether memory of the matrix lies behind the last number of rows up to `row` of x; behind W's of expert `set` up to column `col` and k `k`.
__device__ inline bool x_follows(const Product& p, int64_t row) { return row < p.rows && p.x.line > 0; }
template <Adjacent AB>
__device__ inline bool w_follows(const Product& p, int set, int col, int64_t k) {
    return (col < p.cols && (AB == Adjacent::L || p.w.line > 0)) || (AB == Adjacent::L && k < p.width) || (set + 1 < p.experts && p.w.set > 0);
}

// out = act(x W + b) + add, a tile for each workgroup.  24000 x 4096 x 4096 bf16 672 us with a bias and a residual (1.2 PFLOP/s), 609 without
// both; 48000 rows of 64 experts of 4096 x 4096 1.6 ms (1.0: an expert's last tile, and W that changes, cost what is missing).
template <typename T, Adjacent AB, typename SHAPE, bool DMA>
__device__ __forceinline__ void linear_tile(char* lds, const Product& p, const Ending& e, int bid) {
    using P = TileProduct<T, Adjacent::K, AB, SHAPE, DMA>;
    constexpr int BM = P::S::kM, BN = P::S::kN;
    const RowTiles<BM> tiles(p.offsets, p.experts, p.rows, p.mtiles);
    const int per = tiles.all * p.ntiles;
    if (bid >= per * p.splits) return;
    const int t = xcd_order(bid, per * p.splits);
    const int split = t / per;
    int ntile = 0;
    const RowTile r = tiles.template tile<true>(t - split * per, p.ntiles, &ntile);
    if (r.first >= r.last) return;
    const int n0 = ntile * BN;
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
    const int alines = (int)min((int64_t)BM, r.last - r.first), blines = min(BN, p.cols - n0);
    // The last tile of an expert: half of it takes half the time (48000 rows of 64 experts, 4096 x 4096 bf16: 6 %).
    const bool afollows = x_follows(p, r.first + alines), bfollows = w_follows<AB>(p, r.set, n0 + blines, k0 + ks);
    if (DMA && SHAPE::kM == 256 && alines <= BM / 2) product.template run<P::NO_SUMS, true>(lds, a, p.x.line, alines, afollows, b, p.w.line, blines, bfollows, ks);
    else product.template run<P::NO_SUMS>(lds, a, p.x.line, alines, afollows, b, p.w.line, blines, bfollows, ks);
    product.end(lds, e, r.set, r.first, min(r.last, r.first + BM), n0, p.splits > 1 ? p.parts + (int64_t)split * p.rows * p.cols : nullptr);
}
template <typename T, Adjacent AB, typename SHAPE, bool DMA>
__global__ __launch_bounds__(SHAPE::kThreads) void linear_kernel(Product p, Ending e) {
    __shared__ __align__(16) char lds[TileProduct<T, Adjacent::K, AB, SHAPE, DMA>::kLds];
    linear_tile<T, AB, SHAPE, DMA>(lds, p, e, blockIdx.x);
}

// The same for few rows (R * 16 of a tile), where the weights' bytes are what counts.  Every wave has all of the tile (NF * 16 columns) and
// every KW-th step of k, for which it keeps D stages of its own in LDS under way, without a barrier; the waves' sums are added in order.
// W goes past the caches: one row, 4096 x 16384 bf16 that no cache holds, k adjacent 28.7 us, so 25.3; 128 experts of 4096 x 1024 with a row
// each 189 and 171 us (6.3 TB/s).
template <typename T, Adjacent AB, int R, int NF, int KW, int D>
__global__ __launch_bounds__(KW * 64) void linear_short_kernel(Product p, Ending e) {
    using A = Tile<T, Adjacent::K, R * 16, 64>;
    using B = Tile<T, AB, NF * 16, 64>;
    constexpr int kStage = A::kBytes + B::kBytes, kOwn = D * kStage, kSums = R * 16 * NF * 64;
    static_assert(kSums <= kOwn);
    constexpr int BM = R * 16, BN = NF * 16;
    __shared__ __align__(16) char lds[KW * kOwn];
    const RowTiles<BM> tiles(p.offsets, p.experts, p.rows, p.mtiles);
    const int per = tiles.all * p.ntiles;
    if ((int)blockIdx.x >= per * p.splits) return;
    const int t = xcd_order(blockIdx.x, per * p.splits);
    const int split = t / per;
    int ntile = 0;
    const RowTile r = tiles.template tile<false>(t - split * per, p.ntiles, &ntile);
    if (r.first >= r.last) return;
    const int n0 = ntile * BN;
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
    da.begin(p.x.line, x_follows(p, r.first + alines), lane);
    db.begin(p.w.line, w_follows<AB>(p, r.set, n0 + blines, min((int64_t)p.width, (split + 1) * p.per_split)), lane);
    char* const own = lds + wave * kOwn;
    const auto load = [&](int stage) {
        da.load(a, own + stage * kStage, alines, ks, lane, 0);
        db.template load<true>(b, own + stage * kStage + A::kBytes, blines, ks, lane, 0);
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
    const int64_t last = ks - (steps - 1) * (KW * A::kStep);  // k from this wave's last step on
    const int rest = last < A::kStep ? (int)last : 0;
    const int tail = (int)min(last, (int64_t)A::kStep);
    const bool mend = last <= A::kStep && (rest % A::kChunk || da.misses(alines, tail) || db.misses(blines, tail));
    const char* const alast = a + (steps - 1) * astep;
    const char* const blast = b + (steps - 1) * bstep;
#pragma unroll
    for (int i = 0; i < D; ++i) load(i);
    int stage = 0;
    for (; steps > 0; --steps) {
        constexpr int kLater = (D - 1) * (A::kChunks + B::kChunks);  // loads that were asked for behind this stage's
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLater) : "memory");
        if (steps == 1 && mend) {
            if (rest % A::kChunk) {
                da.clear(own + stage * kStage, rest, lane);
                db.clear(own + stage * kStage + A::kBytes, rest, lane);
            }
            da.patch(alast, own + stage * kStage, alines, tail, lane);
            db.patch(blast, own + stage * kStage + A::kBytes, blines, tail, lane);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
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
            Biases<T> bias;
            Added<T> added;
            bias.load(e, r.set, col);
            added.load(e, row, col);
            if (col + kEnd <= e.cols)
                end_sums<T>(e, Places<T>(e, r.set, row, col), sum, bias, added);
            else
                end_rest<T>(e, r.set, row, col, [&](int j) {
                    float one = 0;
#pragma unroll
                    for (int w = 0; w < KW; ++w) one += *reinterpret_cast<const float*>(lds + w * kOwn + line * (NF * 64) + ((c + j / 4) ^ (line % (NF * 4))) * 16 + j % 4 * 4);
                    return one;
                });
        } else {
            float* const to = p.parts + ((int64_t)split * p.rows + row) * p.cols + col;
#pragma unroll
            for (int j = 0; j < kEnd; ++j)
                if (col + j < p.cols) to[j] = sum[j];
        }
    }
}

// Parts of a sum added up in order, eight of them under way.  (64 parts of 256 x 42 sums: one after the other 61 us.)
__device__ __forceinline__ float sum_parts(const float* from, int64_t stride, int splits) {
    float sum = 0;
    int s = 0;
    for (; s + 8 <= splits; s += 8) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = from[(s + i) * stride];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[i];
    }
    for (; s < splits; ++s) sum += from[s * stride];
    return sum;
}
// The last of `sets` experts that begins at the row or before, or the first.
__device__ inline int set_of(const int32_t* offsets, int sets, int64_t row) {
    int lo = 0, hi = sets;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (offsets[mid] <= row) lo = mid;
        else hi = mid;
    }
    return lo;
}
template <typename T>
__global__ __launch_bounds__(256) void linear_join_kernel(Product p, Ending e) {
    const int64_t items = (int64_t)p.rows * p.cols;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / p.cols;
        const int col = (int)(i - row * p.cols);
        const int set = p.offsets ? set_of(p.offsets, p.experts + 1, row) : 0;
        const bool f32 = sizeof(T) == 4 || e.out_f32;
        if (set == p.experts) {
            for (char* to : {e.out, e.pre})
                if (to) {
                    char* const line = to + row * (to == e.out ? e.out_line : e.pre_line);
                    if (f32) reinterpret_cast<float*>(line)[col] = 0.0f;
                    else reinterpret_cast<T*>(line)[col] = (T)0.0f;
                }
            continue;
        }
        const float sum = sum_parts(p.parts + i, items, p.splits);
        if (f32) end_one<T, float>(e, set, row, col, sum);
        else end_one<T, T>(e, set, row, col, sum);
    }
}

// --- gradients --------------------------------------------------------------

// d[r] = dout[r] * act'(pre[r]) in the rows' type, rows of no expert left out: what both products of the gradient take.  The matrix
// instructions take 16 bits a number: this is where the slope's product is rounded to them.  Bound by memory: 8000 x 16384 bf16 133 us (5.9 TB/s);
// formed in the products' loads instead, dout and pre would both be read there, by every tile beside another.
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
                for (int j = 0; j < V; ++j) y[j] *= act_slope<sizeof(T) == 4>((float)z[j], act);
            }
            store_vec<V, T>(to, rounded_vec<T, V>(y), false);
        } else {
            for (int j = 0; col + j < cols; ++j) to[j] = rounded<T>((float)from[j] * (at ? act_slope<sizeof(T) == 4>((float)at[j], act) : 1.0f));
        }
    }
}

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

// The same with dbias[e] = sum over the rows of expert e of d[r], taken of d before it is rounded: 16 bits a number are for the matrix
// instructions, which dbias does not need.  A workgroup has `each` rows, of which teams of `lanes` lanes (a power of two, up to 64) take one after
// the other, eight columns a lane; where an expert's rows end the teams are added in order.  Parts [chunk of rows + expert][column]: chunks and
// experts that have rows in common go up together, so no two pairs meet in one.  parts: null where one chunk has
// all rows of one matrix, whose sums are dbias.  d: null where only dbias is asked for.  Bound by memory:
// 8000 x 16384 bf16, gelu, 162 us and 5 for the parts, beside which dW without these sums takes 121 instead of 145 (256 k); without d 117.
template <typename T, typename D>
__global__ __launch_bounds__(256) void slope_sums_kernel(const D* dout, int64_t dout_stride, const D* pre, int64_t pre_stride, int act, int32_t rows,
                                                         int32_t cols, const int32_t* offsets, int32_t experts, T* d, int64_t d_stride, int32_t each,
                                                         int32_t lanes, float* parts, void* dbias, bool f32) {
    constexpr int V = 8, AHEAD = 4;
    __shared__ float lds[V][256];
    const int teams = 256 / lanes, lane = threadIdx.x % lanes, team = threadIdx.x / lanes;
    const int col0 = blockIdx.x * lanes * V, col = col0 + lane * V, here = min(V, cols - col);
    const int64_t used = offsets ? min(max(offsets[experts], 0), rows) : rows;
    const int64_t end = min((int64_t)(blockIdx.y + 1) * each, used);
    int64_t first = (int64_t)blockIdx.y * each;
    while (first < end) {
        int set = 0;
        int64_t last = end;
        if (offsets) {
            set = set_of(offsets, experts, first);
            last = min(max((int64_t)offsets[set + 1], first + 1), end);
        }
        float sum[V] = {};
        if (here == V) {
            for (int64_t row = first + team; row < last; row += teams * AHEAD) {
                Pack<D, V> x[AHEAD], z[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    if (row + teams * u >= last) continue;
                    x[u] = load_vec<V>(dout + (row + teams * u) * dout_stride + col);
                    if (pre) z[u] = load_vec<V>(pre + (row + teams * u) * pre_stride + col);
                }
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    if (row + teams * u >= last) continue;
                    float y[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        y[j] = (float)x[u][j];
                        if (pre) y[j] *= act_slope<false>((float)z[u][j], act);
                        sum[j] += y[j];
                    }
                    if (d) store_vec<V, T>(d + (row + teams * u) * d_stride + col, rounded_vec<T, V>(y), false);
                }
            }
        } else {
            for (int64_t row = first + team; row < last; row += teams)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (j >= here) continue;
                    float y = (float)dout[row * dout_stride + col + j];
                    if (pre) y *= act_slope<false>((float)pre[row * pre_stride + col + j], act);
                    sum[j] += y;
                    if (d) d[row * d_stride + col + j] = rounded<T>(y);
                }
        }
        __syncthreads();  // what the last expert's sums left has been read
#pragma unroll
        for (int j = 0; j < V; ++j) lds[j][threadIdx.x] = sum[j];
        __syncthreads();
        const int64_t at = ((int64_t)blockIdx.y + set) * cols;
        for (int c = threadIdx.x; c < min(lanes * V, cols - col0); c += 256) {
            float all = 0;
            for (int t = 0; t < teams; ++t) all += lds[c % V][t * lanes + c / V];
            if (parts) parts[at + col0 + c] = all;
            else if (f32) ((float*)dbias)[col0 + c] = all;
            else ((T*)dbias)[col0 + c] = rounded<T>(all);
        }
        first = last;
    }
}
// The parts added up: a workgroup has 64 columns of an expert, its 16 waves every 16th part, added in order.
template <typename T>
__global__ __launch_bounds__(1024) void slope_join_kernel(const float* parts, int32_t rows, int32_t cols, const int32_t* offsets, int32_t experts,
                                                          int32_t each, void* dbias, bool f32) {
    constexpr int WAVES = 16;
    __shared__ float sums[WAVES][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int set = blockIdx.y;
    for (int block = blockIdx.x; block <= (cols - 1) / 64; block += gridDim.x) {
        const int col = block * 64 + lane;
        const int first = offsets ? min(max(offsets[set], 0), rows) : 0, last = offsets ? min(max(offsets[set + 1], first), rows) : rows;
        const int chunk = first / each + wave, chunks = last > first ? (last - 1) / each + 1 : 0;
        float sum = 0;
        if (col < cols && chunk < chunks) sum = sum_parts(parts + ((int64_t)chunk + set) * cols + col, WAVES * (int64_t)cols, (chunks - chunk + WAVES - 1) / WAVES);
        sums[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && col < cols) {
#pragma unroll
            for (int w = 1; w < WAVES; ++w) sum += sums[w][lane];
            const int64_t at = (int64_t)set * cols + col;
            if (f32) ((float*)dbias)[at] = sum;
            else ((T*)dbias)[at] = rounded<T>(sum);
        }
        __syncthreads();
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
    float* bias_parts;
    void* dbias;  // null: not asked for here
    bool bias_f32;
    bool d_is_a;
    bool sorted;  // long experts first
};

// The expert with the `rank`-th largest number of rows: long tiles that begin last would leave the chip to themselves (dW of 12 experts:
// 10007 x 1500 x 777 floats, dx and dW 437 us in order of experts, 422 so).  Up to 64 experts; more are many tiles anyway, and stay
// in order, as do small ones (the order takes 6 us: 64 experts with a row each, 4764 x 80 96 us and 67).
__device__ inline int by_load(const int32_t* offsets, int experts, int rank, bool sorted) {
    if (!sorted) return rank;
    const int lane = threadIdx.x % 64, e = min(lane, experts - 1);
    const int load = max(offsets[e + 1], 0) - max(offsets[e], 0);
    int before = 0;
    for (int j = 0; j < experts; ++j) {
        const int other = __builtin_amdgcn_readlane(load, j);
        before += other > load || (other == load && j < lane);
    }
    const uint64_t found = __ballot(lane < experts && before == rank);
    return found ? __ffsll((unsigned long long)found) - 1 : rank;
}

// A tile of dW, k being the rows: both operands have k as their stored rows, which the transposing reads of LDS turn, and nothing is transposed in memory.
// 8192 x 8192 x 8192 bf16 1416 TFLOP/s (the library's best for this layout 1080); 12 experts of 10007 x 1500 x 777 floats with dx 415 us.
template <typename T, typename SHAPE, bool DMA>
__device__ __forceinline__ void weight_grad_tile(char* lds, const WeightGrad& p, const Ending& e, int bid) {
    using P = TileProduct<T, Adjacent::L, Adjacent::L, SHAPE, DMA>;
    constexpr int MF = P::MF, NF = P::NF, WN = P::WN;
    constexpr int BM = P::S::kM, BN = P::S::kN;
    const int per = p.mtiles * p.ntiles;
    // An expert's tiles and parts at a time, each expert's shared out to the XCDs.
    const int each = per * p.splits;
    const int set = by_load(p.offsets, p.experts, bid / each, p.sorted);
    const int t = xcd_order(bid % each, each), split = t / per;
    const TileAt tile = banded(t % per, p.mtiles, p.ntiles, 8);
    const RowRange r = grad_rows<P::A::kStep>(p.offsets, p.rows, set, split, p.splits);
    const int m0 = tile.m * BM, n0 = tile.n * BN;
    const char* const a = p.a.p + r.first * p.a.line + m0 * sizeof(T);
    const char* const b = p.b.p + r.first * p.b.line + n0 * sizeof(T);
    P product;
    const auto run = [&](auto of) __attribute__((always_inline)) {
        const int alines = min(BM, p.m - m0), blines = min(BN, p.n - n0);
        const bool more = r.last < p.rows;
        product.template run<decltype(of)::value>(lds, a, p.a.line, alines, more || m0 + alines < p.m, b, p.b.line, blines, more || n0 + blines < p.n, r.last - r.first);
    };
    // The sums of d's columns (where d is not rounded here, or of 32 bits): the workgroups of the first tiles along W's other side multiply d with ones besides.  (A pass over d of its
    // own took 225 us for 8000 x 16384 bf16, beside 920 for the product.)
    const auto put = [&](int col, int cols, float sum) {
        if (col >= cols) return;
        const int64_t at = (int64_t)set * cols + col;
        if (p.splits > 1) p.bias_parts[split * (int64_t)p.experts * cols + at] = sum;
        else if (p.bias_f32) ((float*)p.dbias)[at] = sum;
        else ((T*)p.dbias)[at] = rounded<T>(sum);
    };
    const int lane = threadIdx.x % 64, wm = threadIdx.x / 64 / WN, wn = threadIdx.x / 64 % WN;
    if (p.dbias && !p.d_is_a && tile.m == 0) {
        run(std::integral_constant<int, P::OF_B>{});
        if (wm == 0 && lane % 16 == 0)
#pragma unroll
            for (int n = 0; n < NF; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) put(n0 + (wn * NF + n) * 16 + lane / 4 + q, p.n, product.sums[n][q]);
    } else if (p.dbias && p.d_is_a && tile.n == 0) {
        run(std::integral_constant<int, P::OF_A>{});
        if (wn < MF / 2 && lane < 16)
#pragma unroll
            for (int part = 0; part < 2; ++part) put(m0 + (wm * MF + part * (MF / 2) + wn) * 16 + lane, p.m, product.sums[part][0]);
    } else {
        run(std::integral_constant<int, P::NO_SUMS>{});
    }
    product.end(lds, e, set, m0, min(p.m, m0 + BM), n0, p.splits > 1 ? p.parts + ((int64_t)split * p.experts + set) * p.m * p.n : nullptr);
}
template <typename T, typename SHAPE, bool DMA>
__global__ __launch_bounds__(SHAPE::kThreads) void weight_grad_kernel(WeightGrad p, Ending e) {
    __shared__ __align__(16) char lds[TileProduct<T, Adjacent::L, Adjacent::L, SHAPE, DMA>::kLds];
    weight_grad_tile<T, SHAPE, DMA>(lds, p, e, blockIdx.x);
}

// dx and dW in one launch, where both have tiles of 64 x 64 and k in one part: each alone leaves CUs with one or two workgroups, whose waves
// wait for what those of others would hide.  first: dx's workgroups, a multiple of 8.  (777 x 1500 x 1021 floats 85.5 us
// in two launches, 62.9 in one; 1000 x 1024 x 1024 bf16 21.9 and 15.8; 16 experts of 2000 x 1024 x 1024 floats 96.4 and 89.6.)
template <typename T, Adjacent AB, typename SHAPE>
__global__ __launch_bounds__(SHAPE::kThreads) void grads_kernel(Product x, Ending ex, WeightGrad w, Ending ew, int first) {
    using P = TileProduct<T, Adjacent::K, AB, SHAPE, true>;
    using Q = TileProduct<T, Adjacent::L, Adjacent::L, SHAPE, true>;
    __shared__ __align__(16) char lds[P::kLds > Q::kLds ? P::kLds : Q::kLds];
    if ((int)blockIdx.x < first) linear_tile<T, AB, SHAPE, true>(lds, x, ex, blockIdx.x);
    else weight_grad_tile<T, SHAPE, true>(lds, w, ew, blockIdx.x - first);
}

template <typename T>
__global__ __launch_bounds__(256) void weight_grad_join_kernel(WeightGrad p, Ending e) {
    const int64_t items = (int64_t)p.experts * p.m * p.n;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
        const int64_t line = i / p.n;
        const float sum = sum_parts(p.parts + i, items, p.splits);
        if (sizeof(T) == 4 || e.out_f32) end_one<T, float>(e, (int)(line / p.m), line % p.m, (int)(i - line * p.n), sum);
        else end_one<T, T>(e, (int)(line / p.m), line % p.m, (int)(i - line * p.n), sum);
    }
}

// dbias[e][c] = sum over the rows of expert e of d[r][c]: a workgroup has 64 columns; its four waves add every fourth row, and
// their sums are added in order.  (Only where dW is not asked for.)
template <typename T>
__global__ __launch_bounds__(256) void bias_grad_kernel(const T* d, int64_t d_stride, const int32_t* offsets, int32_t rows, int32_t cols, int32_t splits,
                                                        float* parts, void* dbias, bool f32) {
    __shared__ float sums[4][64];
    const int set = blockIdx.y, split = blockIdx.z, wave = threadIdx.x / 64;
    const RowRange r = grad_rows<1>(offsets, rows, set, split, splits);
    for (int block = blockIdx.x; block <= (cols - 1) / 64; block += gridDim.x) {
        const int col = block * 64 + threadIdx.x % 64;
        float sum = 0;
        if (col < cols)
            for (int64_t row = r.first + wave; row < r.last; row += 4) sum += (float)d[row * d_stride + col];
        sums[wave][threadIdx.x % 64] = sum;
        __syncthreads();
        if (wave == 0 && col < cols) {
            for (int w = 1; w < 4; ++w) sum += sums[w][threadIdx.x];
            const int64_t at = (int64_t)set * cols + col;
            if (splits > 1) parts[split * ((int64_t)gridDim.y * cols) + at] = sum;
            else if (f32) ((float*)dbias)[at] = sum;
            else ((T*)dbias)[at] = rounded<T>(sum);
        }
        __syncthreads();
    }
}
template <typename T>
__global__ __launch_bounds__(256) void bias_grad_join_kernel(const float* parts, int32_t splits, int64_t n, void* dbias, bool f32) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const float sum = sum_parts(parts + i, n, splits);
    if (f32) ((float*)dbias)[i] = sum;
    else ((T*)dbias)[i] = rounded<T>(sum);
}

}  // namespace spdnn
