// What the kernels of the row operators and of the dense products share: vectors of a row, rounding, sums over a team of lanes.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

// Products and sums are rounded to 32 bits where they are written; fused ones are spelled fmaf.
#pragma clang fp contract(off)

namespace spdnn {

// A number of 32 bits rounded to the rows' type.  The empty asm keeps the compiler from making one v_fma_mixlo_f16 of the
// operation that gave x and the conversion: that rounds once where every other type rounds twice.
template <typename S>
__device__ inline S rounded(float x) {
    if constexpr (sizeof(S) == 2) asm("" : "+v"(x));
    return (S)x;
}

// Rows may start at any element: vectors are only aligned like one (global memory takes such loads and stores whole).
template <typename T, int V>
using Pack __attribute__((ext_vector_type(V), aligned(sizeof(T)))) = T;

template <int V, typename T>
__device__ inline Pack<T, V> load_vec(const T* p) {
    if constexpr (V == 1) return Pack<T, V>(*p);
    else return *reinterpret_cast<const Pack<T, V>*>(p);
}
// past: the same for all lanes.  The empty asm on both sides of that branch keeps the compiler from making one access of the two,
// an ordinary one.
template <int V, typename T>
__device__ inline Pack<T, V> load_vec(const T* p, bool past) {
    Pack<T, V> x;
    if (past) {
        asm volatile("");
        x = __builtin_nontemporal_load(reinterpret_cast<const Pack<T, V>*>(p));
        asm volatile("");
    } else {
        x = *reinterpret_cast<const Pack<T, V>*>(p);
    }
    return x;
}
template <int V, typename T>
__device__ inline void store_vec(T* p, Pack<T, V> x, bool past) {
    if (past) {
        asm volatile("");
        __builtin_nontemporal_store(x, reinterpret_cast<Pack<T, V>*>(p));
        asm volatile("");
    } else {
        *reinterpret_cast<Pack<T, V>*>(p) = x;
    }
}
template <typename T, int V>
__device__ inline Pack<T, V> rounded_vec(const float (&from)[V]) {
    Pack<T, V> x;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = rounded<T>(from[i]);
    return x;
}
// U of them, with one branch; at(u) is where vector u goes.
template <int V, typename T, int U, typename F>
__device__ inline void store_all(const Pack<T, V> (&x)[U], bool past, F at) {
    if (past) {
        asm volatile("");
#pragma unroll
        for (int u = 0; u < U; ++u) __builtin_nontemporal_store(x[u], reinterpret_cast<Pack<T, V>*>(at(u)));
        asm volatile("");
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) *reinterpret_cast<Pack<T, V>*>(at(u)) = x[u];
    }
}

// x of another lane, in steps that together reach all G lanes of a team: 1, 2 (the lane's number with that bit turned), 4 and 8
// (mirrored within 8 and 16 lanes: another four, another eight), 16 and 32.
template <int STEP>
__device__ inline int other(int x) {
    if constexpr (STEP == 1) return __builtin_amdgcn_mov_dpp(x, 0xB1, 0xf, 0xf, true);
    else if constexpr (STEP == 2) return __builtin_amdgcn_mov_dpp(x, 0x4E, 0xf, 0xf, true);
    else if constexpr (STEP == 4) return __builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true);
    else if constexpr (STEP == 8) return __builtin_amdgcn_mov_dpp(x, 0x140, 0xf, 0xf, true);
    else return __shfl_xor(x, STEP);
}
template <int STEP>
__device__ inline float other(float x) {
    return __int_as_float(other<STEP>(__float_as_int(x)));
}
template <int STEP>
__device__ inline double other(double x) {
    return __hiloint2double(other<STEP>(__double2hiint(x)), other<STEP>(__double2loint(x)));
}
// f(x, y) over a team's lanes, the same in all of them.
template <int G, int STEP = 1, typename T, typename F>
__device__ inline T team_reduce(T x, F f) {
    if constexpr (STEP < G) return team_reduce<G, 2 * STEP>(f(x, other<STEP>(x)), f);
    else return x;
}
template <int G>
__device__ inline float team_sum(float x) {
    return team_reduce<G>(x, [](float a, float b) { return a + b; });
}
template <int G>
__device__ inline float team_max(float x) {
    return team_reduce<G>(x, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace spdnn
