// Sums over the lanes of a wave without the LDS: rotations within rows of 16 lanes, then rows and halves of the wave swapped.
#pragma once

#include "common.h"

namespace moe {

// v moved between the lanes of a row by a data-parallel primitive (4- and 8-byte types)
template <int CTRL, typename T>
__device__ __forceinline__ T dpp(T v) {
    if constexpr (sizeof(T) == 8) {
        const u32x2 w = __builtin_bit_cast(u32x2, v);
        const u32x2 r = {(uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[0], CTRL, 0xf, 0xf, true),
                         (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[1], CTRL, 0xf, 0xf, true)};
        return __builtin_bit_cast(T, r);
    } else {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
    }
}

// f of a lane's value and that of the lane 16 (HALVES: 32) away, in both
template <bool HALVES, typename T, typename F>
__device__ __forceinline__ T with_swapped(T v, F&& f) {
    auto swap = [](uint32_t a) {
        if constexpr (HALVES) return __builtin_amdgcn_permlane32_swap(a, a, false, false);
        else return __builtin_amdgcn_permlane16_swap(a, a, false, false);
    };
    if constexpr (sizeof(T) == 8) {
        const u32x2 w = __builtin_bit_cast(u32x2, v);
        const auto lo = swap(w[0]), hi = swap(w[1]);
        return f(__builtin_bit_cast(T, u32x2{lo[0], hi[0]}), __builtin_bit_cast(T, u32x2{lo[1], hi[1]}));
    } else {
        const auto r = swap(__builtin_bit_cast(uint32_t, v));
        const uint32_t a = r[0], b = r[1];   // numbers of their own: a bit cast of a vector's element takes its first
        return f(__builtin_bit_cast(T, a), __builtin_bit_cast(T, b));
    }
}

// Sum over the lanes that are congruent modulo FROM (a power of two up to 64), in all of them.
template <int FROM, typename T>
__device__ __forceinline__ T sum_congruent(T v) {
    auto add = [](T a, T b) { return a + b; };
    if constexpr (FROM <= 1) v += dpp<0x121>(v);   // row_ror 1, 2, 4, 8
    if constexpr (FROM <= 2) v += dpp<0x122>(v);
    if constexpr (FROM <= 4) v += dpp<0x124>(v);
    if constexpr (FROM <= 8) v += dpp<0x128>(v);
    if constexpr (FROM <= 16) v = with_swapped<false>(v, add);
    if constexpr (FROM <= 32) v = with_swapped<true>(v, add);
    return v;
}

template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
    return sum_congruent<1>(v);
}

}  // namespace moe
