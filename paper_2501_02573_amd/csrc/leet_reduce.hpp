// Sums and largest values over neighbouring lanes of a wave.
#pragma once

#include "leet_common.hpp"

namespace leet {

template <int kCtrl>
__device__ __forceinline__ float dpp(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), kCtrl, 0xf, 0xf, true));
}
// Sum over the 2^kLog neighbouring lanes that hold a row; every one of them gets it, with the same bits.
template <int kLog>
__device__ __forceinline__ float row_sum(float v) {
    if constexpr (kLog >= 1) v += dpp<0xB1>(v);   // quad_perm 1 0 3 2
    if constexpr (kLog >= 2) v += dpp<0x4E>(v);   // quad_perm 2 3 0 1
    if constexpr (kLog >= 3) v += dpp<0x141>(v);  // row_half_mirror: the quads of eight lanes swap
    if constexpr (kLog >= 4) v += dpp<0x140>(v);  // row_mirror: the halves of sixteen lanes swap
    if constexpr (kLog >= 5) v += __shfl_xor(v, 16, 64);
    if constexpr (kLog >= 6) v += __shfl_xor(v, 32, 64);
    return v;
}
// Largest value over 4, 8, 16 or 64 neighbouring lanes (kLog 2, 3, 4, 6).
template <int kLog>
__device__ __forceinline__ float row_max(float v) {
    v = fmaxf(v, dpp<0xB1>(v));
    v = fmaxf(v, dpp<0x4E>(v));
    if constexpr (kLog >= 3) v = fmaxf(v, dpp<0x141>(v));
    if constexpr (kLog >= 4) v = fmaxf(v, dpp<0x140>(v));
    if constexpr (kLog >= 6) {
        v = fmaxf(v, __shfl_xor(v, 16, 64));
        v = fmaxf(v, __shfl_xor(v, 32, 64));
    }
    return v;
}

}  // namespace leet
