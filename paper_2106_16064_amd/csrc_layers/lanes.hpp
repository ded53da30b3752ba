// Exchanges between the lanes of a wave.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace dgsp {

// v of the lane that differs by the pattern, for sums over 2, 4, 8, 16 lanes
template <int kPattern>
__device__ __forceinline__ float moved(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kPattern, 0xf, 0xf, true));
}

template <int kPattern>
__device__ __forceinline__ double moved(double v) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    const int low = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, kPattern, 0xf, 0xf, true), high = __builtin_amdgcn_update_dpp(0, (int)(bits >> 32), kPattern, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)high << 32 | (uint32_t)low);
}

// over `lanes` (a power of two up to 64) neighbouring lanes; every lane has the sum
template <typename V>
__device__ __forceinline__ V lanes_sum(V v, int lanes) {
    if (lanes > 1) v += moved<0xb1>(v);          // neighbours of a pair
    if (lanes > 2) v += moved<0x4e>(v);          // pairs of four
    if (lanes > 4) v += moved<0x141>(v);         // eight, mirrored
    if (lanes > 8) v += moved<0x140>(v);         // sixteen, mirrored
    if (lanes > 16) v += __shfl_xor(v, 16, 64);
    if (lanes > 32) v += __shfl_xor(v, 32, 64);
    return v;
}

template <int kPattern>
__device__ __forceinline__ uint32_t moved_bits(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kPattern, 0xf, 0xf, true);
}

}  // namespace dgsp
