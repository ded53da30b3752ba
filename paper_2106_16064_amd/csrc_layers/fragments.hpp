// Operands of the matrix instructions for kernels that hold rows in registers and weights in LDS.
#pragma once

#include "element_types.hpp"
#include "matrix_tiles.hpp"

namespace dgsp {

__device__ __forceinline__ s16x8 join(s16x4 low, s16x4 high) { return __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7); }

// p: eight, or four, elements of this lane's row
__device__ __forceinline__ s16x8 read8(const uint16_t* p) { return *reinterpret_cast<const s16x8*>(p); }
__device__ __forceinline__ s16x4 read4(const uint16_t* p) { return *reinterpret_cast<const s16x4*>(p); }
// p: where this lane's group of 16 finds four rows of 16 elements; the lane receives the four elements of its column (l % 16)
__device__ __forceinline__ s16x4 read_column(const uint16_t* rows, int ld, int lane) {
    const uint16_t* p = rows + (lane % 16 / 4) * ld + lane % 4 * 4;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
}

template <typename E>
__device__ __forceinline__ s16x4 pack(f32x4 v) {
    using E4 = E __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(s16x4, E4{from_float<E>(v[0]), from_float<E>(v[1]), from_float<E>(v[2]), from_float<E>(v[3])});
}

}  // namespace dgsp
