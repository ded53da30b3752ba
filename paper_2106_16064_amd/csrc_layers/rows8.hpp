// Rows in 8 bits: blocks of 32 columns of a row, each with a power of two as its scale.
//
// A block's scale is the least 2^e with amax <= 448 2^e, or amax <= 127 2^e, of its finite elements; what is stored is each element / 2^e
// as e4m3 or as a whole number, rounded to nearest, ties to even.  Dividing by a power of two is exact, so that a value is rounded once.  e4m3
// is what the matrix instructions read; whole numbers are nearer to what they stand for (an error of at most amax / 127 against
// 2^-4 of the element), and are what activations are kept in.
//
// Memory bounds both ways (bfloat16, 8192 x 4096: to whole numbers 18.5 us, 5.5 TB/s, to e4m3 20.5 us, 4.9, back 17 us, 5.9).
//
// Values: rows of whole blocks, the last one filled up with zeros.  Scales: bytes b for 2^(b - 127); block k of row r at
// ((k / 4) * ld + r) * 4 + k % 4, so that what a product's stage of 128 columns reads lies together.  Places of a group of four
// beyond the last block hold 127.
#pragma once

#include "../../include/dgsp_layers.h"
#include "chunks.hpp"
#include "lanes.hpp"

namespace dgsp {

constexpr int kBlock = 32, kBlockLanes = kBlock / kChunk;     // lanes that share a block

struct Rows8 {
    uint8_t* values;        // null: not wanted
    int64_t ldv;            // bytes; a multiple of 16
    uint8_t* scales;
    int64_t lds;            // rows from a group of four blocks to the next
    int64_t blocks;         // of a row
};

// Of the four lanes of a block.
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
    v = max(v, moved_bits<0xb1>(v));        // neighbours of a pair
    return max(v, moved_bits<0x4e>(v));     // pairs of four
}

// Least and largest scale.  At the lower end scales stay normal numbers, of float16 steps of its own smallest one; at the upper end what
// a block reads back stays in the range of the type that it came from (largest elements are then cut off at 448 or 127).
struct ScaleRange {
    int least, most;
};

__host__ __device__ inline ScaleRange scale_range(int kind, int type) {
    if (kind == DGSP_E4M3) return {1, 246};
    return type == DGSP_F16 ? ScaleRange{127 - 24, 127 + 9} : ScaleRange{1, 248};
}

// the scale's byte; `amax`: bits of the largest finite magnitude
template <bool kE4m3>
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax, ScaleRange range) {
    const int exponent = (int)(amax >> 23);
    const int up = (amax & 0x7fffffu) > (kE4m3 ? 0x600000u : 0x7e0000u);      // 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6
    return amax == 0 ? 127u : (uint32_t)min(max(exponent - (kE4m3 ? 8 : 6) + up, range.least), range.most);
}

// four numbers as floats whose lowest byte they are -> the bytes
__device__ __forceinline__ uint32_t lowest_bytes(const uint32_t (&bits)[4]) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(bits[3], bits[2], 0x0c0c0400u), __builtin_amdgcn_perm(bits[1], bits[0], 0x0c0c0400u), 0x05040100u);
}

// Four numbers times `factor` as whole numbers in a byte each, to nearest even.  Adding 1.5 * 2^23 in the same step rounds to whole numbers, which are
// then the lowest byte.
__device__ __forceinline__ uint32_t whole_word(const float (&v)[4], float factor) {
    uint32_t bits[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) bits[j] = __builtin_bit_cast(uint32_t, fmaf(v[j], factor, 12582912.0f));
    return lowest_bytes(bits);
}

// Eight of them; `cut`: some may lie beyond 127 (a scale at the end of its range).
__device__ __forceinline__ uint2 whole_bytes(const float (&v)[kChunk], float inverse, bool cut) {
    if (!cut) return {whole_word({v[0], v[1], v[2], v[3]}, inverse), whole_word({v[4], v[5], v[6], v[7]}, inverse)};
    uint32_t out[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        uint32_t bits[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) bits[j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(rintf(v[4 * q + j] * inverse), -127.0f, 127.0f) + 12582912.0f);
        out[q] = lowest_bytes(bits);
    }
    return {out[0], out[1]};
}

// Eight elements of a row as a lane holds them -> eight bytes, and the scale's byte.  All four lanes of a block call it; elements beyond
// the row are 0.  A NaN or an infinity is a NaN in e4m3, which has no infinity; of whole numbers, which have neither, it makes the
// block's scale 255, a NaN.
template <bool kE4m3>
__device__ __forceinline__ uint2 to_8bit(const float (&v)[kChunk], ScaleRange range, uint32_t& scale) {
    uint32_t largest = 0;
#pragma unroll
    for (int j = 0; j < kChunk; ++j) {
        const uint32_t magnitude = __builtin_bit_cast(uint32_t, v[j]) & 0x7fffffffu;
        if (kE4m3)
            largest = max(largest, magnitude < 0x7f800000u ? magnitude : 0u);
        else
            largest = max(largest, magnitude);
    }
    largest = block_max(largest);
    const bool finite = largest < 0x7f800000u;
    scale = scale_byte<kE4m3>(finite ? largest : 0u, range);
    const float inverse = __builtin_bit_cast(float, (254u - scale) << 23);
    if constexpr (!kE4m3) {
        if (finite) return whole_bytes(v, inverse, __builtin_amdgcn_ballot_w64((int)scale == range.most) != 0);
        scale = 255u;
        return {0u, 0u};
    }
    uint32_t out[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        float s[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float scaled = v[4 * q + j] * inverse;
            s[j] = fabsf(v[4 * q + j]) < __builtin_inff() ? __builtin_amdgcn_fmed3f(scaled, -448.0f, 448.0f) : __builtin_nanf("");
        }
        const int low = __builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[1], 0, false);
        out[q] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(s[2], s[3], low, true);
    }
    return {out[0], out[1]};
}

// A lane's eight bytes and, by the first lane of each group of four blocks, their scales.  `lanes`: that hold the row, a power of two of
// at least 4, or any number of whole 16; all of them call it.  `chunk`: which eight columns.
__device__ __forceinline__ void store_8bit(const Rows8& to, int64_t row, int64_t chunk, int lanes, bool inside, uint2 bytes, uint32_t scale) {
    const int64_t block = chunk / kBlockLanes;
    const bool here = inside && block < to.blocks;
    if (here) *reinterpret_cast<uint2*>(to.values + row * to.ldv + chunk * kChunk) = bytes;
    uint32_t word = here && chunk % kBlockLanes == 0 ? scale << (8 * (block % 4)) : 0u;
    if (lanes > 4) word |= moved_bits<0x141>(word);                                  // eight, mirrored
    word |= moved_bits<0xb1>(word);
    word |= moved_bits<0x4e>(word);
    if (lanes > 8) word |= moved_bits<0x140>(word);                                  // sixteen, mirrored
    if (here && chunk % (4 * kBlockLanes) == 0) {
        const int64_t left = to.blocks - block;
        if (left < 4) word |= 0x7f7f7f7fu << (8 * left);
        *reinterpret_cast<uint32_t*>(to.scales + ((block / 4) * to.lds + row) * 4) = word;
    }
}

// Eight bytes back; `scale` as stored.
template <bool kE4m3>
__device__ __forceinline__ void from_8bit(uint2 bytes, uint32_t scale, float (&v)[kChunk]) {
    using F2 = float __attribute__((ext_vector_type(2)));
    const float factor = scale == 255u ? __builtin_nanf("") : scale == 0u ? 0x1p-127f : __builtin_bit_cast(float, scale << 23);
    const uint32_t in[2] = {bytes.x, bytes.y};
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        if constexpr (kE4m3) {
            const F2 low = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[q], false), high = __builtin_amdgcn_cvt_pk_f32_fp8((int)in[q], true);
            v[4 * q] = low[0] * factor;
            v[4 * q + 1] = low[1] * factor;
            v[4 * q + 2] = high[0] * factor;
            v[4 * q + 3] = high[1] * factor;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * q + j] = (float)(int8_t)(in[q] >> (8 * j) & 0xffu) * factor;
        }
    }
}

// ---------------------------------------------------------------- kernels

template <typename T>
struct Rows8Args {
    int64_t rows, width;
    int lanes;              // of a row, a power of two from 4 to 256
    ScaleRange range;
    T* matrix;
    int64_t ld;
    Rows8 rows8;
};

// A team of lanes takes a row (rows beyond 2048 columns in several steps), as many teams side by side as a workgroup of 256 has.
template <typename T, bool kE4m3>
__global__ __launch_bounds__(256) void quantise_kernel(Rows8Args<T> a) {
    const int teams = 256 / a.lanes, lane = threadIdx.x & (a.lanes - 1);
    const int64_t chunks = a.rows8.blocks * kBlockLanes, step = (int64_t)gridDim.x * teams;
    for (int64_t base = (int64_t)blockIdx.x * teams; base < a.rows; base += step) {   // the same turns for all lanes
        const int64_t row = base + threadIdx.x / a.lanes;
        const bool inside = row < a.rows;
        for (int64_t c = lane; c - lane < chunks; c += a.lanes) {
            float v[kChunk];
            const int64_t here = a.width - c * kChunk;
            widen(load_chunk(a.matrix + (inside && here > 0 ? row * a.ld + c * kChunk : 0), inside ? (here > 0 ? here : 0) : 0), v);
            uint32_t scale;
            const uint2 bytes = to_8bit<kE4m3>(v, a.range, scale);
            store_8bit(a.rows8, row, c, a.lanes, inside, bytes, scale);
        }
    }
}

// The other way; a lane takes eight columns of a row.
template <typename T, bool kE4m3>
__global__ __launch_bounds__(256) void dequantise_kernel(Rows8Args<T> a) {
    const int teams = 256 / a.lanes, lane = threadIdx.x & (a.lanes - 1);
    const int64_t chunks = (a.width + kChunk - 1) / kChunk;
    for (int64_t row = (int64_t)blockIdx.x * teams + threadIdx.x / a.lanes; row < a.rows; row += (int64_t)gridDim.x * teams)
        for (int64_t c = lane; c < chunks; c += a.lanes) {
            const int64_t block = c / kBlockLanes;
            const uint2 bytes = *reinterpret_cast<const uint2*>(a.rows8.values + row * a.rows8.ldv + c * kChunk);
            const uint32_t scale = a.rows8.scales[((block / 4) * a.rows8.lds + row) * 4 + block % 4];
            float v[kChunk];
            from_8bit<kE4m3>(bytes, scale, v);
            store_chunk(a.matrix + row * a.ld + c * kChunk, a.width - c * kChunk, v);
        }
}

}  // namespace dgsp
