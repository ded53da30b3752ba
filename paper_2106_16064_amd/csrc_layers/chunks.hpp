// Eight neighbouring elements of a row: what a lane reads at a time, and what one counter of dropout's generator serves.
#pragma once

#include "drop_mask.hpp"
#include "element_types.hpp"

namespace dgsp {

constexpr int kChunk = kDropGroup;

using u32x4 = uint32_t __attribute__((ext_vector_type(4)));

// As it lies in memory: 16 bytes of 16-bit types, 32 of float.  Addresses need the alignment of T only: the memory system takes
// vectors at any address.
template <typename T>
struct RawChunk {
    static constexpr int kQuads = sizeof(T) / 2;
    u32x4 q[kQuads];
    __device__ __forceinline__ float at(int j) const {
        if constexpr (sizeof(T) == 4)
            return __builtin_bit_cast(float, (uint32_t)q[j / 4][j % 4]);
        else
            return to_float(__builtin_bit_cast(T, (uint16_t)(q[0][j / 2] >> (j % 2 * 16))));
    }
};

template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) ChunkInMemory {
    u32x4 q[RawChunk<T>::kQuads];
};

// `here`: how many of the eight belong to the row; the rest are 0
template <typename T>
__device__ __forceinline__ RawChunk<T> load_chunk(const T* p, int64_t here) {
    RawChunk<T> out;
    if (here >= kChunk) {
        const auto* from = reinterpret_cast<const ChunkInMemory<T>*>(p);
#pragma unroll
        for (int i = 0; i < RawChunk<T>::kQuads; ++i) out.q[i] = from->q[i];
    } else {
#pragma unroll
        for (int i = 0; i < RawChunk<T>::kQuads; ++i) out.q[i] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            if (j >= here) break;
            if constexpr (sizeof(T) == 4)
                out.q[j / 4][j % 4] = __builtin_bit_cast(uint32_t, p[j]);
            else
                out.q[0][j / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, p[j]) << (j % 2 * 16);
        }
    }
    return out;
}

template <typename T>
__device__ __forceinline__ void store_chunk(T* p, int64_t here, const float (&v)[kChunk]) {
    if (here >= kChunk) {
        auto* to = reinterpret_cast<ChunkInMemory<T>*>(p);
#pragma unroll
        for (int i = 0; i < RawChunk<T>::kQuads; ++i) {
            u32x4 q;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 4)
                    q[j] = __builtin_bit_cast(uint32_t, v[4 * i + j]);
                else
                    q[j] = __builtin_bit_cast(uint16_t, from_float<T>(v[2 * j])) | (uint32_t)__builtin_bit_cast(uint16_t, from_float<T>(v[2 * j + 1])) << 16;
            }
            to->q[i] = q;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
            if (j < here) p[j] = from_float<T>(v[j]);
    }
}

template <typename T>
__device__ __forceinline__ void widen(const RawChunk<T>& raw, float (&v)[kChunk]) {
#pragma unroll
    for (int j = 0; j < kChunk; ++j) v[j] = raw.at(j);
}

// eight parameters in T or, if `wide`, in float; `otherwise` where there are none
template <typename T>
__device__ __forceinline__ void load_params(const void* p, bool wide, int64_t col, int64_t here, float otherwise, float (&v)[kChunk]) {
    if (!p) {
#pragma unroll
        for (int j = 0; j < kChunk; ++j) v[j] = otherwise;
    } else if (wide) {
        widen(load_chunk(static_cast<const float*>(p) + col, here), v);
    } else {
        widen(load_chunk(static_cast<const T*>(p) + col, here), v);
    }
}

__device__ __forceinline__ void keep(uint32_t bits, float scale, float (&v)[kChunk]) {
#pragma unroll
    for (int j = 0; j < kChunk; ++j) v[j] = bits >> j & 1 ? v[j] * scale : 0.0f;
}

__device__ __forceinline__ void drop(const DropMask& mask, uint64_t offset, int64_t row, int64_t chunk, float (&v)[kChunk]) {
    keep(keep_bits(mask, offset, (uint32_t)row, (uint32_t)chunk), mask.scale, v);
}

}  // namespace dgsp
