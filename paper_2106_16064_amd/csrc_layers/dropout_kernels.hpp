// y = dropout(x) (+ residual): a lane takes the eight elements of one counter, kEach times.
#pragma once

#include "chunks.hpp"

namespace dgsp {

constexpr int kDropThreads = 256;

// quotient of numbers below 2^31 by a constant (Granlund, Montgomery, PLDI 1994): (a * magic + a * 2^32) >> 32 >> shift
struct Divisor {
    uint32_t by, magic, shift;
    explicit Divisor(uint32_t d) : by(d), magic(0), shift(0) {
        while (shift < 31 && (1u << shift) < d) ++shift;
        magic = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ uint32_t quotient(uint32_t a) const { return (uint32_t)(((uint64_t)a * magic >> 32) + a) >> shift; }
};

template <typename T, int kEach>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(int64_t rows, int64_t width, Divisor chunks, DropMask mask, const T* x, int64_t ldx,
                                                               const T* residual, int64_t ldr, T* y, int64_t ldy) {
    const uint64_t offset = mask.device_offset ? *mask.device_offset : mask.offset;
    const int64_t total = rows * (int64_t)chunks.by;
    for (int64_t first = (int64_t)blockIdx.x * (kDropThreads * kEach); first < total; first += (int64_t)gridDim.x * (kDropThreads * kEach)) {
        const int64_t row0 = first / chunks.by;
        const uint32_t in_row = (uint32_t)(first - row0 * chunks.by);
        RawChunk<T> a[kEach], b[kEach];
        int64_t row[kEach];
        uint32_t chunk[kEach];
        bool inside[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const uint32_t at = in_row + e * kDropThreads + threadIdx.x, down = chunks.quotient(at);
            row[e] = row0 + down;
            chunk[e] = at - down * chunks.by;
            inside[e] = row[e] < rows;
            const int64_t col = (int64_t)chunk[e] * kChunk;
            if (inside[e]) {
                a[e] = load_chunk(x + row[e] * ldx + col, width - col);
                if (residual) b[e] = load_chunk(residual + row[e] * ldr + col, width - col);
            }
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            if (!inside[e]) continue;
            const int64_t col = (int64_t)chunk[e] * kChunk;
            float v[kChunk];
            widen(a[e], v);
            if (mask.dropped) drop(mask, offset, row[e], chunk[e], v);
            if (residual) {
                float r[kChunk];
                widen(b[e], r);
#pragma unroll
                for (int j = 0; j < kChunk; ++j) v[j] += r[j];
            }
            store_chunk(y + row[e] * ldy + col, width - col, v);
        }
    }
}

}  // namespace dgsp
