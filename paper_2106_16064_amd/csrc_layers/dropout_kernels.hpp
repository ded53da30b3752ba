// y = dropout(x) (+ residual): a lane takes the eight elements of one counter, in 16-byte accesses.  Memory bounds it: bfloat16, 2^20 rows
// of 128 with a residual, 805 MB, 142 us, 5.7 TB/s (a large copy: 4.96).  The full machine of lanes with one chunk each has enough on its
// way; four chunks a lane took 147 us there, and 81 us against 68 for float rows of 32.
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

template <typename T>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(int64_t rows, int64_t width, Divisor chunks, DropMask mask, const T* x, int64_t ldx,
                                                               const T* residual, int64_t ldr, T* y, int64_t ldy) {
    const uint64_t offset = mask.device_offset ? *mask.device_offset : mask.offset;
    const int64_t total = rows * (int64_t)chunks.by;
    for (int64_t first = (int64_t)blockIdx.x * kDropThreads; first < total; first += (int64_t)gridDim.x * kDropThreads) {
        const int64_t row0 = first / chunks.by;
        const uint32_t at = (uint32_t)(first - row0 * chunks.by) + threadIdx.x, down = chunks.quotient(at), chunk = at - down * chunks.by;
        const int64_t row = row0 + down, col = (int64_t)chunk * kChunk, here = width - col;
        if (row >= rows) continue;
        const RawChunk<T> in = load_chunk(x + row * ldx + col, here);
        RawChunk<T> other;
        if (residual) other = load_chunk(residual + row * ldr + col, here);
        float v[kChunk];
        widen(in, v);
        if (mask.dropped) drop(mask, offset, row, chunk, v);
        if (residual) {
            float r[kChunk];
            widen(other, r);
#pragma unroll
            for (int j = 0; j < kChunk; ++j) v[j] += r[j];
        }
        store_chunk(y + row * ldy + col, here, v);
    }
}

}  // namespace dgsp
