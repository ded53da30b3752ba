// Sums over the rows of a matrix whose workgroups have left theirs: a parameter's gradient.
#pragma once

#include "element_types.hpp"

namespace dgsp {

constexpr int kSumColumns = 32, kSumSlices = 32, kSumAhead = 8;
constexpr int64_t kSumGroups = 1 << 20;         // at most: a launch has fewer than 2^32 threads, and drops what is beyond without an error

// out[c] = sum over g of partial[g][c], in order.  Few columns and many sums: what takes time is waiting for memory, so a lane asks for
// eight sums at a time.
template <typename T>
__global__ __launch_bounds__(kSumColumns* kSumSlices) void column_sums_kernel(int64_t width, int64_t groups, const float* partial, void* out, bool wide) {
    __shared__ float part[kSumSlices][kSumColumns];
    const int column = threadIdx.x % kSumColumns, slice = threadIdx.x / kSumColumns;
    for (int64_t first = (int64_t)blockIdx.x * kSumColumns; first < width; first += (int64_t)gridDim.x * kSumColumns) {
        const int64_t at = first + column;
        float v = 0.0f;
        if (at < width)
            for (int64_t g = slice; g < groups; g += kSumSlices * kSumAhead) {
                float ahead[kSumAhead];
#pragma unroll
                for (int i = 0; i < kSumAhead; ++i) ahead[i] = g + i * kSumSlices < groups ? partial[(g + i * kSumSlices) * width + at] : 0.0f;
#pragma unroll
                for (int i = 0; i < kSumAhead; ++i) v += ahead[i];
            }
        part[slice][column] = v;
        __syncthreads();
        if (slice == 0 && at < width) {
#pragma unroll
            for (int i = 1; i < kSumSlices; ++i) v += part[i][column];
            store_param<T>(out, at, wide, v);
        }
        __syncthreads();
    }
}

template <typename T>
void launch_column_sums(int64_t width, int64_t groups, const float* partial, void* out, bool wide, hipStream_t stream) {
    const int64_t needed = (width + kSumColumns - 1) / kSumColumns;
    column_sums_kernel<T><<<(unsigned)(needed < kSumGroups ? needed : kSumGroups), kSumColumns * kSumSlices, 0, stream>>>(width, groups, partial, out, wide);
}

}  // namespace dgsp
