// y = dropout(x) (+ residual): a thread takes the eight elements of one counter.
#pragma once

#include "drop_mask.hpp"
#include "element_types.hpp"

namespace dgsp {

template <typename T>
__global__ void dropout_kernel(int64_t rows, int64_t width, DropMask drop, const T* x, int64_t ldx, const T* residual, int64_t ldr,
                               T* y, int64_t ldy) {
    const int64_t groups = (width + kDropGroup - 1) / kDropGroup;
    const uint64_t offset = drop.device_offset ? *drop.device_offset : drop.offset;
    const int64_t step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < rows * groups; i += step) {
        const int64_t row = i / groups, group = i - row * groups;
        const uint32_t keep = keep_bits(drop, offset, (uint32_t)row, (uint32_t)group);
        for (int j = 0; j < kDropGroup; ++j) {
            const int64_t col = group * kDropGroup + j;
            if (col >= width) break;
            float v = (keep >> j & 1) ? to_float(x[row * ldx + col]) * drop.scale : 0.0f;
            if (residual) v += to_float(residual[row * ldr + col]);
            y[row * ldy + col] = from_float<T>(v);
        }
    }
}

}  // namespace dgsp
