// Layer norm and its gradient: a wave takes a row.
#pragma once

#include "drop_mask.hpp"
#include "element_types.hpp"

namespace dgsp {

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

template <typename T>
struct NormInput {
    const T* x;
    int64_t ldx;
    const T* residual;
    int64_t ldr;
    DropMask drop;
    // s = x, or residual + dropout(x)
    __device__ float at(int64_t row, int64_t col, uint64_t offset) const {
        float v = to_float(x[row * ldx + col]);
        if (residual) {
            if (drop.dropped) v = (keep_bits(drop, offset, (uint32_t)row, (uint32_t)(col / 8)) >> (col % 8) & 1) ? v * drop.scale : 0.0f;
            v += to_float(residual[row * ldr + col]);
        }
        return v;
    }
};

template <typename T>
__global__ void layer_norm_kernel(int64_t rows, int64_t width, NormInput<T> in, const void* weight, const void* bias, bool wide,
                                  float eps, T* y, int64_t ldy, T* sum, int64_t lds, float* stats) {
    const int lane = threadIdx.x & 63;
    const uint64_t offset = in.drop.device_offset ? *in.drop.device_offset : in.drop.offset;
    const int64_t waves = (int64_t)gridDim.x * blockDim.x >> 6;
    for (int64_t row = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 6; row < rows; row += waves) {
        float total = 0.0f;
        for (int64_t c = lane; c < width; c += 64) total += in.at(row, c, offset);
        const float mean = wave_sum(total) / (float)width;
        float squares = 0.0f;
        for (int64_t c = lane; c < width; c += 64) {
            const float d = in.at(row, c, offset) - mean;
            squares += d * d;
        }
        const float rstd = 1.0f / sqrtf(wave_sum(squares) / (float)width + eps);
        for (int64_t c = lane; c < width; c += 64) {
            const float s = in.at(row, c, offset);
            float v = (s - mean) * rstd;
            if (weight) v *= load_param<T>(weight, c, wide);
            if (bias) v += load_param<T>(bias, c, wide);
            y[row * ldy + c] = from_float<T>(v);
            if (sum) sum[row * lds + c] = from_float<T>(s);
        }
        if (stats && lane == 0) {
            stats[2 * row] = mean;
            stats[2 * row + 1] = rstd;
        }
    }
}

template <typename T>
__global__ void layer_norm_backward_kernel(int64_t rows, int64_t width, const T* s, int64_t lds, const float* stats,
                                           const void* weight, bool wide, const T* dy, int64_t lddy, const T* ds, int64_t ldds,
                                           DropMask drop, T* dsum, T* dx) {
    const int lane = threadIdx.x & 63;
    const uint64_t offset = drop.device_offset ? *drop.device_offset : drop.offset;
    const int64_t waves = (int64_t)gridDim.x * blockDim.x >> 6;
    for (int64_t row = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 6; row < rows; row += waves) {
        const float mean = stats[2 * row], rstd = stats[2 * row + 1];
        float a = 0.0f, b = 0.0f;
        for (int64_t c = lane; c < width; c += 64) {
            const float dhat = to_float(dy[row * lddy + c]) * (weight ? load_param<T>(weight, c, wide) : 1.0f);
            a += dhat;
            b += dhat * (to_float(s[row * lds + c]) - mean) * rstd;
        }
        a = wave_sum(a) / (float)width;
        b = wave_sum(b) / (float)width;
        for (int64_t c = lane; c < width; c += 64) {
            const float dhat = to_float(dy[row * lddy + c]) * (weight ? load_param<T>(weight, c, wide) : 1.0f);
            const float hat = (to_float(s[row * lds + c]) - mean) * rstd;
            float v = (dhat - a - hat * b) * rstd;
            if (ds) v += to_float(ds[row * ldds + c]);
            dsum[row * width + c] = from_float<T>(v);
            if (dx) {
                const bool keep = keep_bits(drop, offset, (uint32_t)row, (uint32_t)(c / 8)) >> (c % 8) & 1;
                dx[row * width + c] = from_float<T>(keep ? v * drop.scale : 0.0f);
            }
        }
    }
}

constexpr int kNormSlices = 256;        // of the rows, for the parameters' gradients

// partial[slice][0 or 1][col]: sums over the slice's rows of dy hat and of dy
template <typename T>
__global__ void layer_norm_param_partials_kernel(int64_t rows, int64_t width, const T* s, int64_t lds, const float* stats, const T* dy,
                                                 int64_t lddy, float* partial) {
    const int64_t col = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (col >= width) return;
    float a = 0.0f, b = 0.0f;
    for (int64_t row = blockIdx.y; row < rows; row += kNormSlices) {
        const float d = to_float(dy[row * lddy + col]);
        a += d * (to_float(s[row * lds + col]) - stats[2 * row]) * stats[2 * row + 1];
        b += d;
    }
    partial[(2 * (int64_t)blockIdx.y) * width + col] = a;
    partial[(2 * (int64_t)blockIdx.y + 1) * width + col] = b;
}

template <typename T>
__global__ void layer_norm_param_sums_kernel(int64_t width, const float* partial, void* dweight, void* dbias, bool wide) {
    const int64_t col = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (col >= width) return;
    float a = 0.0f, b = 0.0f;
    for (int64_t i = 0; i < kNormSlices; ++i) {
        a += partial[2 * i * width + col];
        b += partial[(2 * i + 1) * width + col];
    }
    if (dweight) store_param<T>(dweight, col, wide, a);
    if (dbias) store_param<T>(dbias, col, wide, b);
}

}  // namespace dgsp
