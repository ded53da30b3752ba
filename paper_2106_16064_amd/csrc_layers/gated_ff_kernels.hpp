// The products of the gated feed-forward block: C = sum of A_s B_s over one or two pairs of operands, tiles of C in registers,
// tiles of A and B in LDS, matrix instructions.
#pragma once

#include "../../include/dgsp_layers.h"
#include "element_types.hpp"

namespace dgsp {

template <typename T>
struct Operand {                // element (i, k) at p[i * outer + k * inner]
    const T* p;
    int64_t outer, inner;
};

using f32x4 = float __attribute__((ext_vector_type(4)));

template <typename T>
struct Matrix;
template <>
struct Matrix<bf16_t> {
    static constexpr int kLane = 8, kDepth = 32;        // elements per lane, depth of one instruction
    using Fragment = bf16_t __attribute__((ext_vector_type(8)));
    static __device__ f32x4 multiply(Fragment a, Fragment b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Matrix<f16_t> {
    static constexpr int kLane = 8, kDepth = 32;
    using Fragment = f16_t __attribute__((ext_vector_type(8)));
    static __device__ f32x4 multiply(Fragment a, Fragment b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Matrix<float> {
    static constexpr int kLane = 1, kDepth = 4;
    using Fragment = float __attribute__((ext_vector_type(1)));
    static __device__ f32x4 multiply(Fragment a, Fragment b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a[0], b[0], c, 0, 0, 0); }
};

// act(g) and its derivative
__device__ __forceinline__ void activate(int kind, float g, float& value, float& slope) {
    if (kind == DGSP_ACT_RELU) {
        value = g > 0.0f ? g : (g != g ? g : 0.0f);
        slope = g > 0.0f ? 1.0f : 0.0f;
    } else if (kind == DGSP_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-g));
        value = g * s;
        slope = s * (1.0f + g * (1.0f - s));
    } else {
        const float c = 0.5f * (1.0f + erff(g * 0.70710678f));
        value = g * c;
        slope = c + g * expf(-0.5f * g * g) * 0.39894228f;
    }
}

constexpr int kTile = 64, kTileDepth = 32, kTilePad = 8;

// rows [i0, i0 + 64), depth [k0, k0 + 32) of an operand, zeros beyond its ends
template <typename T>
__device__ void stage(T (*lds)[kTileDepth + kTilePad], const Operand<T>& a, int64_t i0, int64_t n, int64_t k0, int64_t depth) {
    for (int e = threadIdx.x; e < kTile * kTileDepth; e += 256) {
        const int i = a.inner == 1 ? e / kTileDepth : e % kTile, k = a.inner == 1 ? e % kTileDepth : e / kTile;
        lds[i][k] = i0 + i < n && k0 + k < depth ? a.p[(i0 + i) * a.outer + (k0 + k) * a.inner] : from_float<T>(0.0f);
    }
}

// Four waves, each 32 x 32 of the tile: lane l holds row l % 16 and depths l / 16 * kLane ... of an operand's fragment, and
// rows 4 * (l / 16) ... + 3 of column l % 16 of a result's.
template <typename T, int kProducts>
__device__ void tile_products(f32x4 (&acc)[kProducts][2][2], const Operand<T>& a, const Operand<T> (&b)[kProducts], int64_t m0, int64_t m,
                              int64_t n0, int64_t n, int64_t depth) {
    using M = Matrix<T>;
    __shared__ T as[kTile][kTileDepth + kTilePad], bs[kProducts][kTile][kTileDepth + kTilePad];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
    for (int64_t k0 = 0; k0 < depth; k0 += kTileDepth) {
        __syncthreads();
        stage(as, a, m0, m, k0, depth);
        for (int p = 0; p < kProducts; ++p) stage(bs[p], b[p], n0, n, k0, depth);
        __syncthreads();
        for (int k = 0; k < kTileDepth; k += M::kDepth) {
            typename M::Fragment fa[2], fb[2];
            for (int i = 0; i < 2; ++i)
                for (int j = 0; j < M::kLane; ++j) fa[i][j] = as[wm + 16 * i + lane % 16][k + lane / 16 * M::kLane + j];
            for (int p = 0; p < kProducts; ++p) {
                for (int i = 0; i < 2; ++i)
                    for (int j = 0; j < M::kLane; ++j) fb[i][j] = bs[p][wn + 16 * i + lane % 16][k + lane / 16 * M::kLane + j];
                for (int i = 0; i < 2; ++i)
                    for (int j = 0; j < 2; ++j) acc[p][i][j] = M::multiply(fa[i], fb[j], acc[p][i][j]);
            }
        }
    }
}

// calls f(row, column, i, j, r) for the elements that this lane holds
template <typename F>
__device__ void each_element(int64_t m0, int64_t m, int64_t n0, int64_t n, F&& f) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j)
            for (int r = 0; r < 4; ++r) {
                const int64_t row = m0 + wm + 16 * i + lane / 16 * 4 + r, col = n0 + wn + 16 * j + lane % 16;
                if (row < m && col < n) f(row, col, i, j, r);
            }
}

// g, u and h = act(g) u, rows x hidden each; g and u are written only where the backward pass wants them
template <typename T>
__global__ __launch_bounds__(256) void gated_up_kernel(int64_t rows, int64_t width, int64_t hidden, int activation, Operand<T> x,
                                                       Operand<T> w_gate, Operand<T> w_up, T* g, T* u, T* h) {
    const int64_t tiles = (hidden + kTile - 1) / kTile, m0 = blockIdx.x / tiles * kTile, n0 = blockIdx.x % tiles * kTile;
    f32x4 acc[2][2][2] = {};
    const Operand<T> b[2] = {w_gate, w_up};
    tile_products<T, 2>(acc, x, b, m0, rows, n0, hidden, width);
    each_element(m0, rows, n0, hidden, [&](int64_t row, int64_t col, int i, int j, int r) {
        const float gate = acc[0][i][j][r], up = acc[1][i][j][r];
        float value, slope;
        activate(activation, gate, value, slope);
        const int64_t at = row * hidden + col;
        if (g) {
            g[at] = from_float<T>(gate);
            u[at] = from_float<T>(up);
        }
        h[at] = from_float<T>(value * up);
    });
}

// dg and du in place of g and u, from dh = dy w_down
template <typename T>
__global__ __launch_bounds__(256) void gated_down_gradient_kernel(int64_t rows, int64_t hidden, int64_t out_width, int activation,
                                                                  Operand<T> dy, Operand<T> w_down, const T* g, const T* u, T* dg, T* du) {
    const int64_t tiles = (hidden + kTile - 1) / kTile, m0 = blockIdx.x / tiles * kTile, n0 = blockIdx.x % tiles * kTile;
    f32x4 acc[1][2][2] = {};
    const Operand<T> b[1] = {w_down};
    tile_products<T, 1>(acc, dy, b, m0, rows, n0, hidden, out_width);
    each_element(m0, rows, n0, hidden, [&](int64_t row, int64_t col, int i, int j, int r) {
        const int64_t at = row * hidden + col;
        float value, slope;
        activate(activation, to_float(g[at]), value, slope);
        const float dh = acc[0][i][j][r];
        dg[at] = from_float<T>(dh * to_float(u[at]) * slope);
        du[at] = from_float<T>(dh * value);
    });
}

// c = a b^T, or a b^T + a2 b2^T
template <typename T>
__global__ __launch_bounds__(256) void product_kernel(int64_t m, int64_t n, int64_t depth, Operand<T> a, Operand<T> b, Operand<T> a2,
                                                      Operand<T> b2, T* c, int64_t ldc) {
    const int64_t tiles = (n + kTile - 1) / kTile, m0 = blockIdx.x / tiles * kTile, n0 = blockIdx.x % tiles * kTile;
    f32x4 acc[1][2][2] = {};
    for (int s = 0; s < 2; ++s) {
        if (s && !a2.p) break;
        const Operand<T> bs[1] = {s ? b2 : b};
        tile_products<T, 1>(acc, s ? a2 : a, bs, m0, m, n0, n, depth);
    }
    each_element(m0, m, n0, n, [&](int64_t row, int64_t col, int i, int j, int r) { c[row * ldc + col] = from_float<T>(acc[0][i][j][r]); });
}

}  // namespace dgsp
