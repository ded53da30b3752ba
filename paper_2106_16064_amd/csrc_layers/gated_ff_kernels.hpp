// The gated feed-forward block on matrix_tiles.hpp: what becomes of the products of a tile.
#pragma once

#include "product_kernels.hpp"

namespace dgsp {

// h = act(g) u, and for the backward pass act(g) and u act'(g), which it multiplies by dh.  Of 16-bit types h is rounded, as the matrix
// instructions take it; the other two are kept in 32 bits: rounded to 16 they would double the squared error of the gates' gradients.
template <typename T>
struct GatedUpOut {
    static constexpr bool kReadLate = false;
    Kept<T> h;
    float *act, *mul;           // null: not wanted
    int activation;
    float* partial;             // not null: split results, [split][g, u][m][h.ld], for gated_join_kernel
    // four neighbours
    __device__ __forceinline__ void finish(int64_t at, f32x4 g, f32x4 u) const {
        float in[4] = {g[0], g[1], g[2], g[3]}, value[4], slope[4];
        activate<sizeof(T) == 4>(activation, in, value, slope);
        put(at, value, slope, u);
    }
    __device__ __forceinline__ void put(int64_t at, const float* value, const float* slope, f32x4 u) const {
        const f32x4 a = {value[0], value[1], value[2], value[3]}, b = {slope[0], slope[1], slope[2], slope[3]};
        if (act) {
            *reinterpret_cast<f32x4*>(act + at) = a;
            *reinterpret_cast<f32x4*>(mul + at) = b * u;
        }
        h.store(at, a * u);
    }
    template <int kEach>
    __device__ __forceinline__ Nothing ask(const ProductArgs<T>&, int64_t, int64_t) const {
        return {};
    }
    template <int kEach>
    __device__ __forceinline__ void row(const ProductArgs<T>& args, const TileIndex& tile, int64_t m, int64_t n, Nothing, const f32x4 (&v)[kEach][2]) const {
        if (m >= args.m) return;
        const int64_t at = m * h.ld + n;
        if (partial) {
            float* to = partial + 2 * tile.split * args.m * h.ld + at;
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                if (n + 16 * j >= h.ld) break;
                *reinterpret_cast<f32x4*>(to + 16 * j) = v[j][0];
                *reinterpret_cast<f32x4*>(to + args.m * h.ld + 16 * j) = v[j][1];
            }
            return;
        }
        float g[4 * kEach], value[4 * kEach], slope[4 * kEach];
#pragma unroll
        for (int i = 0; i < 4 * kEach; ++i) g[i] = v[i / 4][0][i % 4];
        activate<sizeof(T) == 4>(activation, g, value, slope);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (n + 16 * j >= h.ld) break;
            put(at + 16 * j, value + 4 * j, slope + 4 * j, v[j][1]);
        }
    }
};

// dg = dh u act'(g) and du = dh act(g), dh = dy w_down; of 16-bit types rounded, as the matrix instructions take them in the next products.
// dh itself is not.
template <typename T>
struct GatedSlopeOut {
    static constexpr bool kReadLate = false;
    const float *act, *mul;
    Kept<T> dg, du;
    template <int kEach>
    struct Factors {
        f32x4 act[kEach], mul[kEach];
    };
    template <int kEach>
    __device__ __forceinline__ Factors<kEach> ask(const ProductArgs<T>& args, int64_t m, int64_t n) const {
        Factors<kEach> out;
        const int64_t at = m * dg.ld + n;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const bool inside = m < args.m && n + 16 * j < dg.ld;
            out.act[j] = inside ? *reinterpret_cast<const f32x4*>(act + at + 16 * j) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            out.mul[j] = inside ? *reinterpret_cast<const f32x4*>(mul + at + 16 * j) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        return out;
    }
    template <int kEach>
    __device__ __forceinline__ void row(const ProductArgs<T>& args, const TileIndex&, int64_t m, int64_t n, const Factors<kEach>& kept,
                                        const f32x4 (&v)[kEach][1]) const {
        if (m >= args.m) return;
        const int64_t at = m * dg.ld + n;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (n + 16 * j >= dg.ld) break;
            f32x4 g, u;
#pragma unroll
            for (int r = 0; r < 4; ++r) {               // beyond the hidden width a transposed operand holds whatever lies there
                const bool inside = n + 16 * j + r < args.n;
                g[r] = inside ? v[j][0][r] * kept.mul[j][r] : 0.0f;
                u[r] = inside ? v[j][0][r] * kept.act[j][r] : 0.0f;
            }
            dg.store(at + 16 * j, g);
            du.store(at + 16 * j, u);
        }
    }
};

// the same of the projections' splits, and what becomes of them; rows of `out` are padded
template <typename T>
__global__ __launch_bounds__(256) void gated_join_kernel(int64_t m, int splits, GatedUpOut<T> out) {
    const int64_t one = m * out.h.ld, step = (int64_t)gridDim.x * blockDim.x * 4;
    for (int64_t at = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * 4; at < one; at += step) {
        f32x4 g = {0.0f, 0.0f, 0.0f, 0.0f}, u = g;
        for (int s = 0; s < splits; s += kJoinAhead) {
            f32x4 a[kJoinAhead], b[kJoinAhead];
#pragma unroll
            for (int j = 0; j < kJoinAhead; ++j) {
                const float* from = out.partial + 2 * (s + j < splits ? s + j : 0) * one + at;
                a[j] = *reinterpret_cast<const f32x4*>(from);
                b[j] = *reinterpret_cast<const f32x4*>(from + one);
            }
#pragma unroll
            for (int j = 0; j < kJoinAhead; ++j) {
                if (s + j >= splits) break;
                g += a[j];
                u += b[j];
            }
        }
        out.finish(at, g, u);
    }
}

}  // namespace dgsp
