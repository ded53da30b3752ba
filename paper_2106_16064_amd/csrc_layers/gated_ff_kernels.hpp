// The gated feed-forward block on matrix_tiles.hpp: what becomes of the products of a tile, and how operands are laid out for it.
#pragma once

#include "../../include/dgsp_layers.h"
#include "chunks.hpp"
#include "float_tiles.hpp"
#include "matrix_tiles.hpp"

namespace dgsp {

// act(g) and its derivative, kCount numbers at once (one branch on the kind for all of them): exp2 and the reciprocal of the hardware
// (one unit in the last place of float each; the argument of the exponential is off by g 2^-24), and erf to 1.5e-7 (Abramowitz, Stegun,
// Handbook of Mathematical Functions, 7.1.26), which is what 1 + erf(z) keeps of it in float anyway.  A third of the instructions of
// the library's functions, which took longer than the products where the depth is small.  kFloat: results are float, and the rounding of
// the sigmoid's argument is made up for; the sigmoid counts as 0 from -87.3 on below, where silu is less than 1.1e-36.
template <bool kFloat, int kCount>
__device__ __forceinline__ void activate(int kind, const float (&g)[kCount], float (&value)[kCount], float (&slope)[kCount]) {
    if (kind == DGSP_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            value[i] = g[i] > 0.0f ? g[i] : (g[i] != g[i] ? g[i] : 0.0f);
            slope[i] = g[i] > 0.0f ? 1.0f : 0.0f;
        }
    } else if (kind == DGSP_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            float s;
            if constexpr (kFloat) {
                const float power = -1.44269504f * g[i], inside = fminf(power, 126.0f);
                const float rest = fabsf(power) < 126.0f ? fmaf(-1.44269504f, g[i], -power) - 1.925963e-8f * g[i] : 0.0f;
                const float e = __builtin_amdgcn_exp2f(inside);
                s = power < 126.0f ? __builtin_amdgcn_rcpf(1.0f + fmaf(e, 0.69314718f * rest, e)) : 0.0f;       // 2^-126 and less: not times a large g
            } else {
                s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * g[i]));
            }
            value[i] = g[i] * s;
            slope[i] = s + value[i] * (1.0f - s);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const float z = fabsf(g[i]) * 0.70710678f, t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * z);
            const float e = __builtin_amdgcn_exp2f(-1.44269504f * (z * z));
            const float tail = 0.5f * e * t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
            const float c = g[i] < 0.0f ? tail : 1.0f - tail;
            value[i] = g[i] * c;
            slope[i] = c + g[i] * e * 0.39894228f;
        }
    }
}

// A matrix that the block keeps between its products; ld is a multiple of 8.
template <typename T>
struct Kept {
    T* p;
    int64_t ld;
    // four neighbours
    __device__ __forceinline__ void store(int64_t at, f32x4 v) const {
        using T4 = T __attribute__((ext_vector_type(4)));
        *reinterpret_cast<T4*>(p + at) = T4{from_float<T>(v[0]), from_float<T>(v[1]), from_float<T>(v[2]), from_float<T>(v[3])};
    }
};

// ---------------------------------------------------------------- laying out

// A matrix of 16-bit elements whose rows are padded to a multiple of 8 with zeros.
template <typename T>
struct Layout {
    const T* from;
    int64_t rows, cols, ld;
    T* to;
    int64_t to_ld;
    unsigned groups;            // workgroups that work on it
};

constexpr int kMostLayouts = 5;

template <typename T>
struct Layouts {
    Layout<T> each[kMostLayouts];
    int count;
};

// all matrices of a call in one launch (float16, one of 1000 x 2731: 11 MB in 5.5 us)
template <typename T>
__global__ __launch_bounds__(256) void lay_out_kernel(Layouts<T> all) {
    unsigned group = blockIdx.x;
    Layout<T> l = all.each[0];
#pragma unroll
    for (int i = 1; i < kMostLayouts; ++i)
        if (i < all.count && group >= l.groups) {
            group -= l.groups;
            l = all.each[i];
        }
    const int64_t chunks = l.to_ld / 8, step = (int64_t)l.groups * blockDim.x;
    for (int64_t i = (int64_t)group * blockDim.x + threadIdx.x; i < l.rows * chunks; i += step) {
        const int64_t row = i / chunks, col = (i - row * chunks) * 8;
        *reinterpret_cast<u32x4*>(l.to + row * l.to_ld + col) = load_chunk(l.from + row * l.ld + col, l.cols - col).q[0];
    }
}

// ---------------------------------------------------------------- products

// h = act(g) u, and for the backward pass act(g) and u act'(g), which it multiplies by dh.  Of 16-bit types h is rounded, as the matrix
// instructions take it; the other two are kept in 32 bits: rounded to 16 they would double the squared error of the gates' gradients.
template <typename T>
struct GatedUpOut {
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

template <typename T>
struct ProductOut {
    T* c[2];                    // one per batch
    int64_t ld;
    bool vectors;               // four neighbours may be written at once
    float* partial;             // not null: split results, [split][batch][m][n padded to 4]
    template <int kEach>
    __device__ __forceinline__ Nothing ask(const ProductArgs<T>&, int64_t, int64_t) const {
        return {};
    }
    template <int kEach>
    __device__ __forceinline__ void row(const ProductArgs<T>& args, const TileIndex& tile, int64_t m, int64_t n, Nothing, const f32x4 (&v)[kEach][1]) const {
        using T4 = T __attribute__((ext_vector_type(4)));
        if (m >= args.m) return;
        const int64_t padded = (args.n + 3) / 4 * 4;
        float* split = partial ? partial + (((int64_t)tile.split * args.batch + tile.batch) * args.m + m) * padded + n : nullptr;
        T* to = (tile.batch ? c[1] : c[0]) + m * ld + n;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const f32x4 x = v[j][0];
            if (n + 16 * j >= args.n) break;
            if (partial) {
                *reinterpret_cast<f32x4*>(split + 16 * j) = x;
            } else if (vectors && n + 16 * j + 4 <= args.n) {
                *reinterpret_cast<T4*>(to + 16 * j) = T4{from_float<T>(x[0]), from_float<T>(x[1]), from_float<T>(x[2]), from_float<T>(x[3])};
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (n + 16 * j + r < args.n) to[16 * j + r] = from_float<T>(x[r]);
            }
        }
    }
};

constexpr int kJoinAhead = 8;

// The sum of the splits, in order; eight are asked for at a time, as what takes time is waiting for memory (4096 sums of 4 splits: 4 us).
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(int64_t m, int64_t n, int batch, int splits, const float* partial, ProductOut<T> out) {
    const int64_t quads = (n + 3) / 4, count = m * quads, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < count * batch; i += step) {
        const int64_t b = i / count, row = (i - b * count) / quads, col = (i - b * count - row * quads) * 4;
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < splits; s += kJoinAhead) {
            f32x4 ahead[kJoinAhead];
#pragma unroll
            for (int j = 0; j < kJoinAhead; ++j)
                ahead[j] = s + j < splits ? *reinterpret_cast<const f32x4*>(partial + 4 * ((s + j) * count * batch + i)) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < kJoinAhead; ++j) sum += ahead[j];
        }
        T* to = (b ? out.c[1] : out.c[0]) + row * out.ld + col;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (col + r < n) to[r] = from_float<T>(sum[r]);
    }
}

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
