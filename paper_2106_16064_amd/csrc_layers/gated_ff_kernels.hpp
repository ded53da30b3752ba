// The gated feed-forward block on matrix_tiles.hpp: what becomes of the products of a tile, and how operands are laid out for it.
#pragma once

#include "../../include/dgsp_layers.h"
#include "matrix_tiles.hpp"

namespace dgsp {

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

// The same for results of 16 bits, kCount numbers at once (one branch on the kind for all of them): exp2 and the reciprocal of the
// hardware (one unit in the last place of float each; the argument of the exponential is off by g 2^-24), and erf to 1.5e-7 (Abramowitz,
// Stegun, Handbook of Mathematical Functions, 7.1.26).  A third of the instructions.
template <int kCount>
__device__ __forceinline__ void activate_short(int kind, const float (&g)[kCount], float (&value)[kCount], float (&slope)[kCount]) {
    if (kind == DGSP_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) activate(DGSP_ACT_RELU, g[i], value[i], slope[i]);
    } else if (kind == DGSP_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * g[i]));
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

// v as the sum of three bf16 numbers, each the rest rounded to nearest: what is left is below 2^-26 of v.  Where rounding would pass
// the largest bf16 number the first one is cut off instead; what is not finite stays in the first one.
__device__ __forceinline__ void split3(float v, bf16_t (&out)[3]) {
    out[0] = (bf16_t)v;
    float rest = v - (float)out[0];
    if (!(fabsf((float)out[0]) < __builtin_inff())) {
        if (fabsf(v) < __builtin_inff()) {
            out[0] = __builtin_bit_cast(bf16_t, (uint16_t)(__builtin_bit_cast(uint32_t, v) >> 16));
            rest = v - (float)out[0];
        } else {
            rest = 0.0f;
        }
    }
    out[1] = (bf16_t)rest;
    out[2] = (bf16_t)(rest - (float)out[1]);
}

// A matrix that later products read, in planes of E.  ld is a multiple of 8.
template <typename E>
struct Planes {
    E* p;
    int64_t ld, plane;          // plane 0: one plane
    // four neighbours
    __device__ __forceinline__ void store(int64_t at, f32x4 v) const {
        using E4 = E __attribute__((ext_vector_type(4)));
        E* to = p + at;
        if (plane) {
            if constexpr (sizeof(E) == 2 && !__is_same(E, f16_t)) {
                E4 out[3];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    bf16_t parts[3];
                    split3(v[r], parts);
                    for (int q = 0; q < 3; ++q) out[q][r] = parts[q];
                }
#pragma unroll
                for (int q = 0; q < 3; ++q) *reinterpret_cast<E4*>(to + q * plane) = out[q];
            }
        } else {
            *reinterpret_cast<E4*>(to) = E4{from_float<E>(v[0]), from_float<E>(v[1]), from_float<E>(v[2]), from_float<E>(v[3])};
        }
    }
};

// ---------------------------------------------------------------- laying out

// `from`, rows x cols, as planes whose rows are padded to a multiple of 8 with zeros
template <typename T, typename E>
__global__ void lay_out_kernel(int64_t rows, int64_t cols, const T* from, int64_t ld, E* to, int64_t to_ld, int64_t plane) {
    using E8 = E __attribute__((ext_vector_type(8)));
    const int64_t chunks = to_ld / 8, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < rows * chunks; i += step) {
        const int64_t row = i / chunks, col = (i - row * chunks) * 8;
        const T* at = from + row * ld + col;
        E8 out[3];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const T v = col + j < cols ? at[j] : (T)0.0f;
            if constexpr (sizeof(T) == 4) {
                bf16_t parts[3];
                split3(v, parts);
                for (int q = 0; q < 3; ++q) out[q][j] = parts[q];
            } else {
                out[0][j] = v;
            }
        }
        for (int q = 0; q < (sizeof(T) == 4 ? 3 : 1); ++q) *reinterpret_cast<E8*>(to + q * plane + row * to_ld + col) = out[q];
    }
}

// ---------------------------------------------------------------- products

// h = act(g) u, and for the backward pass act(g) and u act'(g), which it multiplies by dh.  These two are kept in 32 bits: rounded to
// 16 they would double the squared error of the gates' gradients, and the 8 bytes an element cost 3 % of a large block's step.
// kShort: of a 16-bit type.
template <typename E, bool kShort>
struct GatedUpOut {
    Planes<E> h;
    float *act, *mul;           // null: not wanted
    int activation;
    template <int kEach>
    __device__ __forceinline__ Nothing ask(const ProductArgs&, int64_t, int64_t) const {
        return {};
    }
    template <int kEach>
    __device__ __forceinline__ void row(const ProductArgs& args, const TileIndex&, int64_t m, int64_t n, Nothing, const f32x4 (&v)[kEach][2]) const {
        if (m >= args.m) return;
        float g[4 * kEach], value[4 * kEach], slope[4 * kEach];
#pragma unroll
        for (int i = 0; i < 4 * kEach; ++i) g[i] = v[i / 4][0][i % 4];
        if constexpr (kShort) {
            activate_short(activation, g, value, slope);
        } else {
#pragma unroll
            for (int i = 0; i < 4 * kEach; ++i) activate(activation, g[i], value[i], slope[i]);
        }
        const int64_t at = m * h.ld + n;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (n + 16 * j >= h.ld) break;
            const f32x4 a = {value[4 * j], value[4 * j + 1], value[4 * j + 2], value[4 * j + 3]};
            const f32x4 b = {slope[4 * j], slope[4 * j + 1], slope[4 * j + 2], slope[4 * j + 3]};
            if (act) {
                *reinterpret_cast<f32x4*>(act + at + 16 * j) = a;
                *reinterpret_cast<f32x4*>(mul + at + 16 * j) = b * v[j][1];
            }
            h.store(at + 16 * j, a * v[j][1]);
        }
    }
};

// dg = dh u act'(g) and du = dh act(g), dh = dy w_down
template <typename E>
struct GatedSlopeOut {
    const float *act, *mul;
    Planes<E> dg, du;
    template <int kEach>
    struct Kept {
        f32x4 act[kEach], mul[kEach];
    };
    template <int kEach>
    __device__ __forceinline__ Kept<kEach> ask(const ProductArgs& args, int64_t m, int64_t n) const {
        Kept<kEach> out;
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
    __device__ __forceinline__ void row(const ProductArgs& args, const TileIndex&, int64_t m, int64_t n, const Kept<kEach>& kept,
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
    __device__ __forceinline__ Nothing ask(const ProductArgs&, int64_t, int64_t) const {
        return {};
    }
    template <int kEach>
    __device__ __forceinline__ void row(const ProductArgs& args, const TileIndex& tile, int64_t m, int64_t n, Nothing, const f32x4 (&v)[kEach][1]) const {
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

// the sum of the splits, in order
template <typename T>
__global__ void join_kernel(int64_t m, int64_t n, int batch, int splits, const float* partial, ProductOut<T> out) {
    const int64_t quads = (n + 3) / 4, count = m * quads, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < count * batch; i += step) {
        const int64_t b = i / count, row = (i - b * count) / quads, col = (i % quads) * 4;
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < splits; ++s) sum += *reinterpret_cast<const f32x4*>(partial + 4 * (s * count * batch + i));
        for (int r = 0; r < 4; ++r)
            if (col + r < n) out.c[b][row * out.ld + col + r] = from_float<T>(sum[r]);
    }
}

}  // namespace dgsp
