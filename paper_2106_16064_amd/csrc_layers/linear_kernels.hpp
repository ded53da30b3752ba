// y = act(x w^T + bias) + residual on matrix_tiles.hpp: what becomes of the product of a tile, and what the backward pass makes of dy first.
//
// The epilogue adds the bias to the sum in 32 bits, applies the activation, adds the residual and rounds once.  For the backward pass it
// leaves what the activation's derivative is made of: z in the bias's type, or act'(z) in steps of 1/112 in 8 bits, which has 0 and 1 exactly: all of relu's, and what
// gelu (-0.13 ... 1.13) and silu (-0.10 ... 1.10) come to far from 0.  Where z is kept in 16 bits its rounding moves act'(z) by |z act''(z)| half a step, about a third of
// what rounding dz itself costs (z of deviation 0.5 to 2: 0.27 to 0.38 of it); a float bias's gradient is not rounded, and would lose by it.
//
// What it costs beside the product, bfloat16, 8192 x 4096 -> 16384, gelu, z kept: 1010 to 1100 us against 900 of the product alone, of which
// 110 is writing y and z (960 without z); nothing runs beside it, as a tile of 256 takes a CU.  dz, from dy and z: 200 us, 4.0 TB/s.
#pragma once

#include "product_kernels.hpp"
#include "rows8.hpp"

namespace dgsp {

constexpr float kSlopeSteps = 112.0f;

// act(z) alone (activate() without the derivative, which is then never made)
template <bool kFloat, int kCount>
__device__ __forceinline__ void activate_only(int kind, const float (&z)[kCount], float (&value)[kCount]) {
    if (kind == DGSP_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) value[i] = z[i];
    } else {
        float slope[kCount];
        activate<kFloat>(kind, z, value, slope);
    }
}

// A NaN has a code of its own, below all slopes.
__device__ __forceinline__ uint32_t slope_code(float slope) { return slope == slope ? (uint32_t)(int)rintf(slope * kSlopeSteps) & 0xffu : 0x80u; }

// the codes of groups of four, together where none is NaN
template <int kCount>
__device__ __forceinline__ void slope_words(const float (&slope)[4 * kCount], uint32_t (&words)[kCount]) {
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < kCount; ++j) {
        words[j] = whole_word({slope[4 * j], slope[4 * j + 1], slope[4 * j + 2], slope[4 * j + 3]}, kSlopeSteps);
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += slope[4 * j + r];
    }
    if (__builtin_amdgcn_ballot_w64(sum != sum) == 0) return;
#pragma unroll
    for (int j = 0; j < kCount; ++j) {
        words[j] = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) words[j] |= slope_code(slope[4 * j + r]) << (8 * r);
    }
}

// of eight codes the j-th
__device__ __forceinline__ float slope_of(uint2 codes, int j) {
    const int code = (int8_t)((j < 4 ? codes.x : codes.y) >> (8 * (j % 4)) & 0xffu);
    return code == -128 ? __builtin_nanf("") : (float)code * (1.0f / kSlopeSteps);
}

// z as it was kept: an infinity, of z or of its rounding, has the slope of a number far from 0
template <typename T>
__device__ __forceinline__ float inside_range(float z) {
    constexpr float kMost = std::is_same_v<T, f16_t> ? 65504.0f : 3.38953139e38f;
    return fabsf(z) > kMost ? __builtin_copysignf(kMost, z) : z;
}

// How many columns there are from n on.  Rows of fragments ask each for itself: the comparisons with it, kept for all of them, would be more than
// the scalar registers hold.
__device__ __forceinline__ int columns_left(int64_t columns, int64_t n) {
    int left = (int)(columns - n);
    asm volatile("" : "+v"(left));
    return left;
}

// four neighbours, at once where they lie so; `here` of them are there
template <typename T>
__device__ __forceinline__ f32x4 load4(const T* p, bool vectors, int here) {
    using T4 = T __attribute__((ext_vector_type(4)));
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (vectors && here >= 4) {
        const T4 t = *reinterpret_cast<const T4*>(p);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = to_float((T)t[r]);
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (r < here) v[r] = to_float(p[r]);
    }
    return v;
}

// kKeeps: may something be left for a backward pass?  What cannot be is not compiled: the kernels in 8 bits have no registers to spare.
template <typename T, bool kKeeps = true>
struct LinearOut {
    static constexpr bool kReadLate = true;
    T* y;
    int64_t ldy;
    bool vectors, bias_vectors, residual_vectors;       // four neighbours may be read or written at once
    bool wide;                  // the bias, and z, in float
    const void* bias;           // null: none
    const T* residual;          // null: none
    int64_t ldr;
    int activation;
    void* z;                    // in T or, if `wide`, in float; null: not wanted; ld is `kept_ld`, a multiple of 8
    uint8_t* codes;             // null: not wanted; likewise
    int64_t kept_ld;
    float* partial;             // not null: split results, [split][m][n padded to 4], for linear_join_kernel

    // `left` of its elements are there from n on
    __device__ __forceinline__ f32x4 bias_at(int64_t n, int left) const {
        if (!bias) return f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        return wide ? load4(static_cast<const float*>(bias) + n, bias_vectors, left) : load4(static_cast<const T*>(bias) + n, bias_vectors, left);
    }
    // kCount groups of four neighbours, kStep apart: z -> what is kept, and y
    template <bool kWhole, int kCount, int kStep>
    __device__ __forceinline__ void finish(int64_t m, int64_t n, int left, const float (&in)[4 * kCount], const f32x4 (&add)[kCount]) const {
        using T4 = T __attribute__((ext_vector_type(4)));
        float value[4 * kCount];
        if (kKeeps && codes) {
            float slope[4 * kCount];
            uint32_t words[kCount];
            activate<sizeof(T) == 4, true>(activation, in, value, slope);
            slope_words(slope, words);
            uint8_t* to = codes + m * kept_ld + n;
#pragma unroll
            for (int j = 0; j < kCount; ++j)
                if (kWhole || left > kStep * j) *reinterpret_cast<uint32_t*>(to + kStep * j) = words[j];
        } else {
            activate_only<sizeof(T) == 4>(activation, in, value);
        }
        if (kKeeps && z && wide) {
            float* to = static_cast<float*>(z) + m * kept_ld + n;
#pragma unroll
            for (int j = 0; j < kCount; ++j)
                if (kWhole || left > kStep * j) *reinterpret_cast<f32x4*>(to + kStep * j) = f32x4{in[4 * j], in[4 * j + 1], in[4 * j + 2], in[4 * j + 3]};
        } else if (kKeeps && z) {
            T* to = static_cast<T*>(z) + m * kept_ld + n;
#pragma unroll
            for (int j = 0; j < kCount; ++j)
                if (kWhole || left > kStep * j)
                    *reinterpret_cast<T4*>(to + kStep * j) = T4{from_float<T>(in[4 * j]), from_float<T>(in[4 * j + 1]), from_float<T>(in[4 * j + 2]), from_float<T>(in[4 * j + 3])};
        }
        T* to = y + m * ldy + n;
#pragma unroll
        for (int j = 0; j < kCount; ++j) {
            if (!kWhole && left <= kStep * j) break;
            T4 out;
#pragma unroll
            for (int r = 0; r < 4; ++r) out[r] = from_float<T>(value[4 * j + r] + add[j][r]);
            if (kWhole || (vectors && left - kStep * j >= 4)) {
                *reinterpret_cast<T4*>(to + kStep * j) = out;
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (kStep * j + r < left) to[kStep * j + r] = out[r];
            }
        }
    }

    // The results of a tile; kWhole: all of it is inside, and lies in whole vectors.
    template <bool kWhole, typename Shape, typename E>
    __device__ __forceinline__ void rows(const f32x4 (&acc)[Shape::kFragsN][Shape::kFragsM], const ProductArgs<E>& args, const TileIndex& tile, int64_t m, int64_t n) const {
        constexpr int kEach = Shape::kFragsN;
        const int all = columns_left(args.n, n);
        f32x4 b[kEach], add[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) b[j] = bias_at(n + 16 * j, kWhole ? 4 : all - 16 * j);
        auto ask = [&](int i) {
            const int left = columns_left(args.n, n);
            const T* from = residual + (m + 16 * i) * ldr + n;
            const bool wanted = kWhole || m + 16 * i < args.m;
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                add[j] = wanted && (kWhole || left > 16 * j) ? load4(from + 16 * j, kWhole || residual_vectors, kWhole ? 4 : left - 16 * j) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        };
#pragma unroll
        for (int j = 0; j < kEach; ++j) add[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (residual) ask(0);
#pragma unroll
        for (int i = 0; i < Shape::kFragsM; ++i) {
            float in[4 * kEach];
            f32x4 now[kEach];
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                now[j] = add[j];
#pragma unroll
                for (int r = 0; r < 4; ++r) in[4 * j + r] = acc[j][i][r] + b[j][r];
            }
            if (residual && i + 1 < Shape::kFragsM) ask(i + 1);
            if (kWhole || m + 16 * i < args.m) finish<kWhole, kEach, 16>(m + 16 * i, n, columns_left(args.n, n), in, now);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    template <typename Shape, typename E>
    __device__ __forceinline__ void store(const f32x4 (&acc)[Shape::kFragsN][Shape::kFragsM], const ProductArgs<E>& args, const TileIndex& tile) const {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int64_t m = tile.m * Shape::kM + wave / Shape::kWavesN * Shape::kFragsM * 16 + lane % 16;
        const int64_t n = tile.n * Shape::kColumns + wave % Shape::kWavesN * Shape::kFragsN * 16 + lane / 16 * 4;
        if (partial) {
            const int64_t padded = (args.n + 3) / 4 * 4;
#pragma unroll
            for (int i = 0; i < Shape::kFragsM; ++i) {
                if (m + 16 * i >= args.m) break;
                float* to = partial + ((int64_t)tile.split * args.m + m + 16 * i) * padded + n;
                const int left = columns_left(args.n, n);
#pragma unroll
                for (int j = 0; j < Shape::kFragsN; ++j)
                    if (left > 16 * j) *reinterpret_cast<f32x4*>(to + 16 * j) = acc[j][i];
            }
        } else if ((tile.m + 1) * Shape::kM <= args.m && (tile.n + 1) * Shape::kColumns <= args.n && vectors && (!residual || residual_vectors)) {
            rows<true, Shape>(acc, args, tile, m, n);
        } else {
            rows<false, Shape>(acc, args, tile, m, n);
        }
    }
};

// The sum of the splits, in order, and the epilogue.
template <typename T, bool kKeeps>
__global__ __launch_bounds__(256) void linear_join_kernel(int64_t m, int64_t n, int splits, LinearOut<T, kKeeps> out) {
    const int64_t quads = (n + 3) / 4, count = m * quads, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < count; i += step) {
        const int64_t row = i / quads, col = (i - row * quads) * 4;
        const int left = (int)(n - col);
        f32x4 sum = out.bias_at(col, left);
        const f32x4 add = out.residual ? load4(out.residual + row * out.ldr + col, out.residual_vectors, left) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < splits; s += kJoinAhead) {
            f32x4 ahead[kJoinAhead];
#pragma unroll
            for (int j = 0; j < kJoinAhead; ++j)
                ahead[j] = s + j < splits ? *reinterpret_cast<const f32x4*>(out.partial + 4 * ((s + j) * count + i)) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < kJoinAhead; ++j) sum += ahead[j];
        }
        const float in[4] = {sum[0], sum[1], sum[2], sum[3]};
        const f32x4 adds[1] = {add};
        out.template finish<false, 1, 16>(row, col, left, in, adds);
    }
}

// ---------------------------------------------------------------- the backward pass

template <typename T>
struct LinearSlopeArgs {
    int64_t rows, columns;
    int lanes;                  // of a row, a power of two up to 256
    const T* dy;
    int64_t lddy;
    const void* z;              // one of these two, or none: the slope is 1
    bool wide;                  // z in float
    const uint8_t* codes;
    int64_t kept_ld;
    int activation;
    T* dz;                      // null: not wanted; ld is `kept_ld`, and what is beyond the columns is 0
    float* partial;             // [workgroup's slice of the rows][columns]: sums of dz before it is rounded; null: not wanted
};

// dz = dy act'(z), and the workgroup's sums of it over its rows.  A lane keeps eight columns and walks down the rows; workgroups stand side by
// side where a row is longer than 2048 columns.
template <typename T>
__global__ __launch_bounds__(256) void linear_slope_kernel(LinearSlopeArgs<T> a) {
    __shared__ float sums[256 * kChunk];
    const int teams = 256 / a.lanes, lane = threadIdx.x & (a.lanes - 1), team = threadIdx.x / a.lanes;
    const int64_t col = ((int64_t)blockIdx.x * a.lanes + lane) * kChunk, here = a.columns - col;
    float db[kChunk];
#pragma unroll
    for (int j = 0; j < kChunk; ++j) db[j] = 0.0f;
    if (here > 0)
        for (int64_t row = (int64_t)blockIdx.y * teams + team; row < a.rows; row += (int64_t)gridDim.y * teams) {
            float d[kChunk], slope[kChunk];
            widen(load_chunk(a.dy + row * a.lddy + col, here), d);
            if (a.codes) {
                const uint2 codes = *reinterpret_cast<const uint2*>(a.codes + row * a.kept_ld + col);
#pragma unroll
                for (int j = 0; j < kChunk; ++j) slope[j] = slope_of(codes, j);
            } else if (a.z) {
                float z[kChunk], value[kChunk];
                if (a.wide) {
                    widen(load_chunk(static_cast<const float*>(a.z) + row * a.kept_ld + col, kChunk), z);
                } else {
                    widen(load_chunk(static_cast<const T*>(a.z) + row * a.kept_ld + col, kChunk), z);
                }
#pragma unroll
                for (int j = 0; j < kChunk; ++j) z[j] = a.wide ? inside_range<float>(z[j]) : inside_range<T>(z[j]);
                activate<sizeof(T) == 4>(a.activation, z, value, slope);
            } else {
#pragma unroll
                for (int j = 0; j < kChunk; ++j) slope[j] = 1.0f;
            }
#pragma unroll
            for (int j = 0; j < kChunk; ++j) {
                d[j] = j < here ? d[j] * slope[j] : 0.0f;
                db[j] += d[j];
            }
            if (a.dz) store_chunk(a.dz + row * a.kept_ld + col, kChunk, d);
        }
    if (!a.partial) return;
#pragma unroll
    for (int j = 0; j < kChunk; ++j) sums[threadIdx.x * kChunk + j] = db[j];
    __syncthreads();
    for (int c = threadIdx.x; c < a.lanes * kChunk; c += 256) {
        float v = 0.0f;
        for (int t = 0; t < teams; ++t) v += sums[t * a.lanes * kChunk + c];
        const int64_t column = (int64_t)blockIdx.x * a.lanes * kChunk + c;
        if (column < a.columns) a.partial[blockIdx.y * a.columns + column] = v;
    }
}

}  // namespace dgsp
