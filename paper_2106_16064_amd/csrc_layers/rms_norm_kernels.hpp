// Root-mean-square norm and its gradient, held as layer_norm_kernels.hpp holds rows: a team of lanes, a chunk of eight elements a lane, read
// once; one sum a row.  Forms: with the residual's addition, with dropout in front of it, and with a result in 8 bits (rows8.hpp), whose
// blocks are four neighbouring lanes of the team.  Memory bounds it (a large copy: 4.93 TB/s):
//     float, 2^20 rows of 32:        forward 52 us, 5.2 TB/s; gradient 77 us, 5.2 TB/s, and 5 us for the weight's sums
//     bfloat16, 8192 rows of 8192, with the residual:  forward 91 us, 5.9 TB/s; gradient 140 us, 4.8 TB/s (x, residual, dy, ds read)
//     bfloat16, 8192 rows of 4096, with the residual, into 8 bits:  41 us where a cache has the rows, 52 to 69 from memory, 3.4 to 4.5 TB/s
//     bfloat16, 4096 rows of 16384, read again:  forward 65 us, with the residual into 8 bits 163 us; gradient 220 us, with the residual 350
#pragma once

#include "layer_norm_kernels.hpp"
#include "rows8.hpp"

namespace dgsp {

template <typename T>
struct RmsArgs {
    int64_t rows, width;
    int lanes;
    const T *x, *residual;
    int64_t ldx, ldr;
    DropMask mask;
    const void* weight;
    bool wide;              // the weight in float
    float eps;
    T *y, *sum;
    int64_t ldy, lds;
    float* rstd;
    Rows8 rows8;            // in place of y
};

constexpr ScaleRange kE4m3Range{1, 246};

// The squares of a row held in registers, their sum and the root are made in 64 bits: the squares of numbers from 2^64 on, and of those below 2^-75, have no place in
// 32.  Memory bounds the kernels either way (2^20 rows of 32 floats 41.5 us both, 8192 rows of 8192 bfloat16 44 in 32 bits and 45.5; with a second sum only where
// the one in 32 bits says that it is needed 43 and 45).

// What the products of s, the root and the weight are made in.  Before a rounding to 8 bits 64 bits: an error of y is a hundred times as likely as its own size to
// carry an element across a border between two steps (of 4099 x 1001 in 32 bits two or three; rounded from 64 to 32 in between, one).
template <bool k8bit>
using Wide = std::conditional_t<k8bit, double, float>;

// A number on its way to 8 bits: what 32 bits cannot hold of it leaves a 1 in the last place, so that the second rounding is that of the whole.
__device__ __forceinline__ float narrowed(float v) { return v; }
__device__ __forceinline__ float narrowed(double v) {
    constexpr uint32_t kRest = (1u << 29) - 1;
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    const uint32_t low = (uint32_t)bits, odd = (((low & kRest) + kRest) | low) & ~kRest;
    return (float)__builtin_bit_cast(double, (bits & ~0xffffffffull) | odd);
}

// 1 / sqrt(mean + eps); `part`: 1 / width.  By the hardware's first guess, good to 2^-24 or better, and a step of Newton's, which squares its error.
__device__ __forceinline__ double reciprocal_root(double squares, double part, float eps) {
    const double mean = squares * part + eps, guess = __builtin_amdgcn_rsq(mean), better = guess + 0.5 * guess * fma(-mean * guess, guess, 1.0);
    return guess > 0.0 && guess < __builtin_inf() ? better : guess;
}

template <typename T, bool kWhole, bool kAdd, bool k8bit>
__global__ __launch_bounds__(kWhole ? 1024 : 256) void rms_norm_kernel(RmsArgs<T> a) {
    const Team<kWhole> team(a.lanes);
    const uint64_t offset = kAdd && a.mask.device_offset ? *a.mask.device_offset : a.mask.offset;
    const int64_t col = (int64_t)team.lane * kChunk, here = a.width - col;
    float w[kChunk];
    RawChunk<T> x, r;
    auto ask = [&](int64_t row) {
        if (row >= a.rows || here <= 0) return;
        x = load_chunk(a.x + row * a.ldx + col, here);
        if constexpr (kAdd) r = load_chunk(a.residual + row * a.ldr + col, here);
    };
    ask(team.row);
    if (here > 0) load_params<T>(a.weight, a.wide, col, here, 1.0f, w);
    const double part = 1.0 / (double)a.width;
    int turn = 0;
    // all teams of a workgroup make the same number of turns
    const int64_t base = team.row - (kWhole ? 0 : threadIdx.x / team.lanes);
    for (int64_t at = base, row = team.row; at < a.rows; at += team.step, row += team.step) {
        const bool inside = row < a.rows && here > 0;
        float s[kChunk];
        double squares[1] = {0.0};
#pragma unroll
        for (int j = 0; j < kChunk; ++j) s[j] = 0.0f;
        if (inside) {
            widen(x, s);
            if constexpr (kAdd) {
                if (a.mask.dropped) drop(a.mask, offset, row, team.lane, s);
                float add[kChunk];
                widen(r, add);
#pragma unroll
                for (int j = 0; j < kChunk; ++j) s[j] += add[j];
            }
        }
        ask(row + team.step);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) squares[0] += (double)s[j] * (double)s[j];
        team.sum(squares, turn);
        const auto rstd = (Wide<k8bit>)reciprocal_root(squares[0], part, a.eps);
        float out[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) out[j] = inside && j < here ? narrowed(s[j] * rstd * w[j]) : 0.0f;
        if constexpr (k8bit) {                              // all lanes of a block, of which the last may lie behind the row
            uint32_t scale;
            const uint2 bytes = to_8bit<true>(out, kE4m3Range, scale);
            store_8bit(a.rows8, row, team.lane, team.lanes, row < a.rows, bytes, scale);
        }
        if (!inside) continue;
        if constexpr (!k8bit) store_chunk(a.y + row * a.ldy + col, here, out);
        if constexpr (kAdd) store_chunk(a.sum + row * a.lds + col, here, s);
        if (a.rstd && team.lane == 0) a.rstd[row] = (float)rstd;
    }
}

template <typename T>
struct RmsBackwardArgs {
    int64_t rows, width;
    int lanes;
    const T *s, *residual, *dy, *ds;        // with a residual `s` is x
    int64_t lds, ldr, lddy, ldds;
    const float* rstd;
    const void* weight;
    bool wide;
    DropMask mask;
    T *dsum, *dx;
    float* partial;         // [workgroup][width]; null: not wanted
};

// The sum is made again from x and the residual where the one written is rounded, as in layer_norm_backward_kernel.
template <typename T, bool kWhole, bool kAdd>
__global__ __launch_bounds__(kWhole ? 1024 : 256) void rms_norm_backward_kernel(RmsBackwardArgs<T> a) {
    const Team<kWhole> team(a.lanes);
    const uint64_t offset = kAdd && a.mask.device_offset ? *a.mask.device_offset : a.mask.offset;
    const int64_t col = (int64_t)team.lane * kChunk, here = a.width - col;
    float w[kChunk], dw[kChunk];
    RawChunk<T> s, r, g, more;
    float next_rstd = 0.0f;
    auto ask = [&](int64_t row) {
        if (row >= a.rows || here <= 0) return;
        s = load_chunk(a.s + row * a.lds + col, here);
        g = load_chunk(a.dy + row * a.lddy + col, here);
        if constexpr (kAdd) {
            if (a.residual) r = load_chunk(a.residual + row * a.ldr + col, here);
            if (a.ds) more = load_chunk(a.ds + row * a.ldds + col, here);
        }
        next_rstd = a.rstd[row];
    };
    ask(team.row);
    if (here > 0) load_params<T>(a.weight, a.wide, col, here, 1.0f, w);
#pragma unroll
    for (int j = 0; j < kChunk; ++j) dw[j] = 0.0f;
    const float part = 1.0f / (float)a.width;
    int turn = 0;
    const int64_t base = team.row - (kWhole ? 0 : threadIdx.x / team.lanes);
    for (int64_t at = base, row = team.row; at < a.rows; at += team.step, row += team.step) {
        const float rstd = next_rstd;
        const bool inside = row < a.rows && here > 0;
        float hat[kChunk], dhat[kChunk], add[kChunk], sums[1] = {0.0f};
        uint32_t kept = 0;
        if (inside) {
            float d[kChunk];
            widen(s, hat);
            widen(g, d);
            if constexpr (kAdd) {
                if (a.mask.dropped) kept = keep_bits(a.mask, offset, (uint32_t)row, (uint32_t)team.lane);
                if (a.residual) {
                    if (a.mask.dropped) keep(kept, a.mask.scale, hat);
                    widen(r, add);
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) hat[j] += add[j];
                }
                if (a.ds) widen(more, add);
            }
#pragma unroll
            for (int j = 0; j < kChunk; ++j) {
                hat[j] = j < here ? hat[j] * rstd : 0.0f;
                dw[j] += d[j] * hat[j];
                dhat[j] = j < here ? d[j] * w[j] : 0.0f;
                sums[0] += dhat[j] * hat[j];
            }
        }
        ask(row + team.step);
        team.sum(sums, turn);
        if (!inside) continue;
        const float q = sums[0] * part;
        const int64_t to = row * a.width + col;
        float out[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) out[j] = (dhat[j] - hat[j] * q) * rstd;
        if constexpr (kAdd) {
            if (a.ds)
#pragma unroll
                for (int j = 0; j < kChunk; ++j) out[j] += add[j];
        }
        store_chunk(a.dsum + to, here, out);
        if constexpr (kAdd) {
            if (a.dx) {
                if (a.mask.dropped) keep(kept, a.mask.scale, out);
                store_chunk(a.dx + to, here, out);
            }
        }
    }
    if (!a.partial) return;
    float* to = a.partial + (int64_t)blockIdx.x * a.width;
    if constexpr (kWhole) {
        if (here > 0) store_chunk(to + col, here, dw);
    } else {
        // over the teams of a wave by exchanges, over the waves in LDS
        __shared__ float waves_sums[4][64 * kChunk];
        const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, columns = team.lanes * kChunk;
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            float v = dw[j];
            for (int d = team.lanes; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
            if ((threadIdx.x & 63) < team.lanes) waves_sums[wave][team.lane * kChunk + j] = v;
        }
        __syncthreads();
        for (int c = threadIdx.x; c < columns; c += blockDim.x) {
            float v = 0.0f;
            for (int i = 0; i < waves; ++i) v += waves_sums[i][c];
            if (c < a.width) to[c] = v;
        }
    }
}

// ---------------------------------------------------------------- rows beyond what registers hold

// Squares in 32 bits have lost some: at the upper end, or, where eps does not outweigh it, below 2^-90, where steps of 2^-149 for each of up to 2^31 elements
// are no longer small beside the sum.
__device__ __forceinline__ bool beyond_32_bits(float squares, float eps) { return !(squares < __builtin_inff()) || (squares < 0x1p-90f && eps < 0x1p-60f); }

// One workgroup a row, which it reads twice.  Not into 8 bits the squares are held in 32, and made again where that says so (4096 x 16384 bfloat16 65 us;
// held in 64 at all times 69, in 32 alone 63).
template <typename T, bool k8bit>
__global__ __launch_bounds__(1024) void rms_norm_long_kernel(RmsArgs<T> a) {
    const uint64_t offset = a.mask.device_offset ? *a.mask.device_offset : a.mask.offset;
    const Team<true> team(1024);
    int turn = 0;
    const double part = 1.0 / (double)a.width;
    const int64_t chunks = k8bit ? (a.rows8.blocks + 3) / 4 * 4 * kBlockLanes : (a.width + kChunk - 1) / kChunk;
    for (int64_t row = team.row; row < a.rows; row += team.step) {
        auto at = [&](int64_t chunk, float (&v)[kChunk]) {
            const int64_t col = chunk * kChunk, here = a.width - col;
            widen(load_chunk(a.x + row * a.ldx + col, here), v);
            if (!a.residual) return;
            float add[kChunk];
            widen(load_chunk(a.residual + row * a.ldr + col, here), add);
            if (a.mask.dropped) drop(a.mask, offset, row, chunk, v);
            for (int j = 0; j < kChunk; ++j) v[j] += add[j];
        };
        Wide<k8bit> squares[1] = {0};
        float v[kChunk];
        for (int64_t c = threadIdx.x; c * kChunk < a.width; c += blockDim.x) {
            at(c, v);
            for (int j = 0; j < kChunk; ++j) squares[0] += c * kChunk + j < a.width ? (Wide<k8bit>)v[j] * (Wide<k8bit>)v[j] : Wide<k8bit>(0);
        }
        team.sum(squares, turn);
        Wide<k8bit> rstd = (Wide<k8bit>)reciprocal_root(squares[0], part, a.eps);
        if constexpr (!k8bit) {
            if (__builtin_amdgcn_ballot_w64(beyond_32_bits(squares[0], a.eps)) != 0) {          // all waves see the same sum
                double again[1] = {0.0};
                for (int64_t c = threadIdx.x; c * kChunk < a.width; c += blockDim.x) {
                    at(c, v);
                    for (int j = 0; j < kChunk; ++j) again[0] += c * kChunk + j < a.width ? (double)v[j] * (double)v[j] : 0.0;
                }
                team.sum(again, turn);
                rstd = (float)reciprocal_root(again[0], part, a.eps);
            }
        }
        for (int64_t c = threadIdx.x; c < chunks; c += blockDim.x) {
            const int64_t col = c * kChunk, here = a.width - col;
            float w[kChunk], out[kChunk];
            for (int j = 0; j < kChunk; ++j) out[j] = 0.0f;
            if (here > 0) {
                at(c, v);
                load_params<T>(a.weight, a.wide, col, here, 1.0f, w);
                for (int j = 0; j < kChunk; ++j) out[j] = j < here ? narrowed(v[j] * rstd * w[j]) : 0.0f;
            }
            if constexpr (k8bit) {
                uint32_t scale;
                const uint2 bytes = to_8bit<true>(out, kE4m3Range, scale);
                store_8bit(a.rows8, row, c, 64, true, bytes, scale);
            } else {
                store_chunk(a.y + row * a.ldy + col, here, out);
            }
            if (a.sum && here > 0) store_chunk(a.sum + row * a.lds + col, here, v);
        }
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = (float)rstd;
    }
}

template <typename T>
__global__ __launch_bounds__(1024) void rms_norm_backward_long_kernel(RmsBackwardArgs<T> a) {
    const uint64_t offset = a.mask.device_offset ? *a.mask.device_offset : a.mask.offset;
    const Team<true> team(1024);
    int turn = 0;
    const float part = 1.0f / (float)a.width;
    for (int64_t row = team.row; row < a.rows; row += team.step) {
        const float rstd = a.rstd[row];
        auto at = [&](int64_t c, float (&hat)[kChunk], float (&dhat)[kChunk]) {
            const int64_t col = c * kChunk, here = a.width - col;
            float w[kChunk];
            widen(load_chunk(a.s + row * a.lds + col, here), hat);
            if (a.residual) {
                if (a.mask.dropped) drop(a.mask, offset, row, c, hat);
                widen(load_chunk(a.residual + row * a.ldr + col, here), dhat);
                for (int j = 0; j < kChunk; ++j) hat[j] += dhat[j];
            }
            widen(load_chunk(a.dy + row * a.lddy + col, here), dhat);
            load_params<T>(a.weight, a.wide, col, here, 1.0f, w);
            for (int j = 0; j < kChunk; ++j) {
                hat[j] *= rstd;
                dhat[j] *= w[j];
            }
        };
        float sums[1] = {0.0f}, hat[kChunk], dhat[kChunk];
        for (int64_t c = threadIdx.x; c * kChunk < a.width; c += blockDim.x) {
            at(c, hat, dhat);
            for (int j = 0; j < kChunk; ++j)
                if (c * kChunk + j < a.width) sums[0] += dhat[j] * hat[j];
        }
        team.sum(sums, turn);
        const float q = sums[0] * part;
        for (int64_t c = threadIdx.x; c * kChunk < a.width; c += blockDim.x) {
            const int64_t col = c * kChunk, here = a.width - col, to = row * a.width + col;
            float out[kChunk];
            at(c, hat, dhat);
            for (int j = 0; j < kChunk; ++j) out[j] = (dhat[j] - hat[j] * q) * rstd;
            if (a.ds) {
                float add[kChunk];
                widen(load_chunk(a.ds + row * a.ldds + col, here), add);
                for (int j = 0; j < kChunk; ++j) out[j] += add[j];
            }
            store_chunk(a.dsum + to, here, out);
            if (a.dx) {
                if (a.mask.dropped) drop(a.mask, offset, row, c, out);
                store_chunk(a.dx + to, here, out);
            }
        }
    }
}

// partial sums of dy hat over the rows of a slice
template <typename T>
__global__ __launch_bounds__(256) void rms_norm_long_params_kernel(RmsBackwardArgs<T> a) {
    const int64_t col = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (col >= a.width) return;
    const uint64_t offset = a.mask.device_offset ? *a.mask.device_offset : a.mask.offset;
    float dw = 0.0f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        float s = to_float(a.s[row * a.lds + col]);
        if (a.residual) {
            if (a.mask.dropped) s = keep_bits(a.mask, offset, (uint32_t)row, (uint32_t)(col / kChunk)) >> (col % kChunk) & 1 ? s * a.mask.scale : 0.0f;
            s += to_float(a.residual[row * a.ldr + col]);
        }
        dw += to_float(a.dy[row * a.lddy + col]) * (s * a.rstd[row]);
    }
    a.partial[(int64_t)blockIdx.y * a.width + col] = dw;
}

}  // namespace dgsp
