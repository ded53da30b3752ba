// Layer norm and its gradient.  A team of lanes holds a row in registers, a chunk of eight elements a lane: 1 to 64 lanes of a wave,
// several rows side by side, or a whole workgroup.  The row is read once; the mean comes first and the squares are of what is left
// after it, both from the registers (the difference of two sums of squares would lose what a large mean hides).  Teams go on to further
// rows, whose elements are asked for a row ahead.  With two and four chunks a lane the parameters and their sums no longer fit the
// registers of a full CU.  Memory bounds it (a large copy: 4.96 TB/s):
//     float, 2^20 rows of 32:               forward 54 us, 5.0 TB/s; gradient 80 us, 5.0 TB/s, and 4 us for the parameters' sums
//     bfloat16, 8192 rows of 8192:          forward 70 us, 3.8 TB/s; gradient 77 us, 5.2 TB/s, and 5 us: two barriers a row, 16 waves
//     bfloat16, 32768 rows of 1024, residual and dropout:  forward 53 us, 5.1 TB/s; gradient 85 us, 4.7 TB/s (with ds and dx)
#pragma once

#include "chunks.hpp"
#include "lanes.hpp"

namespace dgsp {

constexpr int kMostWaves = 16;

// How a workgroup holds rows.
template <bool kWhole>
struct Team {
    int lanes;              // of a team
    int lane;               // in the team
    int64_t row, step;      // first row of the team, rows to the next one
    __device__ __forceinline__ explicit Team(int lanes_) : lanes(lanes_) {
        if constexpr (kWhole) {
            lane = threadIdx.x;
            row = blockIdx.x;
            step = gridDim.x;
        } else {
            const int teams = blockDim.x / lanes;
            lane = threadIdx.x & (lanes - 1);
            row = (int64_t)blockIdx.x * teams + threadIdx.x / lanes;
            step = (int64_t)gridDim.x * teams;
        }
    }
    // Sums of kValues numbers over the team.  `turn` alternates, so that one barrier a sum is enough for a workgroup.
    template <typename V, int kValues>
    __device__ __forceinline__ void sum(V (&v)[kValues], int& turn) const {
        if constexpr (kWhole) {
            __shared__ V part[2][kValues][kMostWaves];
#pragma unroll
            for (int i = 0; i < kValues; ++i) v[i] = lanes_sum(v[i], 64);
            const int waves = blockDim.x >> 6;
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int i = 0; i < kValues; ++i) part[turn][i][threadIdx.x >> 6] = v[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kValues; ++i) {             // a wave's sum a lane, in every 16 lanes: read one by one they took a third of the time
                const int w = threadIdx.x % kMostWaves;
                v[i] = lanes_sum(w < waves ? part[turn][i][w] : V(0), kMostWaves);
            }
            turn ^= 1;
        } else {
#pragma unroll
            for (int i = 0; i < kValues; ++i) v[i] = lanes_sum(v[i], lanes);
        }
    }
};

template <typename T>
struct NormArgs {
    int64_t rows, width;
    int lanes;
    const T *x, *residual;
    int64_t ldx, ldr;
    DropMask mask;
    const void *weight, *bias;
    bool wide;              // parameters in float
    float eps;
    T *y, *sum;
    int64_t ldy, lds;
    float* stats;
};

template <typename T, bool kWhole, bool kAdd>
__global__ __launch_bounds__(kWhole ? 1024 : 256) void layer_norm_kernel(NormArgs<T> a) {
    const Team<kWhole> team(a.lanes);
    const uint64_t offset = kAdd && a.mask.device_offset ? *a.mask.device_offset : a.mask.offset;
    const int64_t col = (int64_t)team.lane * kChunk, here = a.width - col;
    float w[kChunk], b[kChunk];
    RawChunk<T> x, r;
    auto ask = [&](int64_t row) {
        if (row >= a.rows || here <= 0) return;
        x = load_chunk(a.x + row * a.ldx + col, here);
        if constexpr (kAdd) r = load_chunk(a.residual + row * a.ldr + col, here);
    };
    ask(team.row);
    if (here > 0) {
        load_params<T>(a.weight, a.wide, col, here, 1.0f, w);
        load_params<T>(a.bias, a.wide, col, here, 0.0f, b);
    }
    const float part = 1.0f / (float)a.width;
    int turn = 0;
    // all teams of a workgroup make the same number of turns
    const int64_t base = team.row - (kWhole ? 0 : threadIdx.x / team.lanes);
    for (int64_t at = base, row = team.row; at < a.rows; at += team.step, row += team.step) {
        const bool inside = row < a.rows && here > 0;
        float s[kChunk], total[1] = {0.0f};
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
        for (int j = 0; j < kChunk; ++j) total[0] += s[j];
        team.sum(total, turn);
        const float mean = total[0] * part;
        float squares[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            const float d = j < here ? s[j] - mean : 0.0f;
            squares[0] += d * d;
        }
        team.sum(squares, turn);
        const float rstd = 1.0f / sqrtf(squares[0] * part + a.eps);
        if (!inside) continue;
        float out[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) out[j] = (s[j] - mean) * rstd * w[j] + b[j];
        store_chunk(a.y + row * a.ldy + col, here, out);
        if constexpr (kAdd) store_chunk(a.sum + row * a.lds + col, here, s);
        if (a.stats && team.lane == 0) {
            a.stats[2 * row] = mean;
            a.stats[2 * row + 1] = rstd;
        }
    }
}

template <typename T>
struct NormBackwardArgs {
    int64_t rows, width;
    int lanes;
    const T *s, *residual, *dy, *ds;        // with a residual `s` is x
    int64_t lds, ldr, lddy, ldds;
    const float* stats;
    const void* weight;
    bool wide;
    DropMask mask;
    T *dsum, *dx;
    float* partial;         // [workgroup][dweight, dbias][width]; null: not wanted
};

// Where s is given as the residual and x it is made again: rounded to 16 bits it would add as much to the error of dweight as the rounding
// of the result does.  A third more is read (bfloat16, 32768 rows of 1024: 85 us against 61).
//
// A lane adds up dy hat and dy of its columns over the rows it meets; a workgroup's lanes with the same columns meet in LDS, and the
// workgroups' sums in memory, in the order of the workgroups (layer_norm_params_kernel).
template <typename T, bool kWhole, bool kAdd>
__global__ __launch_bounds__(kWhole ? 1024 : 256) void layer_norm_backward_kernel(NormBackwardArgs<T> a) {
    const Team<kWhole> team(a.lanes);
    const uint64_t offset = kAdd && a.mask.device_offset ? *a.mask.device_offset : a.mask.offset;
    const int64_t col = (int64_t)team.lane * kChunk, here = a.width - col;
    float w[kChunk], dw[kChunk], db[kChunk];
    RawChunk<T> s, r, g, more;
    float next_mean = 0.0f, next_rstd = 0.0f;
    auto ask = [&](int64_t row) {
        if (row >= a.rows || here <= 0) return;
        s = load_chunk(a.s + row * a.lds + col, here);
        g = load_chunk(a.dy + row * a.lddy + col, here);
        if constexpr (kAdd) {
            if (a.residual) r = load_chunk(a.residual + row * a.ldr + col, here);
            if (a.ds) more = load_chunk(a.ds + row * a.ldds + col, here);
        }
        next_mean = a.stats[2 * row];
        next_rstd = a.stats[2 * row + 1];
    };
    ask(team.row);
    if (here > 0) load_params<T>(a.weight, a.wide, col, here, 1.0f, w);
#pragma unroll
    for (int j = 0; j < kChunk; ++j) dw[j] = db[j] = 0.0f;
    const float part = 1.0f / (float)a.width;
    int turn = 0;
    const int64_t base = team.row - (kWhole ? 0 : threadIdx.x / team.lanes);
    for (int64_t at = base, row = team.row; at < a.rows; at += team.step, row += team.step) {
        const float mean = next_mean, rstd = next_rstd;
        const bool inside = row < a.rows && here > 0;
        float hat[kChunk], dhat[kChunk], add[kChunk], sums[2] = {0.0f, 0.0f};
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
                hat[j] = j < here ? (hat[j] - mean) * rstd : 0.0f;
                dw[j] += d[j] * hat[j];
                db[j] += d[j];
                dhat[j] = j < here ? d[j] * w[j] : 0.0f;
                sums[0] += dhat[j];
                sums[1] += dhat[j] * hat[j];
            }
        }
        ask(row + team.step);
        team.sum(sums, turn);
        if (!inside) continue;
        const float p = sums[0] * part, q = sums[1] * part;
        const int64_t to = row * a.width + col;
        float out[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) out[j] = (dhat[j] - p - hat[j] * q) * rstd;
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
    float* to = a.partial + 2 * (int64_t)blockIdx.x * a.width;
    if constexpr (kWhole) {
        if (here <= 0) return;
        store_chunk(to + col, here, dw);
        store_chunk(to + a.width + col, here, db);
    } else {
        // over the teams of a wave by exchanges, over the waves in LDS
        __shared__ float waves_sums[2][4][64 * kChunk];
        const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, columns = team.lanes * kChunk;
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            float v = dw[j], u = db[j];
            for (int d = team.lanes; d < 64; d <<= 1) {
                v += __shfl_xor(v, d, 64);
                u += __shfl_xor(u, d, 64);
            }
            if ((threadIdx.x & 63) < team.lanes) {
                waves_sums[0][wave][team.lane * kChunk + j] = v;
                waves_sums[1][wave][team.lane * kChunk + j] = u;
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * columns; c += blockDim.x) {
            const int kind = c >= columns, column = kind ? c - columns : c;
            float v = 0.0f;
            for (int i = 0; i < waves; ++i) v += waves_sums[kind][i][column];
            if (column < a.width) to[kind * a.width + column] = v;
        }
    }
}

constexpr int kParamColumns = 32, kParamSlices = 32, kParamAhead = 8;
constexpr int64_t kParamGroups = 1 << 20;       // at most: a launch has fewer than 2^32 threads, and drops what is beyond without an error

// dweight and dbias from the workgroups' sums.  Few columns and many sums: what takes time is waiting for memory, so a lane asks for
// eight sums at a time (one at a time: 17 to 38 us where this takes 4 to 8).
template <typename T>
__global__ __launch_bounds__(kParamColumns* kParamSlices) void layer_norm_params_kernel(int64_t width, int64_t groups, const float* partial, void* dweight,
                                                                                         void* dbias, bool wide) {
    __shared__ float part[kParamSlices][kParamColumns];
    const int column = threadIdx.x % kParamColumns, slice = threadIdx.x / kParamColumns;
    for (int64_t first = (int64_t)blockIdx.x * kParamColumns; first < 2 * width; first += (int64_t)gridDim.x * kParamColumns) {
        const int64_t at = first + column;
        float v = 0.0f;
        if (at < 2 * width)
            for (int64_t g = slice; g < groups; g += kParamSlices * kParamAhead) {
                float ahead[kParamAhead];
#pragma unroll
                for (int i = 0; i < kParamAhead; ++i) ahead[i] = g + i * kParamSlices < groups ? partial[(g + i * kParamSlices) * 2 * width + at] : 0.0f;
#pragma unroll
                for (int i = 0; i < kParamAhead; ++i) v += ahead[i];
            }
        part[slice][column] = v;
        __syncthreads();
        if (slice == 0 && at < 2 * width) {
#pragma unroll
            for (int i = 1; i < kParamSlices; ++i) v += part[i][column];
            void* to = at < width ? dweight : dbias;
            if (to) store_param<T>(to, at < width ? at : at - width, wide, v);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- rows beyond what registers hold

// One workgroup a row, which it reads three times.  4096 rows of 16384: forward 84 us in bfloat16, 151 in float, forward and backward pass
// 285 and 469, the rows being small enough for the caches to hold them meanwhile.
template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_long_kernel(NormArgs<T> a) {
    const uint64_t offset = a.mask.device_offset ? *a.mask.device_offset : a.mask.offset;
    const Team<true> team(1024);
    int turn = 0;
    const float part = 1.0f / (float)a.width;
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
        float total[1] = {0.0f}, squares[1] = {0.0f}, v[kChunk];
        for (int64_t c = threadIdx.x; c * kChunk < a.width; c += blockDim.x) {
            at(c, v);
            for (int j = 0; j < kChunk; ++j) total[0] += c * kChunk + j < a.width ? v[j] : 0.0f;
        }
        team.sum(total, turn);
        const float mean = total[0] * part;
        for (int64_t c = threadIdx.x; c * kChunk < a.width; c += blockDim.x) {
            at(c, v);
            for (int j = 0; j < kChunk; ++j) squares[0] += c * kChunk + j < a.width ? (v[j] - mean) * (v[j] - mean) : 0.0f;
        }
        team.sum(squares, turn);
        const float rstd = 1.0f / sqrtf(squares[0] * part + a.eps);
        for (int64_t c = threadIdx.x; c * kChunk < a.width; c += blockDim.x) {
            const int64_t col = c * kChunk, here = a.width - col;
            float w[kChunk], b[kChunk], out[kChunk];
            at(c, v);
            load_params<T>(a.weight, a.wide, col, here, 1.0f, w);
            load_params<T>(a.bias, a.wide, col, here, 0.0f, b);
            for (int j = 0; j < kChunk; ++j) out[j] = (v[j] - mean) * rstd * w[j] + b[j];
            store_chunk(a.y + row * a.ldy + col, here, out);
            if (a.sum) store_chunk(a.sum + row * a.lds + col, here, v);
        }
        if (a.stats && threadIdx.x == 0) {
            a.stats[2 * row] = mean;
            a.stats[2 * row + 1] = rstd;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_backward_long_kernel(NormBackwardArgs<T> a) {
    const uint64_t offset = a.mask.device_offset ? *a.mask.device_offset : a.mask.offset;
    const Team<true> team(1024);
    int turn = 0;
    const float part = 1.0f / (float)a.width;
    for (int64_t row = team.row; row < a.rows; row += team.step) {
        const float mean = a.stats[2 * row], rstd = a.stats[2 * row + 1];
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
                hat[j] = (hat[j] - mean) * rstd;
                dhat[j] *= w[j];
            }
        };
        float sums[2] = {0.0f, 0.0f}, hat[kChunk], dhat[kChunk];
        for (int64_t c = threadIdx.x; c * kChunk < a.width; c += blockDim.x) {
            at(c, hat, dhat);
            for (int j = 0; j < kChunk; ++j)
                if (c * kChunk + j < a.width) {
                    sums[0] += dhat[j];
                    sums[1] += dhat[j] * hat[j];
                }
        }
        team.sum(sums, turn);
        const float p = sums[0] * part, q = sums[1] * part;
        for (int64_t c = threadIdx.x; c * kChunk < a.width; c += blockDim.x) {
            const int64_t col = c * kChunk, here = a.width - col, to = row * a.width + col;
            float out[kChunk];
            at(c, hat, dhat);
            for (int j = 0; j < kChunk; ++j) out[j] = (dhat[j] - p - hat[j] * q) * rstd;
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

// partial sums of dy hat and dy over the rows of a slice
template <typename T>
__global__ __launch_bounds__(256) void layer_norm_long_params_kernel(NormBackwardArgs<T> a) {
    const int64_t col = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (col >= a.width) return;
    const uint64_t offset = a.mask.device_offset ? *a.mask.device_offset : a.mask.offset;
    float dw = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float d = to_float(a.dy[row * a.lddy + col]);
        float s = to_float(a.s[row * a.lds + col]);
        if (a.residual) {
            if (a.mask.dropped) s = keep_bits(a.mask, offset, (uint32_t)row, (uint32_t)(col / kChunk)) >> (col % kChunk) & 1 ? s * a.mask.scale : 0.0f;
            s += to_float(a.residual[row * a.ldr + col]);
        }
        dw += d * ((s - a.stats[2 * row]) * a.stats[2 * row + 1]);
        db += d;
    }
    a.partial[2 * (int64_t)blockIdx.y * a.width + col] = dw;
    a.partial[(2 * (int64_t)blockIdx.y + 1) * a.width + col] = db;
}

}  // namespace dgsp
