// The gated feed-forward block where its weights fit a CU's LDS: the features of many vertices, narrow rows.  What bounds it is reading
// x and writing y, so nothing that is as long as the rows goes to memory in between: g, u and h live in registers, and the backward pass
// makes them again.  h, dg and du are rounded to 16 bits, as the matrix instructions take their operands; sums are held in 32.
// bfloat16, 2^20 rows, 64 -> 128 -> 64: forward 85 us (268 MB, 3.2 TB/s; 52 GFLOP, 0.6 PFLOP/s), gradient 200 us (403 MB; 137 GFLOP, 0.69
// PFLOP/s) and 6 us for the weights' sums: between the two bounds, and the reads of LDS come to as much as the products.  The products of
// matrix_tiles.hpp, one after the other, take 242 and 1010 us; 2^18 rows, 128 -> 128 -> 128: 73 and 385 us against 45 and 174.
//
// The products are arranged so that a result is an operand of the next one where it lies.  A 16 x 16 result of the matrix instructions
// holds, in lane l, rows 4 q ... 4 q + 3 (q = l / 16) of column l % 16; an operand holds eight consecutive k's of its row or column
// l % 16.  With weights as rows and vertices as columns, two results of 16 hidden values each are the eight k's of a lane for a product
// over 32 hidden values, in the order 4 q ... 4 q + 3, 16 + 4 q ... + 3, and the weights are read in the same order.  Only the gradients
// of the weights, which are sums over the vertices, take their operands through LDS.
#pragma once

#include "chunks.hpp"
#include "gated_ff_kernels.hpp"

namespace dgsp {

// kP: width and out_width, kH: hidden, each padded
template <typename E, int kP, int kH, int kWaves>
struct NarrowShape {
    static constexpr int kThreads = 64 * kWaves;
    // rows of LDS are 16 bytes longer than a power of two: neighbouring rows start in different banks
    static constexpr int kLdUp = kP + 8, kLdDown = kH + 8, kLdHidden = 32 + 8;
    static constexpr int kUp = kH * kLdUp, kDown = kP * kLdDown;       // elements of w_gate, of w_up; of w_down
    static constexpr int kRows = 16 * kWaves;                          // of a tile of the backward pass
    static constexpr int kInput = kRows * kLdUp, kHidden = kRows * kLdHidden;
    static constexpr int kForwardLds = (2 * kUp + kDown) * 2, kBackwardLds = kForwardLds + (2 * kInput + 3 * kHidden) * 2;
    static constexpr int kGradients = 3 * kH * kP;                     // of a workgroup's sums: gate, up [kH][kP], down [kP][kH]
};

template <typename E>
struct NarrowArgs {
    int64_t rows, width, hidden, out_width;
    int activation;
    const E *x, *w_gate, *w_up, *w_down, *dy;
    int64_t ldx, ldg, ldu, ldd, lddy;
    E *y, *dx;                  // dx is packed; null: not wanted
    int64_t ldy;
    float* partial;             // [workgroup][kGradients]; null: not wanted
};

using LdsElement = __attribute__((address_space(3))) uint16_t;

__device__ __forceinline__ s16x8 join(s16x4 low, s16x4 high) { return __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7); }

// p: eight, or four, elements of this lane's row
__device__ __forceinline__ s16x8 read8(const uint16_t* p) { return *reinterpret_cast<const s16x8*>(p); }
__device__ __forceinline__ s16x4 read4(const uint16_t* p) { return *reinterpret_cast<const s16x4*>(p); }
// p: where this lane's group of 16 finds four rows of 16 elements; the lane receives the four elements of its column (l % 16)
__device__ __forceinline__ s16x4 read_column(const uint16_t* rows, int ld, int lane) {
    const uint16_t* p = rows + (lane % 16 / 4) * ld + lane % 4 * 4;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
}

template <typename E>
__device__ __forceinline__ s16x4 pack(f32x4 v) {
    using E4 = E __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(s16x4, E4{from_float<E>(v[0]), from_float<E>(v[1]), from_float<E>(v[2]), from_float<E>(v[3])});
}

// rows x cols of a matrix into LDS, zeros up to padded_rows x padded_cols
template <typename E>
__device__ __forceinline__ void stage(uint16_t* lds, int lds_ld, int padded_rows, int padded_cols, const E* from, int64_t ld, int64_t rows, int64_t cols) {
    const int chunks = padded_cols / 8;
    for (int i = threadIdx.x; i < padded_rows * chunks; i += blockDim.x) {
        const int row = i / chunks, col = i % chunks * 8;
        u32x4 v = {0u, 0u, 0u, 0u};
        if (row < rows && col < cols) v = load_chunk(from + row * ld + col, cols - col).q[0];
        *reinterpret_cast<u32x4*>(lds + row * lds_ld + col) = v;
    }
}

// The fragments of 16 rows along the columns: lane l has row l % 16, columns 32 s + 8 (l / 16) ... + 7.  `tile`: first of the wave's rows.
// kFull: all columns are there and in whole 16-byte pieces; reads beyond the last row give 0 by the bounds of the buffer.
template <typename E, int kSteps, bool kFull>
__device__ __forceinline__ void ask_rows(s16x8 (&out)[kSteps], const E* from, int64_t ld, int64_t tile, int64_t rows, int64_t cols, int lane) {
    if constexpr (kFull) {
        const int64_t left = tile < rows ? ((rows - 1 - tile) * ld + cols) * 2 : 0;
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<E*>(from + (tile < rows ? tile * ld : 0)), 0,
                                                                           (int)(left < 0x7fffffff ? left : 0x7fffffff), 0x00020000);
        const int offset = (int)((lane % 16) * ld + 8 * (lane / 16)) * 2;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) out[s] = __builtin_bit_cast(s16x8, __builtin_amdgcn_raw_buffer_load_b128(r, offset + 64 * s, 0, 0));
    } else {
        const int64_t row = tile + lane % 16;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int64_t col = 32 * s + 8 * (lane / 16);
            out[s] = s16x8{};
            if (row < rows && col < cols) out[s] = __builtin_bit_cast(s16x8, load_chunk(from + row * ld + col, cols - col).q[0]);
        }
    }
}

// four neighbours of a row
template <typename E, bool kFull>
__device__ __forceinline__ void store4(E* to, int64_t col, int64_t cols, f32x4 v) {
    using E4 = E __attribute__((ext_vector_type(4), aligned(2)));
    if (kFull || col + 4 <= cols) {
        *reinterpret_cast<E4*>(to + col) = E4{from_float<E>(v[0]), from_float<E>(v[1]), from_float<E>(v[2]), from_float<E>(v[3])};
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (col + r < cols) to[col + r] = from_float<E>(v[r]);
    }
}

// A wave takes 32 rows at a time and needs nothing of the others.
template <typename E, int kP, int kH, int kWaves, bool kFull>
__global__ __launch_bounds__(64 * kWaves) void narrow_forward_kernel(NarrowArgs<E> a) {
#if defined(__HIP_DEVICE_COMPILE__)
    using Shape = NarrowShape<E, kP, kH, kWaves>;
    constexpr int kSteps = kP / 32, kOut = kP / 16;
    __shared__ __attribute__((aligned(16))) uint16_t lds[Shape::kForwardLds / 2];
    uint16_t *gate = lds, *up = lds + Shape::kUp, *down = lds + 2 * Shape::kUp;
    stage(gate, Shape::kLdUp, kH, kP, a.w_gate, a.ldg, a.hidden, a.width);
    stage(up, Shape::kLdUp, kH, kP, a.w_up, a.ldu, a.hidden, a.width);
    stage(down, Shape::kLdDown, kP, kH, a.w_down, a.ldd, a.out_width, a.hidden);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane / 16, own = lane % 16;
    const int64_t step = (int64_t)gridDim.x * kWaves * 32;
    int64_t row0 = ((int64_t)blockIdx.x * kWaves + wave) * 32;
    s16x8 next[2][kSteps];
#pragma unroll
    for (int b = 0; b < 2; ++b) ask_rows<E, kSteps, kFull>(next[b], a.x, a.ldx, row0 + 16 * b, a.rows, a.width, lane);
    __syncthreads();
    for (; row0 < a.rows; row0 += step) {
        s16x8 x[2][kSteps];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int s = 0; s < kSteps; ++s) x[b][s] = next[b][s];
#pragma unroll
        for (int b = 0; b < 2; ++b) ask_rows<E, kSteps, kFull>(next[b], a.x, a.ldx, row0 + step + 16 * b, a.rows, a.width, lane);
        f32x4 y[kOut][2] = {};
#pragma unroll 1
        for (int h0 = 0; h0 < kH; h0 += 32) {
            s16x4 h[2][2];
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const int at = (h0 + 16 * part + own) * Shape::kLdUp + 8 * q;
                f32x4 g[2] = {}, u[2] = {};
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    const s16x8 wg = read8(gate + at + 32 * s), wu = read8(up + at + 32 * s);
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        g[b] = multiply<E>(wg, x[b][s], g[b]);
                        u[b] = multiply<E>(wu, x[b][s], u[b]);
                    }
                }
                float in[8], value[8], slope[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) in[i] = g[i / 4][i % 4];
                activate<false>(a.activation, in, value, slope);
#pragma unroll
                for (int b = 0; b < 2; ++b) h[b][part] = pack<E>(f32x4{value[4 * b], value[4 * b + 1], value[4 * b + 2], value[4 * b + 3]} * u[b]);
            }
#pragma unroll
            for (int o = 0; o < kOut; ++o) {
                const uint16_t* at = down + (16 * o + own) * Shape::kLdDown + h0 + 4 * q;
                const s16x8 wd = join(read4(at), read4(at + 16));
#pragma unroll
                for (int b = 0; b < 2; ++b) y[o][b] = multiply<E>(wd, join(h[b][0], h[b][1]), y[o][b]);
            }
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int64_t row = row0 + 16 * b + own;
            if (row >= a.rows) continue;
#pragma unroll
            for (int o = 0; o < kOut; ++o) store4<E, kFull>(a.y + row * a.ldy, 16 * o + 4 * q, a.out_width, y[o][b]);
        }
    }
#endif
}

// A workgroup takes 16 rows a wave.  For 32 hidden values at a time each wave makes g, u, dh and from them dg, du and h of its rows,
// adds to dx, and leaves dg, du and h in LDS; then each wave adds the rows of all waves to its own blocks of the weights' gradients,
// which stay in registers until the workgroup's last tile.  For up to 256 hidden values: 64 -> 256 -> 64 at 2^18 rows 220 us, some of the
// sums spilled (41 registers, 48 where rows are not in whole pieces; forward and backward pass 262 us, through matrix_tiles.hpp 626, 60 -> 256
// -> 60 288); 32 -> 256 -> 32 92 us.
template <typename E, int kP, int kH, int kWaves, bool kFull>
__global__ __launch_bounds__(64 * kWaves) void narrow_backward_staged_kernel(NarrowArgs<E> a) {
#if defined(__HIP_DEVICE_COMPILE__)
    using Shape = NarrowShape<E, kP, kH, kWaves>;
    constexpr int kSteps = kP / 32, kOut = kP / 16, kParts = kH / 32, kBlocks = 2 * kOut;
    // blocks of 16 x 16 of each gradient that a wave holds per 32 hidden values
    constexpr int kOwn = kBlocks > kWaves ? kBlocks / kWaves : 1;
    __shared__ __attribute__((aligned(16))) uint16_t lds[Shape::kBackwardLds / 2];
    uint16_t *gate = lds, *up = lds + Shape::kUp, *down = lds + 2 * Shape::kUp;
    uint16_t *x_rows = down + Shape::kDown, *dy_rows = x_rows + Shape::kInput;
    uint16_t *dg_rows = dy_rows + Shape::kInput, *du_rows = dg_rows + Shape::kHidden, *h_rows = du_rows + Shape::kHidden;
    stage(gate, Shape::kLdUp, kH, kP, a.w_gate, a.ldg, a.hidden, a.width);
    stage(up, Shape::kLdUp, kH, kP, a.w_up, a.ldu, a.hidden, a.width);
    stage(down, Shape::kLdDown, kP, kH, a.w_down, a.ldd, a.out_width, a.hidden);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane / 16, own = lane % 16;
    const int64_t step = (int64_t)gridDim.x * Shape::kRows;
    f32x4 dw[kParts][3][kOwn] = {};
    s16x8 next_x[kSteps], next_dy[kSteps];
    int64_t first = (int64_t)blockIdx.x * Shape::kRows + 16 * wave;
    ask_rows<E, kSteps, kFull>(next_x, a.x, a.ldx, first, a.rows, a.width, lane);
    ask_rows<E, kSteps, kFull>(next_dy, a.dy, a.lddy, first, a.rows, a.out_width, lane);
    for (int64_t tile = (int64_t)blockIdx.x * Shape::kRows; tile < a.rows; tile += step, first += step) {
        s16x8 x[kSteps], dy[kSteps];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            x[s] = next_x[s];
            dy[s] = next_dy[s];
            const int at = (16 * wave + own) * Shape::kLdUp + 32 * s + 8 * q;
            *reinterpret_cast<s16x8*>(x_rows + at) = x[s];
            *reinterpret_cast<s16x8*>(dy_rows + at) = dy[s];
        }
        ask_rows<E, kSteps, kFull>(next_x, a.x, a.ldx, first + step, a.rows, a.width, lane);
        ask_rows<E, kSteps, kFull>(next_dy, a.dy, a.lddy, first + step, a.rows, a.out_width, lane);
        __syncthreads();                                               // the weights, and these rows, are there
        f32x4 dx[kOut] = {};
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            const int h0 = 32 * p;
            s16x4 dg[2], du[2];
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const int at = (h0 + 16 * part + own) * Shape::kLdUp + 8 * q;
                f32x4 g = {}, u = {}, dh = {};
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    g = multiply<E>(read8(gate + at + 32 * s), x[s], g);
                    u = multiply<E>(read8(up + at + 32 * s), x[s], u);
                    const uint16_t* rows = down + (32 * s + 8 * q) * Shape::kLdDown + h0 + 16 * part;
                    dh = multiply<E>(join(read_column(rows, Shape::kLdDown, lane), read_column(rows + 4 * Shape::kLdDown, Shape::kLdDown, lane)),
                                     dy[s], dh);
                }
                float in[4] = {g[0], g[1], g[2], g[3]}, value[4], slope[4];
                activate<false>(a.activation, in, value, slope);
                f32x4 gs, us, hs;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    gs[r] = dh[r] * u[r] * slope[r];
                    us[r] = dh[r] * value[r];
                    hs[r] = value[r] * u[r];
                }
                dg[part] = pack<E>(gs);
                du[part] = pack<E>(us);
                const int to = (16 * wave + own) * Shape::kLdHidden + 16 * part + 4 * q;
                *reinterpret_cast<s16x4*>(dg_rows + to) = dg[part];
                *reinterpret_cast<s16x4*>(du_rows + to) = du[part];
                *reinterpret_cast<s16x4*>(h_rows + to) = pack<E>(hs);
            }
            if (a.dx) {
#pragma unroll
                for (int d = 0; d < kOut; ++d) {
                    const int at = (h0 + 4 * q) * Shape::kLdUp + 16 * d;
                    dx[d] = multiply<E>(join(read_column(gate + at, Shape::kLdUp, lane), read_column(gate + at + 16 * Shape::kLdUp, Shape::kLdUp, lane)),
                                        join(dg[0], dg[1]), dx[d]);
                    dx[d] = multiply<E>(join(read_column(up + at, Shape::kLdUp, lane), read_column(up + at + 16 * Shape::kLdUp, Shape::kLdUp, lane)),
                                        join(du[0], du[1]), dx[d]);
                }
            }
            __syncthreads();                                           // dg, du and h of all waves are there
            if (a.partial && wave * kOwn < kBlocks) {
                // rows of LDS are the vertices, over which is summed: an operand is columns of them
                auto column = [&](const uint16_t* rows, int ld, int k, int col) {
                    const uint16_t* at = rows + (k + 8 * q) * ld + col;
                    return join(read_column(at, ld, lane), read_column(at + 4 * ld, ld, lane));
                };
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    const int block = wave * kOwn + i, hid = block / kOut * 16, col = block % kOut * 16;
#pragma unroll
                    for (int k = 0; k < Shape::kRows; k += 32) {
                        const s16x8 xs = column(x_rows, Shape::kLdUp, k, col), dys = column(dy_rows, Shape::kLdUp, k, col);
                        dw[p][0][i] = multiply<E>(column(dg_rows, Shape::kLdHidden, k, hid), xs, dw[p][0][i]);
                        dw[p][1][i] = multiply<E>(column(du_rows, Shape::kLdHidden, k, hid), xs, dw[p][1][i]);
                        dw[p][2][i] = multiply<E>(dys, column(h_rows, Shape::kLdHidden, k, hid), dw[p][2][i]);
                    }
                }
            }
            __syncthreads();                                           // and may be written over
        }
        if (a.dx && first + own < a.rows) {
#pragma unroll
            for (int d = 0; d < kOut; ++d) store4<E, kFull>(a.dx + (first + own) * a.width, 16 * d + 4 * q, a.width, dx[d]);
        }
    }
    if (!a.partial || wave * kOwn >= kBlocks) return;
    float* to = a.partial + (int64_t)blockIdx.x * Shape::kGradients;
#pragma unroll
    for (int p = 0; p < kParts; ++p)
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int block = wave * kOwn + i, hid = 32 * p + block / kOut * 16, col = block % kOut * 16;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                to[(hid + 4 * q + r) * kP + col + own] = dw[p][0][i][r];
                to[kH * kP + (hid + 4 * q + r) * kP + col + own] = dw[p][1][i][r];
                to[2 * kH * kP + (col + 4 * q + r) * kH + hid + own] = dw[p][2][i][r];
            }
        }
#endif
}

// The same with the weights in registers, where they and the sums fit: a wave takes 16 hidden values of all rows, so that it reads x and dy
// where the kernel above reads weights, and the three gradients of its weights need nothing of other waves.  Here vertices are the rows of
// g, u and dh, and the results are operands of a sum over the vertices where they lie.  dg and du go to LDS, transposed, for dx, of which
// a wave takes 16 columns, 32 where waves are few.  128 -> 128 -> 128 at 2^18 rows: 174 us, though 157 registers of weights are spilled,
// against 393 us of the kernel above; 64 -> 128 -> 64 at 2^20: 200 against 307.  Where rows are not in whole pieces or widths are between 65
// and 127 the form of 128 x 128 spills 544: forward and backward pass 100 -> 128 -> 100 291 us, 127 -> 128 -> 65 341, 128 -> 128 -> 128 212;
// 60 -> 128 -> 60 at 2^20, which spills none, 321 against 282.
template <typename E, int kP, int kWaves, bool kFull>
__global__ __launch_bounds__(64 * kWaves) void narrow_backward_kernel(NarrowArgs<E> a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kH = 16 * kWaves, kRows = 16 * kWaves, kSteps = kP / 32, kOut = kP / 16, kParts = kH / 32;
    constexpr int kLd = kP + 8, kLdT = kRows + 8;
    constexpr int kShare = kWaves / kOut > 0 ? kWaves / kOut : 1;          // waves that share 16 columns of dx
    constexpr int kTurns = kOut / kWaves > 0 ? kOut / kWaves : 1;          // blocks of 16 columns that a wave takes
    using Shape = NarrowShape<E, kP, kH, kWaves>;
    __shared__ __attribute__((aligned(16))) uint16_t x_rows[kRows * kLd], dy_rows[kRows * kLd], dg_columns[kH * kLdT], du_columns[kH * kLdT];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane / 16, own = lane % 16;
    const int64_t step = (int64_t)gridDim.x * kRows;

    // one element of a matrix, 0 beyond its ends
    auto element = [](const E* w, int64_t ld, int64_t row, int64_t rows, int64_t col, int64_t cols) {
        return row < rows && col < cols ? __builtin_bit_cast(short, w[row * ld + col]) : (short)0;
    };
    // weights: of this wave's hidden values along width and out_width, and of its columns of dx along hidden
    s16x8 gate[kSteps], up[kSteps], down[kSteps], gate_columns[kTurns][kParts], up_columns[kTurns][kParts];
    const int64_t hid = 16 * wave + own;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t k = 32 * s + 8 * q + j;
            gate[s][j] = element(a.w_gate, a.ldg, hid, a.hidden, k, a.width);
            up[s][j] = element(a.w_up, a.ldu, hid, a.hidden, k, a.width);
            down[s][j] = element(a.w_down, a.ldd, k, a.out_width, hid, a.hidden);
        }
#pragma unroll
    for (int c = 0; c < kTurns; ++c)
#pragma unroll
        for (int t = 0; t < kParts; ++t)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t k = 32 * t + 8 * q + j, col = 16 * (wave / kShare + c * kWaves) + own;
                gate_columns[c][t][j] = element(a.w_gate, a.ldg, k, a.hidden, col, a.width);
                up_columns[c][t][j] = element(a.w_up, a.ldu, k, a.hidden, col, a.width);
            }

    f32x4 dw[3][kOut] = {};
    s16x8 next_x[kSteps], next_dy[kSteps];
    int64_t tile = (int64_t)blockIdx.x * kRows;
    auto ask = [&](int64_t at) {
        ask_rows<E, kSteps, kFull>(next_x, a.x, a.ldx, at + 16 * wave, a.rows, a.width, lane);
        ask_rows<E, kSteps, kFull>(next_dy, a.dy, a.lddy, at + 16 * wave, a.rows, a.out_width, lane);
    };
    auto leave = [&] {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int at = (16 * wave + own) * kLd + 32 * s + 8 * q;
            *reinterpret_cast<s16x8*>(x_rows + at) = next_x[s];
            *reinterpret_cast<s16x8*>(dy_rows + at) = next_dy[s];
        }
    };
    ask(tile);
    leave();
    for (; tile < a.rows; tile += step) {
        ask(tile + step);
        __syncthreads();                                                    // x and dy are there, the last tile's dg and du are read
#pragma unroll
        for (int r0 = 0; r0 < kRows; r0 += 32) {
            f32x4 g[2] = {}, u[2] = {}, dh[2] = {};
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    const int at = (r0 + 16 * b + own) * kLd + 32 * s + 8 * q;
                    const s16x8 x = read8(x_rows + at), dy = read8(dy_rows + at);
                    g[b] = multiply<E>(x, gate[s], g[b]);
                    u[b] = multiply<E>(x, up[s], u[b]);
                    dh[b] = multiply<E>(dy, down[s], dh[b]);
                }
            float in[8], value[8], slope[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) in[i] = g[i / 4][i % 4];
            activate<false>(a.activation, in, value, slope);
            s16x4 dg[2], du[2], h[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const f32x4 v = {value[4 * b], value[4 * b + 1], value[4 * b + 2], value[4 * b + 3]};
                const f32x4 m = {slope[4 * b], slope[4 * b + 1], slope[4 * b + 2], slope[4 * b + 3]};
                h[b] = pack<E>(v * u[b]);
                du[b] = pack<E>(dh[b] * v);
                dg[b] = pack<E>(dh[b] * u[b] * m);
                const int at = (16 * wave + own) * kLdT + r0 + 16 * b + 4 * q;
                *reinterpret_cast<s16x4*>(dg_columns + at) = dg[b];
                *reinterpret_cast<s16x4*>(du_columns + at) = du[b];
            }
            // the 32 vertices in the order of the results: 4 q ... 4 q + 3, 16 + 4 q ... + 3
#pragma unroll
            for (int c = 0; c < kOut; ++c) {
                const int at = (r0 + 4 * q) * kLd + 16 * c;
                const s16x8 x = join(read_column(x_rows + at, kLd, lane), read_column(x_rows + at + 16 * kLd, kLd, lane));
                const s16x8 dy = join(read_column(dy_rows + at, kLd, lane), read_column(dy_rows + at + 16 * kLd, kLd, lane));
                dw[0][c] = multiply<E>(join(dg[0], dg[1]), x, dw[0][c]);
                dw[1][c] = multiply<E>(join(du[0], du[1]), x, dw[1][c]);
                dw[2][c] = multiply<E>(dy, join(h[0], h[1]), dw[2][c]);
            }
        }
        __syncthreads();                                                    // dg and du are there, x and dy are read
        leave();
        if (a.dx && wave / kShare < kOut) {
#pragma unroll
            for (int r0 = wave % kShare * 16; r0 < kRows; r0 += kShare * 16) {
                f32x4 dx[kTurns] = {};
#pragma unroll
                for (int t = 0; t < kParts; ++t) {
                    const int at = (32 * t + 8 * q) * kLdT + r0;
                    const s16x8 dg = join(read_column(dg_columns + at, kLdT, lane), read_column(dg_columns + at + 4 * kLdT, kLdT, lane));
                    const s16x8 du = join(read_column(du_columns + at, kLdT, lane), read_column(du_columns + at + 4 * kLdT, kLdT, lane));
#pragma unroll
                    for (int c = 0; c < kTurns; ++c) {
                        dx[c] = multiply<E>(gate_columns[c][t], dg, dx[c]);
                        dx[c] = multiply<E>(up_columns[c][t], du, dx[c]);
                    }
                }
                const int64_t row = tile + r0 + own;
                if (row < a.rows)
#pragma unroll
                    for (int c = 0; c < kTurns; ++c) store4<E, kFull>(a.dx + row * a.width, 16 * (wave / kShare + c * kWaves) + 4 * q, a.width, dx[c]);
            }
        }
    }
    if (!a.partial) return;
    float* to = a.partial + (int64_t)blockIdx.x * Shape::kGradients;
#pragma unroll
    for (int c = 0; c < kOut; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            to[(16 * wave + 4 * q + r) * kP + 16 * c + own] = dw[0][c][r];
            to[kH * kP + (16 * wave + 4 * q + r) * kP + 16 * c + own] = dw[1][c][r];
            to[2 * kH * kP + (16 * c + 4 * q + r) * kH + 16 * wave + own] = dw[2][c][r];
        }
#endif
}

constexpr int kNarrowColumns = 32, kNarrowSlices = 8, kNarrowAhead = 8;

// The weights' gradients from the workgroups' sums, in the order of the workgroups.  256 sums of 24576 numbers, 25 MB: 6 us; eight are
// asked for at a time, as what takes time is waiting for memory.
template <typename E>
__global__ __launch_bounds__(kNarrowColumns* kNarrowSlices) void narrow_join_kernel(int padded, int padded_hidden, int64_t width, int64_t hidden,
                                                                                     int64_t out_width, int groups, const float* partial, E* dw_gate,
                                                                                     E* dw_up, E* dw_down) {
    __shared__ float part[kNarrowSlices][kNarrowColumns];
    const int column = threadIdx.x % kNarrowColumns, slice = threadIdx.x / kNarrowColumns;
    const int one = padded * padded_hidden, count = 3 * one, at = blockIdx.x * kNarrowColumns + column;
    float v = 0.0f;
    for (int g = slice; g < groups; g += kNarrowSlices * kNarrowAhead) {
        float ahead[kNarrowAhead];
#pragma unroll
        for (int i = 0; i < kNarrowAhead; ++i) ahead[i] = g + i * kNarrowSlices < groups ? partial[(int64_t)(g + i * kNarrowSlices) * count + at] : 0.0f;
#pragma unroll
        for (int i = 0; i < kNarrowAhead; ++i) v += ahead[i];
    }
    part[slice][column] = v;
    __syncthreads();
    if (slice) return;
#pragma unroll
    for (int i = 1; i < kNarrowSlices; ++i) v += part[i][column];
    const int which = at / one, in = at % one;
    if (which < 2) {
        const int64_t row = in / padded, col = in % padded;
        E* to = which ? dw_up : dw_gate;
        if (to && row < hidden && col < width) to[row * width + col] = from_float<E>(v);
    } else {
        const int64_t row = in / padded_hidden, col = in % padded_hidden;
        if (dw_down && row < out_width && col < hidden) dw_down[row * hidden + col] = from_float<E>(v);
    }
}

}  // namespace dgsp
