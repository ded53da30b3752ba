// y = act(x w^T + bias) + residual for up to 64 rows of x: one token, a small batch, sums that are not too deep.  What bounds it is the weight's
// way from memory, so it passes through no LDS: a fragment of the matrix instructions is 16 rows of the weight and, in each lane, 16 bytes of
// one of them, which a lane reads itself, wherever they lie.  A workgroup has 16 or 32 columns of y and all of the sum, of which its waves
// take pieces in turn, so that nothing is left for another launch; their parts are added in order.  One token, 4096 -> 16384, a new weight a
// call: bfloat16 25 us, 5.3 TB/s, in 8 bits 15.4 us, 4.4 TB/s (tiles of 64: 35 and 18.5).
#pragma once

#include "chunks.hpp"
#include "fragments.hpp"
#include "linear_kernels.hpp"
#include "tiles_8bit.hpp"

namespace dgsp {

constexpr int kFewRows = 64;

// kSets: 16 rows of x each; kOuts: 16 columns of y each; kWaves of a workgroup
template <int kSets, int kOuts, int kWaves>
struct FewSums {
    f32x4 acc[kOuts][kSets];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int o = 0; o < kOuts; ++o)
#pragma unroll
            for (int s = 0; s < kSets; ++s) acc[o][s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // the waves' sums, each fragment's by one of them, and what becomes of it
    template <typename Out>
    __device__ __forceinline__ void finish(int64_t rows, int64_t out_width, int64_t first, const Out& out) const {
        __shared__ f32x4 parts[kWaves][kOuts * kSets][64];
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int o = 0; o < kOuts; ++o)
#pragma unroll
            for (int s = 0; s < kSets; ++s) parts[wave][o * kSets + s][lane] = acc[o][s];
        __syncthreads();
        if (wave >= kOuts * kSets) return;
        static_assert(kOuts * kSets <= kWaves);
        const int64_t m = wave % kSets * 16 + lane % 16, n = first + wave / kSets * 16 + lane / 16 * 4;
        if (m >= rows || n >= out_width) return;
        const int left = (int)(out_width - n);
        f32x4 sum = out.bias_at(n, left);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += parts[w][wave][lane];
        const float z[4] = {sum[0], sum[1], sum[2], sum[3]};
        const f32x4 add[1] = {out.residual ? load4(out.residual + m * out.ldr + n, out.residual_vectors, left) : f32x4{0.0f, 0.0f, 0.0f, 0.0f}};
        out.template finish<false, 1, 16>(m, n, left, z, add);
    }
};

template <typename E>
struct FewRowsArgs {
    int64_t rows, width, out_width;
    const E *x, *weight;
    int64_t ldx, ldw;
};

template <typename E, int kSets, int kOuts, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 4) void few_rows_kernel(FewRowsArgs<E> a, LinearOut<E> out) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kAhead = kOuts * kSets > 2 ? 4 : 8;                   // pieces of 32 columns that are asked for together
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t first = (int64_t)blockIdx.x * 16 * kOuts;
    // Rows that are not there are read as the last one: what comes of them is not written.
    const E *w[kOuts], *x[kSets];
#pragma unroll
    for (int o = 0; o < kOuts; ++o) w[o] = a.weight + min(first + 16 * o + lane % 16, a.out_width - 1) * a.ldw + lane / 16 * 8;
#pragma unroll
    for (int s = 0; s < kSets; ++s) x[s] = a.x + min((int64_t)(16 * s + lane % 16), a.rows - 1) * a.ldx + lane / 16 * 8;
    FewSums<kSets, kOuts, kWaves> sums;
    sums.clear();
    constexpr int kPiece = 32 * kAhead;
    int64_t k = (int64_t)wave * kPiece;
    for (; k + kPiece <= a.width; k += kWaves * kPiece) {
        s16x8 of_w[kAhead][kOuts], of_x[kAhead][kSets];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int o = 0; o < kOuts; ++o) of_w[i][o] = __builtin_bit_cast(s16x8, load_chunk(w[o] + k + 32 * i, kChunk).q[0]);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
#pragma unroll
            for (int s = 0; s < kSets; ++s) of_x[i][s] = __builtin_bit_cast(s16x8, load_chunk(x[s] + k + 32 * i, kChunk).q[0]);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int o = 0; o < kOuts; ++o)
#pragma unroll
                for (int s = 0; s < kSets; ++s) sums.acc[o][s] = multiply<E>(of_w[i][o], of_x[i][s], sums.acc[o][s]);
    }
    if (k < a.width)                                                    // one wave's: the end of the rows
        for (; k < a.width; k += 32) {
            const int64_t here = a.width - k - lane / 16 * 8;
            s16x8 of_x[kSets];
#pragma unroll
            for (int s = 0; s < kSets; ++s) of_x[s] = __builtin_bit_cast(s16x8, load_chunk(here > 0 ? x[s] + k : a.x, here > 0 ? here : 0).q[0]);
#pragma unroll
            for (int o = 0; o < kOuts; ++o) {
                const s16x8 of_w = __builtin_bit_cast(s16x8, load_chunk(here > 0 ? w[o] + k : a.weight, here > 0 ? here : 0).q[0]);
#pragma unroll
                for (int s = 0; s < kSets; ++s) sums.acc[o][s] = multiply<E>(of_w, of_x[s], sums.acc[o][s]);
            }
        }
    sums.finish(a.rows, a.out_width, first, out);
#endif
}

// Of rows in 8 bits: a lane has the chunks of 16 columns and the scale that Tile8Product's fragments have.
struct FewRows8Args {
    int64_t rows, width, out_width;     // width: filled up to whole blocks
    const uint8_t *x, *weight;
    int64_t ldx, ldw;
    Scales8 scales;                     // a: of x
};

template <typename T, int kSets, int kOuts, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 4) void few_rows_8bit_kernel(FewRows8Args a, LinearOut<T, false> out) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kAhead = kOuts * kSets > 2 ? 1 : kSets * kOuts > 1 ? 2 : 4;      // stages of 128 columns that are asked for together
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), chunk = lane / 16;
    const int64_t first = (int64_t)blockIdx.x * 16 * kOuts, stages = (a.width + 127) / 128;
    int64_t w_row[kOuts], x_row[kSets];
#pragma unroll
    for (int o = 0; o < kOuts; ++o) w_row[o] = min(first + 16 * o + lane % 16, a.out_width - 1);
#pragma unroll
    for (int s = 0; s < kSets; ++s) x_row[s] = min((int64_t)(16 * s + lane % 16), a.rows - 1);
    struct Fragment {
        i32x8 elements;
        int scale;
    };
    // chunks beyond the row are 0, as the loaders of tiles read them
    auto fragment = [&](const uint8_t* values, int64_t ld, const uint8_t* scales, int64_t rows, int64_t row, int64_t stage) {
        const uint8_t* from = values + row * ld + stage * 128;
        const int64_t here = (a.width - stage * 128) / 16;
        u32x4 low = {0u, 0u, 0u, 0u}, high = low;
        if (chunk < here) low = *reinterpret_cast<const u32x4*>(from + chunk * 16);
        if (chunk + 4 < here) high = *reinterpret_cast<const u32x4*>(from + chunk * 16 + 64);
        return Fragment{i32x8{(int)low[0], (int)low[1], (int)low[2], (int)low[3], (int)high[0], (int)high[1], (int)high[2], (int)high[3]},
                        scales[(stage * rows + row) * 4 + chunk]};
    };
    FewSums<kSets, kOuts, kWaves> sums;
    sums.clear();
    for (int64_t stage = wave * kAhead; stage < stages; stage += kWaves * kAhead) {
        Fragment of_w[kAhead][kOuts], of_x[kAhead][kSets];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t at = min(stage + i, stages - 1);              // stages behind the last are read as it, and left out
#pragma unroll
            for (int o = 0; o < kOuts; ++o) of_w[i][o] = fragment(a.weight, a.ldw, a.scales.b, a.scales.rows_b, w_row[o], at);
#pragma unroll
            for (int s = 0; s < kSets; ++s) of_x[i][s] = fragment(a.x, a.ldx, a.scales.a, a.scales.rows_a, x_row[s], at);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (stage + i < stages)
#pragma unroll
                for (int o = 0; o < kOuts; ++o)
#pragma unroll
                    for (int s = 0; s < kSets; ++s)
                        sums.acc[o][s] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(of_w[i][o].elements, of_x[i][s].elements, sums.acc[o][s], 0, 0, 0,
                                                                                          of_w[i][o].scale, 0, of_x[i][s].scale);
    }
    sums.finish(a.rows, a.out_width, first, out);
#endif
}

// Where one launch without splits of the sum is faster than tiles, which split it and read a row of the weight once for 64 rows of x.  Against it are
// deep sums of few columns, which few workgroups add up, the deeper the more rows there are; from some rows on weights that are long in coming; and short
// sums of so many columns that its workgroups, each of which waits once for all it reads, take turns.  bfloat16, us, this and tiles, a new weight a call:
//     1 row     4096 -> 16384 22 and 25    4096 -> 1024 7.3 and 7.9     8192 -> 4096 15 and 16       8192 -> 256 11.3 and 7.7     256 -> 16384 4.8 and 5.8     256 -> 65536 13 and 12     1024 -> 65536 30 and 34
//     16 rows   4096 -> 16384 31 and 26    4096 -> 4096 10.4 and 12.6   8192 -> 2048 17 and 13       2048 -> 256 5.9 and 7.1      512 -> 20000 9.9 and 8.7    128 -> 65536 15 and 9
//     24 rows   2048 -> 512 7.1 and 7.2    2048 -> 4096 8.3 and 10.8    4096 -> 512 12 and 8.6       256 -> 20000 6.1 and 6.9     256 -> 32768 9.7 and 7.5
//     32 rows   1024 -> 16384 14 and 15    2048 -> 4096 9.2 and 11.4    2048 -> 512 7.7 and 7.2      2048 -> 2048 8.8 and 9.0     512 -> 16384 7.7 and 8.2
//     48 rows   512 -> 16384 8.8 and 8.4   256 -> 16384 6.3 and 6.5     1024 -> 8192 8.6 and 12.9    256 -> 24576 10.4 and 7.4
//     64 rows   512 -> 16384 9.7 and 8.1   1024 -> 8192 9.3 and 14.0    1024 -> 1024 7.2 and 7.6     2048 -> 512 11.4 and 7.5     512 -> 10240 9.3 and 7.8
// In 8 bits the same holds of widths twice as large: 1 row 8192 -> 1024 7.6 and 8.1, 16384 -> 512 12 and 9; 64 rows 2048 -> 2048 8.0 and 8.5, 4096 -> 1024 13.5 and 8.6.
// Of 970 sizes measured the choice costs more than 7 % in 21, the most 4 rows in 8 bits 2048 -> 32768 (22 and 17) and 4 rows 512 -> 16384 (7.5 and 6.2).
inline bool few_rows(int64_t rows, int64_t width, int64_t out_width, int64_t element_bytes) {
    const int64_t depth = width * element_bytes, weight = depth * out_width;
    if (rows <= 16)
        return (out_width <= 16384 || depth >= 2048) && (out_width >= 4096 || depth * (rows <= 4 ? 1 : 2) < 16384) && (rows <= 8 || weight < (64 << 20));
    if (rows <= 32) return out_width <= 24576 && depth <= 4096 && weight <= (32 << 20) && (rows * depth <= 24 * 4096 || out_width >= 2048);
    return rows <= kFewRows && depth <= 2048 && weight <= (16 << 20) && (out_width <= 8192 || (out_width <= 16384 && rows * depth <= 48 * 512));
}

// launch(sets, outs, waves): how the rows and columns are cut.  Columns beyond 8192 fill the GPU by workgroups of 8 waves; fewer take 16 (one token, bfloat16,
// 16384 -> 4096: 36 and 31 us with 8 and 16; 4096 -> 16384: 25 and 30).  In 8 bits more than 4 rows pay for 32 columns a workgroup, which read x half as
// often (8 rows 4096 -> 16384: 18.9 and 17.0 us with 16 and 32; bfloat16 30.0 and 33.3), and so do more than 16 rows of both (40 rows 512 -> 8192 6.8 and
// 5.9; where they leave CUs without work they do not: 37 rows 1000 -> 2731 float16 6.3 and 7.7).
template <typename F>
void with_few_rows(int64_t rows, int64_t out_width, bool in_8bit, F&& launch) {
    std::integral_constant<int, 1> one;
    std::integral_constant<int, 2> two;
    std::integral_constant<int, 4> four;
    std::integral_constant<int, 8> eight;
    std::integral_constant<int, 16> sixteen;
    if (rows > 32 && out_width < 8192)
        launch(four, one, eight);
    else if (rows > 32)
        launch(four, two, eight);
    else if (rows > 16 && out_width < 8192)
        launch(two, one, eight);
    else if (rows > 16)
        launch(two, two, eight);
    else if (in_8bit && rows > 4 && out_width >= 8192)
        launch(one, two, eight);
    else if (out_width >= 8192)
        launch(one, one, eight);
    else
        launch(one, one, sixteen);
}

}  // namespace dgsp
