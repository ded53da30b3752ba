// C(m, n) = sum over k of A(m, k) B(n, k) for float matrices.
//
// A float is the sum of three bf16 numbers, 8 bits of the significand in each, and a product of two the sum of six products of these that
// are larger than 2^-24 of it: six matrix instructions in place of one, of which each is sixteen times as fast as that of float
// (2.5 PFLOP/s against 0.157).  A stage is 32 deep, 64 of small tiles, which wait for memory rather than multiply.  It comes from memory into registers while the stage before is multiplied, is split
// there and goes to LDS as three planes, each laid out as in matrix_tiles.hpp; a wave reads a plane's fragments once for all products that
// they are in.  One buffer in LDS: what a workgroup waits for its two barriers a stage, the CU's other workgroup multiplies.
//
// Six products of 32-bit sums: an error of the sum as of float's own instructions.  An infinity or NaN in an operand gives NaN or an
// infinity in the results that it belongs to, which of the two is not said.
#pragma once

#include "chunks.hpp"
#include "matrix_tiles.hpp"

namespace dgsp {

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

// A stage of one operand: kRows elements along m or n, kStage along k.
template <int kRows, int kStage, bool kAlongK, int kThreads>
struct FloatLoader {
    static constexpr int kChunks = kAlongK ? kStage / 8 : kRows / 8;            // of 8 elements in a row of a plane
    static constexpr int kEach = kRows * kStage / 8 / kThreads;                 // chunks a thread
    static constexpr int kPlane = kRows * kStage * 2;                           // bytes
    RawChunk<float> kept[kEach];

    // with what the number of a row's chunk along k is exchanged
    static __device__ __forceinline__ int turn(int row) { return kStage == 64 ? row & 7 : row >> 1 & 3; }
    static __device__ __forceinline__ int exchange(int k) { return ((k & 3) + 4 * ((k >> 3) & 3)) & (kRows / 16 - 1); }

    // `row0` and the rest as of the half of a dual tile that these rows are of
    __device__ __forceinline__ void ask(int e, const Source<float>& s, int64_t i0, int64_t k0, int first_row) {
        const int c = threadIdx.x + e * kThreads, row = c / kChunks - (kAlongK ? first_row : 0), chunk = c % kChunks;
        const int64_t at = (kAlongK ? i0 : k0) + row, col = (kAlongK ? k0 : i0) + chunk * 8;
        const bool inside = at < s.rows && col < s.cols;
        kept[e] = load_chunk(s.p + (inside ? at * s.ld + col : 0), inside ? s.cols - col : 0);
    }
    // which row of the tile chunk `e` of this thread is of
    static __device__ __forceinline__ int row_of(int e) { return (threadIdx.x + e * kThreads) / kChunks; }

    __device__ __forceinline__ void leave(char* lds) const {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int c = threadIdx.x + e * kThreads, row = c / kChunks, chunk = c % kChunks;
            const int to = kAlongK ? chunk ^ turn(row) : (((chunk >> 1) ^ exchange(row)) << 1) + (chunk & 1);
            using E8 = bf16_t __attribute__((ext_vector_type(8)));
            E8 out[3];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                bf16_t parts[3];
                split3(kept[e].at(j), parts);
                for (int q = 0; q < 3; ++q) out[q][j] = parts[q];
            }
#pragma unroll
            for (int q = 0; q < 3; ++q) *reinterpret_cast<E8*>(lds + q * kPlane + row * kChunks * 16 + to * 16) = out[q];
        }
    }
};

// As Reader, of a plane of a stage.
template <int kRows, int kStage, bool kAlongK>
struct FloatReader {
    uint32_t at;
    __device__ __forceinline__ void init(int lane, int first) {
        using Loader = FloatLoader<kRows, kStage, kAlongK, 256>;
        if constexpr (kAlongK) {
            at = (uint32_t)((first + lane % 16) * (kStage * 2) + (lane / 16 ^ Loader::turn(lane % 16)) * 16);
        } else {
            const int k = lane / 16 * 8 + lane % 16 / 4;
            at = (uint32_t)(k * kRows * 2 + ((first / 16 ^ Loader::exchange(k)) * 32) + (lane & 3) * 8);
        }
    }
    template <typename Lds>
    __device__ __forceinline__ s16x8 read(Lds* lds, int s, int i) const {
        if constexpr (kAlongK) {
            return *reinterpret_cast<const s16x8*>(lds + (at ^ (s * 64)) + i * 16 * kStage * 2);
        } else {
            using P = __attribute__((address_space(3))) s16x4*;
            auto* p = lds + (at ^ (i * 32)) + s * 32 * kRows * 2;
            const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)p);
            const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + 4 * kRows * 2));
            return __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

template <typename Shape, bool kARows, bool kBRows, typename Out>
__global__ __launch_bounds__(Shape::kThreads, 2) void float_tile_kernel(ProductArgs<float> args, Out out) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kStage = Shape::kM == 64 ? 64 : 32;
    using ALoader = FloatLoader<Shape::kM, kStage, kARows, Shape::kThreads>;
    using BLoader = FloatLoader<Shape::kN, kStage, kBRows, Shape::kThreads>;
    __shared__ __attribute__((aligned(16))) char lds[3 * (ALoader::kPlane + BLoader::kPlane)];
    char *const a_lds = lds, *const b_lds = lds + 3 * ALoader::kPlane;
    const TileIndex tile = tile_of(args);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_m = wave / Shape::kWavesN, wave_n = wave % Shape::kWavesN;
    const int64_t k_first = tile.split * args.split_depth, k_end = min(args.depth, k_first + args.split_depth);
    const int64_t i0 = tile.m * Shape::kM, j0 = tile.n * Shape::kColumns;
    constexpr int kEachN = Shape::kDual ? Shape::kFragsN / 2 : Shape::kFragsN;

    ALoader a_loader;
    BLoader b_loader;
    FloatReader<Shape::kM, kStage, kARows> a_reader;
    FloatReader<Shape::kN, kStage, kBRows> b_reader;
    a_reader.init(lane, wave_m * Shape::kFragsM * 16);
    b_reader.init(lane, wave_n * kEachN * 16);
    f32x4 acc[Shape::kFragsN][Shape::kFragsM];
#pragma unroll
    for (int j = 0; j < Shape::kFragsN; ++j)
#pragma unroll
        for (int i = 0; i < Shape::kFragsM; ++i) acc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    auto ask = [&](int pair, int64_t k) {
        const Source<float>& a = args.a[args.batch > 1 ? tile.batch : pair];
#pragma unroll
        for (int e = 0; e < ALoader::kEach; ++e) a_loader.ask(e, a, i0, k, 0);
#pragma unroll
        for (int e = 0; e < BLoader::kEach; ++e) {
            // the first half of a dual tile's rows is of b[0], the second of b[1]
            const int half = Shape::kDual && BLoader::row_of(e) >= Shape::kN / 2;
            b_loader.ask(e, args.b[Shape::kDual ? half : pair], j0, k, half * (Shape::kN / 2));
        }
    };
    int pair = 0;
    int64_t k = k_first;
    bool more = k < k_end;
    if (more) ask(pair, k);
    while (more) {
        __syncthreads();                                        // the last stage has been read
        a_loader.leave(a_lds);
        b_loader.leave(b_lds);
        __syncthreads();
        k += kStage;
        if (k >= k_end) {
            k = k_first;
            ++pair;
        }
        more = pair < args.pairs;
        if (more) ask(pair, k);
#pragma unroll
        for (int s = 0; s < kStage / 32; ++s) {
            s16x8 b[3][Shape::kFragsN];
#pragma unroll
            for (int j = 0; j < Shape::kFragsN; ++j)
#pragma unroll
                for (int q = 0; q < 3; ++q)                      // the second half's rows lie kN / 2 rows on
                    b[q][j] = b_reader.read(b_lds + q * BLoader::kPlane + j / kEachN * (BLoader::kPlane / 2), s, j % kEachN);
#pragma unroll
            for (int i = 0; i < Shape::kFragsM; ++i) {
                s16x8 a[3];
#pragma unroll
                for (int q = 0; q < 3; ++q) a[q] = a_reader.read(a_lds + q * ALoader::kPlane, s, i);
                // the smallest first
                constexpr int kA[6] = {1, 0, 2, 0, 1, 0}, kB[6] = {1, 2, 0, 1, 0, 0};
#pragma unroll
                for (int p = 0; p < 6; ++p)
#pragma unroll
                    for (int j = 0; j < Shape::kFragsN; ++j) acc[j][i] = multiply<bf16_t>(b[kB[p]][j], a[kA[p]], acc[j][i]);
            }
        }
    }
    store_tile<Shape>(acc, args, tile, out);
#endif
}

}  // namespace dgsp
