// C(m, n) = sum over k of A(m, k) B(n, k) for float matrices.
//
// A float is the sum of three bf16 numbers, 8 bits of the significand in each, and a product of two the sum of six products of these that
// are larger than 2^-24 of it: six matrix instructions in place of one, of which each is sixteen times as fast as that of float
// (2.5 PFLOP/s against 0.157).  A stage is 32 deep, 64 of small tiles, which wait for memory rather than multiply.  It comes from memory
// into registers while the stage before is multiplied, is split there and goes to LDS as three planes, each laid out as in
// matrix_tiles.hpp; a wave reads a plane's fragments once for all products that they are in.  One buffer in LDS: what a workgroup waits
// for its two barriers a stage, the CU's other workgroup multiplies.
//
// 65536 rows, 128 -> 512 -> 128: the last product of the block 65 us, 132 TFLOP/s of float (a library's: 154), dx 119 us, 144, the weights'
// gradients 138 us (two) and 60 us, 125 and 143; the projections 175 us, 98, and the slopes 155 us, 55, which move 0.44 and 0.57 GB.
// Splitting is a fifth of the instructions; the rest is the six products, and memory at short sums.
//
// Six products of 32-bit sums: an error of the sum as of float's own instructions.  An infinity or NaN in an operand gives NaN or an
// infinity in the results that it belongs to, which of the two is not said.
#pragma once

#include "chunks.hpp"
#include "matrix_tiles.hpp"
#include "rows8.hpp"

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

// Eight of them.  Two at a time, 6 instructions each; where that made an infinity, or met one or a NaN, the last rest is NaN, and they are split one by
// one (with each tested by itself the splitting took twice as long as the products).
__device__ __forceinline__ void split_chunk(const RawChunk<float>& v, u32x4 (&out)[3]) {
    using F2 = float __attribute__((ext_vector_type(2)));
    using E2 = bf16_t __attribute__((ext_vector_type(2)));
    float rests = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float low = v.at(2 * j), high = v.at(2 * j + 1);
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            const uint32_t part = __builtin_bit_cast(uint32_t, __builtin_convertvector((F2{low, high}), E2));
            out[q][j] = part;
            if (q == 2) break;
            low -= __builtin_bit_cast(float, part << 16);
            high -= __builtin_bit_cast(float, part & 0xffff0000u);
        }
        rests += low + high;
    }
    if (__builtin_amdgcn_ballot_w64(rests != rests) == 0) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        bf16_t parts[3];
        split3(v.at(j), parts);
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            const uint32_t part = __builtin_bit_cast(uint16_t, parts[q]);
            out[q][j / 2] = j % 2 ? (out[q][j / 2] & 0xffffu) | part << 16 : part;
        }
    }
}

// A stage of one operand: kRows elements along m or n, kStage along k.  Where all of it is inside the matrix a load is an address of the
// whole stage's plus an offset of the thread's, which stays; else every chunk is looked at.
template <int kRows, int kStage, bool kAlongK, int kThreads>
struct FloatLoader {
    static constexpr int kChunks = kAlongK ? kStage / 8 : kRows / 8;            // of 8 elements in a row of a plane
    static constexpr int kRowsEach = kThreads / kChunks;                        // that the threads take at a time
    static constexpr int kEach = kRows * kStage / 8 / kThreads;                 // chunks a thread
    static constexpr int kPlane = kRows * kStage * 2;                           // bytes
    static constexpr int64_t kMostLd = (1LL << 22) - 8;                         // 128 rows span less than 2^31 bytes
    RawChunk<float> kept[kEach];
    uint32_t offset[kEach];

    // with what the number of a row's chunk along k is exchanged
    static __device__ __forceinline__ int turn(int row) { return kStage == 64 ? row & 7 : row >> 1 & 3; }
    static __device__ __forceinline__ int exchange(int k) { return ((k & 3) + 4 * ((k >> 3) & 3)) & (kRows / 16 - 1); }

    __device__ __forceinline__ void init(int e, int64_t ld, int first_row) {
        const int row = threadIdx.x / kChunks + e * kRowsEach - first_row, chunk = threadIdx.x % kChunks;
        offset[e] = ((uint32_t)row * (uint32_t)ld + chunk * 8) * 4;
    }
    // `count` of the tile's elements along m or n from i0 on, and the stage from k0 on
    static __device__ __forceinline__ bool whole(const Source<float>& s, int64_t i0, int64_t k0, int count) {
        return s.ld <= kMostLd && (kAlongK ? i0 : k0) + (kAlongK ? count : kStage) <= s.rows && (kAlongK ? k0 : i0) + (kAlongK ? kStage : count) <= s.cols;
    }
    static __device__ __forceinline__ const float* begin(const Source<float>& s, int64_t i0, int64_t k0) {
        return s.p + (kAlongK ? i0 * s.ld + k0 : k0 * s.ld + i0);
    }
    __device__ __forceinline__ void ask_whole(int e, const float* from) {
        const auto* p = reinterpret_cast<const ChunkInMemory<float>*>(reinterpret_cast<const char*>(from) + offset[e]);
#pragma unroll
        for (int i = 0; i < RawChunk<float>::kQuads; ++i) kept[e].q[i] = p->q[i];
    }
    __device__ __forceinline__ void ask(int e, const Source<float>& s, int64_t i0, int64_t k0, int first_row) {
        const int row = threadIdx.x / kChunks + e * kRowsEach - first_row, chunk = threadIdx.x % kChunks;
        const int64_t at = (kAlongK ? i0 : k0) + row, col = (kAlongK ? k0 : i0) + chunk * 8;
        const bool inside = at < s.rows && col < s.cols;
        kept[e] = load_chunk(s.p + (inside ? at * s.ld + col : 0), inside ? s.cols - col : 0);
    }

    // the thread's part of the sums over k, of its eight columns
    __device__ __forceinline__ void add(float (&sums)[kChunk]) const {
        static_assert(!kAlongK && kThreads % kChunks == 0);
#pragma unroll
        for (int e = 0; e < kEach; ++e)
#pragma unroll
            for (int j = 0; j < kChunk; ++j) sums[j] += kept[e].at(j);
    }

    // `rows` of an operand along k are there: what comes of others is not stored, and they are left out
    __device__ __forceinline__ void leave(char* lds, int rows) const {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int c = threadIdx.x + e * kThreads, row = c / kChunks, chunk = c % kChunks;
            if (kAlongK && row >= rows) continue;
            const int to = kAlongK ? chunk ^ turn(row) : (((chunk >> 1) ^ exchange(row)) << 1) + (chunk & 1);
            u32x4 out[3];
            split_chunk(kept[e], out);
#pragma unroll
            for (int q = 0; q < 3; ++q) *reinterpret_cast<u32x4*>(lds + q * kPlane + row * kChunks * 16 + to * 16) = out[q];
        }
    }
};

// What a weight's gradient takes besides: its second operand in whole numbers of 8 bits, which with their powers of two are bf16 numbers as they are
// (three products in place of six), and the sums over k of its first operand, which pass through its registers anyway.
// 65536 rows, 128 -> 512: 46 us, and 59 as float, beside 34 of the sums and 12 of reading x back on their own.
template <bool k8bit_>
struct WeightGradient {
    static constexpr bool k8bit = k8bit_;
    Rows8 b;
    float* sums;                // [split][m]; null: not wanted
};

// A stage of an operand in whole numbers, its rows along k.
template <int kRows, int kStage, int kThreads>
struct WholeLoader {
    using Float = FloatLoader<kRows, kStage, false, kThreads>;
    uint2 bytes[Float::kEach];
    uint32_t scale[Float::kEach];
    __device__ __forceinline__ void ask(const Rows8& s, int64_t rows, int64_t i0, int64_t k0) {
#pragma unroll
        for (int e = 0; e < Float::kEach; ++e) {
            const int64_t row = k0 + threadIdx.x / Float::kChunks + e * Float::kRowsEach, block = (i0 + threadIdx.x % Float::kChunks * 8) / kBlock;
            const bool inside = row < rows && block < s.blocks;
            bytes[e] = inside ? *reinterpret_cast<const uint2*>(s.values + row * s.ldv + i0 + threadIdx.x % Float::kChunks * 8) : uint2{0u, 0u};
            scale[e] = inside ? s.scales[((block / 4) * s.lds + row) * 4 + block % 4] : 127u;
        }
    }
    __device__ __forceinline__ void leave(char* lds) const {
#pragma unroll
        for (int e = 0; e < Float::kEach; ++e) {
            const int row = threadIdx.x / Float::kChunks + e * Float::kRowsEach, chunk = threadIdx.x % Float::kChunks;
            float v[kChunk];
            from_8bit<false>(bytes[e], scale[e], v);
            u32x4 out;
#pragma unroll
            for (int j = 0; j < 4; ++j)                         // nothing is in the lower halves
                out[j] = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, v[2 * j + 1]), __builtin_bit_cast(uint32_t, v[2 * j]), 0x07060302u);
            *reinterpret_cast<u32x4*>(lds + row * Float::kChunks * 16 + ((((chunk >> 1) ^ Float::exchange(row)) << 1) + (chunk & 1)) * 16) = out;
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

template <typename Shape, bool kARows, bool kBRows, typename Out, typename More = Nothing>
__global__ __launch_bounds__(Shape::kThreads, 2) void float_tile_kernel(ProductArgs<float> args, Out out, More with) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kStage = Shape::kM == 64 ? 64 : 32;
    constexpr bool kMore = !std::is_same_v<More, Nothing>;
    constexpr bool k8bit = [] {
        if constexpr (kMore) return More::k8bit;
        return false;
    }();
    using ALoader = FloatLoader<Shape::kM, kStage, kARows, Shape::kThreads>;
    using BLoader = FloatLoader<Shape::kN, kStage, kBRows, Shape::kThreads>;
    constexpr int kBPlanes = k8bit ? 1 : 3;
    __shared__ __attribute__((aligned(16))) char lds[3 * ALoader::kPlane + kBPlanes * BLoader::kPlane];
    char *const a_lds = lds, *const b_lds = lds + 3 * ALoader::kPlane;
    const TileIndex tile = tile_of(args);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_m = wave / Shape::kWavesN, wave_n = wave % Shape::kWavesN;
    const int64_t k_first = tile.split * args.split_depth, k_end = min(args.depth, k_first + args.split_depth);
    const int64_t i0 = tile.m * Shape::kM, j0 = tile.n * Shape::kColumns;
    constexpr int kEachN = Shape::kDual ? Shape::kFragsN / 2 : Shape::kFragsN;

    ALoader a_loader;
    BLoader b_loader;
    std::conditional_t<k8bit, WholeLoader<Shape::kN, kStage, Shape::kThreads>, Nothing> whole_loader;
    float sums[kChunk] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    FloatReader<Shape::kM, kStage, kARows> a_reader;
    FloatReader<Shape::kN, kStage, kBRows> b_reader;
    a_reader.init(lane, wave_m * Shape::kFragsM * 16);
    b_reader.init(lane, wave_n * kEachN * 16);
    // small tiles may have few rows, and do nothing for fragments that have none
    constexpr bool kFew = Shape::kM == 64;
    const int rows = kFew ? (int)min(args.m - i0, (int64_t)Shape::kM) : Shape::kM, here_m = rows - wave_m * Shape::kFragsM * 16;
    f32x4 acc[Shape::kFragsN][Shape::kFragsM];
#pragma unroll
    for (int j = 0; j < Shape::kFragsN; ++j)
#pragma unroll
        for (int i = 0; i < Shape::kFragsM; ++i) acc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // the first half of a dual tile's rows is of b[0], the second of b[1]
    constexpr int kSides = Shape::kDual ? 2 : 1, kSideRows = Shape::kN / kSides;
    static_assert(kSideRows % BLoader::kRowsEach == 0 || !Shape::kDual);
    constexpr int kEachSide = Shape::kDual ? kSideRows / BLoader::kRowsEach : BLoader::kEach;
    Source<float> a_now, b_now[kSides];
    int pair = 0;
    int64_t k = k_first;
    auto enter = [&] {
        a_now = args.a[args.batch > 1 ? tile.batch : pair];
#pragma unroll
        for (int e = 0; e < ALoader::kEach; ++e) a_loader.init(e, a_now.ld, 0);
#pragma unroll
        for (int side = 0; side < kSides; ++side) b_now[side] = args.b[Shape::kDual ? side : pair];
        if constexpr (Shape::kDual) b_now[1] = {b_now[1].p, b_now[0].rows, b_now[0].cols, b_now[1].ld};     // of equal extents
#pragma unroll
        for (int e = 0; e < BLoader::kEach; ++e) b_loader.init(e, b_now[e / kEachSide].ld, e / kEachSide * kSideRows);
    };
    auto ask = [&] {
        if (ALoader::whole(a_now, i0, k, Shape::kM)) {
#pragma unroll
            for (int e = 0; e < ALoader::kEach; ++e) a_loader.ask_whole(e, ALoader::begin(a_now, i0, k));
        } else {
#pragma unroll
            for (int e = 0; e < ALoader::kEach; ++e) a_loader.ask(e, a_now, i0, k, 0);
        }
        if constexpr (k8bit) {
            whole_loader.ask(with.b, args.depth, j0, k);
            return;
        }
        bool whole = true;
#pragma unroll
        for (int side = 0; side < kSides; ++side) whole = whole && BLoader::whole(b_now[side], j0, k, kSideRows);
        if (whole) {
#pragma unroll
            for (int e = 0; e < BLoader::kEach; ++e) b_loader.ask_whole(e, BLoader::begin(b_now[e / kEachSide], j0, k));
        } else {
#pragma unroll
            for (int e = 0; e < BLoader::kEach; ++e) b_loader.ask(e, b_now[e / kEachSide], j0, k, e / kEachSide * kSideRows);
        }
    };
    bool more = k < k_end;
    if (more) {
        enter();
        ask();
    }
    while (more) {
        __syncthreads();                                        // the last stage has been read
        a_loader.leave(a_lds, rows);
        if constexpr (k8bit)
            whole_loader.leave(b_lds);
        else
            b_loader.leave(b_lds, Shape::kN);
        if constexpr (kMore)
            if (with.sums && tile.n == 0) a_loader.add(sums);
        __syncthreads();
        k += kStage;
        if (k >= k_end) {
            k = k_first;
            more = ++pair < args.pairs;
            if (more) enter();
        }
        if (more) ask();
#pragma unroll
        for (int s = 0; s < kStage / 32; ++s) {
            if (kFew && here_m <= 0) break;
            s16x8 b[kBPlanes][Shape::kFragsN];
#pragma unroll
            for (int j = 0; j < Shape::kFragsN; ++j)
#pragma unroll
                for (int q = 0; q < kBPlanes; ++q)                      // the second half's rows lie kN / 2 rows on
                    b[q][j] = b_reader.read(b_lds + q * BLoader::kPlane + j / kEachN * (BLoader::kPlane / 2), s, j % kEachN);
#pragma unroll
            for (int i = 0; i < Shape::kFragsM; ++i) {
                if (kFew && i * 16 >= here_m) break;
                s16x8 a[3];
#pragma unroll
                for (int q = 0; q < 3; ++q) a[q] = a_reader.read(a_lds + q * ALoader::kPlane, s, i);
                // the smallest first
                constexpr int kProducts = k8bit ? 3 : 6, kA[6] = {k8bit ? 2 : 1, k8bit ? 1 : 0, k8bit ? 0 : 2, 0, 1, 0}, kB[6] = {k8bit ? 0 : 1, k8bit ? 0 : 2, 0, 1, 0, 0};
#pragma unroll
                for (int p = 0; p < kProducts; ++p)
#pragma unroll
                    for (int j = 0; j < Shape::kFragsN; ++j) acc[j][i] = multiply<bf16_t>(b[kB[p]][j], a[kA[p]], acc[j][i]);
            }
        }
    }
    if constexpr (kMore)
        if (with.sums && tile.n == 0) {
            float(*part)[Shape::kM] = reinterpret_cast<float(*)[Shape::kM]>(lds);
            static_assert(ALoader::kRowsEach * Shape::kM * 4 <= sizeof(lds));
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kChunk; ++j) part[threadIdx.x / ALoader::kChunks][threadIdx.x % ALoader::kChunks * 8 + j] = sums[j];
            __syncthreads();
            if (threadIdx.x < Shape::kM && i0 + threadIdx.x < args.m) {
                float v = 0.0f;
#pragma unroll
                for (int r = 0; r < ALoader::kRowsEach; ++r) v += part[r][threadIdx.x];
                with.sums[(int64_t)tile.split * args.m + i0 + threadIdx.x] = v;
            }
        }
    if constexpr (Out::kReadLate)
        argument_behind<Out, ProductArgs<float>>().template store<Shape>(acc, args, tile);
    else
        store_tile<Shape>(acc, args, tile, out);
#endif
}

}  // namespace dgsp
