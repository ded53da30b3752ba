// C(m, n) = sum over k of A(m, k) B(n, k) for rows in e4m3 with a scale for every 32 columns (rows8.hpp): the matrix instructions take the
// scales with the elements, 128 columns at a time.
//
// What bounds it: the matrix instructions, at the clock that the card holds under them; reading the fragments from LDS takes as long.  8192 x 8192 x 8192
// 455 us, 2.4 PFLOP/s, 8192 x 4096 x 16384 530 to 560 us by the card's power, 2.0 to 2.1 (a library's: 2.7 and 2.5); of a few rows the weights' way from memory.
//
// As in matrix_tiles.hpp, whose loaders move a stage of 128 bytes a row: here 128 columns, with four scales a row, which go to LDS beside it.
// Lane l of a fragment has row l % 16, of the 16-byte chunks of its stage those numbered l / 16 and l / 16 + 4, exchanged by the row as the loader
// leaves them, and the scale of block l / 16, which belongs to chunks 2 (l / 16) and 2 (l / 16) + 1: the instruction hands it to the lanes
// that have those.
//
// Sums: the instruction adds the products of eight neighbouring columns aligned to the largest of them and cuts off what lies 2^-13 below its power of two (it does so
// in its form without scales as well); sums of these are held in 32 bits.  That is a 500th of what rounding the elements to e4m3
// costs, and the only way to the rate of 8 bits: widened to 16 bits the operands would take the instructions that are half as fast.
#pragma once

#include "matrix_tiles.hpp"
#include "rows8.hpp"

namespace dgsp {

using i32x8 = int __attribute__((ext_vector_type(8)));

using Pair8 = uint16_t;                 // what the loaders count in: two elements

struct Scales8 {
    const uint8_t *a, *b;
    int64_t rows_a, rows_b;             // from a group of four blocks to the next
    int64_t groups;
};

// c += a b in place, written out for the same reasons as accumulate(); the wait is for operands and scales that vector instructions wrote.
__device__ __forceinline__ void accumulate8(i32x8 a, i32x8 b, f32x4& c, int scale_a, int scale_b) {
    asm volatile("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]"
                 : "+v"(c)
                 : "v"(a), "v"(b), "v"(scale_a), "v"(scale_b));
}

template <typename Shape>
struct Tile8Product {
    static constexpr int kStageBytes = 128;                             // of a row
    static constexpr int kABytes = Shape::kM * kStageBytes, kBBytes = Shape::kN * kStageBytes;
    static constexpr int kAScales = Shape::kM * 4, kBScales = Shape::kN * 4;
    static constexpr int kStage = kABytes + kBBytes + kAScales + kBScales;
    using ALoader = Loader<Shape::kM, true, Shape::kWaves>;
    using BLoader = Loader<Shape::kN, true, Shape::kWaves>;
    f32x4 acc[Shape::kFragsN][Shape::kFragsM];

    __device__ __forceinline__ void run(const ProductArgs<Pair8>& args, const Scales8& scales, const TileIndex& tile) {
        constexpr uint32_t kRing = Shape::kBuffers * kStage;
        __shared__ __attribute__((aligned(1024))) char lds[kRing];
        const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wave_m = wave / Shape::kWavesN, wave_n = wave % Shape::kWavesN;
        const int64_t k_first = tile.split * args.split_depth, k_end = min(args.depth, k_first + args.split_depth);
        const int64_t i0 = tile.m * Shape::kM, j0 = tile.n * Shape::kN;
#pragma unroll
        for (int j = 0; j < Shape::kFragsN; ++j)
#pragma unroll
            for (int i = 0; i < Shape::kFragsM; ++i) acc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        const int total = k_end > k_first ? (int)((k_end - k_first + kDepth - 1) / kDepth) : 0;
        if (total == 0) return;

        ALoader a_loader;
        BLoader b_loader;
        constexpr int kARowsEach = ALoader::kInstructions * ALoader::kRowsEach, kBRowsEach = BLoader::kInstructions * BLoader::kRowsEach;
        a_loader.init(lane, wave * kARowsEach, args.a[0].ld);
        b_loader.init(lane, wave * kBRowsEach, args.b[0].ld);
        const uint32_t a_lds = lds_at + wave * ALoader::kInstructions * kWaveBytes, b_lds = lds_at + kABytes + wave * BLoader::kInstructions * kWaveBytes;
        auto a_from = ALoader::begin(args.a[0], i0, k_first, wave * kARowsEach);
        auto b_from = BLoader::begin(args.b[0], j0, k_first, wave * kBRowsEach);

        // the first half of the waves brings A's scales, the second B's, 64 rows each; where there are more waves than that, some the same
        constexpr int kHalf = Shape::kWaves / 2;
        const bool of_a = wave < kHalf;
        const int part = of_a ? wave % (Shape::kM / 64) : (wave - kHalf) % (Shape::kN / 64);
        const int64_t scale_rows = of_a ? scales.rows_a : scales.rows_b, scale_row = (of_a ? i0 : j0) + 64 * part;
        int64_t group = k_first / kDepth;
        const char* const scales_from = reinterpret_cast<const char*>(of_a ? scales.a : scales.b);
        const uint32_t scales_lds = lds_at + kABytes + kBBytes + (of_a ? 0 : kAScales) + part * 256;

        typename ALoader::Stage a_stage;
        typename BLoader::Stage b_stage;
        u32x4 scales_stage;
        uint32_t into = 0;
        auto begin_load = [&](uint32_t buffer) {
            a_stage = a_loader.stage(a_from, args.a[0].ld);
            b_stage = b_loader.stage(b_from, args.b[0].ld);
            const int64_t at = (group * scale_rows + scale_row) * 4, left = scales.groups * scale_rows * 4 - at;
            const uint64_t address = reinterpret_cast<uint64_t>(scales_from + at);
            scales_stage = {(uint32_t)address, (uint32_t)(address >> 32) & 0xffffu, left > 256 ? 256u : left > 0 ? (uint32_t)left : 0u, 0x00020000u};
            ++group;
            into = buffer;
        };
        auto load_piece = [&](int i) {
            if (i < ALoader::kInstructions)
                a_loader.issue(i, a_stage, a_lds + into);
            else if (i < ALoader::kInstructions + BLoader::kInstructions)
                b_loader.issue(i - ALoader::kInstructions, b_stage, b_lds + into);
            else if (i == ALoader::kInstructions + BLoader::kInstructions)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(scales_lds + into), "v"(lane * 4), "s"(scales_stage)
                             : "memory", "m0");
        };
        constexpr int kOfAStage = ALoader::kInstructions + BLoader::kInstructions + 1;
        auto arrive = [&](int later) {
            if (later <= 0)
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            else if (Shape::kBuffers == 2 || later == 1)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kOfAStage) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * kOfAStage) : "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        // Where a fragment's chunks and scale stand in a stage; those of further fragments are constants away.
        struct Places {
            uint32_t low, high, scale;
            __device__ __forceinline__ Places in(uint32_t buffer) const {
                Places p = {low + buffer, high + buffer, scale + buffer};
                asm volatile("" : "+v"(p.low), "+v"(p.high), "+v"(p.scale));        // one addition a stage, not one a fragment
                return p;
            }
        };
        const int row = lane % 16, a_first = wave_m * Shape::kFragsM * 16 + row, b_first = wave_n * Shape::kFragsN * 16 + row;
        const uint32_t in_row = (lane / 16 ^ (row & 7)) * 16;
        const Places of_a_stage = {lds_at + a_first * kStageBytes + in_row, lds_at + a_first * kStageBytes + (in_row ^ 64), lds_at + kABytes + kBBytes + a_first * 4 + lane / 16};
        const Places of_b_stage = {lds_at + kABytes + b_first * kStageBytes + in_row, lds_at + kABytes + b_first * kStageBytes + (in_row ^ 64),
                                   lds_at + kABytes + kBBytes + kAScales + b_first * 4 + lane / 16};
        struct Fragment {
            i32x8 elements;
            int scale;
        };
        auto fragment = [&](const Places& at, int i) {
            using Quads = const __attribute__((address_space(3))) u32x4*;
            using Byte = const __attribute__((address_space(3))) uint8_t*;
            const u32x4 low = *(Quads)(uintptr_t)(at.low + i * 16 * kStageBytes), high = *(Quads)(uintptr_t)(at.high + i * 16 * kStageBytes);
            return Fragment{i32x8{(int)low[0], (int)low[1], (int)low[2], (int)low[3], (int)high[0], (int)high[1], (int)high[2], (int)high[3]},
                            *(Byte)(uintptr_t)(at.scale + i * 64)};
        };
        // Fragments of B stay for a stage and have a second place for the next one's; the two change roles from stage to stage (moving them
        // instead took a fifth more time).  Those of A come kAhead rows before they are multiplied; when
        // the last ones of a stage are there all waves meet, and from then on fragments are read of the next stage, which has arrived, while
        // the last rows are multiplied, and the buffer takes the stage after that.
        constexpr int kAhead = 2, kRows = Shape::kFragsM, kPieces = (kOfAStage + kAhead - 1) / kAhead;
        static_assert(kRows % kAhead == 0);
        using Columns = Fragment[Shape::kFragsN];
        Fragment a[kAhead];
        Columns b_even, b_odd;
        auto multiply_row = [&](int i, const Columns& b) {
#pragma unroll
            for (int j = 0; j < Shape::kFragsN; ++j)
                accumulate8(b[j].elements, a[i % kAhead].elements, acc[j][i], b[j].scale, a[i % kAhead].scale);
        };
        auto first_rows = [&](const Places& at, const Columns& b) {
#pragma unroll
            for (int i = 0; i < kRows - kAhead; ++i) {
                multiply_row(i, b);
                a[i % kAhead] = fragment(at, i + kAhead);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        for (int i = 0; i < min(total, Shape::kBuffers); ++i) {
            begin_load(i * kStage);
#pragma unroll
            for (int piece = 0; piece < kOfAStage; ++piece) load_piece(piece);
        }
        arrive(min(total, Shape::kBuffers) - 1);
        uint32_t here = 0;
        int step = 0;
        const auto a_first_at = of_a_stage.in(0), b_first_at = of_b_stage.in(0);
#pragma unroll
        for (int j = 0; j < Shape::kFragsN; ++j) b_even[j] = fragment(b_first_at, j);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) a[i] = fragment(a_first_at, i);
        first_rows(a_first_at, b_even);
        auto advance = [&](const Columns& b, Columns& b_next) {
            const uint32_t next = here + kStage == kRing ? 0 : here + kStage;
            arrive(min(total - 2 - step, Shape::kBuffers - 2));
            const bool more = step + Shape::kBuffers < total;
            if (more) begin_load(here);
            const Places a_at = of_a_stage.in(next), b_at = of_b_stage.in(next);
#pragma unroll
            for (int j = 0; j < Shape::kFragsN; ++j) b_next[j] = fragment(b_at, j);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = kRows - kAhead; i < kRows; ++i) {
                multiply_row(i, b);
                a[i % kAhead] = fragment(a_at, i - (kRows - kAhead));
                if (more)
#pragma unroll
                    for (int piece = 0; piece < kPieces; ++piece) load_piece((i - (kRows - kAhead)) * kPieces + piece);
                __builtin_amdgcn_sched_barrier(0);
            }
            here = next;
            ++step;
            first_rows(a_at, b_next);
        };
        // Other instructions may read a result 19 cycles after its matrix instruction has begun; the compiler does not see these, and may move results
        // as soon as the ways meet again.
        auto last_rows = [&](const Columns& b) {
#pragma unroll
            for (int i = kRows - kAhead; i < kRows; ++i) multiply_row(i, b);
            asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
            for (int i = 0; i < Shape::kFragsM; ++i)
#pragma unroll
                for (int j = 0; j < Shape::kFragsN; ++j) asm volatile("" : "+v"(acc[j][i]));
        };
        if (total % 2 == 0) {
            advance(b_even, b_odd);
#pragma unroll
            for (int j = 0; j < Shape::kFragsN; ++j) b_even[j] = b_odd[j];
        }
        while (step + 1 < total) {
            advance(b_even, b_odd);
            advance(b_odd, b_even);
        }
        last_rows(b_even);
    }
};

// A workgroup per tile.
template <typename Shape, typename Out>
__global__ __launch_bounds__(Shape::kThreads, Shape::kWavesASimd) void product_8bit_kernel(ProductArgs<Pair8> args, Scales8 scales, Out out) {
#if defined(__HIP_DEVICE_COMPILE__)
    const TileIndex tile = tile_of(args);
    Tile8Product<Shape> product;
    product.run(args, scales, tile);
    argument_behind<Out, ProductArgs<Pair8>, Scales8>().template store<Shape>(product.acc, args, tile);
#endif
}

}  // namespace dgsp
