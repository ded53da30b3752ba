// C(m, n) = sum over k of A(m, k) B(n, k) for rows in e4m3 with a scale for every 32 columns (rows8.hpp): the matrix instructions take the
// scales with the elements, 128 columns at a time.
//
// As in matrix_tiles.hpp, whose loaders move a stage of 128 bytes a row: here 128 columns, with four scales a row, which go to LDS beside it.
// Lane l of a fragment has row l % 16, of the 16-byte chunks of its stage those numbered l / 16 and l / 16 + 4, exchanged by the row as the loader
// leaves them, and the scale of block l / 16, which belongs to chunks 2 (l / 16) and 2 (l / 16) + 1: the instruction hands it to the lanes
// that have those.
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

#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ f32x4 multiply8(i32x8 a, i32x8 b, f32x4 c, int scale_a, int scale_b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, scale_a, 0, scale_b);
}
#endif

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
        auto a_at = ALoader::begin(args.a[0], i0, k_first, wave * kARowsEach);
        auto b_at = BLoader::begin(args.b[0], j0, k_first, wave * kBRowsEach);

        // the first half of the waves brings A's scales, the second B's, 64 rows each; where there are more waves than that, some the same
        constexpr int kHalf = Shape::kWaves / 2;
        const bool of_a = wave < kHalf;
        const int part = of_a ? wave % (Shape::kM / 64) : (wave - kHalf) % (Shape::kN / 64);
        const int64_t scale_rows = of_a ? scales.rows_a : scales.rows_b, scale_row = (of_a ? i0 : j0) + 64 * part;
        int64_t group = k_first / kDepth;
        const char* const scales_from = reinterpret_cast<const char*>(of_a ? scales.a : scales.b);
        const uint32_t scales_lds = lds_at + kABytes + kBBytes + (of_a ? 0 : kAScales) + part * 256;

        auto load = [&](uint32_t buffer) {
            a_loader.issue(a_at, args.a[0].ld, a_lds + buffer);
            b_loader.issue(b_at, args.b[0].ld, b_lds + buffer);
            const int64_t at = (group * scale_rows + scale_row) * 4, left = scales.groups * scale_rows * 4 - at;
            const uint64_t address = reinterpret_cast<uint64_t>(scales_from + at);
            const u32x4 resource = {(uint32_t)address, (uint32_t)(address >> 32) & 0xffffu, left > 256 ? 256u : left > 0 ? (uint32_t)left : 0u, 0x00020000u};
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(scales_lds + buffer), "v"(lane * 4), "s"(resource)
                         : "memory", "m0");
            ++group;
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
        // of a fragment's row, block lane / 16
        const int row = lane % 16, a_first = wave_m * Shape::kFragsM * 16 + row, b_first = wave_n * Shape::kFragsN * 16 + row;
        const int in_row = ((lane / 16) ^ (row & 7)) * 16;
        auto fragment = [&](const char* from) {
            const u32x4 low = *reinterpret_cast<const u32x4*>(from + in_row), high = *reinterpret_cast<const u32x4*>(from + (in_row ^ 64));
            return i32x8{(int)low[0], (int)low[1], (int)low[2], (int)low[3], (int)high[0], (int)high[1], (int)high[2], (int)high[3]};
        };
        for (int i = 0; i < min(total, Shape::kBuffers); ++i) load(i * kStage);
        uint32_t here = 0;
        for (int step = 0; step < total; ++step) {
            arrive(min(total - 1 - step, Shape::kBuffers - 1));
            const char* const stage = lds + here;
            const uint8_t* const stage_scales = reinterpret_cast<const uint8_t*>(stage + kABytes + kBBytes) + lane / 16;
            i32x8 b[Shape::kFragsN];
            int b_scale[Shape::kFragsN];
#pragma unroll
            for (int j = 0; j < Shape::kFragsN; ++j) {
                b[j] = fragment(stage + kABytes + (b_first + 16 * j) * kStageBytes);
                b_scale[j] = stage_scales[kAScales + (b_first + 16 * j) * 4];
            }
#pragma unroll
            for (int i = 0; i < Shape::kFragsM; ++i) {
                const i32x8 a = fragment(stage + (a_first + 16 * i) * kStageBytes);
                const int a_scale = stage_scales[(a_first + 16 * i) * 4];
#pragma unroll
                for (int j = 0; j < Shape::kFragsN; ++j) acc[j][i] = multiply8(b[j], a, acc[j][i], b_scale[j], a_scale);
            }
            // all waves have read the stage
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (step + Shape::kBuffers < total) load(here);
            here = here + kStage == kRing ? 0 : here + kStage;
        }
    }
};

// A workgroup per tile.
template <typename Shape, typename Out>
__global__ __launch_bounds__(Shape::kThreads, Shape::kWavesASimd) void product_8bit_kernel(ProductArgs<Pair8> args, Scales8 scales, Out out) {
#if defined(__HIP_DEVICE_COMPILE__)
    const TileIndex tile = tile_of(args);
    Tile8Product<Shape> product;
    product.run(args, scales, tile);
    store_tile<Shape>(product.acc, args, tile, argument_behind<Out, ProductArgs<Pair8>, Scales8>());
#endif
}

}  // namespace dgsp
