// C(m, n) = sum over k of A(m, k) B(n, k) for matrices of 16-bit elements: tiles of C in registers, tiles of A and B in LDS.
//
// A stage is 64 deep.  Its tiles go from memory to LDS without passing through registers, 1 KB per wave and instruction, into one of
// two buffers while the other one is multiplied; a barrier per stage hands the buffers over.  Each lane chooses which 16 bytes of
// memory its 16 bytes of LDS receive, and the choice spreads what the fragments' reads touch over all banks:
//   rows of k     an operand that is contiguous along k: 128 bytes a row, 16-byte chunk c of row r at chunk c ^ (r % 8).  Fragments are
//                 8 elements a lane, one 16-byte read.
//   rows of m/n   an operand that is contiguous along m or n (transposed): rows of one k, pairs of chunks (16 elements) exchanged by k.
//                 Fragments come from the transposing reads: 16 lanes read 4 k's of 16 elements and receive 4 k's of one element each.
// A product of float matrices takes each as the sum of three bf16 planes, 8 bits of the significand in each, and adds the six products
// of planes that are larger than 2^-24 of the whole, smallest first: six times the matrix instructions, but these are sixteen times as
// fast as those of float (2.5 PFLOP/s to 0.157).
#pragma once

#include "element_types.hpp"

namespace dgsp {

using f32x4 = float __attribute__((ext_vector_type(4)));
using s16x4 = short __attribute__((ext_vector_type(4)));
using s16x8 = short __attribute__((ext_vector_type(8)));

constexpr int kDepth = 64;                  // of a stage
constexpr int kWaveBytes = 1024;            // that one instruction of a wave moves to LDS
constexpr uint32_t kNowhere = 0x80000000u;  // an offset beyond every buffer: reads 0

template <typename E>
__device__ __forceinline__ f32x4 multiply(s16x8 a, s16x8 b, f32x4 c);
template <>
__device__ __forceinline__ f32x4 multiply<bf16_t>(s16x8 a, s16x8 b, f32x4 c) {
    using V = bf16_t __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x4 multiply<f16_t>(s16x8 a, s16x8 b, f32x4 c) {
    using V = f16_t __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
}

// A matrix of 16-bit elements in memory, or three planes of one.  Address, ld, cols and plane are multiples of 8 elements, ld >= cols,
// and 256 rows span less than 2^31 bytes.
struct Source {
    const uint16_t* p;
    int64_t rows, cols, ld, plane;
};

struct ProductArgs {
    Source a[2], b[2];          // the sum runs over `pairs` of them, of equal ld; or see TileShape::kDual, `batch`
    int pairs, planes;          // planes: 1 or 3
    int64_t m, n, depth;
    int64_t tiles_m, tiles_n;
    int batch;                  // 2: two products, of a[0] and of a[1], with b[0]
    int splits;                 // of the depth: each its own result
    int64_t split_depth;        // a multiple of kDepth
};

template <int kM_, int kN_, int kWavesM_, int kWavesN_, bool kDual_ = false>
struct TileShape {
    static constexpr int kM = kM_, kN = kN_, kWavesM = kWavesM_, kWavesN = kWavesN_, kWaves = kWavesM * kWavesN, kThreads = 64 * kWaves;
    static constexpr int kFragsM = kM / kWavesM / 16, kFragsN = kN / kWavesN / 16;
    // the first half of a tile's kN rows is of b[0], the second of b[1], for the same kN / 2 columns of two results
    static constexpr bool kDual = kDual_;
    static constexpr int kColumns = kDual ? kN / 2 : kN;
};

// Moves a stage of one operand to LDS: kRows elements along m or n.
template <int kRows, bool kAlongK, int kWaves>
struct Loader {
    static constexpr int kInstructions = kRows * kDepth * 2 / kWaveBytes / kWaves;
    static constexpr int kChunks = kAlongK ? kDepth / 8 : kRows / 8;        // of 16 bytes in a row of LDS
    static constexpr int kRowsEach = 64 / kChunks;                          // rows of LDS per instruction
    uint32_t offset[kInstructions];
    int chunk;                                                              // along k

    static __device__ __forceinline__ int exchange(int k) { return ((k & 3) + 4 * ((k >> 3) & 3)) & (kRows / 16 - 1); }

    // `row0`: the first row of LDS that this wave fills, as a row of the source's tile
    __device__ __forceinline__ void init(int lane, int row0, int64_t ld) {
#pragma unroll
        for (int j = 0; j < kInstructions; ++j) {
            const int row = row0 + j * kRowsEach + lane / kChunks, c = lane % kChunks;
            const int from = kAlongK ? c ^ (row & 7) : (((c >> 1) ^ exchange(row)) << 1) + (c & 1);
            offset[j] = (uint32_t)(row * ld + from * 8) * 2u;
            chunk = from;
        }
    }

    // tile origin (row i0 along m or n, k0); `lds`: where the wave's rows begin
    __device__ __forceinline__ void issue(const Source& s, int plane, int64_t i0, int64_t k0, char* lds) const {
        const int64_t origin = (kAlongK ? i0 * s.ld + k0 : k0 * s.ld + i0), end = (s.rows - 1) * s.ld + s.cols;
        const int64_t left = (end - origin) * 2;
        const uint32_t bytes = left <= 0 ? 0u : left < 0x7fffffff ? (uint32_t)left : 0x7fffffffu;
        const __amdgpu_buffer_rsrc_t r =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(s.p + plane * s.plane + origin), 0, bytes, 0x00020000);
        const bool beyond = kAlongK && k0 + chunk * 8 >= s.cols;            // the next row lies there
#pragma unroll
        for (int j = 0; j < kInstructions; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + j * kWaveBytes), 16,
                                                     beyond ? kNowhere : offset[j], 0, 0, 0);
    }
};

// Reads fragments of a stage: for 16 elements along m or n and 32 k's, lane l has element l % 16 and k's 8 * (l / 16) ... + 7.
template <int kRows, bool kAlongK, int kFrags>
struct Reader {
    uint32_t at[kAlongK ? 2 : kFrags];
    __device__ __forceinline__ void init(int lane, int first) {
        if constexpr (kAlongK) {
#pragma unroll
            for (int s = 0; s < 2; ++s) at[s] = (uint32_t)((first + lane % 16) * (kDepth * 2) + ((s * 4 + lane / 16) ^ (lane & 7)) * 16);
        } else {
            const int k = lane / 16 * 8 + lane % 16 / 4;
#pragma unroll
            for (int i = 0; i < kFrags; ++i)
                at[i] = (uint32_t)(k * kRows * 2 + (((first / 16 + i) ^ Loader<kRows, false, 1>::exchange(k)) * 32) + (lane & 3) * 8);
        }
    }
    template <typename Lds>
    __device__ __forceinline__ s16x8 read(Lds* lds, int s, int i) const {
        if constexpr (kAlongK) {
            return *reinterpret_cast<const s16x8*>(lds + at[s] + i * 16 * kDepth * 2);
        } else {
            using P = __attribute__((address_space(3))) s16x4*;
            auto* p = lds + at[i] + s * 32 * kRows * 2;
            const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)p);
            const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + 4 * kRows * 2));
            return __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

// Which tile a workgroup takes.  Workgroups are dealt out to the 8 XCDs in turn; each XCD gets a contiguous range of tiles, in blocks
// of 8 rows of tiles, so that what its L2 holds of A and B is used by its neighbours.
struct TileIndex {
    int64_t m, n;
    int batch, split;
};

__device__ __forceinline__ TileIndex tile_of(const ProductArgs& args) {
    const uint32_t count = gridDim.x, id = blockIdx.x;
    const uint32_t each = count / 8, more = count % 8, xcd = id % 8;
    uint32_t t = xcd * each + (xcd < more ? xcd : more) + id / 8;
    TileIndex out;
    const uint32_t tiles = (uint32_t)(args.tiles_m * args.tiles_n);
    const uint32_t layer = t / tiles;
    t -= layer * tiles;
    out.batch = (int)(layer % args.batch);
    out.split = (int)(layer / args.batch);
    const uint32_t group = 8 * (uint32_t)args.tiles_n, first = t / group * 8;
    const uint32_t height = min(8u, (uint32_t)args.tiles_m - first), in = t % group;
    out.m = first + in % height;
    out.n = in / height;
    return out;
}

// The products of a tile: acc[j][i] holds, in lane l, elements m = 16 i + l % 16 and n = 16 j + 4 (l / 16) ... + 3 of the wave's part.
template <typename E, typename Shape, bool kARows, bool kBRows>
struct TileProduct {
    static constexpr int kABytes = Shape::kM * kDepth * 2, kBBytes = Shape::kN * kDepth * 2;
    using ALoader = Loader<Shape::kM, kARows, Shape::kWaves>;
    using BLoader = Loader<Shape::kN, kBRows, Shape::kWaves>;
    f32x4 acc[Shape::kFragsN][Shape::kFragsM];

    __device__ __forceinline__ void run(const ProductArgs& args, const TileIndex& tile) {
        // apart, so that the compiler sees that reads of one do not wait for what is on its way to the other
        __shared__ __attribute__((aligned(1024))) char first[kABytes + kBBytes];
        __shared__ __attribute__((aligned(1024))) char second[kABytes + kBBytes];
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wave_m = wave / Shape::kWavesN, wave_n = wave % Shape::kWavesN;

        const int64_t k_first = tile.split * args.split_depth, k_end = min(args.depth, k_first + args.split_depth);
        const int64_t i0 = tile.m * Shape::kM, j0 = tile.n * Shape::kColumns;
        // which half of a dual tile's rows this wave loads
        constexpr int kHalf = Shape::kWaves / 2;
        const int side = Shape::kDual ? wave / kHalf : 0, b_wave = Shape::kDual ? wave % kHalf : wave;
        ALoader a_loader;
        BLoader b_loader;
        constexpr int kARowsEach = ALoader::kInstructions * ALoader::kRowsEach, kBRowsEach = BLoader::kInstructions * BLoader::kRowsEach;
        const uint32_t a_lds = wave * ALoader::kInstructions * kWaveBytes, b_lds = kABytes + wave * BLoader::kInstructions * kWaveBytes;

        Reader<Shape::kM, kARows, Shape::kFragsM> a_reader;
        Reader<Shape::kN, kBRows, Shape::kFragsN / (Shape::kDual ? 2 : 1)> b_reader;
        a_reader.init(lane, wave_m * Shape::kFragsM * 16);
        b_reader.init(lane, wave_n * Shape::kFragsN * 16 / (Shape::kDual ? 2 : 1));

#pragma unroll
        for (int j = 0; j < Shape::kFragsN; ++j)
#pragma unroll
            for (int i = 0; i < Shape::kFragsM; ++i) acc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

        const int64_t steps = k_end > k_first ? (k_end - k_first + kDepth - 1) / kDepth : 0;
        const int products = args.planes == 3 ? 6 : 1;
        const int64_t total = steps * products * args.pairs;
        // products of planes (1,1) (0,2) (2,0) (0,1) (1,0) (0,0), two bits each
        constexpr uint32_t kPlanesA = 1u | 0u << 2 | 2u << 4 | 0u << 6 | 1u << 8 | 0u << 10;
        constexpr uint32_t kPlanesB = 1u | 2u << 2 | 0u << 4 | 1u << 6 | 0u << 8 | 0u << 10;
        int pair = 0, product = 0;
        int64_t k = k_first;
        a_loader.init(lane, wave * kARowsEach, args.a[args.batch > 1 ? tile.batch : 0].ld);
        b_loader.init(lane, b_wave * kBRowsEach, args.b[side].ld);

        auto load = [&](char* lds) {
            const int plane_a = args.planes == 3 ? (kPlanesA >> (2 * product)) & 3 : 0, plane_b = args.planes == 3 ? (kPlanesB >> (2 * product)) & 3 : 0;
            a_loader.issue(args.a[args.batch > 1 ? tile.batch : pair], plane_a, i0, k, lds + a_lds);
            b_loader.issue(args.b[Shape::kDual ? side : pair], plane_b, j0, k, lds + b_lds);
            k += kDepth;
            if (k >= k_end) {
                k = k_first;
                if (++product == products) {
                    product = 0;
                    ++pair;
                }
            }
        };
        auto compute = [&](const char* lds) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                s16x8 fa[Shape::kFragsM], fb[Shape::kFragsN];
#pragma unroll
                for (int i = 0; i < Shape::kFragsM; ++i) fa[i] = a_reader.read(lds, s, i);
#pragma unroll
                for (int j = 0; j < Shape::kFragsN; ++j) {
                    constexpr int kEach = Shape::kDual ? Shape::kFragsN / 2 : Shape::kFragsN;
                    const int half = j / kEach;                             // the second half's rows lie kN / 2 rows on
                    fb[j] = b_reader.read(lds + kABytes + half * (kBBytes / 2), s, j % kEach);
                }
#pragma unroll
                for (int j = 0; j < Shape::kFragsN; ++j)
#pragma unroll
                    for (int i = 0; i < Shape::kFragsM; ++i) acc[j][i] = multiply<E>(fb[j], fa[i], acc[j][i]);
                __builtin_amdgcn_sched_barrier(0);      // the other half's fragments would not fit the registers
            }
        };
        // what a wave has asked for has arrived, and all waves are here
        auto arrive = [&] {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        if (total > 0) load(first);
        int64_t step = 0;
        for (; step + 2 <= total; step += 2) {
            arrive();
            load(second);
            compute(first);
            arrive();
            if (step + 2 < total) load(first);
            compute(second);
        }
        if (step < total) {
            arrive();
            compute(first);
        }
    }

    // hands the elements to out.store(args, tile, m, n, four neighbours along n), or out.store(..., four of each result) of a dual tile
    template <typename Out>
    __device__ __forceinline__ void store(const ProductArgs& args, const TileIndex& tile, const Out& out) {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int wave_m = wave / Shape::kWavesN, wave_n = wave % Shape::kWavesN;
        constexpr int kEach = Shape::kDual ? Shape::kFragsN / 2 : Shape::kFragsN;
#pragma unroll
        for (int i = 0; i < Shape::kFragsM; ++i)
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const int64_t m = tile.m * Shape::kM + (wave_m * Shape::kFragsM + i) * 16 + lane % 16;
                const int64_t n = tile.n * Shape::kColumns + (wave_n * kEach + j) * 16 + lane / 16 * 4;
                if constexpr (Shape::kDual)
                    out.store(args, tile, m, n, acc[j][i], acc[j + kEach][i]);
                else
                    out.store(args, tile, m, n, acc[j][i]);
            }
    }
};

// A workgroup per tile.  Two waves a SIMD, or four where tiles are small.
template <typename E, typename Shape, bool kARows, bool kBRows, typename Out>
__global__ __launch_bounds__(Shape::kThreads, Shape::kM == 64 ? 4 : 2) void tile_kernel(ProductArgs args, Out out) {
#if defined(__HIP_DEVICE_COMPILE__)         // the host's half knows neither buffers nor matrix instructions
    const TileIndex tile = tile_of(args);
    TileProduct<E, Shape, kARows, kBRows> product;
    product.run(args, tile);
    product.store(args, tile, out);
#endif
}

}  // namespace dgsp
