// C(m, n) = sum over k of A(m, k) B(n, k) for matrices of 16-bit elements: tiles of C in registers, tiles of A and B in LDS.
//
// A stage is 64 deep.  Its tiles go from memory to LDS without passing through registers, 1 KB per wave and instruction, into one of
// two buffers (three of small tiles) while another one is multiplied; a barrier per stage hands the buffers over.  Each lane chooses
// which 16 bytes of memory its 16 bytes of LDS receive, and the choice spreads what the fragments' reads touch over all banks:
//   rows of k     an operand that is contiguous along k: 128 bytes a row, 16-byte chunk c of row r at chunk c ^ (r % 8).  Fragments are
//                 8 elements a lane, one 16-byte read.
//   rows of m/n   an operand that is contiguous along m or n (transposed): rows of one k, pairs of chunks (16 elements) exchanged by k.
//                 Fragments come from the transposing reads: 16 lanes read 4 k's of 16 elements and receive 4 k's of one element each.
//
// What bounds it: of a long sum the matrix instructions, at the 2.0 GHz that the card holds under them.  bfloat16, 8192 x 4096 x 16384:
// both along k 0.90 ms, 1.22 PFLOP/s; one transposed, two pairs 1.69 ms, 1.30; both transposed 0.94 ms, 1.17; with the epilogues of
// gated_ff_kernels.hpp, 1.6 GB each, that nothing runs beside: both projections 2.06 ms, 1.07, the slopes 1.25 ms, 0.88.  A library's
// products reach 1.35 to 1.58 and 1.05 to 1.15.  Of a few rows the weights' way from memory: one token, 4096 x 16384, 400 MB in 80 us,
// 5.0 TB/s.
#pragma once

#include "chunks.hpp"

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

// c += a b in place.  The builtin leaves the compiler free to put each result into other registers than c's; with the accumulators
// filling half of the registers, two thirds of them moved around and others were spilled.  A matrix instruction may read
// a register two cycles after another vector instruction has written it; the compiler does not know that this is one and puts nothing
// between them.  The wait is over before the matrix unit is free again.
template <typename E>
__device__ __forceinline__ void accumulate(s16x8 a, s16x8 b, f32x4& c);
template <>
__device__ __forceinline__ void accumulate<bf16_t>(s16x8 a, s16x8 b, f32x4& c) {
    asm volatile("s_nop 1\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "v"(b));
}
template <>
__device__ __forceinline__ void accumulate<f16_t>(s16x8 a, s16x8 b, f32x4& c) {
    asm volatile("s_nop 1\n\tv_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "v"(b));
}

// A matrix in memory.  Of 16-bit elements, address, ld and cols are multiples of 8 elements, ld >= cols, and 256 rows span less than 2^31
// bytes.
template <typename T>
struct Source {
    const T* p;
    int64_t rows, cols, ld;
};

template <typename T>
struct ProductArgs {
    Source<T> a[2], b[2];       // the sum runs over `pairs` of them, of equal ld; or see TileShape::kDual, `batch`
    int pairs;
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
    static constexpr int kWavesASimd = kM == 64 ? 3 : 2;
    // Small tiles are of products that read more than they multiply, by few workgroups: for one token at width 4096 the projections'
    // weights come at 4.2 TB/s with one stage on its way and at 5.3 with two.
    static constexpr int kBuffers = kM == 64 ? 3 : 2;
};

// Moves a stage of one operand to LDS: kRows elements along m or n.
template <int kRows, bool kAlongK, int kWaves>
struct Loader {
    static constexpr int kInstructions = kRows * kDepth * 2 / kWaveBytes / kWaves;
    static constexpr int kChunks = kAlongK ? kDepth / 8 : kRows / 8;        // of 16 bytes in a row of LDS
    static constexpr int kRowsEach = 64 / kChunks;                          // rows of LDS per instruction
    // Which chunk a lane takes depends on the instruction in the first or in the second bit of its number, or not at all.
    static constexpr int kPatternBit = kAlongK || kRows == 64 ? -1 : kRows == 256 ? 0 : 1;
    static constexpr int kPatterns = kPatternBit < 0 ? 1 : 2;
    uint32_t offset[kPatterns];             // of the lane in the rows of an instruction
    int chunk;                              // along k

    static __device__ __forceinline__ int exchange(int k) { return ((k & 3) + 4 * ((k >> 3) & 3)) & (kRows / 16 - 1); }

    // `row0`: the first row of LDS that this wave fills
    __device__ __forceinline__ void init(int lane, int row0, int64_t ld) {
        const int row = lane / kChunks, c = lane % kChunks;
#pragma unroll
        for (int p = 0; p < kPatterns; ++p) {
            const int k = row0 + (kPatternBit > 0 ? p << kPatternBit : p) * kRowsEach + row;
            chunk = kAlongK ? c ^ (k & 7) : (((c >> 1) ^ exchange(k)) << 1) + (c & 1);
            offset[p] = (uint32_t)(row * ld + chunk * 8) * 2u;
        }
    }

    // Where the wave's rows of a stage begin in the source and how much of it is left there; all lanes alike.
    struct Cursor {
        const char* at;
        int64_t left;           // bytes
        int depth_left;         // elements of a row, along k
    };
    // row i0 along m or n, k0; `row0`: the wave's first row of the tile
    template <typename T>
    static __device__ __forceinline__ Cursor begin(const Source<T>& s, int64_t i0, int64_t k0, int row0) {
        const int64_t origin = kAlongK ? (i0 + row0) * s.ld + k0 : (k0 + row0) * s.ld + i0, end = (s.rows - 1) * s.ld + s.cols;
        return {reinterpret_cast<const char*>(s.p + origin), (end - origin) * 2, (int)(s.cols - k0)};
    }
    // A stage on its way to byte `lds` of LDS, where the wave's rows begin.  The instruction is written out because the compiler waits for
    // one of its own before any read of LDS that it cannot tell from where it goes; the waits are arrive()'s.  It has no result in
    // registers.
    __device__ __forceinline__ void issue(Cursor& c, int64_t ld, uint32_t lds) const {
        const bool beyond = kAlongK && chunk * 8 >= c.depth_left;           // the next row lies there
        const char* at = c.at;
        int64_t left = c.left;
#pragma unroll
        for (int j = 0; j < kInstructions; ++j) {
            // in halves, as there are no 64-bit comparisons of scalars
            const int high = (int)(left >> 32);
            const uint32_t low = (uint32_t)left, some = high > 0 ? 0x7fffffffu : low < 0x7fffffffu ? low : 0x7fffffffu;
            const uint64_t address = reinterpret_cast<uint64_t>(at);
            const u32x4 buffer = {(uint32_t)address, (uint32_t)(address >> 32) & 0xffffu, high < 0 ? 0u : some, 0x00020000u};
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds + j * kWaveBytes),
                         "v"(beyond ? kNowhere : offset[kPatternBit < 0 ? 0 : j >> kPatternBit & 1]), "s"(buffer)
                         : "memory", "m0");
            at += kRowsEach * 2 * ld;
            left -= kRowsEach * 2 * ld;
        }
        const int64_t step = kAlongK ? kDepth * 2 : kDepth * 2 * ld;
        c.at += step;
        c.left -= step;
        c.depth_left -= kDepth;
    }
};

// Reads fragments of a stage: for 16 elements along m or n and 32 k's, lane l has element l % 16 and k's 8 * (l / 16) ... + 7.
template <int kRows, bool kAlongK, int kFrags>
struct Reader {
    uint32_t at;
    __device__ __forceinline__ void init(int lane, int first) {
        if constexpr (kAlongK) {
            at = (uint32_t)((first + lane % 16) * (kDepth * 2) + (lane / 16 ^ (lane & 7)) * 16);
        } else {
            const int k = lane / 16 * 8 + lane % 16 / 4;
            at = (uint32_t)(k * kRows * 2 + ((first / 16 ^ Loader<kRows, false, 1>::exchange(k)) * 32) + (lane & 3) * 8);
        }
    }
    // half s of the stage, 16 elements i; `first` is a multiple of 16 kFrags, so that the chunks' exchanges are those of `at`
    template <typename Lds>
    __device__ __forceinline__ s16x8 read(Lds* lds, int s, int i) const {
        if constexpr (kAlongK) {
            return *reinterpret_cast<const s16x8*>(lds + (at ^ (s * 64)) + i * 16 * kDepth * 2);
        } else {
            static_assert((kFrags & (kFrags - 1)) == 0);
            using P = __attribute__((address_space(3))) s16x4*;
            auto* p = lds + (at ^ (i * 32)) + s * 32 * kRows * 2;
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

template <typename T>
__device__ __forceinline__ TileIndex tile_of(const ProductArgs<T>& args) {
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

    __device__ __forceinline__ void run(const ProductArgs<E>& args, const TileIndex& tile) {
        constexpr uint32_t kStage = kABytes + kBBytes, kRing = Shape::kBuffers * kStage;
        __shared__ __attribute__((aligned(1024))) char lds[kRing];
        const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
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
        const uint32_t a_lds = lds_at + wave * ALoader::kInstructions * kWaveBytes, b_lds = lds_at + kABytes + wave * BLoader::kInstructions * kWaveBytes;

        Reader<Shape::kM, kARows, Shape::kFragsM> a_reader;
        Reader<Shape::kN, kBRows, Shape::kFragsN / (Shape::kDual ? 2 : 1)> b_reader;
        a_reader.init(lane, wave_m * Shape::kFragsM * 16);
        b_reader.init(lane, wave_n * Shape::kFragsN * 16 / (Shape::kDual ? 2 : 1));

#pragma unroll
        for (int j = 0; j < Shape::kFragsN; ++j)
#pragma unroll
            for (int i = 0; i < Shape::kFragsM; ++i) acc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

        const int steps = k_end > k_first ? (int)((k_end - k_first + kDepth - 1) / kDepth) : 0;
        const int total = steps * args.pairs;
        if (total == 0) return;
        const int64_t a_ld = args.a[args.batch > 1 ? tile.batch : 0].ld, b_ld = args.b[side].ld;
        a_loader.init(lane, wave * kARowsEach, a_ld);
        b_loader.init(lane, b_wave * kBRowsEach, b_ld);

        // stages are loaded in order: along the depth, then the next pair
        int pair = 0;
        int stages_left = steps;
        typename ALoader::Cursor a_at;
        typename BLoader::Cursor b_at;
        auto enter = [&] {
            a_at = ALoader::begin(args.a[args.batch > 1 ? tile.batch : pair], i0, k_first, wave * kARowsEach);
            b_at = BLoader::begin(args.b[Shape::kDual ? side : pair], j0, k_first, b_wave * kBRowsEach);
        };
        enter();
        auto load = [&](uint32_t buffer) {
            if (stages_left == 0) {
                ++pair;
                stages_left = steps;
                enter();
            }
            --stages_left;
            a_loader.issue(a_at, a_ld, a_lds + buffer);
            b_loader.issue(b_at, b_ld, b_lds + buffer);
        };
        auto read_a = [&](uint32_t buffer, int s, int i) { return a_reader.read(lds + buffer, s, i); };
        auto read_b = [&](uint32_t buffer, int s, s16x8 (&f)[Shape::kFragsN]) {
#pragma unroll
            for (int j = 0; j < Shape::kFragsN; ++j) {
                constexpr int kEach = Shape::kDual ? Shape::kFragsN / 2 : Shape::kFragsN;
                f[j] = b_reader.read(lds + buffer + kABytes + j / kEach * (kBBytes / 2), s, j % kEach);     // the second half's rows lie kN / 2 rows on
            }
        };
        // what this wave has asked for has arrived, but for the latest `later` stages, and all waves are here
        constexpr int kOfAStage = ALoader::kInstructions + BLoader::kInstructions;
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
        // A fragment of A is multiplied by all of B's and makes room for the one of the next half stage at once; B's have a second place.
        // A little into the second half all waves have read the whole stage and the next one has arrived: from there on fragments are of
        // the next one, and this one's buffer takes the one after that, which has a whole stage's time on its way.
        constexpr int kEarly = Shape::kFragsM >= 8 ? 2 : 1;
        s16x8 a[Shape::kFragsM], b_low[Shape::kFragsN], b_high[Shape::kFragsN];
        auto multiply_row = [&](int i, const s16x8 (&b)[Shape::kFragsN]) {
#pragma unroll
            for (int j = 0; j < Shape::kFragsN; ++j) accumulate<E>(b[j], a[i], acc[j][i]);
        };
        for (int i = 0; i < min(total, Shape::kBuffers); ++i) load(i * kStage);
        arrive(min(total, Shape::kBuffers) - 1);
        read_b(0, 0, b_low);
#pragma unroll
        for (int i = 0; i < Shape::kFragsM; ++i) a[i] = read_a(0, 0, i);
        // the first half, and as much of the second as its last fragments take to arrive
        auto first_half = [&](uint32_t buffer) {
            read_b(buffer, 1, b_high);
#pragma unroll
            for (int i = 0; i < Shape::kFragsM; ++i) {
                multiply_row(i, b_low);
                a[i] = read_a(buffer, 1, i);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < kEarly; ++i) multiply_row(i, b_high);
            __builtin_amdgcn_sched_barrier(0);
        };
        uint32_t here = 0;
        first_half(here);
        for (int step = 0; step + 1 < total; ++step) {          // begins where no read is on its way that has to be waited for
            const uint32_t next = here + kStage == kRing ? 0 : here + kStage;
            arrive(min(total - 2 - step, Shape::kBuffers - 2));
            if (step + Shape::kBuffers < total) load(here);
            read_b(next, 0, b_low);
#pragma unroll
            for (int i = 0; i < kEarly; ++i) a[i] = read_a(next, 0, i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = kEarly; i < Shape::kFragsM; ++i) {
                multiply_row(i, b_high);
                a[i] = read_a(next, 0, i);
                __builtin_amdgcn_sched_barrier(0);
            }
            here = next;
            first_half(here);
        }
#pragma unroll
        for (int i = kEarly; i < Shape::kFragsM; ++i) multiply_row(i, b_high);
        // other instructions may read a result 11 cycles after its matrix instruction has begun; the compiler does not see these
#pragma unroll
        for (int i = 0; i < Shape::kFragsM; ++i)
#pragma unroll
            for (int j = 0; j < Shape::kFragsN; ++j) {
                if (i == 0 && j == 0) asm volatile("s_nop 15\n\ts_nop 15" : "+v"(acc[0][0]));
                asm volatile("" : "+v"(acc[j][i]));
            }
    }
};

// Hands the results of a tile to out.row(args, tile, m, n, more, v[j][...]), a row of fragments at a time: element m and, for fragment j,
// four elements from n + 16 j on; of a dual tile v[j][0] and v[j][1] are of the two results.  `more` is what out.ask(args, m, n) gave for
// them a row earlier.
template <typename Shape, typename T, typename Out>
__device__ __forceinline__ void store_tile(const f32x4 (&acc)[Shape::kFragsN][Shape::kFragsM], const ProductArgs<T>& args, const TileIndex& tile, const Out& out) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_m = wave / Shape::kWavesN, wave_n = wave % Shape::kWavesN;
    constexpr int kEach = Shape::kDual ? Shape::kFragsN / 2 : Shape::kFragsN, kResults = Shape::kDual ? 2 : 1;
    const int64_t m = tile.m * Shape::kM + wave_m * Shape::kFragsM * 16 + lane % 16;
    const int64_t n = tile.n * Shape::kColumns + wave_n * kEach * 16 + lane / 16 * 4;
    auto more = out.template ask<kEach>(args, m, n);
#pragma unroll
    for (int i = 0; i < Shape::kFragsM; ++i) {
        const auto have = more;
        if (i + 1 < Shape::kFragsM) more = out.template ask<kEach>(args, m + 16 * (i + 1), n);
        f32x4 v[kEach][kResults];
#pragma unroll
        for (int j = 0; j < kEach; ++j)
#pragma unroll
            for (int r = 0; r < kResults; ++r) v[j][r] = acc[j + r * kEach][i];
        out.row(args, tile, m + 16 * i, n, have, v);
    }
}

struct Nothing {};

// A workgroup per tile.
template <typename E, typename Shape, bool kARows, bool kBRows, typename Out>
__global__ __launch_bounds__(Shape::kThreads, Shape::kWavesASimd) void tile_kernel(ProductArgs<E> args, Out out) {
#if defined(__HIP_DEVICE_COMPILE__)         // the host's half knows neither buffers nor matrix instructions
    const TileIndex tile = tile_of(args);
    TileProduct<E, Shape, kARows, kBRows> product;
    product.run(args, tile);
    store_tile<Shape>(product.acc, args, tile, out);
#endif
}

}  // namespace dgsp
