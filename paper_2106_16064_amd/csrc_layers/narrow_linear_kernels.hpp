// y = act(x w^T + bias) + residual where the weight fits a CU's LDS: the features of many vertices in narrow rows.  What bounds it is
// reading and writing the matrices that are as long as the rows, so each is touched once: the forward pass writes y and what is kept, x in 8 bits
// among it, and the backward pass makes dz = dy act'(z) in registers and all three gradients of it.
//
// 2^20 vertices, bfloat16, with residual: 64 -> 64 forward 105 us (537 MB, 5.1 TB/s), gradient 128 us (537 MB, 4.2 TB/s); 128 -> 128 with
// activations kept in 8 bits 250 to 265 us (1.08 GB, 4.1 to 4.3 TB/s; gelu and what becomes 8 bits are 150 us of vector instructions beside that) and
// 220 to 270 us (0.81 GB).  The products of matrix_tiles.hpp one after the other: 183 and 270 us, 417 and 560 us.  Float, gelu, 32 -> 32 forward 92 us
// (403 MB, 4.4 TB/s), gradient 116 us (537 MB, 4.6 TB/s), by tiles of 64 167 and 325 us; 64 -> 64 166 and 224 us; 64 -> 128 with residual 371 and 467 us,
// by tiles 428 and 762.
//
// A lane has a vertex (l % 16 of 16) and, q = l / 16, columns 32 t + 8 q ... + 7 of every 32: a piece of 16 bytes, which is also what the matrix
// instructions take of it as an operand, and 16 lanes of a block of 32 columns are 64 bytes of a row.  The weight's rows are put in such an order
// that a lane's results are neighbours as well: row 4 q + i of a 16 x 16 result is its column 32 t + 8 q + 4 h + i, for two results h.  Float numbers are
// three bf16 ones each, and their products six (float_tiles.hpp); weights and, for the weight's gradient, rows lie in LDS as planes of these.
#pragma once

#include "chunks.hpp"
#include "float_tiles.hpp"
#include "fragments.hpp"
#include "lanes.hpp"
#include "linear_kernels.hpp"
#include "rows8.hpp"

namespace dgsp {

template <typename E>
struct NarrowLinearArgs {
    int64_t rows, width, out_width;
    int activation;
    const E *x, *weight;
    int64_t ldx, ldw;
    const void* bias;
    bool wide;                  // the bias, and z, in float
    const E* residual;
    int64_t ldr;
    E* y;
    int64_t ldy;
    void* z;                    // kept: one of these two, or none; ld is `kept_ld`, a multiple of 8
    uint8_t* codes;
    int64_t kept_ld;
    Rows8 x8;                   // x in whole numbers of 8 bits: written by the forward pass, read by the backward pass; or not
    ScaleRange range;
};

// Which row of the weight a fragment's row is, among 32.
__device__ __forceinline__ int place_in_32(int row, int half) { return 8 * (row / 4) + 4 * half + row % 4; }

// eight 16-bit numbers as they are rounded
template <typename E>
__device__ __forceinline__ s16x8 pack8(const float (&v)[kChunk]) {
    return join(pack<E>(f32x4{v[0], v[1], v[2], v[3]}), pack<E>(f32x4{v[4], v[5], v[6], v[7]}));
}

// Eight neighbours as the matrix instructions take them: 16-bit ones as they are, float ones as three bf16 numbers each (float_tiles.hpp).
template <typename E>
constexpr int kPlanes = sizeof(E) == 4 ? 3 : 1;

template <int kCount>
struct Planes {
    s16x8 q[kCount];
};

template <typename E>
__device__ __forceinline__ Planes<kPlanes<E>> planes_of(const RawChunk<E>& raw) {
    Planes<kPlanes<E>> out;
    if constexpr (kPlanes<E> == 3) {
        u32x4 parts[3];
        split_chunk(raw, parts);
#pragma unroll
        for (int p = 0; p < 3; ++p) out.q[p] = __builtin_bit_cast(s16x8, parts[p]);
    } else {
        out.q[0] = __builtin_bit_cast(s16x8, raw.q[0]);
    }
    return out;
}

// of 16-bit types they are rounded
template <typename E>
__device__ __forceinline__ Planes<kPlanes<E>> planes_of(const float (&v)[kChunk]) {
    if constexpr (kPlanes<E> == 3)
        return planes_of<float>(RawChunk<float>{{__builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]}), __builtin_bit_cast(u32x4, f32x4{v[4], v[5], v[6], v[7]})}});
    else
        return {{pack8<E>(v)}};
}

// c += a b, of float the six products that are larger than 2^-24 of it, the smallest first, or three where b is exact in bf16
template <typename E, int kA, int kB>
__device__ __forceinline__ f32x4 multiply_planes(const Planes<kA>& a, const Planes<kB>& b, f32x4 c) {
    if constexpr (kA == 3 && kB == 3) {
        constexpr int kFirst[6] = {1, 0, 2, 0, 1, 0}, kSecond[6] = {1, 2, 0, 1, 0, 0};
#pragma unroll
        for (int p = 0; p < 6; ++p) c = multiply<bf16_t>(a.q[kFirst[p]], b.q[kSecond[p]], c);
        return c;
    } else if constexpr (kA == 3) {
        return multiply<bf16_t>(a.q[0], b.q[0], multiply<bf16_t>(a.q[1], b.q[0], multiply<bf16_t>(a.q[2], b.q[0], c)));
    } else {
        return multiply<E>(a.q[0], b.q[0], c);
    }
}

// the largest of the four lanes that have a vertex's block
__device__ __forceinline__ uint32_t vertex_max(uint32_t v) {
    const auto far = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max((uint32_t)far[0], (uint32_t)far[1]);
    const auto near = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return max((uint32_t)near[0], (uint32_t)near[1]);
}

// A lane's eight elements of a vertex -> whole numbers of 8 bits, as to_8bit() of a row's four neighbouring lanes.
template <typename E>
__device__ __forceinline__ uint2 vertex_bytes(const RawChunk<E>& raw, ScaleRange range, uint32_t& scale) {
    float amax;                                                // magnitudes are in the order of their bits
    if constexpr (sizeof(E) == 4) {
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < kChunk; ++j) most = max(most, raw.q[j / 4][j % 4] & 0x7fffffffu);
        amax = __builtin_bit_cast(float, vertex_max(most));
    } else {
        using Pair = uint16_t __attribute__((ext_vector_type(2)));
        Pair most = {0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(Pair, raw.q[0][j] & 0x7fff7fffu));
        amax = to_float(__builtin_bit_cast(E, (uint16_t)vertex_max(max(most[0], most[1]))));
    }
    const bool finite = amax < __builtin_inff();
    scale = scale_byte<false>(finite ? __builtin_bit_cast(uint32_t, amax) : 0u, range);
    const float inverse = __builtin_bit_cast(float, (254u - scale) << 23);
    float v[kChunk];
    widen(raw, v);
    uint2 bytes = whole_bytes(v, inverse, __builtin_amdgcn_ballot_w64((int)scale == range.most) != 0);
    if (!finite) {
        scale = 255u;
        bytes = {0u, 0u};
    }
    return bytes;
}

// slope_words() of eight neighbours
__device__ __forceinline__ uint2 slope_bytes(const float (&slope)[kChunk]) {
    uint32_t words[2];
    slope_words(slope, words);
    return {words[0], words[1]};
}

// Value and derivative, the one at an infinity as well, in kPieces, one after the other: together eight of them take more registers than the widest rows leave.
template <int kPieces, bool kFloat>
__device__ __forceinline__ void activate_in(int kind, const float (&z)[kChunk], float (&value)[kChunk], float (&slope)[kChunk]) {
    constexpr int kEach = kChunk / kPieces;
#pragma unroll
    for (int p = 0; p < kPieces; ++p) {
        float in[kEach], v[kEach], s[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) in[j] = z[p * kEach + j];
        activate<kFloat, true>(kind, in, v, s);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            value[p * kEach + j] = v[j];
            slope[p * kEach + j] = s[j];
        }
        if constexpr (kPieces > 1) __builtin_amdgcn_sched_barrier(0);
    }
}

// A lane's eight elements of a row at `col`.  Where rows are whole, rows that are not there are read as the first one, and what comes of them is
// not written or counts as 0; else what is not there is 0.
template <bool kWhole, typename E>
__device__ __forceinline__ RawChunk<E> row_chunk(const E* p, int64_t row, int64_t ld, int col, int columns, bool inside) {
    if constexpr (kWhole) return load_chunk(p + (inside ? row * ld : 0) + col, kChunk);
    const bool some = inside && col < columns;
    return load_chunk(p + (some ? row * ld + col : 0), some ? columns - col : 0);
}

// kP: width, kO: out_width, each padded to 32, 64 or 128; kX8: x is written in 8 bits; kWhole: nothing is padded
template <typename E, int kP, int kO, bool kX8, bool kWhole>
__global__ __launch_bounds__(256, (kP * kO * kPlanes<E> > 64 * 64 ? 3 : 4)) void narrow_linear_kernel(NarrowLinearArgs<E> a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kU = kP / 32, kT = kO / 32, kFragments = 2 * kT * kU, kParts = kPlanes<E>;
    constexpr bool kFloat = sizeof(E) == 4;
    __shared__ u32x4 weights[kParts][kFragments * 64];
    __shared__ __attribute__((aligned(16))) float bias[kO];
    for (int c = threadIdx.x; c < kO; c += 256)
        bias[c] = !a.bias || c >= a.out_width ? 0.0f : a.wide ? static_cast<const float*>(a.bias)[c] : to_float(static_cast<const E*>(a.bias)[c]);
    for (int i = threadIdx.x; i < kFragments * 64; i += 256) {
        const int f = i / 64, l = i % 64, u = f % kU, out = f / kU / 2 * 32 + place_in_32(l % 16, f / kU % 2), k = 32 * u + l / 16 * 8;
        const bool there = out < a.out_width && k < a.width;
        const auto planes = planes_of<E>(load_chunk(a.weight + (there ? out * a.ldw + k : 0), there ? a.width - k : 0));
#pragma unroll
        for (int p = 0; p < kParts; ++p) weights[p][i] = __builtin_bit_cast(u32x4, planes.q[p]);
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, first = lane / 16 * 8;           // of the lane's columns in every 32
    const int width = kWhole ? kP : (int)a.width, out_width = kWhole ? kO : (int)a.out_width, blocks = (width + kBlock - 1) / kBlock;
    const int64_t step = (int64_t)gridDim.x * 64;
    int64_t row = (int64_t)blockIdx.x * 64 + threadIdx.x / 64 * 16 + lane % 16;
    RawChunk<E> x[kU];
    auto ask = [&](int64_t at) {
#pragma unroll
        for (int u = 0; u < kU; ++u) x[u] = row_chunk<kWhole>(a.x, at, a.ldx, 32 * u + first, width, at < a.rows);
    };
    ask(row);
    for (int64_t base = (int64_t)blockIdx.x * 64; base < a.rows; base += step, row += step) {
        const bool inside = row < a.rows;
        RawChunk<E> residual[kT];
        if (a.residual)
#pragma unroll
            for (int t = 0; t < kT; ++t) residual[t] = row_chunk<kWhole>(a.residual, row, a.ldr, 32 * t + first, out_width, inside);
        Planes<kParts> operand[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) operand[u] = planes_of<E>(x[u]);
        if constexpr (kX8) {
            uint32_t word = 0;
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                uint32_t scale;
                const uint2 bytes = vertex_bytes<E>(x[u], a.range, scale);
                if (inside && (kWhole || u < blocks)) *reinterpret_cast<uint2*>(a.x8.values + row * a.x8.ldv + 32 * u + first) = bytes;
                word |= (kWhole || u < blocks ? scale : 127u) << (8 * u);
            }
            if (kU < 4) word |= 0x7f7f7f7fu << (8 * kU % 32);
            if (inside && first == 0) *reinterpret_cast<uint32_t*>(a.x8.scales + row * 4) = word;
        }
        ask(row + step);
        int piece = lane;                                               // of a fragment; read again for every row where all would not fit the registers
        if constexpr (kP * kO * kParts >= 64 * 64) asm volatile("" : "+v"(piece));
#pragma unroll
        for (int t = 0; t < kT; ++t) {
            f32x4 part[2] = {*reinterpret_cast<const f32x4*>(bias + 32 * t + piece / 16 * 8), *reinterpret_cast<const f32x4*>(bias + 32 * t + piece / 16 * 8 + 4)};
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    Planes<kParts> w;
#pragma unroll
                    for (int p = 0; p < kParts; ++p) w.q[p] = __builtin_bit_cast(s16x8, weights[p][((t * 2 + h) * kU + u) * 64 + piece]);
                    part[h] = multiply_planes<E>(w, operand[u], part[h]);
                }
            float z[kChunk], value[kChunk];
#pragma unroll
            for (int j = 0; j < kChunk; ++j) z[j] = part[j / 4][j % 4];
            const int col = 32 * t + first, here = kWhole ? kChunk : out_width - col;
            const bool store = inside && here > 0;
            if (a.codes) {
                float slope[kChunk];
                activate_in<(kFloat && !kWhole && kP * kO > 64 * 64 && kP > kO ? 4 : 1), kFloat>(a.activation, z, value, slope);
                const uint2 bytes = slope_bytes(slope);
                if (store) *reinterpret_cast<uint2*>(a.codes + row * a.kept_ld + col) = bytes;
            } else {
                activate_only<kFloat>(a.activation, z, value);
                if (a.z && store) {
                    if (a.wide)
                        store_chunk(static_cast<float*>(a.z) + row * a.kept_ld + col, kChunk, z);
                    else
                        store_chunk(static_cast<E*>(a.z) + row * a.kept_ld + col, kChunk, z);
                }
            }
            if (a.residual) {
                float add[kChunk];
                widen(residual[t], add);
#pragma unroll
                for (int j = 0; j < kChunk; ++j) value[j] += add[j];
            }
            if (store) store_chunk(a.y + row * a.ldy + col, here, value);
        }
    }
#endif
}

template <typename E>
struct NarrowLinearBackwardArgs {
    int64_t rows, width, out_width;
    int activation;
    const E *x, *weight, *dy;
    int64_t ldx, ldw, lddy;
    const void* z;              // what was kept: one of these two, or none
    bool wide;                  // z in float
    const uint8_t* codes;
    int64_t kept_ld;
    Rows8 x8;                   // in place of x
    E* dx;                      // packed; null: not wanted
    float *weight_sums;         // [workgroup and part of the vertices][out_width][width]; null: not wanted
    float *bias_sums;           // [workgroup][out_width]; null: not wanted
};

// How the waves share the weight's gradient: kDown x kAcross of them have a block each, of kParts parts of the vertices.  Of float rows
// wider than 32 a workgroup has half as many vertices, so that two find room in LDS.  kGroups: workgroups that a CU has room for, which is what LDS and, of the eight
// waves of 16-bit rows, registers leave; the compiler is told.  With one of two left out (2^20 rows 64 -> 64 float, kept in 8 bits) the gradient takes
// 175 us in place of 150; with one too many, which waits for its turn, (2^20 rows 64 -> 128 bfloat16) 232 in place of 223.
template <typename E, int kP, int kO, bool kX8, bool kWhole>
struct NarrowShare {
    static constexpr int kWaves = sizeof(E) == 4 && kP * kO > 32 * 32 ? 4 : 8, kTile = 16 * kWaves;          // kTile vertices of a workgroup
    static constexpr int kDown = 2, kAcross = kP / 16 < kWaves / 2 ? kP / 16 : kWaves / 2, kParts = kWaves / (kDown * kAcross);
    static constexpr int kFragsO = kO / 16 / kDown, kFragsP = kP / 16 / kAcross;
    static constexpr int kLdO = kO + 8, kLdP = kP + 8;                  // rows of LDS start in different banks
    static constexpr int kXParts = kX8 ? 1 : kPlanes<E>;                // whole numbers are exact in bf16
    static constexpr int kLds = kPlanes<E> * 2 * kO * kP + 2 * kTile * (kPlanes<E> * kLdO + kXParts * kLdP) + 4 * kWaves * kO;
    static constexpr int kGroups = 2 * kLds <= 163840 && (sizeof(E) == 4 || (kO <= 64 && kP * kO <= (kWhole || kO < 64 ? 64 * 64 : 32 * 64))) ? 2 : 1;
};

// dz stays in registers as an operand for dx; for the weight's gradient, a sum over the vertices, dz and x pass through LDS, which hands them out by
// columns.  Sums over the vertices stay in registers until the end; the workgroups' are added in their order (column_sums.hpp).
// Z: the type that z was kept in
template <typename E, int kP, int kO, bool kX8, bool kWhole, typename Z>
__global__ __launch_bounds__((64 * NarrowShare<E, kP, kO, kX8, kWhole>::kWaves), (NarrowShare<E, kP, kO, kX8, kWhole>::kGroups * NarrowShare<E, kP, kO, kX8, kWhole>::kWaves / 4)) void narrow_linear_backward_kernel(NarrowLinearBackwardArgs<E> a) {
#if defined(__HIP_DEVICE_COMPILE__)
    using Share = NarrowShare<E, kP, kO, kX8, kWhole>;
    constexpr int kNarrowWaves = Share::kWaves, kNarrowTile = Share::kTile;
    constexpr int kU = kP / 32, kT = kO / 32, kFragments = 2 * kT * kU, kParts = kPlanes<E>, kXParts = Share::kXParts;
    constexpr bool kFloat = sizeof(E) == 4;
    __shared__ u32x4 weights[kParts][kFragments * 64];                  // by columns: 16 of width, 32 of out_width
    __shared__ uint16_t dz_rows[kParts][kNarrowTile * Share::kLdO], x_rows[kXParts][kNarrowTile * Share::kLdP];
    if (a.dx)
        for (int i = threadIdx.x; i < kFragments * 64; i += 64 * kNarrowWaves) {
            const int f = i / 64, l = i % 64, t = f % kT, k = f / kT / 2 * 32 + place_in_32(l % 16, f / kT % 2), out = 32 * t + l / 16 * 8;
            RawChunk<E> v;
#pragma unroll
            for (int j = 0; j < RawChunk<E>::kQuads; ++j) v.q[j] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < kChunk; ++j)
                if (k < a.width && out + j < a.out_width) {
                    if constexpr (kFloat)
                        v.q[j / 4][j % 4] = __builtin_bit_cast(uint32_t, a.weight[(out + j) * a.ldw + k]);
                    else
                        v.q[0][j / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, a.weight[(out + j) * a.ldw + k]) << (j % 2 * 16);
                }
            const auto planes = planes_of<E>(v);
#pragma unroll
            for (int p = 0; p < kParts; ++p) weights[p][i] = __builtin_bit_cast(u32x4, planes.q[p]);
        }
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), first = lane / 16 * 8;
    const int in_tile = wave * 16 + lane % 16;
    const int width = kWhole ? kP : (int)a.width, out_width = kWhole ? kO : (int)a.out_width, blocks = (width + kBlock - 1) / kBlock;
    const int down = wave % Share::kDown, across = wave / Share::kDown % Share::kAcross, part = wave / (Share::kDown * Share::kAcross);
    RawChunk<E> dy[kT], x[kU];
    RawChunk<Z> z[kT];
    uint2 codes[kT], x8[kU];
    uint32_t scales = 0;
    auto ask = [&](int64_t row) {
        const bool inside = row < a.rows;
        const int64_t kept_row = inside ? row * a.kept_ld : 0;
#pragma unroll
        for (int t = 0; t < kT; ++t) {
            const int col = 32 * t + first;
            const int64_t at = kWhole || col < out_width ? kept_row + col : 0;
            dy[t] = row_chunk<kWhole>(a.dy, row, a.lddy, col, out_width, inside);
            if (a.codes) codes[t] = *reinterpret_cast<const uint2*>(a.codes + at);
            if (a.z) z[t] = load_chunk(static_cast<const Z*>(a.z) + at, kChunk);
        }
        if (!a.weight_sums) return;
        if constexpr (kX8) scales = *reinterpret_cast<const uint32_t*>(a.x8.scales + (inside ? row * 4 : 0));
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int col = 32 * u + first;
            if constexpr (kX8)
                x8[u] = *reinterpret_cast<const uint2*>(a.x8.values + (inside ? row * a.x8.ldv : 0) + (kWhole || u < blocks ? col : 0));
            else
                x[u] = row_chunk<kWhole>(a.x, row, a.ldx, col, width, inside);
        }
    };
    f32x4 sums[Share::kFragsO][Share::kFragsP];
#pragma unroll
    for (int i = 0; i < Share::kFragsO; ++i)
#pragma unroll
        for (int j = 0; j < Share::kFragsP; ++j) sums[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float db[kT][kChunk];
#pragma unroll
    for (int t = 0; t < kT; ++t)
#pragma unroll
        for (int j = 0; j < kChunk; ++j) db[t][j] = 0.0f;

    const int64_t step = (int64_t)gridDim.x * kNarrowTile;
    int64_t row = (int64_t)blockIdx.x * kNarrowTile + in_tile;
    ask(row);
    for (int64_t base = (int64_t)blockIdx.x * kNarrowTile; base < a.rows; base += step, row += step) {
        Planes<kParts> dz[kT];
#pragma unroll
        for (int t = 0; t < kT; ++t) {
            float d[kChunk], slope[kChunk];
            widen(dy[t], d);
            if (a.codes) {
#pragma unroll
                for (int j = 0; j < kChunk; ++j) slope[j] = slope_of(codes[t], j);
            } else if (a.z) {
                float at[kChunk], value[kChunk];
                widen(z[t], at);
#pragma unroll
                for (int j = 0; j < kChunk; ++j) at[j] = inside_range<Z>(at[j]);
                activate<kFloat>(a.activation, at, value, slope);
            } else {
#pragma unroll
                for (int j = 0; j < kChunk; ++j) slope[j] = 1.0f;
            }
            const int here = row < a.rows ? (kWhole ? kChunk : out_width - 32 * t - first) : 0;
#pragma unroll
            for (int j = 0; j < kChunk; ++j) {
                d[j] = (kWhole ? here > 0 : j < here) ? d[j] * slope[j] : 0.0f;
                db[t][j] += d[j];
            }
            dz[t] = planes_of<E>(d);
        }
        if (a.weight_sums) {
            Planes<kXParts> in[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                if constexpr (kX8) {
                    float v[kChunk];
                    from_8bit<false>(x8[u], scales >> (8 * u) & 0xffu, v);
                    in[u] = {{pack8<std::conditional_t<kFloat, bf16_t, E>>(v)}};
                } else {
                    in[u] = planes_of<E>(x[u]);
                }
                // 0 times what a row that is not there, or columns behind a block's last, read instead could be NaN
                if (row >= a.rows || !(kWhole || !kX8 || u < blocks)) in[u] = {};
            }
            __syncthreads();                                            // the tile before has been read
#pragma unroll
            for (int t = 0; t < kT; ++t)
#pragma unroll
                for (int p = 0; p < kParts; ++p) *reinterpret_cast<s16x8*>(dz_rows[p] + in_tile * Share::kLdO + 32 * t + first) = dz[t].q[p];
#pragma unroll
            for (int u = 0; u < kU; ++u)
#pragma unroll
                for (int p = 0; p < kXParts; ++p) *reinterpret_cast<s16x8*>(x_rows[p] + in_tile * Share::kLdP + 32 * u + first) = in[u].q[p];
        }
        constexpr bool kLate = kFloat && kP * kO > 64 * 64 && kO > 64;         // the next rows and these ones' dz are more than the registers hold
        if constexpr (!kLate) ask(row + step);
        if (a.weight_sums) __syncthreads();
        if (a.dx) {
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                f32x4 out[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    out[h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int t = 0; t < kT; ++t) {
                        Planes<kParts> w;
#pragma unroll
                        for (int p = 0; p < kParts; ++p) w.q[p] = __builtin_bit_cast(s16x8, weights[p][((u * 2 + h) * kT + t) * 64 + lane]);
                        out[h] = multiply_planes<E>(w, dz[t], out[h]);
                    }
                }
                float v[kChunk];
#pragma unroll
                for (int j = 0; j < kChunk; ++j) v[j] = out[j / 4][j % 4];
                const int col = 32 * u + first, here = kWhole ? kChunk : width - col;
                if (row < a.rows && here > 0) store_chunk(a.dx + row * a.width + col, here, v);
            }
        }
        if constexpr (kLate) ask(row + step);
        if (a.weight_sums) {
            // 16 columns of 32 vertices, of each plane
            auto columns = [&](const auto& rows, int ld, int vertex, int column) {
                Planes<(int)std::extent_v<std::remove_reference_t<decltype(rows)>>> out;
#pragma unroll
                for (int p = 0; p < (int)std::extent_v<std::remove_reference_t<decltype(rows)>>; ++p) {
                    const uint16_t* at = rows[p] + (vertex + first) * ld + column;
                    out.q[p] = join(read_column(at, ld, lane), read_column(at + 4 * ld, ld, lane));
                }
                return out;
            };
#pragma unroll
            for (int s = 0; s < kNarrowTile / 32 / Share::kParts; ++s) {
                const int vertex = (part * (kNarrowTile / 32 / Share::kParts) + s) * 32;
                Planes<kXParts> across_x[Share::kFragsP];
#pragma unroll
                for (int j = 0; j < Share::kFragsP; ++j) across_x[j] = columns(x_rows, Share::kLdP, vertex, (across * Share::kFragsP + j) * 16);
#pragma unroll
                for (int i = 0; i < Share::kFragsO; ++i) {
                    const auto of_dz = columns(dz_rows, Share::kLdO, vertex, (down * Share::kFragsO + i) * 16);
#pragma unroll
                    for (int j = 0; j < Share::kFragsP; ++j) sums[i][j] = multiply_planes<E>(of_dz, across_x[j], sums[i][j]);
                }
            }
        }
    }
    if (a.weight_sums) {
        float* to = a.weight_sums + ((int64_t)blockIdx.x * Share::kParts + part) * a.out_width * a.width;
#pragma unroll
        for (int i = 0; i < Share::kFragsO; ++i)
#pragma unroll
            for (int j = 0; j < Share::kFragsP; ++j) {
                const int64_t out = (down * Share::kFragsO + i) * 16 + lane / 16 * 4, k = (across * Share::kFragsP + j) * 16 + lane % 16;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (out + r < a.out_width && k < a.width) to[(out + r) * a.width + k] = sums[i][j][r];
            }
    }
    if (a.bias_sums) {
        __shared__ float waves_sums[kNarrowWaves][kO];
#pragma unroll
        for (int t = 0; t < kT; ++t)
#pragma unroll
            for (int j = 0; j < kChunk; ++j) {
                const float v = lanes_sum(db[t][j], 16);
                if (lane % 16 == 0) waves_sums[wave][32 * t + first + j] = v;
            }
        __syncthreads();
        for (int c = threadIdx.x; c < kO; c += 64 * kNarrowWaves)
            if (c < a.out_width) {
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < kNarrowWaves; ++w) v += waves_sums[w][c];
                a.bias_sums[(int64_t)blockIdx.x * a.out_width + c] = v;
            }
    }
#endif
}

}  // namespace dgsp
