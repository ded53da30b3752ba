// Host side of the products on matrix_tiles.hpp: how they are cut into tiles, how their operands are laid out, launches.
#pragma once

#include "layers_host.hpp"

#include "product_kernels.hpp"

namespace dgsp {

constexpr int64_t kMostWidth = (1LL << 22) - 8;         // 256 rows of it span less than 2^31 bytes (matrix_tiles.hpp)
constexpr int64_t kAlign = 256;
inline int64_t padded(int64_t n, int64_t to) { return ceil_div(n, to) * to; }

inline bool known_activation(int activation) { return activation >= DGSP_ACT_SILU && activation <= DGSP_ACT_RELU; }

inline bool enough(const void* workspace, int64_t bytes, int64_t need) { return need == 0 || (workspace && aligned(workspace, 16) && bytes >= need); }

// Hands out pieces of a buffer, or adds up what they need where there is none.
class Pieces {
public:
    explicit Pieces(void* base) : base_(static_cast<char*>(base)) {}
    void* take(int64_t bytes) {
        void* p = base_ ? base_ + used_ : nullptr;
        used_ += padded(bytes, kAlign);
        return p;
    }
    int64_t used() const { return used_; }

private:
    char* base_;
    int64_t used_ = 0;
};

// ---------------------------------------------------------------- how a product is cut

enum TileSize { kSmall = 64, kMiddle = 128, kLarge = 256 };

struct Cut {
    int size;
    int64_t tiles_m, tiles_n;
    int splits;
    int64_t split_depth;
    int64_t groups(int batch) const { return tiles_m * tiles_n * batch * splits; }
};

// Which tiles.  256 x 256 read half as much per product as 128 x 128, but take a CU each, so that nothing runs while their results leave:
// they pay where the sum is long (`terms` counts pairs of operands), there is one for every CU, and the edges waste little.  64 x 64 are
// for what has fewer than a tile of 128 for every CU and cannot be split along the depth, or is hardly half as wide.  Forward and backward
// pass, bfloat16, us, by this rule, without 256 and with 64 alone:
//     8192 rows, 4096 -> 16384 -> 4096      8900   11000   19300
//     65536 rows, 256 -> 1024 -> 256         739     749     942
//     2048 rows, 1024 -> 4096 -> 1024        221     224     286
//     256 rows, 4096 -> 16384 -> 4096        572     573     821
// and 256 alone in float, 65536 rows, 128 -> 512 -> 128, made the slopes 284 us where 128 took 231: float has no tiles of 256 (with 64
// alone it takes 776 us, by this rule 638).  Where tiles are fewer than CUs the depth is split, to as many workgroups as are resident
// together (two of 128, three of 64 a CU; one token, 4096 -> 16384: 97, 88, 81 and 88 us with one to four a CU), down to 256 each, of
// float matrices 128.  `enough_tiles`: from how many on the depth is not split.
inline Cut cut(int64_t m, int64_t n, int64_t depth, int terms, int batch, int type, bool dual, bool may_split, int64_t enough_tiles = kCus) {
    auto tiles = [&](int size) { return ceil_div(m, size) * ceil_div(n, dual ? size / 2 : size) * batch; };
    const bool splits = may_split && depth >= (type == DGSP_F32 ? 512 : 1024);
    Cut c{kSmall, 0, 0, 1, padded(std::max<int64_t>(depth, 1), kDepth)};
    if (type != DGSP_F32 && tiles(kLarge) >= kCus && depth * terms >= 1024 && 4 * tiles(kLarge) <= tiles(kMiddle) + tiles(kMiddle) / 8)
        c.size = kLarge;
    else if ((tiles(kMiddle) >= kCus || splits) && 2 * (4 * tiles(kMiddle)) <= 3 * tiles(kSmall))
        c.size = kMiddle;
    c.tiles_m = ceil_div(m, c.size);
    c.tiles_n = ceil_div(n, dual ? c.size / 2 : c.size);
    const int64_t count = tiles(c.size);
    if (splits && count > 0 && count < enough_tiles) {               // no tiles: a batch without rows
        const int64_t most = std::min<int64_t>(ceil_div((c.size == kMiddle ? 2 : 3) * kCus, count), depth / (type == DGSP_F32 ? 128 : 256));
        c.split_depth = padded(ceil_div(depth, most), kDepth);
        c.splits = (int)ceil_div(depth, c.split_depth);
    }
    return c;
}

// As cut(), for products of which some are as deep as there are rows.  Splits make at most as many workgroups as are resident together: a few more
// than that are a second turn of the whole GPU.  Deep sums are split also where there is a tile for every CU but not two (three) of them,
// and tiles of 256 take over where cut so they come to 0.8 of the share of the CUs that is busy otherwise: their sums have to stay deep, as
// a CU has nothing else to do while one begins and ends, and their parts few, as each leaves 256 KB.  By cut() and this, us: the weight's gradient,
// bfloat16, 16384 rows, 1024 -> 4096 202 and 123 (128 split in two: 146), 65536 rows, 1024 -> 2048 293 and 241, 32768 rows, 1500 -> 2000 363
// and 237, 50000 rows, 301 -> 777 105 and 79; float, 4096 rows, 2048 -> 2048 244 and 187; the product, 200 rows, 4096 -> 5000 31 and 23.
inline Cut cut_to_fill(int64_t m, int64_t n, int64_t depth, int type, int64_t enough_tiles = kCus) {
    Cut c = cut(m, n, depth, 1, 1, type, false, true, enough_tiles);
    if (c.size == kLarge || m == 0) return c;
    const int64_t count = c.tiles_m * c.tiles_n, resident = (c.size == kMiddle ? 2 : 3) * kCus;
    int64_t splits = c.splits;
    if (count <= resident && (splits > 1 || (2 * count <= resident && depth >= 4096)))
        splits = std::min<int64_t>(resident / count, depth / (type == DGSP_F32 ? 128 : 256));
    const int64_t turns = ceil_div(count * splits, resident), large = ceil_div(m, kLarge) * ceil_div(n, kLarge), of_large = std::min<int64_t>(kCus / large, 16);
    if (type != DGSP_F32 && c.size == kMiddle && of_large > 0 && 4 * large <= count + count / 8 && depth >= 2048 * of_large &&
        10 * (large * of_large) * (turns * resident) >= 8 * (count * splits) * kCus) {
        c.size = kLarge;
        c.tiles_m = ceil_div(m, kLarge);
        c.tiles_n = ceil_div(n, kLarge);
        splits = of_large;
    }
    c.split_depth = padded(ceil_div(std::max<int64_t>(depth, 1), splits), kDepth);
    c.splits = (int)ceil_div(std::max<int64_t>(depth, 1), c.split_depth);
    return c;
}

inline bool launchable(const Cut& c, int batch) { return c.groups(batch) < (1LL << 32) / 512; }

template <bool kDual>
using Large = TileShape<256, 256, 2, 4, kDual>;
template <bool kDual>
using Middle = TileShape<128, 128, 2, 2, kDual>;
template <bool kDual>
using Small = TileShape<64, 64, 2, 2, kDual>;

template <typename T>
ProductArgs<T> product_args(const Cut& c, int64_t m, int64_t n, int64_t depth, int batch) {
    ProductArgs<T> args{};
    args.pairs = 1;
    args.m = m;
    args.n = n;
    args.depth = depth;
    args.tiles_m = c.tiles_m;
    args.tiles_n = c.tiles_n;
    args.batch = batch;
    args.splits = c.splits;
    args.split_depth = c.split_depth;
    return args;
}

inline int64_t partial_bytes(const Cut& c, int64_t m, int64_t n, int batch) {
    return c.splits > 1 ? (int64_t)c.splits * batch * m * padded(n, 4) * 4 : 0;
}

template <typename T, bool kDual, bool kARows, bool kBRows, typename Out>
void launch(const Cut& c, const ProductArgs<T>& args, const Out& out, hipStream_t stream) {
    const auto groups = (unsigned)c.groups(args.batch);
    if constexpr (sizeof(T) == 4) {
        if (c.size == kMiddle)
            float_tile_kernel<Middle<kDual>, kARows, kBRows, Out><<<groups, Middle<kDual>::kThreads, 0, stream>>>(args, out, Nothing{});
        else
            float_tile_kernel<Small<kDual>, kARows, kBRows, Out><<<groups, Small<kDual>::kThreads, 0, stream>>>(args, out, Nothing{});
    } else if (c.size == kLarge) {
        tile_kernel<T, Large<kDual>, kARows, kBRows, Out><<<groups, Large<kDual>::kThreads, 0, stream>>>(args, out);
    } else if (c.size == kMiddle) {
        tile_kernel<T, Middle<kDual>, kARows, kBRows, Out><<<groups, Middle<kDual>::kThreads, 0, stream>>>(args, out);
    } else {
        tile_kernel<T, Small<kDual>, kARows, kBRows, Out><<<groups, Small<kDual>::kThreads, 0, stream>>>(args, out);
    }
}

// c[0 ... batch - 1] = the product (products.hip)
template <typename T, bool kARows, bool kBRows>
void product(const Cut& c, const ProductArgs<T>& args, ProductOut<T> out, void* partial, hipStream_t stream);

// A weight's gradient of float matrices, a[0] rows x m and b[0] rows x n.  `b8`: in place of b[0]; null: b[0].  `sums`: over the rows of a[0], [split][m];
// null: not wanted.
void weight_gradient(const Cut& c, const ProductArgs<float>& args, const Rows8* b8, float* sums, ProductOut<float> out, void* partial, hipStream_t stream);

// ---------------------------------------------------------------- operands

inline int64_t kept_bytes(int64_t rows, int64_t cols, int type) { return rows * padded(cols, 8) * element_bytes(type); }

// what a matrix that does not lie as the products read it takes; float matrices are read as they lie
inline int64_t laid_out_bytes(int64_t rows, int64_t cols, int type) { return type == DGSP_F32 ? 0 : kept_bytes(rows, cols, type); }

// The matrices of a call as its products read them: float matrices as they are, those of 16-bit elements in place if they lie in whole
// 16-byte pieces, else laid out in a piece of memory, all in one launch that has to come before the products'.
template <typename T>
class Operands {
public:
    static bool in_place(const void* p, int64_t rows, int64_t cols, int64_t ld) {
        return sizeof(T) == 4 || (cols % 8 == 0 && (rows == 1 || (ld % 8 == 0 && ld >= cols && ld <= kMostWidth)) && aligned(p, 16));
    }
    Source<T> add(const void* p, int64_t rows, int64_t cols, int64_t ld, void* piece, bool copy = false) {
        if (in_place(p, rows, cols, ld) && !copy) return {static_cast<const T*>(p), rows, cols, rows == 1 ? cols : ld};
        const int64_t to_ld = padded(cols, 8);
        if (rows > 0) {
            const auto groups = (unsigned)std::min<int64_t>(ceil_div(rows * to_ld / 8, 256), 1 << 14);
            all_.each[all_.count++] = {static_cast<const T*>(p), rows, cols, ld, static_cast<T*>(piece), to_ld, groups};
            groups_ += groups;
        }
        return {static_cast<const T*>(piece), rows, to_ld, to_ld};
    }
    void launch(hipStream_t stream) const {
        if constexpr (sizeof(T) == 2)
            if (all_.count) lay_out_kernel<T><<<groups_, 256, 0, stream>>>(all_);
    }

private:
    Layouts<T> all_{};
    unsigned groups_ = 0;
};

template <typename T>
Source<T> source(const Kept<T>& kept, int64_t rows) {
    return {kept.p, rows, kept.ld, kept.ld};
}

template <typename T>
Kept<T> kept(void* p, int64_t hidden) {
    return {static_cast<T*>(p), padded(hidden, 8)};
}

}  // namespace dgsp
