// Host side of the gated feed-forward block: argument checks, how operands are laid out, tile shapes and launches.  The C-ABI is
// documented in include/dgsp_layers.h.
#include "layers_host.hpp"

#include "gated_ff_kernels.hpp"
#include "narrow_ff.hpp"

namespace {

using namespace dgsp;

constexpr int64_t kMostWidth = (1LL << 22) - 8;         // 256 rows of it span less than 2^31 bytes (matrix_tiles.hpp)
constexpr int64_t kAlign = 256;
constexpr int64_t kCus = 256;

int64_t padded(int64_t n, int64_t to) { return ceil_div(n, to) * to; }

bool gated_extents(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type) {
    return rows >= 0 && rows <= kMostRows && width >= 1 && width <= kMostWidth && hidden >= 1 && hidden <= kMostWidth &&
           out_width >= 1 && out_width <= kMostWidth && known_type(type);
}

bool known_activation(int activation) { return activation >= DGSP_ACT_SILU && activation <= DGSP_ACT_RELU; }

bool enough(const void* workspace, int64_t bytes, int64_t need) { return need == 0 || (workspace && aligned(workspace, 16) && bytes >= need); }

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
// float matrices 128.
Cut cut(int64_t m, int64_t n, int64_t depth, int terms, int batch, int type, bool dual, bool may_split) {
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
    if (splits && count > 0 && count < kCus) {               // no tiles: a batch without rows
        const int64_t most = std::min<int64_t>(ceil_div((c.size == kMiddle ? 2 : 3) * kCus, count), depth / (type == DGSP_F32 ? 128 : 256));
        c.split_depth = padded(ceil_div(depth, most), kDepth);
        c.splits = (int)ceil_div(depth, c.split_depth);
    }
    return c;
}

bool launchable(const Cut& c, int batch) { return c.groups(batch) < (1LL << 32) / 512; }

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

int64_t partial_bytes(const Cut& c, int64_t m, int64_t n, int batch) {
    return c.splits > 1 ? (int64_t)c.splits * batch * m * padded(n, 4) * 4 : 0;
}

template <typename T, bool kDual, bool kARows, bool kBRows, typename Out>
void launch(const Cut& c, const ProductArgs<T>& args, const Out& out, hipStream_t stream) {
    const auto groups = (unsigned)c.groups(args.batch);
    if constexpr (sizeof(T) == 4) {
        if (c.size == kMiddle)
            float_tile_kernel<Middle<kDual>, kARows, kBRows, Out><<<groups, Middle<kDual>::kThreads, 0, stream>>>(args, out);
        else
            float_tile_kernel<Small<kDual>, kARows, kBRows, Out><<<groups, Small<kDual>::kThreads, 0, stream>>>(args, out);
    } else if (c.size == kLarge) {
        tile_kernel<T, Large<kDual>, kARows, kBRows, Out><<<groups, Large<kDual>::kThreads, 0, stream>>>(args, out);
    } else if (c.size == kMiddle) {
        tile_kernel<T, Middle<kDual>, kARows, kBRows, Out><<<groups, Middle<kDual>::kThreads, 0, stream>>>(args, out);
    } else {
        tile_kernel<T, Small<kDual>, kARows, kBRows, Out><<<groups, Small<kDual>::kThreads, 0, stream>>>(args, out);
    }
}

// c[0 ... batch - 1] = the product
template <typename T, bool kARows, bool kBRows>
void product(const Cut& c, const ProductArgs<T>& args, ProductOut<T> out, void* partial, hipStream_t stream) {
    if (args.m == 0) return;
    out.vectors = out.ld % 4 == 0 && aligned(out.c[0], 4 * sizeof(T)) && (args.batch < 2 || aligned(out.c[1], 4 * sizeof(T)));
    out.partial = c.splits > 1 ? static_cast<float*>(partial) : nullptr;
    launch<T, false, kARows, kBRows>(c, args, out, stream);
    if (c.splits > 1) {
        const int64_t quads = args.batch * args.m * ceil_div(args.n, 4);
        join_kernel<T><<<(unsigned)std::min<int64_t>(ceil_div(quads, 256), 4096), 256, 0, stream>>>(args.m, args.n, args.batch, c.splits, out.partial, out);
    }
}

// ---------------------------------------------------------------- operands

int64_t kept_bytes(int64_t rows, int64_t cols, int type) { return rows * padded(cols, 8) * element_bytes(type); }

// what a matrix that does not lie as the products read it takes; float matrices are read as they lie
int64_t laid_out_bytes(int64_t rows, int64_t cols, int type) { return type == DGSP_F32 ? 0 : kept_bytes(rows, cols, type); }

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

// what the forward pass leaves: act(g) and u act'(g) in 32 bits, and h
struct Saved {
    void *act, *mul, *h;
    Saved(Pieces& pieces, int64_t rows, int64_t hidden, int type)
        : act(pieces.take(kept_bytes(rows, hidden, DGSP_F32))), mul(pieces.take(kept_bytes(rows, hidden, DGSP_F32))),
          h(pieces.take(kept_bytes(rows, hidden, type))) {}
};

struct ForwardPieces {
    Cut up, down;
    void *x, *gate, *up_weight, *down_weight, *h, *partial;
    ForwardPieces(Pieces& pieces, int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type)
        : up(cut(rows, hidden, width, 1, 1, type, true, true)), down(cut(rows, out_width, hidden, 1, 1, type, false, true)),
          x(pieces.take(laid_out_bytes(rows, width, type))), gate(pieces.take(laid_out_bytes(hidden, width, type))),
          up_weight(pieces.take(laid_out_bytes(hidden, width, type))), down_weight(pieces.take(laid_out_bytes(out_width, hidden, type))),
          h(pieces.take(kept_bytes(rows, hidden, type))),
          partial(pieces.take(std::max(partial_bytes(up, rows, padded(hidden, 8), 2), partial_bytes(down, rows, out_width, 1)))) {}
};

struct BackwardPieces {
    Cut slope, dx, gates, down;
    void *x, *gate, *up_weight, *down_weight, *dy, *dg, *du, *partial;
    BackwardPieces(Pieces& pieces, int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type, int batch)
        : slope(cut(rows, hidden, out_width, 1, 1, type, false, false)), dx(cut(rows, width, hidden, 2, 1, type, false, true)),
          gates(cut(hidden, width, rows, 1, batch, type, false, true)), down(cut(out_width, hidden, rows, 1, 1, type, false, true)),
          x(pieces.take(laid_out_bytes(rows, width, type))), gate(pieces.take(laid_out_bytes(hidden, width, type))),
          up_weight(pieces.take(laid_out_bytes(hidden, width, type))), down_weight(pieces.take(laid_out_bytes(out_width, hidden, type))),
          dy(pieces.take(laid_out_bytes(rows, out_width, type))), dg(pieces.take(kept_bytes(rows, hidden, type))),
          du(pieces.take(kept_bytes(rows, hidden, type))),
          partial(pieces.take(std::max({partial_bytes(dx, rows, width, 1), partial_bytes(gates, hidden, width, batch),
                                        partial_bytes(down, out_width, hidden, 1)}))) {}
};

}  // namespace

extern "C" int64_t dgsp_gated_ff_saved_bytes(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type) {
    if (!gated_extents(rows, width, hidden, out_width, type) || narrow_fits(width, hidden, out_width, type)) return 0;
    Pieces pieces(nullptr);
    Saved saved(pieces, rows, hidden, type);
    return pieces.used();
}

extern "C" int64_t dgsp_gated_ff_workspace_bytes(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type) {
    if (!gated_extents(rows, width, hidden, out_width, type) || narrow_fits(width, hidden, out_width, type)) return 0;
    Pieces pieces(nullptr);
    ForwardPieces need(pieces, rows, width, hidden, out_width, type);
    return pieces.used();
}

extern "C" int64_t dgsp_gated_ff_backward_workspace_bytes(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type) {
    if (!gated_extents(rows, width, hidden, out_width, type)) return 0;
    if (narrow_fits(width, hidden, out_width, type)) return narrow_backward_bytes(rows, width, hidden, out_width);
    Pieces one(nullptr), two(nullptr);
    BackwardPieces need_one(one, rows, width, hidden, out_width, type, 1), need_two(two, rows, width, hidden, out_width, type, 2);
    return std::max(one.used(), two.used());
}

extern "C" int dgsp_gated_ff(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type, int activation, const void* x,
                             int64_t ldx, const void* w_gate, int64_t ldg, const void* w_up, int64_t ldu, const void* w_down, int64_t ldd,
                             void* y, int64_t ldy, void* saved, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!gated_extents(rows, width, hidden, out_width, type) || !known_activation(activation)) return DGSP_ERR_INVALID_ARG;
    if (rows == 0) return DGSP_OK;
    if (!readable(x, rows, width, ldx) || !readable(w_gate, hidden, width, ldg) || !readable(w_up, hidden, width, ldu) ||
        !readable(w_down, out_width, hidden, ldd) || !writable(y, rows, out_width, ldy) || !aligned(saved, 16) ||
        !enough(workspace, workspace_bytes, dgsp_gated_ff_workspace_bytes(rows, width, hidden, out_width, type)))
        return DGSP_ERR_INVALID_ARG;
    if (narrow_fits(width, hidden, out_width, type))
        return narrow_forward({rows, width, hidden, out_width, type, activation, x, ldx, w_gate, ldg, w_up, ldu, w_down, ldd, y, ldy}, stream);
    Pieces pieces(workspace), kept_pieces(saved);
    const ForwardPieces at(pieces, rows, width, hidden, out_width, type);
    const Saved keep(kept_pieces, rows, hidden, type);
    if (!launchable(at.up, 1) || !launchable(at.down, 1)) return DGSP_ERR_UNSUPPORTED;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        const auto on = static_cast<hipStream_t>(stream);
        const Kept<T> h = kept<T>(saved ? keep.h : at.h, hidden);
        Operands<T> operands;
        ProductArgs<T> up = product_args<T>(at.up, rows, hidden, width, 1), down = product_args<T>(at.down, rows, out_width, hidden, 1);
        up.a[0] = operands.add(x, rows, width, ldx, at.x);
        up.b[0] = operands.add(w_gate, hidden, width, ldg, at.gate);
        up.b[1] = operands.add(w_up, hidden, width, ldu, at.up_weight);
        down.a[0] = source(h, rows);
        down.b[0] = operands.add(w_down, out_width, hidden, ldd, at.down_weight);
        operands.launch(on);
        const GatedUpOut<T> out{h, saved ? static_cast<float*>(keep.act) : nullptr, saved ? static_cast<float*>(keep.mul) : nullptr, activation,
                                at.up.splits > 1 ? static_cast<float*>(at.partial) : nullptr};
        launch<T, true, true, true>(at.up, up, out, on);
        if (out.partial)
            gated_join_kernel<T><<<(unsigned)std::min<int64_t>(ceil_div(rows * h.ld / 4, 256), 4096), 256, 0, on>>>(rows, at.up.splits, out);
        product<T, true, true>(at.down, down, {{static_cast<T*>(y), nullptr}, ldy, false, nullptr}, at.partial, on);
        return launched();
    });
}

extern "C" int dgsp_gated_ff_backward(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type, int activation,
                                      const void* x, int64_t ldx, const void* w_gate, int64_t ldg, const void* w_up, int64_t ldu,
                                      const void* w_down, int64_t ldd, const void* dy, int64_t lddy, const void* saved, void* dx,
                                      void* dw_gate, void* dw_up, void* dw_down, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!gated_extents(rows, width, hidden, out_width, type) || !known_activation(activation) ||
        !enough(workspace, workspace_bytes, dgsp_gated_ff_backward_workspace_bytes(rows, width, hidden, out_width, type)))
        return DGSP_ERR_INVALID_ARG;
    const bool narrow = narrow_fits(width, hidden, out_width, type);
    if (rows > 0 && (!readable(x, rows, width, ldx) || !readable(w_gate, hidden, width, ldg) || !readable(w_up, hidden, width, ldu) ||
                     !readable(w_down, out_width, hidden, ldd) || !readable(dy, rows, out_width, lddy) || (!saved && !narrow) || !aligned(saved, 16)))
        return DGSP_ERR_INVALID_ARG;
    if (narrow)
        return narrow_backward({rows, width, hidden, out_width, type, activation, x, ldx, w_gate, ldg, w_up, ldu, w_down, ldd, nullptr, 0, dy, lddy, dx,
                                dw_gate, dw_up, dw_down, workspace}, stream);
    const int batch = dw_gate && dw_up ? 2 : 1;
    Pieces pieces(workspace), kept_pieces(const_cast<void*>(saved));
    const BackwardPieces at(pieces, rows, width, hidden, out_width, type, batch);
    const Saved keep(kept_pieces, rows, hidden, type);
    if (!launchable(at.slope, 1) || !launchable(at.dx, 1) || !launchable(at.gates, batch) || !launchable(at.down, 1))
        return DGSP_ERR_UNSUPPORTED;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        const auto on = static_cast<hipStream_t>(stream);
        const bool gates = (dx || dw_gate || dw_up) && rows > 0;
        Operands<T> operands;
        Source<T> in{}, gate{}, up{}, down{};
        const Source<T> grad = operands.add(dy, rows, out_width, lddy, at.dy);
        if (dw_gate || dw_up) in = operands.add(x, rows, width, ldx, at.x);
        if (dx) {                                       // a pair's operands lie alike
            const bool alike = ldg == ldu && operands.in_place(w_gate, hidden, width, ldg) && operands.in_place(w_up, hidden, width, ldu);
            gate = operands.add(w_gate, hidden, width, ldg, at.gate, sizeof(T) == 2 && !alike);
            up = operands.add(w_up, hidden, width, ldu, at.up_weight, sizeof(T) == 2 && !alike);
        }
        if (gates) down = operands.add(w_down, out_width, hidden, ldd, at.down_weight);
        operands.launch(on);
        const Kept<T> dg = kept<T>(at.dg, hidden), du = kept<T>(at.du, hidden), h = kept<T>(keep.h, hidden);
        if (gates) {
            ProductArgs<T> args = product_args<T>(at.slope, rows, hidden, out_width, 1);
            args.a[0] = grad;
            args.b[0] = down;
            launch<T, false, true, false>(at.slope, args,
                                          GatedSlopeOut<T>{static_cast<const float*>(keep.act), static_cast<const float*>(keep.mul), dg, du}, on);
        }
        if (dx) {
            ProductArgs<T> args = product_args<T>(at.dx, rows, width, hidden, 1);
            args.pairs = 2;
            args.a[0] = source(dg, rows);
            args.a[1] = source(du, rows);
            args.b[0] = gate;
            args.b[1] = up;
            product<T, true, false>(at.dx, args, {{static_cast<T*>(dx), nullptr}, width, false, nullptr}, at.partial, on);
        }
        if (dw_gate || dw_up) {
            ProductArgs<T> args = product_args<T>(at.gates, hidden, width, rows, batch);
            args.a[0] = source(dw_gate ? dg : du, rows);
            args.a[1] = source(du, rows);
            args.b[0] = in;
            product<T, false, false>(at.gates, args, {{static_cast<T*>(dw_gate ? dw_gate : dw_up), static_cast<T*>(dw_up)}, width, false, nullptr},
                                     at.partial, on);
        }
        if (dw_down) {
            ProductArgs<T> args = product_args<T>(at.down, out_width, hidden, rows, 1);
            args.a[0] = grad;
            args.b[0] = source(h, rows);
            product<T, false, false>(at.down, args, {{static_cast<T*>(dw_down), nullptr}, hidden, false, nullptr}, at.partial, on);
        }
        return launched();
    });
}
