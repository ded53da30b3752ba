// Host side of the gated feed-forward block: argument checks, products and launches.  The C-ABI is
// documented in include/dgsp_layers.h.
#include "gated_ff_kernels.hpp"
#include "narrow_ff.hpp"
#include "products.hpp"

namespace {

using namespace dgsp;

bool gated_extents(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type) {
    return rows >= 0 && rows <= kMostRows && width >= 1 && width <= kMostWidth && hidden >= 1 && hidden <= kMostWidth &&
           out_width >= 1 && out_width <= kMostWidth && known_type(type);
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
