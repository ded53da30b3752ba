// Host side of the matrix product with its epilogue: argument checks, products and launches.  The C-ABI is documented in include/dgsp_layers.h.
#include "column_sums.hpp"
#include "few_rows_kernels.hpp"
#include "linear_host.hpp"
#include "narrow_linear.hpp"
#include "rows8_host.hpp"

namespace {

using namespace dgsp;

bool linear_extents(int64_t rows, int64_t width, int64_t out_width, int type) {
    return rows >= 0 && rows <= kMostRows && width >= 1 && width <= kMostWidth && out_width >= 1 && out_width <= kMostWidth && known_type(type);
}

// Products of few rows take kernels of their own, that need no workspace.
bool few_rows(int64_t rows, int64_t width, int64_t out_width, int type) {
    return type != DGSP_F32 && dgsp::few_rows(rows, width, out_width, 2);
}

bool known_epilogue(int activation) { return known_activation(activation) || activation == DGSP_ACT_NONE; }
bool known_keep(int keep) { return keep >= DGSP_KEEP_NOTHING && keep <= DGSP_KEEP_8BIT; }

// what the forward pass leaves of z: nothing, the slope in 8 bits, or z
enum Left { kNothing, kCodes, kZ };
Left left(int activation, int keep) {
    if (activation == DGSP_ACT_NONE || keep == DGSP_KEEP_NOTHING) return kNothing;
    return activation == DGSP_ACT_RELU || keep == DGSP_KEEP_8BIT ? kCodes : kZ;
}

struct ForwardPieces {
    Cut up;
    void *x, *weight, *partial;
    ForwardPieces(Pieces& pieces, int64_t rows, int64_t width, int64_t out_width, int type)
        : up(cut_to_fill(rows, out_width, width, type, rows <= 64 ? 2 * kCus : kCus)), x(pieces.take(laid_out_bytes(rows, width, type))),
          weight(pieces.take(laid_out_bytes(out_width, width, type))), partial(pieces.take(partial_bytes(up, rows, out_width, 1))) {}
};

// How the rows are dealt out for dz and the sums over them.
struct Slices {
    int lanes;
    int64_t across, down;       // workgroups along a row, along the rows
    Slices(int64_t rows, int64_t columns) {
        const int64_t chunks = ceil_div(columns, kChunk);
        lanes = 1;
        while (lanes < chunks && lanes < 256) lanes *= 2;
        across = ceil_div(chunks, lanes);
        down = std::max<int64_t>(1, std::min(ceil_div(rows, (256 / lanes) * 4), ceil_div(8 * kCus, across)));
    }
};

struct BackwardPieces {
    Cut dx, dw;
    Slices slices;
    void *x, *weight, *dz, *partial, *sums;
    BackwardPieces(Pieces& pieces, int64_t rows, int64_t width, int64_t out_width, int type, int activation, int keep)
        : dx(cut_to_fill(rows, width, out_width, type)), dw(cut_to_fill(out_width, width, rows, type)), slices(rows, out_width),
          x(pieces.take(keep == DGSP_KEEP_8BIT && type != DGSP_F32 ? kept_bytes(rows, width, type) : laid_out_bytes(rows, width, type))),
          weight(pieces.take(laid_out_bytes(out_width, width, type))),
          dz(pieces.take(activation != DGSP_ACT_NONE ? kept_bytes(rows, out_width, type) : laid_out_bytes(rows, out_width, type))),
          partial(pieces.take(std::max(partial_bytes(dx, rows, width, 1), partial_bytes(dw, out_width, width, 1)))),
          sums(pieces.take(std::max<int64_t>(slices.down, type == DGSP_F32 ? dw.splits : 0) * out_width * 4)) {}
};

}  // namespace

extern "C" int64_t dgsp_linear_saved_bytes(int64_t rows, int64_t out_width, int type, int bias_type, int activation, int keep) {
    if (!linear_extents(rows, 1, out_width, type) || (bias_type != type && bias_type != DGSP_F32) || !known_epilogue(activation) || !known_keep(keep)) return 0;
    const Left what = left(activation, keep);
    return what == kNothing ? 0 : what == kCodes ? rows * padded(out_width, 8) : kept_bytes(rows, out_width, bias_type);
}

extern "C" int64_t dgsp_linear_workspace_bytes(int64_t rows, int64_t width, int64_t out_width, int type) {
    if (!linear_extents(rows, width, out_width, type) || narrow_linear_fits(width, out_width, type) || few_rows(rows, width, out_width, type)) return 0;
    Pieces pieces(nullptr);
    ForwardPieces need(pieces, rows, width, out_width, type);
    return pieces.used();
}

extern "C" int64_t dgsp_linear_backward_workspace_bytes(int64_t rows, int64_t width, int64_t out_width, int type, int activation, int keep) {
    if (!linear_extents(rows, width, out_width, type) || !known_epilogue(activation) || !known_keep(keep)) return 0;
    if (narrow_linear_fits(width, out_width, type)) return narrow_linear_backward_bytes(rows, width, out_width, type, keep == DGSP_KEEP_8BIT);
    Pieces pieces(nullptr);
    BackwardPieces need(pieces, rows, width, out_width, type, activation, keep);
    return pieces.used();
}

extern "C" int dgsp_linear(int64_t rows, int64_t width, int64_t out_width, int type, int bias_type, int activation, int keep, const void* x,
                           int64_t ldx, const void* weight, int64_t ldw, const void* bias, const void* residual, int64_t ldr, void* y,
                           int64_t ldy, void* saved, void* x_values, int64_t ldv, void* x_scales, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!linear_extents(rows, width, out_width, type) || !known_epilogue(activation) || !known_keep(keep) ||
        (bias_type != type && bias_type != DGSP_F32))
        return DGSP_ERR_INVALID_ARG;
    if (rows == 0) return DGSP_OK;
    const Left what = left(activation, keep);
    if (!readable(x, rows, width, ldx) || !readable(weight, out_width, width, ldw) || (residual && !readable(residual, rows, out_width, ldr)) ||
        !writable(y, rows, out_width, ldy) || (what != kNothing && !saved) || !aligned(saved, 16) ||
        (x_values && (keep != DGSP_KEEP_8BIT || !rows8_lies(x_values, rows, width, ldv, x_scales) || (rows > 1 && ldv < rows8_bytes(width)))) ||
        !enough(workspace, workspace_bytes, dgsp_linear_workspace_bytes(rows, width, out_width, type)))
        return DGSP_ERR_INVALID_ARG;
    if (narrow_linear_fits(width, out_width, type)) {
        return with_type(type, [&](auto element) {
            using T = decltype(element);
            return narrow_linear<T>({rows, width, out_width, activation, static_cast<const T*>(x), static_cast<const T*>(weight), ldx, ldw, bias, bias_type != type,
                                     static_cast<const T*>(residual), ldr, static_cast<T*>(y), ldy, what == kZ ? saved : nullptr,
                                     what == kCodes ? static_cast<uint8_t*>(saved) : nullptr, padded(out_width, 8),
                                     x_values ? rows8(x_values, rows, width, ldv, x_scales) : Rows8{}, scale_range(DGSP_INT8, type)},
                                    static_cast<hipStream_t>(stream));
        });
    }
    if (few_rows(rows, width, out_width, type)) {
        const auto call = [&](auto element) {
            using T = decltype(element);
            const auto on = static_cast<hipStream_t>(stream);
            const LinearOut<T> out = linear_out<T>(y, ldy, bias, bias_type != type, residual, ldr, activation, what == kZ ? saved : nullptr,
                                                   what == kCodes ? saved : nullptr, out_width, nullptr);
            const FewRowsArgs<T> args{rows, width, out_width, static_cast<const T*>(x), static_cast<const T*>(weight), rows == 1 ? 0 : ldx, out_width == 1 ? 0 : ldw};
            with_few_rows(rows, out_width, false, [&](auto sets, auto outs, auto waves) {
                constexpr int kSets = decltype(sets)::value, kOuts = decltype(outs)::value, kWaves = decltype(waves)::value;
                few_rows_kernel<T, kSets, kOuts, kWaves><<<(unsigned)ceil_div(out_width, 16 * kOuts), 64 * kWaves, 0, on>>>(args, out);
            });
            if (x_values) launch_quantise<T>(DGSP_INT8, rows, width, static_cast<const T*>(x), ldx, rows8(x_values, rows, width, ldv, x_scales), on);
            return launched();
        };
        return type == DGSP_BF16 ? call(bf16_t{}) : call(f16_t{});
    }
    Pieces pieces(workspace);
    const ForwardPieces at(pieces, rows, width, out_width, type);
    if (!launchable(at.up, 1)) return DGSP_ERR_UNSUPPORTED;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        const auto on = static_cast<hipStream_t>(stream);
        Operands<T> operands;
        ProductArgs<T> args = product_args<T>(at.up, rows, out_width, width, 1);
        args.a[0] = operands.add(x, rows, width, ldx, at.x);
        args.b[0] = operands.add(weight, out_width, width, ldw, at.weight);
        operands.launch(on);
        const LinearOut<T> out = linear_out<T>(y, ldy, bias, bias_type != type, residual, ldr, activation, what == kZ ? saved : nullptr,
                                               what == kCodes ? saved : nullptr, out_width, at.up.splits > 1 ? at.partial : nullptr);
        launch<T, false, true, true>(at.up, args, out, on);
        if (x_values) launch_quantise<T>(DGSP_INT8, rows, width, static_cast<const T*>(x), ldx, rows8(x_values, rows, width, ldv, x_scales), on);
        if (out.partial)
            linear_join_kernel<<<(unsigned)std::min<int64_t>(ceil_div(rows * ceil_div(out_width, 4), 256), 4096), 256, 0, on>>>(rows, out_width, at.up.splits, out);
        return launched();
    });
}

extern "C" int dgsp_linear_backward(int64_t rows, int64_t width, int64_t out_width, int type, int bias_type, int activation, int keep,
                                    const void* x, int64_t ldx, const void* x_scales, const void* weight, int64_t ldw, const void* saved,
                                    const void* dy, int64_t lddy, void* dx, void* dweight, void* dbias, void* workspace, int64_t workspace_bytes,
                                    void* stream) {
    if (!linear_extents(rows, width, out_width, type) || !known_epilogue(activation) || !known_keep(keep) || keep == DGSP_KEEP_NOTHING ||
        (bias_type != type && bias_type != DGSP_F32) ||
        !enough(workspace, workspace_bytes, dgsp_linear_backward_workspace_bytes(rows, width, out_width, type, activation, keep)))
        return DGSP_ERR_INVALID_ARG;
    const bool in_8bit = keep == DGSP_KEEP_8BIT;
    const Left what = left(activation, keep);
    if (rows > 0 && (!readable(dy, rows, out_width, lddy) || (what != kNothing && !saved) || !aligned(saved, 16) ||
                     (dx && !readable(weight, out_width, width, ldw)) ||
                     (dweight && !(in_8bit ? rows8_lies(x, rows, width, ldx, x_scales) : readable(x, rows, width, ldx)))))
        return DGSP_ERR_INVALID_ARG;
    if (narrow_linear_fits(width, out_width, type)) {
        if (!dx && !dweight && !dbias) return DGSP_OK;
        return with_type(type, [&](auto element) {
            using T = decltype(element);
            return narrow_linear_backward<T>({rows, width, out_width, activation, in_8bit ? nullptr : static_cast<const T*>(x), static_cast<const T*>(weight),
                                              static_cast<const T*>(dy), ldx, ldw, lddy, what == kZ ? saved : nullptr, bias_type != type,
                                              what == kCodes ? static_cast<const uint8_t*>(saved) : nullptr, padded(out_width, 8),
                                              in_8bit && dweight ? rows8(const_cast<void*>(x), rows, width, ldx, const_cast<void*>(x_scales)) : Rows8{},
                                              static_cast<T*>(dx), nullptr, nullptr},
                                             in_8bit, dweight, dbias, bias_type != type, workspace, static_cast<hipStream_t>(stream));
        });
    }
    Pieces pieces(workspace);
    const BackwardPieces at(pieces, rows, width, out_width, type, activation, keep);
    if (!launchable(at.dx, 1) || !launchable(at.dw, 1)) return DGSP_ERR_UNSUPPORTED;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        const auto on = static_cast<hipStream_t>(stream);
        const Slices& slices = at.slices;
        const int64_t kept_ld = padded(out_width, 8);
        Operands<T> operands;
        Source<T> grad{}, in{}, w{};
        if (activation == DGSP_ACT_NONE)
            grad = operands.add(dy, rows, out_width, lddy, at.dz);
        else
            grad = {static_cast<const T*>(at.dz), rows, kept_ld, kept_ld};
        constexpr bool kFloat = sizeof(T) == 4;
        Rows8 x8{};
        if (dweight && in_8bit) x8 = rows8(const_cast<void*>(x), rows, width, ldx, const_cast<void*>(x_scales));
        if (dweight && in_8bit && !kFloat) {
            const int64_t ld = padded(width, 8);
            if (rows > 0)
                launch_dequantise<T>(DGSP_INT8, rows, width, x8, static_cast<T*>(at.x), ld, on);
            in = {static_cast<const T*>(at.x), rows, ld, ld};
        } else if (dweight && !in_8bit) {
            in = operands.add(x, rows, width, ldx, at.x);
        }
        if (dx) w = operands.add(weight, out_width, width, ldw, at.weight);
        operands.launch(on);
        // the sums over the rows: with dz, or with the weight's gradient, or on their own
        const bool sums_beside = kFloat && activation == DGSP_ACT_NONE && dweight && dbias;
        if (rows > 0 && (activation != DGSP_ACT_NONE ? dx || dweight || dbias : dbias && !sums_beside)) {
            const LinearSlopeArgs<T> args{rows, out_width, slices.lanes, static_cast<const T*>(dy), lddy, what == kZ ? saved : nullptr, bias_type != type,
                                          what == kCodes ? static_cast<const uint8_t*>(saved) : nullptr, kept_ld, activation,
                                          activation != DGSP_ACT_NONE && (dx || dweight) ? static_cast<T*>(at.dz) : nullptr,
                                          dbias ? static_cast<float*>(at.sums) : nullptr};
            linear_slope_kernel<T><<<dim3((unsigned)slices.across, (unsigned)slices.down), 256, 0, on>>>(args);
        }
        if (dx) {
            ProductArgs<T> args = product_args<T>(at.dx, rows, width, out_width, 1);
            args.a[0] = grad;
            args.b[0] = w;
            product<T, true, false>(at.dx, args, {{static_cast<T*>(dx), nullptr}, width, false, nullptr}, at.partial, on);
        }
        if (dweight) {
            ProductArgs<T> args = product_args<T>(at.dw, out_width, width, rows, 1);
            args.a[0] = grad;
            args.b[0] = in;
            const ProductOut<T> out{{static_cast<T*>(dweight), nullptr}, width, false, nullptr};
            if constexpr (kFloat)
                weight_gradient(at.dw, args, in_8bit ? &x8 : nullptr, sums_beside ? static_cast<float*>(at.sums) : nullptr, out, at.partial, on);
            else
                product<T, false, false>(at.dw, args, out, at.partial, on);
        }
        if (dbias) launch_column_sums<T>(out_width, rows == 0 ? 0 : sums_beside ? at.dw.splits : slices.down, static_cast<const float*>(at.sums), dbias, bias_type != type, on);
        return launched();
    });
}
