// Host side of the matrix product of rows in 8 bits: argument checks and launches.  The C-ABI is documented in include/dgsp_layers.h.
#include "few_rows_kernels.hpp"
#include "linear_host.hpp"
#include "rows8_host.hpp"
#include "tiles_8bit.hpp"

namespace {

using namespace dgsp;

constexpr int64_t kMostLd = 2 * kMostWidth;             // 256 rows of it span less than 2^31 bytes

bool extents(int64_t rows, int64_t width, int64_t out_width) {
    return rows >= 0 && rows <= kMostRows && width >= 1 && width <= kMostWidth && out_width >= 1 && out_width <= kMostWidth;
}

// a product of pairs of elements
Cut cut8(int64_t rows, int64_t width, int64_t out_width) { return cut_to_fill(rows, out_width, rows8_bytes(width) / 2, DGSP_BF16); }

Source<Pair8> source8(const void* values, int64_t rows, int64_t width, int64_t ld) {
    const int64_t pairs = rows8_bytes(width) / 2;
    return {static_cast<const Pair8*>(values), rows, pairs, rows == 1 ? pairs : ld / 2};
}

template <typename Out>
void launch8(const Cut& c, const ProductArgs<Pair8>& args, const Scales8& scales, const Out& out, hipStream_t stream) {
    const auto groups = (unsigned)c.groups(1);
    if (c.size == kLarge)
        product_8bit_kernel<Large<false>, Out><<<groups, Large<false>::kThreads, 0, stream>>>(args, scales, out);
    else if (c.size == kMiddle)
        product_8bit_kernel<Middle<false>, Out><<<groups, Middle<false>::kThreads, 0, stream>>>(args, scales, out);
    else
        product_8bit_kernel<Small<false>, Out><<<groups, Small<false>::kThreads, 0, stream>>>(args, scales, out);
}

}  // namespace

extern "C" int64_t dgsp_linear_8bit_workspace_bytes(int64_t rows, int64_t width, int64_t out_width) {
    if (!extents(rows, width, out_width) || few_rows(rows, width, out_width, 1)) return 0;
    return partial_bytes(cut8(rows, width, out_width), rows, out_width, 1);
}

extern "C" int dgsp_linear_8bit(int64_t rows, int64_t width, int64_t out_width, int type, int bias_type, int activation, const void* x, int64_t ldx,
                                const void* x_scales, const void* weight, int64_t ldw, const void* weight_scales, const void* bias,
                                const void* residual, int64_t ldr, void* y, int64_t ldy, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!extents(rows, width, out_width) || !known_type(type) || (bias_type != type && bias_type != DGSP_F32) ||
        !(known_activation(activation) || activation == DGSP_ACT_NONE))
        return DGSP_ERR_INVALID_ARG;
    if (rows == 0) return DGSP_OK;
    if (!rows8_lies(x, rows, width, ldx, x_scales) || !rows8_lies(weight, out_width, width, ldw, weight_scales) || (rows > 1 && ldx > kMostLd) ||
        (out_width > 1 && ldw > kMostLd) || (residual && !readable(residual, rows, out_width, ldr)) || !writable(y, rows, out_width, ldy) ||
        !enough(workspace, workspace_bytes, dgsp_linear_8bit_workspace_bytes(rows, width, out_width)))
        return DGSP_ERR_INVALID_ARG;
    const Scales8 scales{static_cast<const uint8_t*>(x_scales), static_cast<const uint8_t*>(weight_scales), rows, out_width, ceil_div(width, 4 * kBlock)};
    if (few_rows(rows, width, out_width, 1))
        return with_type(type, [&](auto element) {
            using T = decltype(element);
            const LinearOut<T, false> out = linear_out<T, false>(y, ldy, bias, bias_type != type, residual, ldr, activation, nullptr, nullptr, out_width, nullptr);
            const FewRows8Args args{rows, rows8_bytes(width), out_width, static_cast<const uint8_t*>(x), static_cast<const uint8_t*>(weight), rows == 1 ? 0 : ldx,
                                    out_width == 1 ? 0 : ldw, scales};
            with_few_rows(rows, out_width, true, [&](auto sets, auto outs, auto waves) {
                constexpr int kSets = decltype(sets)::value, kOuts = decltype(outs)::value, kWaves = decltype(waves)::value;
                few_rows_8bit_kernel<T, kSets, kOuts, kWaves><<<(unsigned)ceil_div(out_width, 16 * kOuts), 64 * kWaves, 0, static_cast<hipStream_t>(stream)>>>(args, out);
            });
            return launched();
        });
    const Cut c = cut8(rows, width, out_width);
    if (!launchable(c, 1)) return DGSP_ERR_UNSUPPORTED;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        const auto on = static_cast<hipStream_t>(stream);
        ProductArgs<Pair8> args = product_args<Pair8>(c, rows, out_width, rows8_bytes(width) / 2, 1);
        args.a[0] = source8(x, rows, width, ldx);
        args.b[0] = source8(weight, out_width, width, ldw);
        const LinearOut<T, false> out = linear_out<T, false>(y, ldy, bias, bias_type != type, residual, ldr, activation, nullptr, nullptr, out_width,
                                               c.splits > 1 ? workspace : nullptr);
        launch8(c, args, scales, out, on);
        if (out.partial)
            linear_join_kernel<<<(unsigned)std::min<int64_t>(ceil_div(rows * ceil_div(out_width, 4), 256), 4096), 256, 0, on>>>(rows, out_width, c.splits, out);
        return launched();
    });
}
