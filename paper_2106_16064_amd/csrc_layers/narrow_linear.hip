// Launches of the matrix product with its epilogue where the weight fits LDS.
#include "narrow_linear.hpp"

#include "column_sums.hpp"
#include "layers_host.hpp"

namespace dgsp {

namespace {

int padded_width(int64_t n) { return n <= 32 ? 32 : n <= 64 ? 64 : 128; }

template <typename F>
void with_width(int64_t width, F&& f) {
    switch (padded_width(width)) {
        case 32: return f(std::integral_constant<int, 32>{});
        case 64: return f(std::integral_constant<int, 64>{});
        default: return f(std::integral_constant<int, 128>{});
    }
}

template <typename F>
void with_flags(bool first, bool second, F&& f) {
    if (first)
        second ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
    else
        second ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}

// workgroups of the backward pass: as many as are resident together
int64_t backward_groups(int64_t rows, int64_t width, int64_t out_width) {
    int64_t a_cu = 1;
    with_width(width, [&](auto p) {
        with_width(out_width, [&](auto o) { a_cu = std::min<int64_t>(2, 163840 / (NarrowShare<decltype(p)::value, decltype(o)::value>::kLds + 4096)); });
    });
    return std::max<int64_t>(1, std::min(ceil_div(rows, kNarrowTile), kCus * a_cu));
}

int64_t parts(int64_t width) { return padded_width(width) == 32 ? 2 : 1; }

}  // namespace

bool narrow_linear_fits(int64_t width, int64_t out_width, int type) { return type != DGSP_F32 && width <= 128 && out_width <= 128; }

template <typename E>
int narrow_linear(const NarrowLinearArgs<E>& args, hipStream_t stream) {
    with_width(args.width, [&](auto p) {
        with_width(args.out_width, [&](auto o) {
            constexpr int kP = decltype(p)::value, kO = decltype(o)::value;
            const auto groups = (unsigned)std::min<int64_t>(ceil_div(args.rows, 64), kCus * (kP * kO > 64 * 64 ? 3 : 4));
            with_flags(args.x8.values != nullptr, args.width == kP && args.out_width == kO, [&](auto x8, auto whole) {
                narrow_linear_kernel<E, kP, kO, decltype(x8)::value, decltype(whole)::value><<<groups, 256, 0, stream>>>(args);
            });
        });
    });
    return launched();
}

int64_t narrow_linear_backward_bytes(int64_t rows, int64_t width, int64_t out_width) {
    return backward_groups(rows, width, out_width) * (parts(width) * out_width * width + out_width) * 4;
}

template <typename E>
int narrow_linear_backward(NarrowLinearBackwardArgs<E> args, void* dweight, void* dbias, bool wide, void* workspace, hipStream_t stream) {
    const int64_t groups = backward_groups(args.rows, args.width, args.out_width), weight_groups = groups * parts(args.width);
    float* const sums = static_cast<float*>(workspace);
    args.weight_sums = dweight ? sums : nullptr;
    args.bias_sums = dbias ? sums + weight_groups * args.out_width * args.width : nullptr;
    if (args.rows > 0)
        with_width(args.width, [&](auto p) {
            with_width(args.out_width, [&](auto o) {
                constexpr int kP = decltype(p)::value, kO = decltype(o)::value;
                with_flags(args.x8.values != nullptr, args.width == kP && args.out_width == kO, [&](auto x8, auto whole) {
                    narrow_linear_backward_kernel<E, kP, kO, decltype(x8)::value, decltype(whole)::value>
                        <<<(unsigned)groups, 64 * kNarrowWaves, 0, stream>>>(args);
                });
            });
        });
    if (dweight) launch_column_sums<E>(args.out_width * args.width, args.rows > 0 ? weight_groups : 0, args.weight_sums, dweight, false, stream);
    if (dbias) launch_column_sums<E>(args.out_width, args.rows > 0 ? groups : 0, args.bias_sums, dbias, wide, stream);
    return launched();
}

template int narrow_linear<bf16_t>(const NarrowLinearArgs<bf16_t>&, hipStream_t);
template int narrow_linear<f16_t>(const NarrowLinearArgs<f16_t>&, hipStream_t);
template int narrow_linear_backward<bf16_t>(NarrowLinearBackwardArgs<bf16_t>, void*, void*, bool, void*, hipStream_t);
template int narrow_linear_backward<f16_t>(NarrowLinearBackwardArgs<f16_t>, void*, void*, bool, void*, hipStream_t);

}  // namespace dgsp
