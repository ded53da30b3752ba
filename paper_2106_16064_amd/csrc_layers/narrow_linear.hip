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

constexpr int kMostFloat = 64 * 128;            // of float weights, padded: three planes of it, and of rows, fill LDS

// f(padded width, padded out_width)
template <typename E, typename F>
void with_widths(int64_t width, int64_t out_width, F&& f) {
    with_width(width, [&](auto p) {
        with_width(out_width, [&](auto o) {
            if constexpr (sizeof(E) == 2 || decltype(p)::value * decltype(o)::value <= kMostFloat) f(p, o);
        });
    });
}

// Of the backward pass: workgroups, as many as are resident together, and the sums that each leaves.  `in_8bit`: x was kept so.
struct Backward {
    int64_t groups = 1, parts = 1;
    template <typename E>
    static Backward of(int64_t rows, int64_t width, int64_t out_width, bool in_8bit) {
        Backward b;
        with_widths<E>(width, out_width, [&](auto p, auto o) {
            constexpr int kP = decltype(p)::value, kO = decltype(o)::value;
            with_flags(in_8bit, width == kP && out_width == kO, [&](auto x8, auto whole) {
                using Share = NarrowShare<E, kP, kO, decltype(x8)::value, decltype(whole)::value>;
                b.groups = std::max<int64_t>(1, std::min(ceil_div(rows, Share::kTile), kCus * Share::kGroups));
                b.parts = Share::kParts;
            });
        });
        return b;
    }
};

}  // namespace

bool narrow_linear_fits(int64_t width, int64_t out_width, int type) { return width <= 128 && out_width <= 128 && (type != DGSP_F32 || padded_width(width) * padded_width(out_width) <= kMostFloat); }

template <typename E>
int narrow_linear(const NarrowLinearArgs<E>& args, hipStream_t stream) {
    with_widths<E>(args.width, args.out_width, [&](auto p, auto o) {
        constexpr int kP = decltype(p)::value, kO = decltype(o)::value;
        const auto groups = (unsigned)std::min<int64_t>(ceil_div(args.rows, 64), kCus * (kP * kO * kPlanes<E> > 64 * 64 ? 3 : 4));
        with_flags(args.x8.values != nullptr, args.width == kP && args.out_width == kO, [&](auto x8, auto whole) {
            narrow_linear_kernel<E, kP, kO, decltype(x8)::value, decltype(whole)::value><<<groups, 256, 0, stream>>>(args);
        });
    });
    return launched();
}

int64_t narrow_linear_backward_bytes(int64_t rows, int64_t width, int64_t out_width, int type, bool in_8bit) {
    const Backward b = type == DGSP_F32 ? Backward::of<float>(rows, width, out_width, in_8bit) : Backward::of<bf16_t>(rows, width, out_width, in_8bit);
    return b.groups * (b.parts * out_width * width + out_width) * 4;
}

template <typename E>
int narrow_linear_backward(NarrowLinearBackwardArgs<E> args, bool in_8bit, void* dweight, void* dbias, bool wide, void* workspace, hipStream_t stream) {
    const Backward b = Backward::of<E>(args.rows, args.width, args.out_width, in_8bit);
    float* const sums = static_cast<float*>(workspace);
    args.weight_sums = dweight ? sums : nullptr;
    args.bias_sums = dbias ? sums + b.groups * b.parts * args.out_width * args.width : nullptr;
    if (args.rows > 0)
        with_widths<E>(args.width, args.out_width, [&](auto p, auto o) {
            constexpr int kP = decltype(p)::value, kO = decltype(o)::value;
            with_flags(args.x8.values != nullptr, args.width == kP && args.out_width == kO, [&](auto x8, auto whole) {
                constexpr bool kX8 = decltype(x8)::value, kWhole = decltype(whole)::value;
                const dim3 groups((unsigned)b.groups), threads(64 * NarrowShare<E, kP, kO, kX8, kWhole>::kWaves);
                if constexpr (sizeof(E) == 2 && !kX8)
                    if (args.wide && args.z) return narrow_linear_backward_kernel<E, kP, kO, kX8, kWhole, float><<<groups, threads, 0, stream>>>(args);
                narrow_linear_backward_kernel<E, kP, kO, kX8, kWhole, E><<<groups, threads, 0, stream>>>(args);
            });
        });
    if (dweight) launch_column_sums<E>(args.out_width * args.width, args.rows > 0 ? b.groups * b.parts : 0, args.weight_sums, dweight, false, stream);
    if (dbias) launch_column_sums<E>(args.out_width, args.rows > 0 ? b.groups : 0, args.bias_sums, dbias, wide, stream);
    return launched();
}

#define NARROW(E)                                                            \
    template int narrow_linear<E>(const NarrowLinearArgs<E>&, hipStream_t); \
    template int narrow_linear_backward<E>(NarrowLinearBackwardArgs<E>, bool, void*, void*, bool, void*, hipStream_t);
NARROW(float)
NARROW(bf16_t)
NARROW(f16_t)
#undef NARROW

}  // namespace dgsp
