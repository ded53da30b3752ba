// The products whose results are written as they are.
#include "products.hpp"

namespace dgsp {

namespace {

// Fewer results than a quarter of the CUs take by join_kernel, and splits enough to be read side by side.
constexpr int64_t kMostDeep = 16384;
constexpr int kLeastDeep = 32;

template <typename T>
void into(ProductOut<T>& out, const Cut& c, const ProductArgs<T>& args, void* partial) {
    out.vectors = out.ld % 4 == 0 && aligned(out.c[0], 4 * sizeof(T)) && (args.batch < 2 || aligned(out.c[1], 4 * sizeof(T)));
    out.partial = c.splits > 1 ? static_cast<float*>(partial) : nullptr;
}

template <typename T>
void join(const Cut& c, const ProductArgs<T>& args, const ProductOut<T>& out, hipStream_t stream) {
    if (c.splits == 1) return;
    const int64_t quads = args.batch * args.m * ceil_div(args.n, 4);
    if (quads <= kMostDeep && c.splits >= kLeastDeep)
        join_deep_kernel<T><<<(unsigned)ceil_div(quads, kDeepQuads), kDeepQuads * kDeepSlices, 0, stream>>>(args.m, args.n, args.batch, c.splits, out.partial, out);
    else
        join_kernel<T><<<(unsigned)std::min<int64_t>(ceil_div(quads, 256), 4096), 256, 0, stream>>>(args.m, args.n, args.batch, c.splits, out.partial, out);
}

template <typename More>
void launch_gradient(const Cut& c, const ProductArgs<float>& args, const ProductOut<float>& out, const More& with, hipStream_t stream) {
    const auto groups = (unsigned)c.groups(1);
    if (c.size == kMiddle)
        float_tile_kernel<Middle<false>, false, false, ProductOut<float>, More><<<groups, Middle<false>::kThreads, 0, stream>>>(args, out, with);
    else
        float_tile_kernel<Small<false>, false, false, ProductOut<float>, More><<<groups, Small<false>::kThreads, 0, stream>>>(args, out, with);
}

}  // namespace

template <typename T, bool kARows, bool kBRows>
void product(const Cut& c, const ProductArgs<T>& args, ProductOut<T> out, void* partial, hipStream_t stream) {
    if (args.m == 0) return;
    into(out, c, args, partial);
    launch<T, false, kARows, kBRows>(c, args, out, stream);
    join(c, args, out, stream);
}

void weight_gradient(const Cut& c, const ProductArgs<float>& args, const Rows8* b8, float* sums, ProductOut<float> out, void* partial, hipStream_t stream) {
    into(out, c, args, partial);
    if (b8)
        launch_gradient(c, args, out, WeightGradient<true>{*b8, sums}, stream);
    else if (sums)
        launch_gradient(c, args, out, WeightGradient<false>{{}, sums}, stream);
    else
        launch<float, false, false, false>(c, args, out, stream);
    join(c, args, out, stream);
}

#define PRODUCTS(T)                                                                                            \
    template void product<T, true, true>(const Cut&, const ProductArgs<T>&, ProductOut<T>, void*, hipStream_t);  \
    template void product<T, true, false>(const Cut&, const ProductArgs<T>&, ProductOut<T>, void*, hipStream_t); \
    template void product<T, false, false>(const Cut&, const ProductArgs<T>&, ProductOut<T>, void*, hipStream_t);
PRODUCTS(float)
PRODUCTS(bf16_t)
PRODUCTS(f16_t)
#undef PRODUCTS

}  // namespace dgsp
