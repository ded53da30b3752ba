// The products whose results are written as they are.
#include "products.hpp"

namespace dgsp {

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

#define PRODUCTS(T)                                                                                            \
    template void product<T, true, true>(const Cut&, const ProductArgs<T>&, ProductOut<T>, void*, hipStream_t);  \
    template void product<T, true, false>(const Cut&, const ProductArgs<T>&, ProductOut<T>, void*, hipStream_t); \
    template void product<T, false, false>(const Cut&, const ProductArgs<T>&, ProductOut<T>, void*, hipStream_t);
PRODUCTS(float)
PRODUCTS(bf16_t)
PRODUCTS(f16_t)
#undef PRODUCTS

}  // namespace dgsp
