// Host side of what becomes of a product in linear_kernels.hpp.
#pragma once

#include "linear_kernels.hpp"
#include "products.hpp"

namespace dgsp {

template <typename T, bool kKeeps = true>
LinearOut<T, kKeeps> linear_out(void* y, int64_t ldy, const void* bias, bool wide, const void* residual, int64_t ldr, int activation, void* z, void* codes, int64_t out_width,
                        void* partial) {
    const auto four = [](const void* p, int64_t ld, int64_t size) { return ld % 4 == 0 && aligned(p, 4 * size); };
    LinearOut<T, kKeeps> out{};
    out.y = static_cast<T*>(y);
    out.ldy = ldy;
    out.vectors = four(y, ldy, sizeof(T));
    out.bias_vectors = four(bias, 0, wide ? 4 : sizeof(T));
    out.residual_vectors = four(residual, ldr, sizeof(T));
    out.wide = wide;
    out.bias = bias;
    out.residual = static_cast<const T*>(residual);
    out.ldr = ldr;
    out.activation = activation;
    out.z = z;
    out.codes = static_cast<uint8_t*>(codes);
    out.kept_ld = padded(out_width, 8);
    out.partial = static_cast<float*>(partial);
    return out;
}

}  // namespace dgsp
