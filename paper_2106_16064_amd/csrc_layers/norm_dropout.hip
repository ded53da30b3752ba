// Host side of layer norm and dropout: argument checks and launches.  The C-ABI is documented in include/dgsp_layers.h.
#include "layers_host.hpp"

#include <cmath>

#include "dropout_kernels.hpp"
#include "layer_norm_kernels.hpp"

namespace {

using namespace dgsp;

bool make_mask(const dgsp_dropout_t* d, DropMask& mask) {
    mask = DropMask{0, 1.0f, 0, 0, 0, nullptr};
    if (!d) return true;
    if (!(d->p >= 0.0 && d->p <= 1.0)) return false;
    mask.dropped = (uint32_t)std::floor(d->p * 65536.0 + 0.5);
    mask.scale = mask.dropped < 65536 ? (float)(65536.0 / (65536.0 - mask.dropped)) : 0.0f;
    mask.key0 = (uint32_t)d->seed;
    mask.key1 = (uint32_t)(d->seed >> 32);
    mask.offset = d->offset;
    mask.device_offset = d->device_offset;
    return true;
}

constexpr int kThreads = 256;

// a wave per row, and several rows per wave where there are very many
unsigned row_blocks(int64_t rows) { return (unsigned)std::min<int64_t>(ceil_div(rows, kThreads / 64), 1 << 20); }

}  // namespace

// ---------------------------------------------------------------- dropout

extern "C" int dgsp_dropout(int64_t rows, int64_t width, int type, const dgsp_dropout_t* dropout, const void* x, int64_t ldx,
                            const void* residual, int64_t ldr, void* y, int64_t ldy, void* stream) {
    DropMask mask;
    if (rows < 0 || width < 0 || rows > kMostRows || width > kMostRows || !known_type(type) || !dropout || !make_mask(dropout, mask))
        return DGSP_ERR_INVALID_ARG;
    if (rows == 0 || width == 0) return DGSP_OK;
    if (!readable(x, rows, width, ldx) || (residual && !readable(residual, rows, width, ldr)) || !writable(y, rows, width, ldy))
        return DGSP_ERR_INVALID_ARG;
    const int64_t groups = rows * ceil_div(width, kDropGroup);
    const unsigned blocks = (unsigned)std::min<int64_t>(ceil_div(groups, kThreads), 1 << 20);
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        dropout_kernel<T><<<blocks, kThreads, 0, static_cast<hipStream_t>(stream)>>>(
            rows, width, mask, static_cast<const T*>(x), ldx, static_cast<const T*>(residual), ldr, static_cast<T*>(y), ldy);
        return launched();
    });
}

// ---------------------------------------------------------------- layer norm

extern "C" int dgsp_layer_norm(int64_t rows, int64_t width, int type, int param_type, const void* x, int64_t ldx, const void* residual,
                               int64_t ldr, const dgsp_dropout_t* dropout, const void* weight, const void* bias, float eps, void* y,
                               int64_t ldy, void* sum, int64_t lds, float* stats, void* stream) {
    DropMask mask;
    if (rows < 0 || width < 1 || rows > kMostRows || width > kMostRows || !known_type(type) ||
        (param_type != type && param_type != DGSP_F32) || !make_mask(dropout, mask))
        return DGSP_ERR_INVALID_ARG;
    if ((residual == nullptr) != (sum == nullptr) && rows > 0) return DGSP_ERR_INVALID_ARG;
    if (dropout && !residual && rows > 0) return DGSP_ERR_INVALID_ARG;
    if (rows == 0) return DGSP_OK;
    if (!readable(x, rows, width, ldx) || !writable(y, rows, width, ldy) ||
        (residual && (!readable(residual, rows, width, ldr) || !writable(sum, rows, width, lds))))
        return DGSP_ERR_INVALID_ARG;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        const NormInput<T> in{static_cast<const T*>(x), ldx, static_cast<const T*>(residual), ldr, mask};
        layer_norm_kernel<T><<<row_blocks(rows), kThreads, 0, static_cast<hipStream_t>(stream)>>>(
            rows, width, in, weight, bias, param_type != type, eps, static_cast<T*>(y), ldy, static_cast<T*>(sum), lds, stats);
        return launched();
    });
}

extern "C" int64_t dgsp_layer_norm_backward_workspace_bytes(int64_t rows, int64_t width) {
    if (rows < 0 || width < 1) return 0;
    return 2 * kNormSlices * width * 4;
}

extern "C" int dgsp_layer_norm_backward(int64_t rows, int64_t width, int type, int param_type, const void* s, int64_t lds,
                                        const float* stats, const void* weight, const void* dy, int64_t lddy, const void* ds,
                                        int64_t ldds, const dgsp_dropout_t* dropout, void* dsum, void* dx, void* dweight, void* dbias,
                                        void* workspace, int64_t workspace_bytes, void* stream) {
    DropMask mask;
    if (rows < 0 || width < 1 || rows > kMostRows || width > kMostRows || !known_type(type) ||
        (param_type != type && param_type != DGSP_F32) || !make_mask(dropout, mask))
        return DGSP_ERR_INVALID_ARG;
    const bool params = dweight || dbias;
    if (rows > 0 && (!readable(s, rows, width, lds) || !readable(dy, rows, width, lddy) || !stats || !dsum ||
                     (ds && !readable(ds, rows, width, ldds)) || (dropout == nullptr) != (dx == nullptr)))
        return DGSP_ERR_INVALID_ARG;
    if (params && (!workspace || !aligned(workspace, 16) || workspace_bytes < dgsp_layer_norm_backward_workspace_bytes(rows, width)))
        return DGSP_ERR_INVALID_ARG;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        const auto on = static_cast<hipStream_t>(stream);
        const bool wide = param_type != type;
        if (rows > 0)
            layer_norm_backward_kernel<T><<<row_blocks(rows), kThreads, 0, on>>>(
                rows, width, static_cast<const T*>(s), lds, stats, weight, wide, static_cast<const T*>(dy), lddy,
                static_cast<const T*>(ds), ldds, mask, static_cast<T*>(dsum), static_cast<T*>(dx));
        if (params) {
            auto* partial = static_cast<float*>(workspace);
            const unsigned columns = (unsigned)ceil_div(width, kThreads);
            layer_norm_param_partials_kernel<T><<<dim3(columns, kNormSlices), kThreads, 0, on>>>(
                rows, width, static_cast<const T*>(s), lds, stats, static_cast<const T*>(dy), lddy, partial);
            layer_norm_param_sums_kernel<T><<<columns, kThreads, 0, on>>>(width, partial, dweight, dbias, wide);
        }
        return launched();
    });
}
