// Host side of layer norm and dropout: argument checks, how rows are held, launches.  The C-ABI is documented in include/dgsp_layers.h.
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

constexpr int64_t kCus = 256;

// How rows of a width are held: up to 512 elements a wave holds one or several, up to 8192 a workgroup holds one.
struct Hold {
    bool whole;             // a workgroup a row
    int lanes, threads;
    bool fits;
    explicit Hold(int64_t width) {
        const int64_t chunks = ceil_div(width, kChunk);
        whole = chunks > 64;
        fits = chunks <= 1024;
        if (!whole) {
            lanes = 1;
            while (lanes < chunks) lanes *= 2;
            threads = 256;
        } else {
            threads = lanes = (int)std::min<int64_t>(1024, ceil_div(chunks, 64) * 64);
        }
    }
    int64_t rows_a_group() const { return whole ? 1 : threads / lanes; }
};

template <typename T, bool kAdd>
void launch_norm(const Hold& hold, const NormArgs<T>& args, hipStream_t stream) {
    const unsigned groups = (unsigned)std::min<int64_t>(ceil_div(args.rows, hold.rows_a_group()), kCus * 2048 / hold.threads);
    if (hold.whole)
        layer_norm_kernel<T, true, kAdd><<<groups, hold.threads, 0, stream>>>(args);
    else
        layer_norm_kernel<T, false, kAdd><<<groups, hold.threads, 0, stream>>>(args);
}

// Workgroups of the backward pass, each with sums of its own for the parameters, as many as the GPU holds at once.  Of many rows the sums
// are a small part of what is read anyway (32768 x 1024, 16 bits: 17 MB beside 268); where a workgroup is left with a row or two they are
// not: 4099 x 1001 has 2048 workgroups, whose sums of 16 MB are written and read again beside 33 MB read and 16 written.
int64_t backward_groups(const Hold& hold, int64_t rows) {
    if (!hold.fits) return std::min<int64_t>(std::max<int64_t>(rows, 1), 64);
    const int64_t most = hold.whole ? kCus * std::max(1, 1024 / hold.threads) : kCus * 4;
    return std::max<int64_t>(1, std::min(ceil_div(rows, hold.rows_a_group()), most));
}

template <typename T, bool kAdd>
void launch_backward(const Hold& hold, const NormBackwardArgs<T>& args, int64_t groups, hipStream_t stream) {
    if (hold.whole)
        layer_norm_backward_kernel<T, true, kAdd><<<(unsigned)groups, hold.threads, 0, stream>>>(args);
    else
        layer_norm_backward_kernel<T, false, kAdd><<<(unsigned)groups, hold.threads, 0, stream>>>(args);
}

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
    const int64_t chunks = ceil_div(width, kChunk), total = rows * chunks;
    const unsigned groups = (unsigned)std::min<int64_t>(ceil_div(total, kDropThreads), 1 << 23);
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        const auto *in = static_cast<const T*>(x), *add = static_cast<const T*>(residual);
        const auto on = static_cast<hipStream_t>(stream);
        const Divisor divisor((uint32_t)chunks);
        dropout_kernel<T><<<groups, kDropThreads, 0, on>>>(rows, width, divisor, mask, in, ldx, add, ldr, static_cast<T*>(y), ldy);
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
        const Hold hold(width);
        const auto on = static_cast<hipStream_t>(stream);
        const NormArgs<T> args{rows,   width, hold.lanes, static_cast<const T*>(x), static_cast<const T*>(residual), ldx, ldr, mask, weight, bias, param_type != type,
                               eps,    static_cast<T*>(y), static_cast<T*>(sum), ldy, lds, stats};
        if (!hold.fits)
            layer_norm_long_kernel<T><<<(unsigned)std::min<int64_t>(rows, kCus * 2), 1024, 0, on>>>(args);
        else if (residual)
            launch_norm<T, true>(hold, args, on);
        else
            launch_norm<T, false>(hold, args, on);
        return launched();
    });
}

extern "C" int64_t dgsp_layer_norm_backward_workspace_bytes(int64_t rows, int64_t width) {
    if (rows < 0 || width < 1 || rows > kMostRows || width > kMostRows) return 0;
    return 2 * backward_groups(Hold(width), rows) * width * 4;
}

extern "C" int dgsp_layer_norm_backward(int64_t rows, int64_t width, int type, int param_type, const void* s, int64_t lds,
                                        const void* residual, int64_t ldr, const float* stats, const void* weight, const void* dy, int64_t lddy, const void* ds,
                                        int64_t ldds, const dgsp_dropout_t* dropout, void* dsum, void* dx, void* dweight, void* dbias,
                                        void* workspace, int64_t workspace_bytes, void* stream) {
    DropMask mask;
    if (rows < 0 || width < 1 || rows > kMostRows || width > kMostRows || !known_type(type) ||
        (param_type != type && param_type != DGSP_F32) || !make_mask(dropout, mask))
        return DGSP_ERR_INVALID_ARG;
    const bool params = dweight || dbias;
    if (rows > 0 && (!readable(s, rows, width, lds) || (residual && !readable(residual, rows, width, ldr)) || !readable(dy, rows, width, lddy) || !stats || !dsum ||
                     (ds && !readable(ds, rows, width, ldds)) || (dropout == nullptr) != (dx == nullptr)))
        return DGSP_ERR_INVALID_ARG;
    if (params && (!workspace || !aligned(workspace, 16) || workspace_bytes < dgsp_layer_norm_backward_workspace_bytes(rows, width)))
        return DGSP_ERR_INVALID_ARG;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        const Hold hold(width);
        const auto on = static_cast<hipStream_t>(stream);
        const bool wide = param_type != type;
        const int64_t groups = backward_groups(hold, rows);
        const NormBackwardArgs<T> args{rows, width, hold.lanes, static_cast<const T*>(s), static_cast<const T*>(residual), static_cast<const T*>(dy), static_cast<const T*>(ds),
                                       lds,  ldr,   lddy,  ldds,       stats, weight, wide, mask, static_cast<T*>(dsum), static_cast<T*>(dx),
                                       params ? static_cast<float*>(workspace) : nullptr};
        if (rows > 0 && !hold.fits) {
            layer_norm_backward_long_kernel<T><<<(unsigned)std::min<int64_t>(rows, kCus * 2), 1024, 0, on>>>(args);
            if (params) layer_norm_long_params_kernel<T><<<dim3((unsigned)ceil_div(width, 256), (unsigned)groups), 256, 0, on>>>(args);
        } else if (rows > 0) {
            if (ds || dx || residual)
                launch_backward<T, true>(hold, args, groups, on);
            else
                launch_backward<T, false>(hold, args, groups, on);
        }
        if (params)
            layer_norm_params_kernel<T><<<(unsigned)std::min(ceil_div(2 * width, kParamColumns), kParamGroups), kParamColumns * kParamSlices, 0, on>>>(
                width, rows > 0 ? groups : 0, args.partial, dweight, dbias, wide);
        return launched();
    });
}
