// Host side of the root-mean-square norm and of rows in 8 bits: argument checks, launches.  The C-ABI is documented in include/dgsp_layers.h.
#include "column_sums.hpp"
#include "norms_host.hpp"
#include "rms_norm_kernels.hpp"
#include "rows8_host.hpp"

namespace {

using namespace dgsp;

bool norm_extents(int64_t rows, int64_t width, int type, int param_type) {
    return rows >= 0 && width >= 1 && rows <= kMostRows && width <= kMostRows && known_type(type) && (param_type == type || param_type == DGSP_F32);
}

template <typename T, bool k8bit>
void launch_norm(const Hold& hold, const RmsArgs<T>& args, hipStream_t stream) {
    // As many workgroups as 2048 threads a CU are, which go on to further rows that they have asked for before.  Two to four times as many rows with a workgroup
    // each take longer, but for float with the residual's addition, whose four matrices come from memory.  us, so and with a workgroup a row:
    //     float16   262144 x 32 9.2 and 10.2      8192 x 1001 10.1 and 10.7, into 8 bits 13.0 and 13.3    4096 x 4096 14.5 and 17.4, into 8 bits 19.2 and 22.2
    //               with the residual: 16384 x 300 15.9 and 16.5    8192 x 2048 26.8 and 24.6, into 8 bits 25.7 and 29.5    2048 x 8192 26.9 and 35.3
    //     float     262144 x 32 12.9 and 14.7     8192 x 1001 12.9 and 13.3                               4096 x 4096 26.1 and 26.2, into 8 bits 22.2 and 25.7
    //               with the residual: 262144 x 32 27.3 and 25.5    8192 x 1001 27.2 and 26.1    4096 x 4096 45.4 and 44.9    2048 x 8192 49 and 52
    const int64_t needed = ceil_div(args.rows, hold.rows_a_group()), resident = kCus * 2048 / hold.threads;
    const bool four = args.residual && !k8bit && sizeof(T) == 4 && hold.threads <= 512;
    const unsigned groups = (unsigned)(needed <= (four ? 4 : 1) * resident ? needed : resident);
    if (!hold.fits)
        rms_norm_long_kernel<T, k8bit><<<(unsigned)std::min<int64_t>(args.rows, kCus * 2), 1024, 0, stream>>>(args);
    else if (hold.whole && args.residual)
        rms_norm_kernel<T, true, true, k8bit><<<groups, hold.threads, 0, stream>>>(args);
    else if (hold.whole)
        rms_norm_kernel<T, true, false, k8bit><<<groups, hold.threads, 0, stream>>>(args);
    else if (args.residual)
        rms_norm_kernel<T, false, true, k8bit><<<groups, hold.threads, 0, stream>>>(args);
    else
        rms_norm_kernel<T, false, false, k8bit><<<groups, hold.threads, 0, stream>>>(args);
}

template <typename T>
void launch_backward(const Hold& hold, const RmsBackwardArgs<T>& args, int64_t groups, hipStream_t stream) {
    const bool add = args.ds || args.dx || args.residual;
    if (hold.whole && add)
        rms_norm_backward_kernel<T, true, true><<<(unsigned)groups, hold.threads, 0, stream>>>(args);
    else if (hold.whole)
        rms_norm_backward_kernel<T, true, false><<<(unsigned)groups, hold.threads, 0, stream>>>(args);
    else if (add)
        rms_norm_backward_kernel<T, false, true><<<(unsigned)groups, hold.threads, 0, stream>>>(args);
    else
        rms_norm_backward_kernel<T, false, false><<<(unsigned)groups, hold.threads, 0, stream>>>(args);
}

}  // namespace

// ---------------------------------------------------------------- the norm

extern "C" int dgsp_rms_norm(int64_t rows, int64_t width, int type, int param_type, const void* x, int64_t ldx, const void* residual,
                             int64_t ldr, const dgsp_dropout_t* dropout, const void* weight, float eps, void* y, int64_t ldy, void* sum,
                             int64_t lds, float* rstd, void* stream) {
    DropMask mask;
    if (!norm_extents(rows, width, type, param_type) || !make_mask(dropout, mask)) return DGSP_ERR_INVALID_ARG;
    if (rows == 0) return DGSP_OK;
    if ((residual == nullptr) != (sum == nullptr) || (dropout && !residual)) return DGSP_ERR_INVALID_ARG;
    if (!readable(x, rows, width, ldx) || !writable(y, rows, width, ldy) ||
        (residual && (!readable(residual, rows, width, ldr) || !writable(sum, rows, width, lds))))
        return DGSP_ERR_INVALID_ARG;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        const Hold hold(width);
        launch_norm<T, false>(hold, {rows, width, hold.lanes, static_cast<const T*>(x), static_cast<const T*>(residual), ldx, ldr, mask, weight,
                                     param_type != type, eps, static_cast<T*>(y), static_cast<T*>(sum), ldy, lds, rstd, {}},
                              static_cast<hipStream_t>(stream));
        return launched();
    });
}

extern "C" int dgsp_rms_norm_8bit(int64_t rows, int64_t width, int type, int param_type, const void* x, int64_t ldx, const void* residual,
                                  int64_t ldr, const void* weight, float eps, void* values, int64_t ldv, void* scales, void* sum, int64_t lds,
                                  void* stream) {
    if (!norm_extents(rows, width, type, param_type)) return DGSP_ERR_INVALID_ARG;
    if (rows == 0) return DGSP_OK;
    if ((residual == nullptr) != (sum == nullptr) || !readable(x, rows, width, ldx) || !rows8_lies(values, rows, width, ldv, scales) ||
        (rows > 1 && ldv < rows8_bytes(width)) || (residual && (!readable(residual, rows, width, ldr) || !writable(sum, rows, width, lds))))
        return DGSP_ERR_INVALID_ARG;
    DropMask mask;
    make_mask(nullptr, mask);
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        Hold hold(rows8_bytes(width));
        if (!hold.whole) hold.lanes = std::max(hold.lanes, kBlockLanes);
        launch_norm<T, true>(hold, {rows, width, hold.lanes, static_cast<const T*>(x), static_cast<const T*>(residual), ldx, ldr, mask, weight,
                                    param_type != type, eps, nullptr, static_cast<T*>(sum), 0, lds, nullptr, rows8(values, rows, width, ldv, scales)},
                             static_cast<hipStream_t>(stream));
        return launched();
    });
}

extern "C" int64_t dgsp_rms_norm_backward_workspace_bytes(int64_t rows, int64_t width) {
    if (rows < 0 || width < 1 || rows > kMostRows || width > kMostRows) return 0;
    return backward_groups(Hold(width), rows) * width * 4;
}

extern "C" int dgsp_rms_norm_backward(int64_t rows, int64_t width, int type, int param_type, const void* s, int64_t lds, const void* residual,
                                      int64_t ldr, const float* rstd, const void* weight, const void* dy, int64_t lddy, const void* ds, int64_t ldds,
                                      const dgsp_dropout_t* dropout, void* dsum, void* dx, void* dweight, void* workspace, int64_t workspace_bytes,
                                      void* stream) {
    DropMask mask;
    if (!norm_extents(rows, width, type, param_type) || !make_mask(dropout, mask)) return DGSP_ERR_INVALID_ARG;
    if (rows > 0 && (!readable(s, rows, width, lds) || (residual && !readable(residual, rows, width, ldr)) || !readable(dy, rows, width, lddy) || !rstd || !dsum ||
                     (ds && !readable(ds, rows, width, ldds)) || (dropout == nullptr) != (dx == nullptr)))
        return DGSP_ERR_INVALID_ARG;
    if (dweight && (!workspace || !aligned(workspace, 16) || workspace_bytes < dgsp_rms_norm_backward_workspace_bytes(rows, width)))
        return DGSP_ERR_INVALID_ARG;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        const Hold hold(width);
        const auto on = static_cast<hipStream_t>(stream);
        const bool wide = param_type != type;
        const int64_t groups = backward_groups(hold, rows);
        const RmsBackwardArgs<T> args{rows, width, hold.lanes, static_cast<const T*>(s), static_cast<const T*>(residual), static_cast<const T*>(dy),
                                      static_cast<const T*>(ds), lds, ldr, lddy, ldds, rstd, weight, wide, mask, static_cast<T*>(dsum), static_cast<T*>(dx),
                                      dweight ? static_cast<float*>(workspace) : nullptr};
        if (rows > 0 && !hold.fits) {
            rms_norm_backward_long_kernel<T><<<(unsigned)std::min<int64_t>(rows, kCus * 2), 1024, 0, on>>>(args);
            if (dweight) rms_norm_long_params_kernel<T><<<dim3((unsigned)ceil_div(width, 256), (unsigned)groups), 256, 0, on>>>(args);
        } else if (rows > 0) {
            launch_backward<T>(hold, args, groups, on);
        }
        if (dweight) launch_column_sums<T>(width, rows > 0 ? groups : 0, args.partial, dweight, wide, on);
        return launched();
    });
}

// ---------------------------------------------------------------- rows in 8 bits

extern "C" int dgsp_quantise(int64_t rows, int64_t width, int type, int kind, const void* x, int64_t ldx, void* values, int64_t ldv, void* scales,
                             void* stream) {
    if (!norm_extents(rows, width, type, type) || !known_kind(kind)) return DGSP_ERR_INVALID_ARG;
    if (rows == 0) return DGSP_OK;
    if (!readable(x, rows, width, ldx) || !rows8_lies(values, rows, width, ldv, scales) || (rows > 1 && ldv < rows8_bytes(width))) return DGSP_ERR_INVALID_ARG;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        launch_quantise<T>(kind, rows, width, static_cast<const T*>(x), ldx, rows8(values, rows, width, ldv, scales), static_cast<hipStream_t>(stream));
        return launched();
    });
}

extern "C" int dgsp_dequantise(int64_t rows, int64_t width, int type, int kind, const void* values, int64_t ldv, const void* scales, void* y,
                               int64_t ldy, void* stream) {
    if (!norm_extents(rows, width, type, type) || !known_kind(kind)) return DGSP_ERR_INVALID_ARG;
    if (rows == 0) return DGSP_OK;
    if (!rows8_lies(values, rows, width, ldv, scales) || !writable(y, rows, width, ldy)) return DGSP_ERR_INVALID_ARG;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        launch_dequantise<T>(kind, rows, width, rows8(const_cast<void*>(values), rows, width, ldv, const_cast<void*>(scales)), static_cast<T*>(y), ldy,
                             static_cast<hipStream_t>(stream));
        return launched();
    });
}
