// Host side of libdgsp_layers: argument checks and launches.  The C-ABI is documented in include/dgsp_layers.h.
#include "../../include/dgsp_layers.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "dropout_kernels.hpp"
#include "gated_ff_kernels.hpp"
#include "layer_norm_kernels.hpp"

namespace {

using namespace dgsp;

constexpr int64_t kMostRows = 2147483647LL - 4096, kMostWidth = (1LL << 28) - 1;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int launched() { return hipGetLastError() == hipSuccess ? DGSP_OK : DGSP_ERR_LAUNCH; }

bool known_type(int type) { return type == DGSP_F32 || type == DGSP_BF16 || type == DGSP_F16; }

int64_t element_bytes(int type) { return type == DGSP_F32 ? 4 : 2; }

template <typename F>
int with_type(int type, F&& f) {
    if (type == DGSP_F32) return f(float{});
    if (type == DGSP_BF16) return f(bf16_t{});
    return f(f16_t{});
}

// Does the matrix lie where it can be read?  ld = 0 repeats one row.
bool readable(const void* p, int64_t rows, int64_t cols, int64_t ld) {
    if (rows <= 0 || cols <= 0) return true;
    return p != nullptr && (rows == 1 || ld == 0 || ld >= cols);
}

bool writable(const void* p, int64_t rows, int64_t cols, int64_t ld) {
    if (rows <= 0 || cols <= 0) return true;
    return p != nullptr && (rows == 1 || ld >= cols);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

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
    if (params && (!workspace || !aligned16(workspace) || workspace_bytes < dgsp_layer_norm_backward_workspace_bytes(rows, width)))
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

// ---------------------------------------------------------------- gated feed-forward block

namespace {

bool gated_extents(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type) {
    return rows >= 0 && rows <= kMostRows && width >= 1 && width <= kMostWidth && hidden >= 1 && hidden <= kMostWidth &&
           out_width >= 1 && out_width <= kMostWidth && known_type(type);
}

int64_t hidden_bytes(int64_t rows, int64_t hidden, int type) { return ceil_div(rows * hidden * element_bytes(type), 256) * 256; }

template <typename T>
Operand<T> operand(const void* p, int64_t outer, int64_t inner) {
    return {static_cast<const T*>(p), outer, inner};
}

int64_t tiles(int64_t m, int64_t n) { return ceil_div(m, kTile) * ceil_div(n, kTile); }

// a launch has fewer than 2^32 threads
bool launchable(int64_t m, int64_t n) { return tiles(m, n) < (1LL << 32) / 256; }

template <typename T>
void product(int64_t m, int64_t n, int64_t depth, Operand<T> a, Operand<T> b, Operand<T> a2, Operand<T> b2, void* c, int64_t ldc,
             hipStream_t stream) {
    if (m > 0) product_kernel<T><<<(unsigned)tiles(m, n), 256, 0, stream>>>(m, n, depth, a, b, a2, b2, static_cast<T*>(c), ldc);
}

}  // namespace

// saved: g, u, h
extern "C" int64_t dgsp_gated_ff_saved_bytes(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type) {
    return gated_extents(rows, width, hidden, out_width, type) ? 3 * hidden_bytes(rows, hidden, type) : 0;
}

extern "C" int64_t dgsp_gated_ff_workspace_bytes(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type) {
    return gated_extents(rows, width, hidden, out_width, type) ? hidden_bytes(rows, hidden, type) : 0;
}

extern "C" int64_t dgsp_gated_ff_backward_workspace_bytes(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type) {
    return gated_extents(rows, width, hidden, out_width, type) ? 2 * hidden_bytes(rows, hidden, type) : 0;
}

extern "C" int dgsp_gated_ff(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type, int activation, const void* x,
                             int64_t ldx, const void* w_gate, int64_t ldg, const void* w_up, int64_t ldu, const void* w_down, int64_t ldd,
                             void* y, int64_t ldy, void* saved, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!gated_extents(rows, width, hidden, out_width, type) || activation < DGSP_ACT_SILU || activation > DGSP_ACT_RELU)
        return DGSP_ERR_INVALID_ARG;
    if (rows == 0) return DGSP_OK;
    if (!readable(x, rows, width, ldx) || !readable(w_gate, hidden, width, ldg) || !readable(w_up, hidden, width, ldu) ||
        !readable(w_down, out_width, hidden, ldd) || !writable(y, rows, out_width, ldy) || !aligned16(saved))
        return DGSP_ERR_INVALID_ARG;
    if (!saved && (!workspace || !aligned16(workspace) ||
                   workspace_bytes < dgsp_gated_ff_workspace_bytes(rows, width, hidden, out_width, type)))
        return DGSP_ERR_INVALID_ARG;
    if (!launchable(rows, std::max({width, hidden, out_width})) || !launchable(hidden, std::max(width, out_width))) return DGSP_ERR_UNSUPPORTED;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        const auto on = static_cast<hipStream_t>(stream);
        const int64_t part = hidden_bytes(rows, hidden, type);
        auto* base = static_cast<char*>(saved);
        T* g = saved ? reinterpret_cast<T*>(base) : nullptr;
        T* u = saved ? reinterpret_cast<T*>(base + part) : nullptr;
        T* h = saved ? reinterpret_cast<T*>(base + 2 * part) : static_cast<T*>(workspace);
        gated_up_kernel<T><<<(unsigned)tiles(rows, hidden), 256, 0, on>>>(rows, width, hidden, activation, operand<T>(x, ldx, 1),
                                                                          operand<T>(w_gate, ldg, 1), operand<T>(w_up, ldu, 1), g, u, h);
        product<T>(rows, out_width, hidden, operand<T>(h, hidden, 1), operand<T>(w_down, ldd, 1), {}, {}, y, ldy, on);
        return launched();
    });
}

extern "C" int dgsp_gated_ff_backward(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type, int activation,
                                      const void* x, int64_t ldx, const void* w_gate, int64_t ldg, const void* w_up, int64_t ldu,
                                      const void* w_down, int64_t ldd, const void* dy, int64_t lddy, const void* saved, void* dx,
                                      void* dw_gate, void* dw_up, void* dw_down, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!gated_extents(rows, width, hidden, out_width, type) || activation < DGSP_ACT_SILU || activation > DGSP_ACT_RELU)
        return DGSP_ERR_INVALID_ARG;
    if (rows > 0 && (!readable(x, rows, width, ldx) || !readable(w_gate, hidden, width, ldg) || !readable(w_up, hidden, width, ldu) ||
                     !readable(w_down, out_width, hidden, ldd) || !readable(dy, rows, out_width, lddy) || !saved || !aligned16(saved) ||
                     !workspace || !aligned16(workspace) ||
                     workspace_bytes < dgsp_gated_ff_backward_workspace_bytes(rows, width, hidden, out_width, type)))
        return DGSP_ERR_INVALID_ARG;
    if (!launchable(rows, std::max({width, hidden, out_width})) || !launchable(hidden, std::max(width, out_width))) return DGSP_ERR_UNSUPPORTED;
    return with_type(type, [&](auto element) {
        using T = decltype(element);
        const auto on = static_cast<hipStream_t>(stream);
        const int64_t part = hidden_bytes(rows, hidden, type);
        const auto* base = static_cast<const char*>(saved);
        const T *g = reinterpret_cast<const T*>(base), *u = reinterpret_cast<const T*>(base + part);
        const auto* h = base + 2 * part;
        T *dg = static_cast<T*>(workspace), *du = reinterpret_cast<T*>(static_cast<char*>(workspace) + part);
        if (rows > 0)
            gated_down_gradient_kernel<T><<<(unsigned)tiles(rows, hidden), 256, 0, on>>>(rows, hidden, out_width, activation,
                                                                                         operand<T>(dy, lddy, 1), operand<T>(w_down, 1, ldd),
                                                                                         g, u, dg, du);
        if (dx)
            product<T>(rows, width, hidden, operand<T>(dg, hidden, 1), operand<T>(w_gate, 1, ldg), operand<T>(du, hidden, 1),
                       operand<T>(w_up, 1, ldu), dx, width, on);
        if (dw_gate) product<T>(hidden, width, rows, operand<T>(dg, 1, hidden), operand<T>(x, 1, ldx), {}, {}, dw_gate, width, on);
        if (dw_up) product<T>(hidden, width, rows, operand<T>(du, 1, hidden), operand<T>(x, 1, ldx), {}, {}, dw_up, width, on);
        if (dw_down) product<T>(out_width, hidden, rows, operand<T>(dy, 1, lddy), operand<T>(h, 1, hidden), {}, {}, dw_down, hidden, on);
        return launched();
    });
}
