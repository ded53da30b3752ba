// Launches of the gated feed-forward block with its weights in LDS.
#include "narrow_ff.hpp"

#include "layers_host.hpp"

#include "narrow_ff_kernels.hpp"

namespace dgsp {

namespace {

// The extents as they are padded: width and out_width to 32, 64 or 128, hidden to 64, 128 or 256, as long as the weights, a tile of
// rows and the hidden values of a tile fit 160 KB.  Four waves a workgroup where eight waves' tiles no longer do (64 x 256), and where
// hidden is at most 64, of which a wave takes 16.
struct Padded {
    int p, h, waves, groups_a_cu;       // waves and resident workgroups of the backward pass
    bool fits;
    Padded(int64_t width, int64_t hidden, int64_t out_width) {
        const int64_t most = std::max(width, out_width);
        p = most <= 32 ? 32 : most <= 64 ? 64 : 128;
        h = hidden <= 64 ? 64 : hidden <= 128 ? 128 : 256;
        fits = most <= 128 && hidden <= 256 && p * h <= 64 * 256;
        waves = (p == 64 && h == 256) || h == 64 ? 4 : 8;
        groups_a_cu = p < 128 && h == 64 ? 2 : 1;
    }
    int64_t groups(int64_t rows) const { return std::max<int64_t>(1, std::min(ceil_div(rows, 16 * waves), kCus * groups_a_cu)); }
    int64_t gradients() const { return 3LL * p * h; }
};

// Do rows start and end on 16-byte pieces, and few enough bytes apart for the offsets of a buffer?
bool whole_pieces(const void* p, int64_t ld) { return aligned(p, 16) && ld % 8 == 0 && ld > 0 && ld < (1 << 22); }

template <typename E, int kP, int kH, int kWaves>
void launch_forward(const NarrowArgs<E>& args, hipStream_t stream) {
    // as many workgroups as are resident together
    const int64_t most = kCus * std::max(1, std::min(16 / kWaves, 163840 / NarrowShape<E, kP, kH, kWaves>::kForwardLds));
    const auto groups = (unsigned)std::min(ceil_div(args.rows, 32 * kWaves), most);
    if (args.width == kP && args.out_width == kP && whole_pieces(args.x, args.ldx))
        narrow_forward_kernel<E, kP, kH, kWaves, true><<<groups, 64 * kWaves, 0, stream>>>(args);
    else
        narrow_forward_kernel<E, kP, kH, kWaves, false><<<groups, 64 * kWaves, 0, stream>>>(args);
}

template <typename E, int kP>
bool backward_in_whole_pieces(const NarrowArgs<E>& args) {
    return args.width == kP && args.out_width == kP && whole_pieces(args.x, args.ldx) && whole_pieces(args.dy, args.lddy);
}

template <typename E, int kP, int kWaves>
void launch_backward(const NarrowArgs<E>& args, int64_t groups, hipStream_t stream) {
    if (backward_in_whole_pieces<E, kP>(args))
        narrow_backward_kernel<E, kP, kWaves, true><<<(unsigned)groups, 64 * kWaves, 0, stream>>>(args);
    else
        narrow_backward_kernel<E, kP, kWaves, false><<<(unsigned)groups, 64 * kWaves, 0, stream>>>(args);
}

template <typename E, int kP, int kH, int kWaves>
void launch_backward_staged(const NarrowArgs<E>& args, int64_t groups, hipStream_t stream) {
    if (backward_in_whole_pieces<E, kP>(args))
        narrow_backward_staged_kernel<E, kP, kH, kWaves, true><<<(unsigned)groups, 64 * kWaves, 0, stream>>>(args);
    else
        narrow_backward_staged_kernel<E, kP, kH, kWaves, false><<<(unsigned)groups, 64 * kWaves, 0, stream>>>(args);
}

template <typename E>
NarrowArgs<E> arguments(const NarrowCall& c) {
    NarrowArgs<E> a{};
    a.rows = c.rows;
    a.width = c.width;
    a.hidden = c.hidden;
    a.out_width = c.out_width;
    a.activation = c.activation;
    a.x = static_cast<const E*>(c.x);
    a.ldx = c.rows == 1 ? c.width : c.ldx;             // of one row it may be anything, and the kernels' buffers end where it says
    a.w_gate = static_cast<const E*>(c.w_gate);
    a.ldg = c.ldg;
    a.w_up = static_cast<const E*>(c.w_up);
    a.ldu = c.ldu;
    a.w_down = static_cast<const E*>(c.w_down);
    a.ldd = c.ldd;
    a.y = static_cast<E*>(c.y);
    a.ldy = c.ldy;
    a.dy = static_cast<const E*>(c.dy);
    a.lddy = c.rows == 1 ? c.out_width : c.lddy;
    a.dx = static_cast<E*>(c.dx);
    return a;
}

template <typename E>
int forward(const NarrowCall& call, hipStream_t stream) {
    const NarrowArgs<E> args = arguments<E>(call);
    const Padded at(call.width, call.hidden, call.out_width);
    if (at.p == 32 && at.h == 64)
        launch_forward<E, 32, 64, 8>(args, stream);
    else if (at.p == 32 && at.h == 128)
        launch_forward<E, 32, 128, 8>(args, stream);
    else if (at.p == 32)
        launch_forward<E, 32, 256, 8>(args, stream);
    else if (at.p == 64 && at.h == 64)
        launch_forward<E, 64, 64, 8>(args, stream);
    else if (at.p == 64 && at.h == 128)
        launch_forward<E, 64, 128, 8>(args, stream);
    else if (at.p == 64)
        launch_forward<E, 64, 256, 8>(args, stream);
    else if (at.h == 64)
        launch_forward<E, 128, 64, 8>(args, stream);
    else
        launch_forward<E, 128, 128, 8>(args, stream);
    return launched();
}

template <typename E>
int backward(const NarrowCall& call, hipStream_t stream) {
    NarrowArgs<E> args = arguments<E>(call);
    const Padded at(call.width, call.hidden, call.out_width);
    const int64_t groups = at.groups(call.rows);
    const bool weights = call.dw_gate || call.dw_up || call.dw_down;
    if (weights) args.partial = static_cast<float*>(call.workspace);
    if (call.rows > 0 && (weights || call.dx)) {
        if (at.p == 32 && at.h == 64)
            launch_backward<E, 32, 4>(args, groups, stream);
        else if (at.p == 32 && at.h == 128)
            launch_backward<E, 32, 8>(args, groups, stream);
        else if (at.p == 32)
            launch_backward_staged<E, 32, 256, 8>(args, groups, stream);
        else if (at.p == 64 && at.h == 64)
            launch_backward<E, 64, 4>(args, groups, stream);
        else if (at.p == 64 && at.h == 128)
            launch_backward<E, 64, 8>(args, groups, stream);
        else if (at.p == 64)
            launch_backward_staged<E, 64, 256, 4>(args, groups, stream);
        else if (at.h == 64)
            launch_backward<E, 128, 4>(args, groups, stream);
        else
            launch_backward<E, 128, 8>(args, groups, stream);
    }
    if (weights)
        narrow_join_kernel<E><<<(unsigned)(at.gradients() / kNarrowColumns), kNarrowColumns * kNarrowSlices, 0, stream>>>(
            at.p, at.h, call.width, call.hidden, call.out_width, call.rows > 0 ? (int)groups : 0, args.partial, static_cast<E*>(call.dw_gate),
            static_cast<E*>(call.dw_up), static_cast<E*>(call.dw_down));
    return launched();
}

}  // namespace

bool narrow_fits(int64_t width, int64_t hidden, int64_t out_width, int type) { return type != DGSP_F32 && Padded(width, hidden, out_width).fits; }

int64_t narrow_backward_bytes(int64_t rows, int64_t width, int64_t hidden, int64_t out_width) {
    const Padded at(width, hidden, out_width);
    return at.groups(rows) * at.gradients() * 4;
}

int narrow_forward(const NarrowCall& call, void* stream) {
    return call.type == DGSP_BF16 ? forward<bf16_t>(call, static_cast<hipStream_t>(stream)) : forward<f16_t>(call, static_cast<hipStream_t>(stream));
}

int narrow_backward(const NarrowCall& call, void* stream) {
    return call.type == DGSP_BF16 ? backward<bf16_t>(call, static_cast<hipStream_t>(stream)) : backward<f16_t>(call, static_cast<hipStream_t>(stream));
}

}  // namespace dgsp
