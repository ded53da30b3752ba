// The gated feed-forward block with its weights in LDS: which blocks it takes, and its launches (narrow_ff.hip).
#pragma once

#include <cstdint>

namespace dgsp {

struct NarrowCall {
    int64_t rows, width, hidden, out_width;
    int type, activation;
    const void* x;
    int64_t ldx;
    const void* w_gate;
    int64_t ldg;
    const void* w_up;
    int64_t ldu;
    const void* w_down;
    int64_t ldd;
    void* y;
    int64_t ldy;
    const void* dy = nullptr;
    int64_t lddy = 0;
    void *dx = nullptr, *dw_gate = nullptr, *dw_up = nullptr, *dw_down = nullptr, *workspace = nullptr;
};

bool narrow_fits(int64_t width, int64_t hidden, int64_t out_width, int type);
int64_t narrow_backward_bytes(int64_t rows, int64_t width, int64_t hidden, int64_t out_width);
int narrow_forward(const NarrowCall& call, void* stream);
int narrow_backward(const NarrowCall& call, void* stream);

}  // namespace dgsp
