/*
 * libdgsp_layers - the layers that stand next to a sparse product in a graph network, for AMD MI355X (gfx950): layer norm,
 * dropout and the gated feed-forward block, each with its gradient.
 *
 * The dense operand of Y = A X holds one row of features per vertex.  Between two products a network adds the result to what
 * was there (a residual), normalises the rows, drops elements while it trains and runs a feed-forward block.
 *
 * Conventions for every entry point
 *   - Pointers are HIP device memory of the current device unless stated otherwise.  The caller owns every buffer,
 *     workspaces included; the library allocates nothing and keeps no state between calls.
 *   - Matrices are row-major: element (r, c) is at r * ld + c, in elements, ld >= number of columns unless there is at most
 *     one row.  Inputs may repeat rows (ld = 0).  Any alignment that the element type has is taken.  Matrices without an ld
 *     argument are packed.  Results must not overlap inputs.
 *   - `type` is the element type of matrices.  Sums, statistics and products are held in 32 bits and rounded once when a
 *     result is written, unless the entry point says otherwise.
 *   - No result depends on the order in which workgroups run: the same call gives the same bits.
 *   - Calls are asynchronous: work is enqueued on `stream` (a hipStream_t as void*, NULL = the default stream) and may be
 *     recorded into a graph.
 *   - Return value: a dgsp_status_t (dgsp.h).  On any error nothing has been enqueued, except that after DGSP_ERR_LAUNCH
 *     earlier launches of the same call may have been.
 */
#ifndef DGSP_LAYERS_H
#define DGSP_LAYERS_H

#include <stdint.h>

#include "dgsp.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { DGSP_F32 = 0, DGSP_BF16 = 1, DGSP_F16 = 2 } dgsp_type_t;

/* silu(g) = g / (1 + exp(-g)); gelu(g) = g (1 + erf(g / sqrt 2)) / 2; relu(g) = max(g, 0), with derivative 0 at 0. */
typedef enum { DGSP_ACT_SILU = 0, DGSP_ACT_GELU = 1, DGSP_ACT_RELU = 2 } dgsp_activation_t;

/*
 * Dropout without a stored mask: whether element (row, col) is kept is a function of seed, offset, row and col, so that the
 * backward pass asks again.  With t = floor(65536 p + 1/2), the element is kept if its 16-bit number is >= t and then
 * multiplied by 65536 / (65536 - t); elsewhere the result is 0 whatever the input holds (p = 1: everywhere).  The number is
 * the (col % 8)-th of the eight 16-bit halves, lower half first, of what Philox4x32 with 10 rounds (Salmon, Moraes, Dror,
 * Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC 2011) makes of the counter (col / 8, row, low word of offset, high
 * word of offset) under the key (low word of seed, high word of seed).  Calls with different offsets are independent.
 * `device_offset`: NULL, or device memory that holds the offset, which the kernels read when they run (for replays of a
 * graph); `offset` is not looked at then.  The structure itself is host memory, read before a call returns.
 */
typedef struct {
    double p; /* 0 <= p <= 1 */
    uint64_t seed, offset;
    const uint64_t *device_offset;
} dgsp_dropout_t;

/*
 * y = dropout(x), or y = residual + dropout(x) if residual is not NULL.  The gradient of x is dropout(dy) with the same
 * seed and offset, the residual's is dy.  rows and width are below 2^31 - 4096.
 */
int dgsp_dropout(int64_t rows, int64_t width, int type, const dgsp_dropout_t *dropout, const void *x, int64_t ldx,
                 const void *residual, int64_t ldr, void *y, int64_t ldy, void *stream);

/*
 * Layer norm over the rows of s, where s = x, or s = residual + dropout(x) if residual is not NULL:
 *     y = (s - mean(s)) / sqrt(var(s) + eps) * weight + bias,    var the mean square of s - mean(s)
 *   weight, bias  width elements of `param_type`, which is `type` or DGSP_F32; NULL: 1, 0
 *   dropout       host, NULL: nothing is dropped; only with a residual
 *   sum           s, rounded to `type`; wanted with a residual, NULL without.  y is made from the sum before it is rounded.
 *   stats         2 floats a row, mean and 1 / sqrt(var + eps), for the backward pass; NULL: not wanted
 * rows and width are below 2^31 - 4096, width is at least 1.
 */
int dgsp_layer_norm(int64_t rows, int64_t width, int type, int param_type, const void *x, int64_t ldx, const void *residual,
                    int64_t ldr, const dgsp_dropout_t *dropout, const void *weight, const void *bias, float eps, void *y,
                    int64_t ldy, void *sum, int64_t lds, float *stats, void *stream);

/*
 * Its gradient.  With hat = (s - mean) / sqrt(var + eps) and dhat = dy * weight:
 *     dsum = (dhat - mean(dhat) - hat mean(dhat hat)) / sqrt(var + eps) + ds
 *     dweight = sum over the rows of dy hat,   dbias = sum over the rows of dy
 *   s          what the forward pass normalised: x, or the sum it wrote, which is rounded
 *   residual   if not NULL, s is the forward pass's x and the sum is made again from both, which costs the reading of one
 *              more matrix; with 16-bit types the rounded one would double the squared error of dweight
 *   stats      the forward pass's statistics
 *   ds         gradient of the result `sum`, NULL: none
 *   dropout    that of the forward pass, NULL: none
 *   dsum       gradient of s: that of x without a residual, that of the residual with one
 *   dx         dropout(dsum), wanted with dropout, else NULL
 *   dweight, dbias   width elements of `param_type`, NULL: not wanted
 *   workspace  dgsp_layer_norm_backward_workspace_bytes(rows, width) bytes, 16-byte aligned
 */
int dgsp_layer_norm_backward(int64_t rows, int64_t width, int type, int param_type, const void *s, int64_t lds,
                             const void *residual, int64_t ldr, const float *stats, const void *weight, const void *dy,
                             int64_t lddy, const void *ds, int64_t ldds,
                             const dgsp_dropout_t *dropout, void *dsum, void *dx, void *dweight, void *dbias, void *workspace,
                             int64_t workspace_bytes, void *stream);
int64_t dgsp_layer_norm_backward_workspace_bytes(int64_t rows, int64_t width);

/*
 * The gated feed-forward block: with g = x w_gate^T and u = x w_up^T,
 *     y = h w_down^T,   h = act(g) * u
 *   x        rows x width;   w_gate, w_up  hidden x width;   w_down  out_width x hidden;   y  rows x out_width
 *   saved    dgsp_gated_ff_saved_bytes(...) bytes, 16-byte aligned, for the backward pass; NULL: not wanted
 *   workspace  dgsp_gated_ff_workspace_bytes(...) bytes, 16-byte aligned
 * Either size may be 0; the pointer is not looked at then.  (Blocks whose weights fit a CU's LDS make g, u and h again.)
 * Of 16-bit types h is rounded to `type`, as the matrix instructions take their operands; act(g) and u act'(g) are saved in
 * 32 bits.  In float16 an h beyond 65504 becomes infinite, whatever w_down would have made of it.  Products of float matrices
 * are sums of products of three bfloat16 parts of each number, as exact as 32-bit arithmetic.  An infinity or NaN in an operand,
 * or a g or u beyond the range of 32 bits, makes infinity or NaN of the results that it belongs to; which of the two is not said.
 * rows is below 2^31 - 4096, the three widths are at least 1 and below 2^22 - 7.  DGSP_ERR_UNSUPPORTED: a product has 2^23 tiles
 * or more, which are 64 x 64 (of the projections 64 x 32) where it is small: float blocks of widths up to 32 from 2^29 - 63 rows on.
 */
int dgsp_gated_ff(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type, int activation, const void *x,
                  int64_t ldx, const void *w_gate, int64_t ldg, const void *w_up, int64_t ldu, const void *w_down, int64_t ldd,
                  void *y, int64_t ldy, void *saved, void *workspace, int64_t workspace_bytes, void *stream);
int64_t dgsp_gated_ff_saved_bytes(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type);
int64_t dgsp_gated_ff_workspace_bytes(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type);

/*
 * Its gradient.  With dh = dy w_down, dg = dh * u * act'(g) and du = dh * act(g):
 *     dx = dg w_gate + du w_up,  dw_gate = dg^T x,  dw_up = du^T x,  dw_down = dy^T h
 * dx is rows x width, the others have the shapes of the weights; NULL: not wanted.  Of 16-bit types dg and du are rounded
 * to `type`: in float16 they become infinite beyond 65504 and lose bits below 2^-14, so that a loss wants scaling.  Limits as above.
 */
int dgsp_gated_ff_backward(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type, int activation,
                           const void *x, int64_t ldx, const void *w_gate, int64_t ldg, const void *w_up, int64_t ldu,
                           const void *w_down, int64_t ldd, const void *dy, int64_t lddy, const void *saved, void *dx,
                           void *dw_gate, void *dw_up, void *dw_down, void *workspace, int64_t workspace_bytes, void *stream);
int64_t dgsp_gated_ff_backward_workspace_bytes(int64_t rows, int64_t width, int64_t hidden, int64_t out_width, int type);

#ifdef __cplusplus
}
#endif
#endif /* DGSP_LAYERS_H */
