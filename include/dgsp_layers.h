/*
 * libdgsp_layers - the layers that stand next to a sparse product in a graph network, for AMD MI355X (gfx950): layer norm,
 * root-mean-square norm, dropout, the matrix product with its epilogue and the gated feed-forward block, each with its gradient, and
 * the norm and the product in 8 bits.
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
typedef enum { DGSP_ACT_SILU = 0, DGSP_ACT_GELU = 1, DGSP_ACT_RELU = 2, DGSP_ACT_NONE = 3 } dgsp_activation_t;

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

/*
 * Root-mean-square norm over the rows of s, where s = x, or s = residual + dropout(x) if residual is not NULL:
 *     y = s / sqrt(mean(s^2) + eps) * weight
 * Squares that 32 bits cannot hold are summed in 64, so that any finite s has its norm; rstd itself passes their range where mean(s^2) + eps is below 2^-256.
 *   rstd   a float a row, 1 / sqrt(mean(s^2) + eps), for the backward pass; NULL: not wanted
 * The other arguments and the limits are those of dgsp_layer_norm.
 */
int dgsp_rms_norm(int64_t rows, int64_t width, int type, int param_type, const void *x, int64_t ldx, const void *residual,
                  int64_t ldr, const dgsp_dropout_t *dropout, const void *weight, float eps, void *y, int64_t ldy, void *sum,
                  int64_t lds, float *rstd, void *stream);

/*
 * Its gradient.  With hat = s / sqrt(mean(s^2) + eps) and dhat = dy * weight:
 *     dsum = (dhat - hat mean(dhat hat)) / sqrt(mean(s^2) + eps) + ds,   dweight = sum over the rows of dy hat
 * The arguments are those of dgsp_layer_norm_backward.
 *   workspace  dgsp_rms_norm_backward_workspace_bytes(rows, width) bytes, 16-byte aligned, if dweight is wanted
 */
int dgsp_rms_norm_backward(int64_t rows, int64_t width, int type, int param_type, const void *s, int64_t lds,
                           const void *residual, int64_t ldr, const float *rstd, const void *weight, const void *dy, int64_t lddy,
                           const void *ds, int64_t ldds, const dgsp_dropout_t *dropout, void *dsum, void *dx, void *dweight,
                           void *workspace, int64_t workspace_bytes, void *stream);
int64_t dgsp_rms_norm_backward_workspace_bytes(int64_t rows, int64_t width);

/*
 * Rows in 8 bits.  A row is cut into blocks of 32 columns, each with a power of two as its scale: the least 2^e with
 * amax <= 448 2^e (DGSP_E4M3) or amax <= 127 2^e (DGSP_INT8), amax being the block's largest finite magnitude.  An element is
 * stored as element / 2^e, in e4m3 (4 bits of exponent, 3 of fraction, no infinities) or as a whole number, rounded to nearest,
 * ties to even.
 *   values  rows of 32 ceil(width / 32) bytes, filled up with zeros, 16-byte aligned, ld a multiple of 16
 *   scales  ceil(width / 128) * rows * 4 bytes, 4-byte aligned: byte b stands for 2^(b - 127), 255 for NaN; block k of row r at
 *           ((k / 4) * rows + r) * 4 + k % 4.  Blocks of zeros have 127, as have places beyond the last block.
 * e is at least -126 and at most 119 (DGSP_E4M3) or 121 (DGSP_INT8), for whole numbers of float16 matrices at least -24 and at
 * most 9: what is read back is then in the range of the type; elements beyond 448 or 127 times the largest scale become that.
 * An infinity or NaN becomes NaN: in e4m3 of the element, of whole numbers of its whole block.
 */
typedef enum { DGSP_E4M3 = 0, DGSP_INT8 = 1 } dgsp_kind_t;

/* `type`: that of x or y.  rows and width are below 2^31 - 4096, width is at least 1. */
int dgsp_quantise(int64_t rows, int64_t width, int type, int kind, const void *x, int64_t ldx, void *values, int64_t ldv,
                  void *scales, void *stream);
int dgsp_dequantise(int64_t rows, int64_t width, int type, int kind, const void *values, int64_t ldv, const void *scales, void *y,
                    int64_t ldy, void *stream);

/* dgsp_rms_norm without dropout, y in DGSP_E4M3: made from s, which is held in 32 bits, in 64 bits and rounded once. */
int dgsp_rms_norm_8bit(int64_t rows, int64_t width, int type, int param_type, const void *x, int64_t ldx, const void *residual,
                       int64_t ldr, const void *weight, float eps, void *values, int64_t ldv, void *scales, void *sum, int64_t lds,
                       void *stream);

/*
 * What a product keeps for its backward pass.  DGSP_KEEP_WHOLE: x, and of z as much as the activation's derivative needs (z in
 * `bias_type`, which is that of its gradient; of relu the derivative in a byte; without an activation nothing).  DGSP_KEEP_8BIT: x in DGSP_INT8, and act'(z) in steps of
 * 1/112 in a byte, which has 0 and 1 exactly and a code for NaN.
 */
typedef enum { DGSP_KEEP_NOTHING = 0, DGSP_KEEP_WHOLE = 1, DGSP_KEEP_8BIT = 2 } dgsp_keep_t;

/*
 * The matrix product with its epilogue:
 *     y = act(z) + residual,   z = x weight^T + bias
 *   x  rows x width;   weight  out_width x width;   residual, y  rows x out_width
 *   bias        out_width elements of `bias_type`, which is `type` or DGSP_F32; NULL: 0
 *   residual    NULL: 0
 *   activation  DGSP_ACT_...
 *   saved       dgsp_linear_saved_bytes(...) bytes, 16-byte aligned, for the backward pass; not looked at if that is 0
 *   x_values, x_scales   x in DGSP_INT8 for the backward pass, only with DGSP_KEEP_8BIT; NULL: not wanted
 *   workspace   dgsp_linear_workspace_bytes(...) bytes, 16-byte aligned; not looked at if that is 0.  Sizes are for operands that lie anywhere: of 16-bit types
 *               there is room for a copy of each, used where rows are no whole 16-byte pieces
 * z, act(z) and the sum with the residual are held in 32 bits.  Float matrices, infinities, NaN and limits: as in dgsp_gated_ff.
 */
int dgsp_linear(int64_t rows, int64_t width, int64_t out_width, int type, int bias_type, int activation, int keep, const void *x,
                int64_t ldx, const void *weight, int64_t ldw, const void *bias, const void *residual, int64_t ldr, void *y,
                int64_t ldy, void *saved, void *x_values, int64_t ldv, void *x_scales, void *workspace, int64_t workspace_bytes, void *stream);
int64_t dgsp_linear_saved_bytes(int64_t rows, int64_t out_width, int type, int bias_type, int activation, int keep);
int64_t dgsp_linear_workspace_bytes(int64_t rows, int64_t width, int64_t out_width, int type);

/*
 * Its gradient.  With dz = dy act'(z):
 *     dx = dz weight,   dweight = dz^T x,   dbias = sum over the rows of dz;   the residual's is dy
 *   keep         what the forward pass kept, not DGSP_KEEP_NOTHING
 *   x, x_scales  DGSP_KEEP_WHOLE: the matrix, NULL.  DGSP_KEEP_8BIT: values and scales of x in DGSP_INT8; ldx is that of the values.
 *   dx, dweight, dbias   NULL: not wanted.  dx is rows x width, dweight out_width x width, both packed; dbias is of `bias_type`.
 * Of 16-bit types dz is rounded to `type`, as the matrix instructions take their operands (dbias is summed before that): in
 * float16 it becomes infinite beyond 65504 and loses bits below 2^-14.  act'(z) of an infinite z is 1 or 0, whatever was kept.
 */
int dgsp_linear_backward(int64_t rows, int64_t width, int64_t out_width, int type, int bias_type, int activation, int keep,
                         const void *x, int64_t ldx, const void *x_scales, const void *weight, int64_t ldw, const void *saved,
                         const void *dy, int64_t lddy, void *dx, void *dweight, void *dbias, void *workspace, int64_t workspace_bytes,
                         void *stream);
int64_t dgsp_linear_backward_workspace_bytes(int64_t rows, int64_t width, int64_t out_width, int type, int activation, int keep);

/*
 * The same product of operands in DGSP_E4M3, for serving: x is rows x width, weight out_width x width.  Products of eight neighbouring
 * columns are added aligned to the largest of them and cut off 2^-13 below its power of two; sums of these are held in 32 bits.
 *   type   of the residual and of y
 *   ldx, ldw   of the values, in bytes, below 2^23
 * Limits as above.
 */
int dgsp_linear_8bit(int64_t rows, int64_t width, int64_t out_width, int type, int bias_type, int activation, const void *x, int64_t ldx,
                     const void *x_scales, const void *weight, int64_t ldw, const void *weight_scales, const void *bias,
                     const void *residual, int64_t ldr, void *y, int64_t ldy, void *workspace, int64_t workspace_bytes, void *stream);
int64_t dgsp_linear_8bit_workspace_bytes(int64_t rows, int64_t width, int64_t out_width);

#ifdef __cplusplus
}
#endif
#endif /* DGSP_LAYERS_H */
