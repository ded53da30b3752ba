// The matrix product with its epilogue where the weight fits LDS (narrow_linear.hip).
#pragma once

#include "narrow_linear_kernels.hpp"

namespace dgsp {

// both widths at most 128, of float not both above 64
bool narrow_linear_fits(int64_t width, int64_t out_width, int type);

template <typename E>
int narrow_linear(const NarrowLinearArgs<E>& args, hipStream_t stream);

// `in_8bit`: x was kept in 8 bits
int64_t narrow_linear_backward_bytes(int64_t rows, int64_t width, int64_t out_width, int type, bool in_8bit);
// `dweight`, `dbias`: null where they are not wanted; args' sums are set here
template <typename E>
int narrow_linear_backward(NarrowLinearBackwardArgs<E> args, bool in_8bit, void* dweight, void* dbias, bool wide, void* workspace, hipStream_t stream);

}  // namespace dgsp
