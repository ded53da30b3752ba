// What the host sides of the layers share: argument checks and types.
#pragma once

#include "../../include/dgsp_layers.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "element_types.hpp"

namespace dgsp {

constexpr int64_t kMostRows = 2147483647LL - 4096;
constexpr int64_t kCus = 256;

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int launched() { return hipGetLastError() == hipSuccess ? DGSP_OK : DGSP_ERR_LAUNCH; }

inline bool known_type(int type) { return type == DGSP_F32 || type == DGSP_BF16 || type == DGSP_F16; }

inline int64_t element_bytes(int type) { return type == DGSP_F32 ? 4 : 2; }

template <typename F>
int with_type(int type, F&& f) {
    if (type == DGSP_F32) return f(float{});
    if (type == DGSP_BF16) return f(bf16_t{});
    return f(f16_t{});
}

// Does the matrix lie where it can be read?  ld = 0 repeats one row.
inline bool readable(const void* p, int64_t rows, int64_t cols, int64_t ld) {
    if (rows <= 0 || cols <= 0) return true;
    return p != nullptr && (rows == 1 || ld == 0 || ld >= cols);
}

inline bool writable(const void* p, int64_t rows, int64_t cols, int64_t ld) {
    if (rows <= 0 || cols <= 0) return true;
    return p != nullptr && (rows == 1 || ld >= cols);
}

inline bool aligned(const void* p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

}  // namespace dgsp
