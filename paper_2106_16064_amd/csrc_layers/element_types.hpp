// Element types of the layers' matrices: memory holds T, arithmetic is float.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace dgsp {

using bf16_t = __bf16;
using f16_t = _Float16;

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16_t v) { return (float)v; }
__device__ __forceinline__ float to_float(f16_t v) { return (float)v; }

// one rounding to nearest, ties to even
template <typename T>
__device__ __forceinline__ T from_float(float v) {
    return (T)v;
}

// an element of a vector that is stored in T or, if `wide`, in float
template <typename T>
__device__ __forceinline__ void store_param(void* p, int64_t i, bool wide, float v) {
    if (wide)
        static_cast<float*>(p)[i] = v;
    else
        static_cast<T*>(p)[i] = from_float<T>(v);
}

}  // namespace dgsp
