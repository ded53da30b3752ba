// Host side of rows in 8 bits, for those that read or write them.
#pragma once

#include "layers_host.hpp"

#include "rows8.hpp"

namespace dgsp {

inline bool known_kind(int kind) { return kind == DGSP_E4M3 || kind == DGSP_INT8; }

inline int64_t rows8_bytes(int64_t width) { return ceil_div(width, kBlock) * kBlock; }          // of a row's values
inline int64_t scales_bytes(int64_t rows, int64_t width) { return ceil_div(width, 4 * kBlock) * rows * 4; }

// Do values and scales lie where they can be read?  ldv = 0 repeats one row.
inline bool rows8_lies(const void* values, int64_t rows, int64_t width, int64_t ldv, const void* scales) {
    return values && scales && aligned(values, 16) && aligned(scales, 4) && (rows == 1 || (ldv % 16 == 0 && (ldv == 0 || ldv >= rows8_bytes(width))));
}

inline Rows8 rows8(void* values, int64_t rows, int64_t width, int64_t ldv, void* scales) {
    return {static_cast<uint8_t*>(values), ldv, static_cast<uint8_t*>(scales), rows, ceil_div(width, kBlock)};
}

inline int team_lanes(int64_t chunks) {
    int lanes = kBlockLanes;
    while (lanes < chunks && lanes < 256) lanes *= 2;
    return lanes;
}

inline unsigned team_groups(int64_t rows, int lanes) { return (unsigned)std::min<int64_t>(ceil_div(rows, 256 / lanes), 1 << 16); }

template <typename T>
void launch_quantise(int kind, int64_t rows, int64_t width, const T* x, int64_t ldx, const Rows8& to, hipStream_t stream) {
    const int lanes = team_lanes(to.blocks * kBlockLanes);
    const int type = sizeof(T) == 4 ? DGSP_F32 : std::is_same_v<T, f16_t> ? DGSP_F16 : DGSP_BF16;
    const Rows8Args<T> args{rows, width, lanes, scale_range(kind, type), const_cast<T*>(x), ldx, to};
    if (kind == DGSP_E4M3)
        quantise_kernel<T, true><<<team_groups(rows, lanes), 256, 0, stream>>>(args);
    else
        quantise_kernel<T, false><<<team_groups(rows, lanes), 256, 0, stream>>>(args);
}

template <typename T>
void launch_dequantise(int kind, int64_t rows, int64_t width, const Rows8& from, T* y, int64_t ldy, hipStream_t stream) {
    const int lanes = team_lanes(ceil_div(width, kChunk));
    const Rows8Args<T> args{rows, width, lanes, {}, y, ldy, from};
    if (kind == DGSP_E4M3)
        dequantise_kernel<T, true><<<team_groups(rows, lanes), 256, 0, stream>>>(args);
    else
        dequantise_kernel<T, false><<<team_groups(rows, lanes), 256, 0, stream>>>(args);
}

}  // namespace dgsp
