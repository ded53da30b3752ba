// What the host sides of the norms share: dropout's mask and how rows are held.
#pragma once

#include "layers_host.hpp"

#include <cmath>

#include "chunks.hpp"

namespace dgsp {

inline bool make_mask(const dgsp_dropout_t* d, DropMask& mask) {
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

// How rows of a width are held: up to 512 elements a wave holds one or several, up to 8192 a workgroup holds one.
struct Hold {
    bool whole;             // a workgroup a row
    int lanes, threads;
    bool fits;
    explicit Hold(int64_t width) {
        const int64_t chunks = ceil_div(width, kChunk);
        whole = chunks > 64;
        fits = chunks <= 1024;
        if (!whole) {
            lanes = 1;
            while (lanes < chunks) lanes *= 2;
            threads = 256;
        } else {
            threads = lanes = (int)std::min<int64_t>(1024, ceil_div(chunks, 64) * 64);
        }
    }
    int64_t rows_a_group() const { return whole ? 1 : threads / lanes; }
};

// Workgroups of the backward pass, each with sums of its own for the parameters, as many as the GPU holds at once.  Of many rows the sums
// are a small part of what is read anyway (32768 x 1024, 16 bits: 17 MB beside 268); where a workgroup is left with a row or two they are
// not: 4099 x 1001 has 2048 workgroups, whose sums of 16 MB are written and read again beside 33 MB read and 16 written.
inline int64_t backward_groups(const Hold& hold, int64_t rows) {
    if (!hold.fits) return std::min<int64_t>(std::max<int64_t>(rows, 1), 64);
    const int64_t most = hold.whole ? kCus * std::max(1, 1024 / hold.threads) : kCus * 4;
    return std::max<int64_t>(1, std::min(ceil_div(rows, hold.rows_a_group()), most));
}

}  // namespace dgsp
