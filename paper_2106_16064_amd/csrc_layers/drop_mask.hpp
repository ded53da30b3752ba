// Which elements dropout keeps: a function of seed, offset, row and column, never stored.
#pragma once

#include <cstdint>

#include "../csrc/host_device.hpp"

namespace dgsp {

// Philox4x32 with 10 rounds (Salmon, Moraes, Dror, Shaw, SC 2011): a bijection of 128-bit counters under a 64-bit key.
struct PhiloxWords {
    uint32_t w[4];
};

DGSP_HOST_DEVICE PhiloxWords philox4x32(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// As kernels take it.  `dropped` of the 65536 16-bit numbers drop their element.
struct DropMask {
    uint32_t dropped;
    float scale;                        // of the kept ones
    uint32_t key0, key1;
    uint64_t offset;
    const uint64_t* device_offset;      // read instead of `offset` unless null
};

// One counter serves eight neighbouring elements of a row with 16 bits each: the generator's 20 wide multiplications cost more
// than the memory accesses of four elements.  Rates are multiples of 1/65536.
constexpr int kDropGroup = 8;

// bit j: element 8 * group + j of the row is kept
DGSP_HOST_DEVICE uint32_t keep_bits(const DropMask& d, uint64_t offset, uint32_t row, uint32_t group) {
    const PhiloxWords r = philox4x32(group, row, (uint32_t)offset, (uint32_t)(offset >> 32), d.key0, d.key1);
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bits |= (uint32_t)((r.w[i] & 0xffffu) >= d.dropped) << (2 * i);
        bits |= (uint32_t)((r.w[i] >> 16) >= d.dropped) << (2 * i + 1);
    }
    return bits;
}

}  // namespace dgsp
