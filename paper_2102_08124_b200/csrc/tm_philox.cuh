// Random numbers of the operators, from a counter: Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel Random Numbers: As Easy as
// 1, 2, 3", 2011).  Key: the two halves of the seed; counter: (block, row, the two halves of the offset), low halves first.  Any element's numbers
// can be had again from its place alone, so no mask is ever stored.
#pragma once
#include <cstdint>

#include "tm_launch.h"

namespace tmask {

// A kernel's generator: the keys of the rounds lie among its arguments, so that they are operands and no instructions
struct Philox {
    const PhiloxKeys& keys;
    uint32_t o0, o1;
    __device__ __forceinline__ Philox(const PhiloxKeys& keys_, unsigned long long offset, const unsigned long long* offset_dev) : keys(keys_) {
        if (offset_dev) offset += *offset_dev;
        o0 = (uint32_t)offset; o1 = (uint32_t)(offset >> 32);
    }
    __device__ __forceinline__ uint4 operator()(uint32_t block, uint32_t row) const {
        uint32_t c0 = block, c1 = row, c2 = o0, c3 = o1;
#pragma unroll
        for (int i = 0; i < kPhiloxRounds; ++i) {
            const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
            c0 = (uint32_t)(b >> 32) ^ c1 ^ keys.k[2 * i];
            c1 = (uint32_t)b;
            c2 = (uint32_t)(a >> 32) ^ c3 ^ keys.k[2 * i + 1];
            c3 = (uint32_t)a;
        }
        return make_uint4(c0, c1, c2, c3);
    }
};

// Dropout: a block is eight columns of a row, sixteen bits each, the low half of the first word first.  Bit j of the result: column j stays,
// its bits being limit or more.  The high half of a word is compared with the low one still below it, which decides nothing.
__device__ __forceinline__ uint32_t kept_bits(const uint4& w, uint32_t limit) {
    const uint32_t high = limit << 16, u[4] = {w.x, w.y, w.z, w.w};
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bits |= ((u[i] << 16) >= high ? 1u : 0u) << (2 * i);
        bits |= (u[i] >= high ? 2u : 0u) << (2 * i);
    }
    return bits;
}

}  // namespace tmask
