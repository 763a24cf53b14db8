// Counter-based random bits for dropout: Philox-4x32 with ten rounds (Salmon,
// Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011).
// A value's bits follow from (seed, offset, row, column) alone, so no mask is kept:
// the backward pass draws it again.
#pragma once

#include "dyad_device.h"

namespace dyad {

// What a kernel needs to draw a mask.  thr of 65536 values of a 16-bit number
// are dropped; scale is 65536 / (65536 - thr), 0 where everything is dropped.
struct DropArgs {
    uint64_t seed, offset;
    const uint64_t *offset_dev;   // added to offset; null: 0
    uint32_t thr;
    float scale;
};

inline DropArgs drop_args(double p, uint64_t seed, uint64_t offset, const uint64_t *offset_dev) {
    DropArgs d;
    d.seed = seed;
    d.offset = offset;
    d.offset_dev = offset_dev;
    // p in [0, 1]; 16 bits a value, so that one evaluation serves eight (at 32 bits
    // each the generator's multiplies take as long as the memory traffic)
    d.thr = (uint32_t)__builtin_rint(p * 65536.0);
    d.scale = d.thr < 65536u ? (float)(65536.0 / (65536.0 - (double)d.thr)) : 0.f;
    return d;
}

__device__ __forceinline__ uint64_t drop_offset(const DropArgs &d) {
    return d.offset + (d.offset_dev ? *d.offset_dev : 0);
}

// The eight 16-bit numbers of octet `octet` as four words, value j in half j % 2 of word j / 2.
__device__ __forceinline__ uint4 philox(uint64_t seed, uint64_t offset, uint64_t octet) {
    uint32_t c0 = (uint32_t)octet, c1 = (uint32_t)(octet >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// Bit j: value j of the octet is kept.
__device__ __forceinline__ uint32_t keep_bits(const uint4 &r, uint32_t thr) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m |= (((w[j >> 1] >> (16 * (j & 1))) & 0xffffu) >= thr ? 1u : 0u) << j;
    return m;
}

// Dropped values are zero whatever they were; the others are scaled.
__device__ __forceinline__ void apply_drop(float (&v)[8], uint32_t keep, float scale) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (keep >> j) & 1u ? v[j] * scale : 0.f;
}

}  // namespace dyad
