// LDS side of the fp4 product's tiles: global-to-LDS loads, waits and barriers
// come with the bf16 tiles' loop.
#pragma once

#include "pp_core.h"

namespace dyad {

// SM fragments from LDS.  One block of instructions that ends in its own wait:
// the compiler orders an LDS read behind every global-to-LDS load in flight.
#define MX4_R(i, off) "ds_read_b128 %[x" #i "], %[p] offset:" #off "\n\t"
#define MX4_O(i) [x##i] "=&v"(v[i])
template <int SM>
__device__ __forceinline__ void mx4_read(uint32_t p, uint4 (&x)[SM]) {
    u32x4_t v[SM];
    static_assert(SM == 8 || SM == 4, "a fragment read exists");
    if constexpr (SM == 8)
        asm volatile(MX4_R(0, 0) MX4_R(1, 1024) MX4_R(2, 2048) MX4_R(3, 3072) MX4_R(4, 4096) MX4_R(5, 5120) MX4_R(6, 6144)
                         MX4_R(7, 7168) "s_waitcnt lgkmcnt(0)"
                     : MX4_O(0), MX4_O(1), MX4_O(2), MX4_O(3), MX4_O(4), MX4_O(5), MX4_O(6), MX4_O(7)
                     : [p] "v"(p)
                     : "memory");
    else
        asm volatile(MX4_R(0, 0) MX4_R(1, 1024) MX4_R(2, 2048) MX4_R(3, 3072) "s_waitcnt lgkmcnt(0)"
                     : MX4_O(0), MX4_O(1), MX4_O(2), MX4_O(3)
                     : [p] "v"(p)
                     : "memory");
#pragma unroll
    for (int i = 0; i < SM; ++i) x[i] = make_uint4(v[i].x, v[i].y, v[i].z, v[i].w);
}

}  // namespace dyad
