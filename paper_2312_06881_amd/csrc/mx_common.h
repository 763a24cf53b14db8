// Device helpers of the microscaled formats: a block of 32 values shares the
// power of two 2^(s - 127) of its scale byte s, the largest one's floor(log2)
// less the element format's (0 for int8's k / 64, 2 for fp4, whose largest
// value is 6).  A block that holds an infinity or a NaN gets the scale byte 255
// and reads back as NaN throughout.
#pragma once

#include "mfma_common.h"
#include "mx_internal.h"

namespace dyad {

// Magnitude bits of a float: they order like the magnitudes, NaN above all.
__device__ __forceinline__ uint32_t mag_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Scale byte of a block from the largest magnitude bits in it.
template <int FMT>
__device__ __forceinline__ uint32_t mx_scale(uint32_t top) {
    const uint32_t e = top >> 23;                       // 0 for zero and subnormals: 2^-127 holds them
    if (e == 255u) return 255u;
    if constexpr (FMT == kMxInt8) return e;
    else return e > 2u ? e - 2u : 0u;
}

// 2^(s - 127), s < 255 (2^-127 is subnormal).
__device__ __forceinline__ float mx_pow(uint32_t s) { return __uint_as_float(s ? s << 23 : 0x00400000u); }

// int8 code of x: rounded to nearest even at 2^(s - 133), |code| <= 127.
__device__ __forceinline__ int mx_int8(float x, uint32_t s) {
    const float k = __builtin_amdgcn_fmed3f(rintf(ldexpf(x, 133 - (int)s)), -127.f, 127.f);
    return s == 255u ? 0 : (int)k;
}

// What the codes of a block are multiplied with: NaN for a non-finite block.
// Products of it with a code are exact in fp32, and in bf16: 7 bits.
__device__ __forceinline__ float mx_int8_step(uint32_t s) {
    return s == 255u ? __uint_as_float(0x7fc00000u) : ldexpf(1.f, (int)s - 133);
}

// fp4 codes of two values, the first in the low nibble (nearest even,
// saturating at 6), into byte BYTE of `old`.
template <int BYTE>
__device__ __forceinline__ uint32_t mx_fp4x2(uint32_t old, float a, float b, float pow) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, a, b, pow, BYTE);
}
// Eight codes.
__device__ __forceinline__ uint32_t mx_fp4x8(const float (&x)[8], float pow) {
    uint32_t w = mx_fp4x2<0>(0u, x[0], x[1], pow);
    w = mx_fp4x2<1>(w, x[2], x[3], pow);
    w = mx_fp4x2<2>(w, x[4], x[5], pow);
    return mx_fp4x2<3>(w, x[6], x[7], pow);
}
// Value of a code times two (a whole number): 0, 1, 2, 3, 4, 6, 8, 12.
__device__ __forceinline__ float mx_fp4_twice(uint32_t c) {
    const float m = (float)((0xc8643210u >> (4u * (c & 7u))) & 15u);
    return c & 8u ? -m : m;
}
__device__ __forceinline__ float mx_fp4_half_step(uint32_t s) {
    return s == 255u ? __uint_as_float(0x7fc00000u) : ldexpf(1.f, (int)s - 128);
}

}  // namespace dyad
