// Device helpers of the microscaled formats: a block of 32 values shares the
// power of two 2^(s - 127) of its scale byte s, the largest one's floor(log2)
// less the element format's (0 for int8's k / 64, 2 for fp4, whose largest
// value is 6).  A block that holds an infinity or a NaN gets the scale byte 255
// and reads back as NaN throughout.
#pragma once

#include "mfma_common.h"
#include "mx_internal.h"

namespace dyad {

typedef __attribute__((ext_vector_type(2))) unsigned short u16x2_t;

// Bytes at any address: rows of an odd width start anywhere (the hardware takes
// vector accesses at every alignment).
template <typename V>
__device__ __forceinline__ V load_any(const void *p) {
    V v;
    __builtin_memcpy(&v, p, sizeof v);
    return v;
}
template <typename V>
__device__ __forceinline__ void store_any(void *p, const V &v) {
    __builtin_memcpy(p, &v, sizeof v);
}

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

// int8 codes of four values: rounded to nearest even at 2^(s - 133) and at most
// 127.  Adding 1.5 * 2^23 leaves the code in the sum's low byte.
__device__ __forceinline__ uint32_t mx_int8x4(float a, float b, float c, float d, uint32_t s) {
    auto code = [&](float x) {
        return __float_as_uint(__builtin_amdgcn_fmed3f(ldexpf(x, 133 - (int)s), -127.f, 127.f) + 12582912.f);
    };
    const uint32_t ab = __builtin_amdgcn_perm(code(b), code(a), 0x0c0c0400u);
    const uint32_t cd = __builtin_amdgcn_perm(code(d), code(c), 0x04000c0cu);
    return s == 255u ? 0u : ab | cd;
}

// What the codes of a block are multiplied with: NaN for a non-finite block.
// Products of it with a code are exact in fp32, and in bf16: 7 bits.
__device__ __forceinline__ float mx_int8_step(uint32_t s) {
    return s == 255u ? __uint_as_float(0x7fc00000u) : ldexpf(1.f, (int)s - 133);
}

// Values of four codes, each a signed byte converted in place (one instruction)
// and multiplied, exactly.  (An offset taken off after the step would leave
// fp32's range in the largest blocks, 128 * 2^121.)
__device__ __forceinline__ void mx_int8_values(uint32_t codes, float step, float (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (float)(int8_t)(codes >> (8 * e)) * step;
}

// Eight codes as packed bf16, which holds each exactly.
__device__ __forceinline__ uint4 mx_int8_bf16(uint32_t lo, uint32_t hi, uint32_t s) {
    const float step = mx_int8_step(s);
    float a[4], b[4];
    mx_int8_values(lo, step, a);
    mx_int8_values(hi, step, b);
    return make_uint4(pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3]), pack_bf16(b[0], b[1]), pack_bf16(b[2], b[3]));
}

// Largest of a value over the four lanes of a quad, and over the four 16-lane rows.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));   // lanes 1, 0, 3, 2
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));   // lanes 2, 3, 0, 1
}
__device__ __forceinline__ uint32_t rows_max(uint32_t v) {
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max((uint32_t)a[0], (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max((uint32_t)b[0], (uint32_t)b[1]);
}

// Magnitude bits of the largest of eight.
__device__ __forceinline__ uint32_t mag_max(const float (&x)[8]) {
    uint32_t top = mag_bits(x[0]);
#pragma unroll
    for (int e = 1; e < 8; ++e) top = max(top, mag_bits(x[e]));
    return top;
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
// 32 values into 32 codes, and their scale byte.
__device__ __forceinline__ uint4 mx4_encode(const float (&x)[32], uint32_t &sb) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 32; ++e) top = max(top, mag_bits(x[e]));
    sb = mx_scale<kMxFp4>(top);
    if (sb == 255u) return make_uint4(0u, 0u, 0u, 0u);
    const float pow = mx_pow(sb);
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        w[q] = mx_fp4x2<0>(0u, x[8 * q], x[8 * q + 1], pow);
        w[q] = mx_fp4x2<1>(w[q], x[8 * q + 2], x[8 * q + 3], pow);
        w[q] = mx_fp4x2<2>(w[q], x[8 * q + 4], x[8 * q + 5], pow);
        w[q] = mx_fp4x2<3>(w[q], x[8 * q + 6], x[8 * q + 7], pow);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// 32 bf16 values as 16 words: magnitudes compared in pairs as whole numbers,
// codes from pairs.
__device__ __forceinline__ uint4 mx4_encode(const uint32_t (&x)[16], uint32_t &sb) {
    u16x2_t top = {0, 0};
#pragma unroll
    for (int e = 0; e < 16; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2_t, x[e] & 0x7fff7fffu));
    sb = mx_scale<kMxFp4>((uint32_t)max(top.x, top.y) << 16);
    if (sb == 255u) return make_uint4(0u, 0u, 0u, 0u);
    const float pow = mx_pow(sb);
    uint32_t w[4];
    auto pair = [&](int e) { return __builtin_bit_cast(bf16x2_t, x[e]); };
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        w[q] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, pair(4 * q), pow, 0);
        w[q] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w[q], pair(4 * q + 1), pow, 1);
        w[q] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w[q], pair(4 * q + 2), pow, 2);
        w[q] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w[q], pair(4 * q + 3), pow, 3);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
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
