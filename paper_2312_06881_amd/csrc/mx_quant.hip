// Microscaled quantisation of row-major matrices, and back.
//
// Quantising is one pass: a block of 32 values is held by four neighbouring
// lanes, eight values each, whose largest magnitude meets over two lane
// exchanges.  Nothing but the traffic bounds either direction (a few
// operations a value), so each lane moves 16 or 32 bytes at a time.  16384 x
// 3072 bf16 to int8 in 30 us and back in 23.5 (5.1 and 6.5 TB/s: part of it stays
// in the last cache); 4099 x 1001 floats to fp4, no row aligned, in 5.7 and back in 7.6.
#include "mx_common.h"

namespace dyad {

namespace {

constexpr int kThreads = 256, kUnits = 4;     // units of 8 values a thread

// Eight values of a row, of which `n` exist.
template <typename T>
__device__ __forceinline__ void load8(const T *p, int n, float (&x)[8]) {
    if (n == 8) {
        if constexpr (sizeof(T) == 2) {
            const uint4 v = load_any<uint4>(p);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = unpack_bf16(word_of(v, e >> 1), e & 1);
        } else {
            const float4 a = load_any<float4>(p), b = load_any<float4>(p + 4);
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
            x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < n ? load_f32<T>(p, e) : 0.f;
    }
}

// A workgroup takes kThreads * kUnits consecutive units of 8 values, `per_row`
// (a multiple of 4) to a row; units past the row's end hold nothing.
struct Units {
    int64_t row0;
    uint32_t rem, per_row;
    int64_t total;
    __device__ Units(int64_t rows, uint32_t pr) : per_row(pr), total(rows * pr) {
        const int64_t base = (int64_t)blockIdx.x * (kThreads * kUnits);
        row0 = base / pr;
        rem = (uint32_t)(base - row0 * pr);
    }
    // unit `q` of this thread: false past the matrix
    __device__ __forceinline__ bool at(int q, int64_t &row, uint32_t &u) const {
        const uint32_t t = rem + (uint32_t)(q * kThreads) + threadIdx.x;
        const uint32_t r = t / per_row;
        row = row0 + r;
        u = t - r * per_row;
        return (int64_t)blockIdx.x * (kThreads * kUnits) + q * kThreads + threadIdx.x < total;
    }
};

template <int FMT, typename T>
__global__ void __launch_bounds__(kThreads) mx_quantize_kernel(int64_t rows, int64_t cols, const T *__restrict__ X,
                                                               uint8_t *__restrict__ codes,
                                                               uint8_t *__restrict__ scales) {
    const int64_t nb = (cols + kMxBlock - 1) / kMxBlock, code_row = FMT == kMxInt8 ? cols : (cols + 1) / 2;
    const Units units(rows, (uint32_t)(4 * nb));
    float x[kUnits][8];
    int64_t row[kUnits];
    uint32_t u[kUnits];
    int n[kUnits];
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
        const bool in = units.at(q, row[q], u[q]);
        const int64_t left = cols - (int64_t)u[q] * 8;
        n[q] = !in || left < 0 ? 0 : left < 8 ? (int)left : 8;
        load8<T>(X + row[q] * cols + (int64_t)u[q] * 8, n[q], x[q]);
    }
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
        const uint32_t s = mx_scale<FMT>(quad_max(mag_max(x[q])));
        if (n[q] > 0 && (u[q] & 3u) == 0u) scales[row[q] * nb + u[q] / 4u] = (uint8_t)s;
        if constexpr (FMT == kMxInt8) {
            uint8_t *dst = codes + row[q] * code_row + (int64_t)u[q] * 8;
            const uint32_t w[2] = {mx_int8x4(x[q][0], x[q][1], x[q][2], x[q][3], s),
                                   mx_int8x4(x[q][4], x[q][5], x[q][6], x[q][7], s)};
            if (n[q] == 8) {
                store_any(dst, make_uint2(w[0], w[1]));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < n[q]) dst[e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
            }
        } else {
            uint8_t *dst = codes + row[q] * code_row + (int64_t)u[q] * 4;
            const uint32_t w = s == 255u ? 0u : mx_fp4x8(x[q], mx_pow(s));
            if (n[q] == 8) {
                store_any(dst, w);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (2 * e < n[q]) dst[e] = (uint8_t)(w >> (8 * e));
            }
        }
    }
}

template <int FMT, typename T, bool GELU>
__global__ void __launch_bounds__(kThreads) mx_dequantize_kernel(int64_t rows, int64_t cols,
                                                                 const uint8_t *__restrict__ codes,
                                                                 const uint8_t *__restrict__ scales,
                                                                 T *__restrict__ Y) {
    const int64_t nb = (cols + kMxBlock - 1) / kMxBlock, code_row = FMT == kMxInt8 ? cols : (cols + 1) / 2;
    const Units units(rows, (uint32_t)(4 * nb));
    uint32_t w[kUnits][2], s[kUnits];
    int64_t row[kUnits];
    uint32_t u[kUnits];
    int n[kUnits];
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
        const bool in = units.at(q, row[q], u[q]);
        const int64_t left = cols - (int64_t)u[q] * 8;
        n[q] = !in || left < 0 ? 0 : left < 8 ? (int)left : 8;
        w[q][0] = w[q][1] = 0u;
        s[q] = n[q] > 0 ? scales[row[q] * nb + u[q] / 4u] : 0u;
        const uint8_t *src = codes + row[q] * code_row + (int64_t)u[q] * (FMT == kMxInt8 ? 8 : 4);
        if (n[q] == 8) {
            if constexpr (FMT == kMxInt8) {
                const uint2 v = load_any<uint2>(src);
                w[q][0] = v.x;
                w[q][1] = v.y;
            } else {
                w[q][0] = load_any<uint32_t>(src);
            }
        } else if constexpr (FMT == kMxInt8) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n[q]) w[q][e >> 2] |= (uint32_t)src[e] << (8 * (e & 3));
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (2 * e < n[q]) w[q][0] |= (uint32_t)src[e] << (8 * e);
        }
    }
#pragma unroll
    for (int q = 0; q < kUnits; ++q) {
        float x[8];
        if constexpr (FMT == kMxInt8) {
            float lo[4], hi[4];
            mx_int8_values(w[q][0], mx_int8_step(s[q]), lo);
            mx_int8_values(w[q][1], mx_int8_step(s[q]), hi);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = lo[e];
                x[4 + e] = hi[e];
            }
        }
        const float half = mx_fp4_half_step(s[q]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (FMT == kMxFp4) x[e] = mx_fp4_twice(w[q][0] >> (4 * e)) * half;
            if constexpr (GELU) x[e] = sizeof(T) == 2 ? gelu(x[e]) : gelu_f32(x[e]);
        }
        T *dst = Y + row[q] * cols + (int64_t)u[q] * 8;
        if (n[q] < 8) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n[q]) store_f32<T>(dst, e, x[e]);
        } else if constexpr (sizeof(T) == 2) {
            store_any(dst, make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])));
        } else {
            store_any(dst, make_float4(x[0], x[1], x[2], x[3]));
            store_any(dst + 4, make_float4(x[4], x[5], x[6], x[7]));
        }
    }
}

// Workgroups for `rows` rows of `cols`; 0 when they are too many for a launch.
unsigned grid_for(int64_t rows, int64_t cols) {
    const int64_t units = rows * ((cols + kMxBlock - 1) / kMxBlock) * 4;
    const int64_t g = (units + kThreads * kUnits - 1) / (kThreads * kUnits);
    return g < ((int64_t)1 << 31) ? (unsigned)g : 0u;
}

}  // namespace

hipError_t launch_mx_quantize(int fmt, int64_t rows, int64_t cols, int dtype, const void *X, void *codes, void *scales,
                              hipStream_t s) {
    const unsigned grid = grid_for(rows, cols);
    if (!grid) return hipErrorInvalidValue;
    auto go = [&](auto f, auto t) {
        using T = decltype(t);
        mx_quantize_kernel<decltype(f)::value, T><<<grid, kThreads, 0, s>>>(
            rows, cols, static_cast<const T *>(X), static_cast<uint8_t *>(codes), static_cast<uint8_t *>(scales));
    };
    auto by_type = [&](auto f) {
        if (dtype == kBF16) go(f, uint16_t{});
        else go(f, float{});
    };
    if (fmt == kMxInt8) by_type(std::integral_constant<int, kMxInt8>{});
    else by_type(std::integral_constant<int, kMxFp4>{});
    return hipGetLastError();
}

hipError_t launch_mx_dequantize(int fmt, int64_t rows, int64_t cols, int dtype, const void *codes, const void *scales,
                                bool gelu, void *Y, hipStream_t s) {
    const unsigned grid = grid_for(rows, cols);
    if (!grid) return hipErrorInvalidValue;
    auto go = [&](auto f, auto t, auto act) {
        using T = decltype(t);
        mx_dequantize_kernel<decltype(f)::value, T, decltype(act)::value><<<grid, kThreads, 0, s>>>(
            rows, cols, static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), static_cast<T *>(Y));
    };
    auto by_type = [&](auto f, auto act) {
        if (dtype == kBF16) go(f, uint16_t{}, act);
        else go(f, float{}, act);
    };
    if (fmt == kMxFp4) by_type(std::integral_constant<int, kMxFp4>{}, std::false_type{});
    else if (gelu) by_type(std::integral_constant<int, kMxInt8>{}, std::true_type{});
    else by_type(std::integral_constant<int, kMxInt8>{}, std::false_type{});
    return hipGetLastError();
}

}  // namespace dyad
