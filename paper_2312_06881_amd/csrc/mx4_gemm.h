// Shared pieces of the fp4 product's kernels.
#pragma once

#include "mx_common.h"

namespace dyad {

typedef __attribute__((ext_vector_type(8))) int i32x8_t;

struct Mx4Args {
    int64_t M, n_in, n_out;
    int D, bi, bo;
    const void *X;
    const uint8_t *wc, *ws, *xc, *xs;    // codes and scales of weights and input
    int w_frags, w_groups, x_frags, x_groups, steps;
    const void *bias;
    void *Y;
    int gelu, in_t;
    int tiles_n, tiles;
    int tiles_m, m_fast; // token panels; whether they are the fastest (small tiles)
    int wave_n;          // waves side by side along the columns
    int group_m;         // large tiles: token panels per run of tiles
};

// Large tiles (mx4_tiles.hip), no output transpose; hipErrorNotSupported, launching
// nothing, where they would leave CUs idle.
hipError_t launch_mx4_tiles(const Mx4Args &a, bool bf16, hipStream_t s);

// Large tiles under an output transpose (mx4_res_tiles.hip), bf16 and weights by
// residue; hipErrorNotSupported, launching nothing, for the others.
hipError_t launch_mx4_res_tiles(const Mx4Args &a, hipStream_t s);

// acc += W fragment (16 outputs) times X fragment (16 tokens) over 128 indices.
// The weights are the first operand: a lane's four sums are outputs
// 4 * (lane / 16) + v of token lane % 16.  BW, BX: bytes of the scale words.
template <int BW, int BX>
__device__ __forceinline__ f32x4_t mx4_mfma(uint4 w, uint4 x, f32x4_t acc, uint32_t sw, uint32_t sx) {
    const i32x8_t wv = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0};
    const i32x8_t xv = {(int)x.x, (int)x.y, (int)x.z, (int)x.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, xv, acc, 4, 4, BW, (int)sw, BX, (int)sx);
}

template <int J, int I, int SN, int SM>
__device__ __forceinline__ void mx4_multiply(const uint4 (&w)[SN], const uint4 (&x)[SM], const uint32_t (&sw)[(SN + 3) / 4],
                                             const uint32_t (&sx)[(SM + 3) / 4], f32x4_t (&acc)[SN][SM]) {
    acc[J][I] = mx4_mfma<J % 4, I % 4>(w[J], x[I], acc[J][I], sw[J / 4], sx[I / 4]);
    if constexpr (I + 1 < SM) mx4_multiply<J, I + 1, SN, SM>(w, x, sw, sx, acc);
    else if constexpr (J + 1 < SN) mx4_multiply<J + 1, 0, SN, SM>(w, x, sw, sx, acc);
}

template <int N, int M>
__device__ __forceinline__ void mx4_zero(f32x4_t (&acc)[N][M]) {
#pragma unroll
    for (int c = 0; c < N; ++c)
#pragma unroll
        for (int t = 0; t < M; ++t) acc[c][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
}

template <typename T>
__device__ __forceinline__ float mx4_act(const Mx4Args &a, float x) {
    return !a.gelu ? x : sizeof(T) == 2 ? gelu(x) : gelu_f32(x);
}

// Up to four consecutive outputs x of token m from column f: `n` of them real.
template <typename T>
__device__ __forceinline__ void mx4_store(const Mx4Args &a, int64_t m, int64_t f, int n, f32x4_t x) {
    if (n <= 0 || m >= a.M) return;
    const T *bias = static_cast<const T *>(a.bias);
    if (bias) {
#pragma unroll
        for (int v = 0; v < 4; ++v) x[v] += v < n ? load_f32<T>(bias, f + v) : 0.f;
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) x[v] = mx4_act<T>(a, x[v]);
    T *dst = static_cast<T *>(a.Y) + m * a.n_out + f;
    if (n >= 4 && ((uintptr_t)dst & (4 * sizeof(T) - 1)) == 0) {
        if constexpr (sizeof(T) == 2)
            *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
        else
            *reinterpret_cast<f32x4_t *>(dst) = x;
    } else {
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (v < n) store_f32<T>(dst, v, x[v]);
    }
}

// Swaps the odd lane rows of a with the even ones of b.
__device__ __forceinline__ void mx4_swap(uint32_t &a, uint32_t &b) {
    typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
    const u32x2_t r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r.x;
    b = r.y;
}

// Two fragments' outputs of token m in bf16, columns f .. f + 31 of a row, all
// real and 16-byte aligned: after the row swap a lane holds eight of them.
__device__ __forceinline__ void mx4_store_pair(const Mx4Args &a, int64_t m, int64_t f, int lane, const float (&b)[8],
                                               f32x4_t x, f32x4_t y) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        x[v] = mx4_act<uint16_t>(a, x[v] + b[v]);
        y[v] = mx4_act<uint16_t>(a, y[v] + b[4 + v]);
    }
    uint32_t d0 = pack_bf16(x[0], x[1]), d1 = pack_bf16(x[2], x[3]);
    uint32_t s0 = pack_bf16(y[0], y[1]), s1 = pack_bf16(y[2], y[3]);
    mx4_swap(d0, s0);
    mx4_swap(d1, s1);
    const int lg = lane >> 4, piece = (lg & 1) * 16 + (lg >> 1) * 8;
    if (m < a.M)
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.Y) + m * a.n_out + f + piece) = make_uint4(d0, d1, s0, s1);
}

// The wave's block without an output transpose: fragments c0.. of block g (SN),
// tokens from fragment t0 (SM).
template <int SN, int SM, typename T>
__device__ __forceinline__ void mx4_epilogue(const Mx4Args &a, int g, int c0, int64_t t0, int lane, const f32x4_t (&acc)[SN][SM]) {
    const int quad = 4 * (lane >> 4), row = lane & 15;
    const int64_t base = (int64_t)g * a.bo;
    int64_t end = base + a.bo < a.n_out ? base + a.bo : a.n_out;      // real columns of the block
    if constexpr (sizeof(T) == 2 && SN % 2 == 0) {
        if (base + (c0 + SN) * 16 <= end && a.n_out % 8 == 0 && a.bo % 8 == 0) {
            const uint16_t *bias = static_cast<const uint16_t *>(a.bias);
#pragma unroll
            for (int j = 0; j < SN; j += 2) {
                const int64_t f = base + (c0 + j) * 16;
                float b[8];
#pragma unroll
                for (int v = 0; v < 8; ++v) b[v] = bias ? bf16_to_f32(bias[f + (v < 4 ? quad + v : 12 + quad + v)]) : 0.f;
#pragma unroll
                for (int i = 0; i < SM; ++i) mx4_store_pair(a, (t0 + i) * 16 + row, f, lane, b, acc[j][i], acc[j + 1][i]);
            }
            return;
        }
    }
#pragma unroll
    for (int j = 0; j < SN; ++j) {
        const int64_t f = base + (c0 + j) * 16 + quad;
#pragma unroll
        for (int i = 0; i < SM; ++i)
            mx4_store<T>(a, (t0 + i) * 16 + row, f, end - f < 4 ? (int)(end - f) : 4, acc[j][i]);
    }
}

}  // namespace dyad
