// Rows of any length and alignment, eight columns a lane.
#pragma once

#include "mfma_common.h"

namespace dyad {

// Eight values from p as fp32.  Rows of a width that 8 does not divide start at any
// element, so the access is declared with the element's alignment; global memory
// takes 16-byte instructions at such addresses, and at aligned ones they are the
// same instructions.
__device__ __forceinline__ void load8(const float *p, float (&v)[8]) { __builtin_memcpy(v, p, 32); }
__device__ __forceinline__ void load8(const uint16_t *p, float (&v)[8]) {
    uint32_t w[4];
    __builtin_memcpy(w, p, 16);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = unpack_bf16(w[e >> 1], e & 1);
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) { __builtin_memcpy(p, v, 32); }
__device__ __forceinline__ void store8(uint16_t *p, const float (&v)[8]) {
    const uint32_t w[4] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    __builtin_memcpy(p, w, 16);
}

// Columns c .. c + 7 of a row of n; columns past it read zero and are not written.
template <class T>
__device__ __forceinline__ void load_cols(const T *row, int c, int n, float (&v)[8]) {
    if (c + 8 <= n) {
        load8(row + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < n ? load_f32(row, c + e) : 0.f;
    }
}
// RAG: n may end inside the eight (element by element; rows of whole vectors have instances without).
template <bool RAG, class T>
__device__ __forceinline__ void store_cols(T *row, int c, int n, const float (&v)[8]) {
    if (c + 8 <= n) {
        store8(row + c, v);
    } else if constexpr (RAG) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < n) store_f32(row, c + e, v[e]);
    }
}

// Eight values as they lie in memory, for operands that wait in registers until they are used.
template <class T>
struct Raw {
    uint32_t w[sizeof(T) * 2];
};
// Columns c .. c + 7 of a row of n >= 8, zeros past it.  RAG: the octet that n ends in is read
// from column n - 8 on and moved down, without a branch (element by element, each a branch of its
// own, 3997 rows of 1001 took a backward pass 60 us, so 57).
template <bool RAG, class T>
__device__ __forceinline__ Raw<T> load_raw(const T *row, int c, int n) {
    constexpr int W = (int)sizeof(T) * 2;
    Raw<T> r;
    if constexpr (!RAG) {
#pragma unroll
        for (int i = 0; i < W; ++i) r.w[i] = 0u;
        if (c < n) __builtin_memcpy(r.w, row + c, sizeof(T) * 8);
    } else {
        const int at = c < n - 8 ? c : n - 8, s = c - at;      // values to drop in front
        __builtin_memcpy(r.w, row + at, sizeof(T) * 8);
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const uint32_t next = i + 1 < W ? r.w[i + 1] : 0u;
                r.w[i] = s & 1 ? __builtin_amdgcn_alignbit(next, r.w[i], 16) : r.w[i];
            }
        }
        // by whole words
        const int words = sizeof(T) == 2 ? s >> 1 : s;
#pragma unroll
        for (int step = 1; step < W; step *= 2)
#pragma unroll
            for (int i = 0; i < W; ++i) r.w[i] = words & step ? (i + step < W ? r.w[i + step] : 0u) : r.w[i];
#pragma unroll
        for (int i = 0; i < W; ++i) r.w[i] = s >= 8 ? 0u : r.w[i];
    }
    return r;
}
__device__ __forceinline__ void unpack8(const Raw<float> &r, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(r.w[e]);
}
__device__ __forceinline__ void unpack8(const Raw<uint16_t> &r, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = unpack_bf16(r.w[e >> 1], e & 1);
}

template <bool RAG, class T>
__device__ __forceinline__ void load_row(const T *row, int c, int n, float (&v)[8]) {
    unpack8(load_raw<RAG>(row, c, n), v);
}

}  // namespace dyad
