// Fragment order of the fp4 product's operands (mx_internal.h): weights once,
// the input within each call.
//
// The input's pass reads every value once and writes its codes once, or twice
// under an input transpose: a workgroup stages 16 tokens x a span of columns in
// LDS, from which the contiguous blocks and the residues k*D + g are taken.
// The lanes of a wave write 1 KB of a fragment in a row.  What bounds it is that
// traffic: 8192 tokens of 4096 in both orders, 25 us (4.1 TB/s), where one wave a
// fragment that loads its values itself took 162.  The weights, once for a model, do
// that all the same: 4096 -> 16384, n_dyad 4, 75 us (1.1 TB/s), 183 in the order of
// residues.
#include "mx_common.h"

namespace dyad {

namespace {

struct Mx4PackArgs {
    int64_t M, n_in, n_out;
    int D, bi, bo, in_t, out_t, by_residue;
    const void *W1, *W2, *X;
    uint8_t *codes, *scales;
    int parts, frags, steps, groups;
    int64_t items;      // fragments times steps (general kernel)
    int span, tiles;    // columns a workgroup stages, and how many of them a row has
};

// Codes and scale byte into row `row`'s block kb of fragment `frag` of part `part`.
__device__ __forceinline__ void mx4_put(const Mx4PackArgs &a, int part, int64_t frag, int row, int kb, uint32_t sb, uint4 c) {
    const int s = kb >> 2, lane = (kb & 3) * 16 + row;
    reinterpret_cast<uint4 *>(a.codes + ((part * (int64_t)a.frags + frag) * a.steps + s) * 1024)[lane] = c;
    a.scales[((part * (int64_t)a.groups + (frag >> 2)) * a.steps + s) * 256 + lane * 4 + (frag & 3)] = (uint8_t)sb;
}

// Wide rows of any blocks, and the weights: a wave a fragment and step, values loaded one by
// one.  WEIGHTS: part = component * D + block of W1 / W2, else block (or, from D
// on, residue) of the input.
template <bool WEIGHTS, typename T>
__global__ void __launch_bounds__(256) mx4_pack_kernel(Mx4PackArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (item >= a.items) return;
    // parts fastest: the waves that read the same rows' residues run together
    const int part = (int)(item % a.parts), s = (int)(item / a.parts % a.steps);
    const int64_t fr = item / a.parts / a.steps;
    const bool second = part >= a.D;
    const int g = second ? part - a.D : part;
    const bool strided = second && a.in_t;                // input columns k*D + g
    int64_t row = fr * 16 + (lane & 15);
    const int k0 = s * 128 + (lane >> 4) * 32;
    const int64_t n = a.n_in;
    float x[32];
    const T *src;
    int64_t step;
    bool real;
    if constexpr (WEIGHTS) {
        if (a.by_residue && !second) row = row % (a.bo / a.D) * a.D + row / (a.bo / a.D);
        src = static_cast<const T *>(second ? a.W2 : a.W1) + ((int64_t)g * a.bo + row) * a.bi;
        const int64_t out = second && a.out_t ? row * a.D + g : (int64_t)g * a.bo + row;
        real = row < a.bo && out < a.n_out;
        step = 1;
    } else {
        src = static_cast<const T *>(a.X) + row * n + (strided ? g : (int64_t)g * a.bi);
        real = row < a.M;
        step = strided ? a.D : 1;
    }
#pragma unroll
    for (int e = 0; e < 32; ++e) {
        const int k = k0 + e;
        const int64_t col = strided ? (int64_t)k * a.D + g : (int64_t)g * a.bi + k;
        x[e] = real && k < a.bi && col < n ? load_f32<T>(src, k * step) : 0.f;
    }
    uint32_t sb;
    const uint4 c = mx4_encode(x, sb);
    mx4_put(a, part, fr, lane & 15, k0 >> 5, sb, c);
}

// Input whose blocks are whole 32s (n_in = D * bi).  RW: residues a lane takes
// from one LDS read, 0 without an input transpose.
template <int RW, typename T>
__global__ void __launch_bounds__(256) mx4_input_kernel(Mx4PackArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    constexpr int E = sizeof(T);
    const int tid = threadIdx.x;
    const int tile = blockIdx.x % a.tiles;
    const int64_t frag = blockIdx.x / a.tiles, m0 = frag * 16;
    const int n = (int)a.n_in, c0 = tile * a.span;
    const int cols = n - c0 < a.span ? n - c0 : a.span;
    const int pitch = a.span * E + 16;                    // rows four banks apart
    const int per_row = cols * E / 16, real = (int)(a.M - m0 < 16 ? a.M - m0 : 16);
    const unsigned char *src = static_cast<const unsigned char *>(a.X) + (m0 * n + c0) * E;
    for (int p = tid; p < 16 * per_row; p += 256) {
        const int row = p / per_row, q = p - row * per_row;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (row < real) v = *reinterpret_cast<const uint4 *>(src + (int64_t)row * n * E + q * 16);
        *reinterpret_cast<uint4 *>(smem + row * pitch + q * 16) = v;
    }
    __syncthreads();
    const int nk = a.bi / 32;                             // blocks of 32 in a block
    // a lane that has written the last of them zeroes the rest of the step
    auto put = [&](int part, int row, int kb, uint32_t sb, uint4 c) {
        mx4_put(a, part, frag, row, kb, sb, c);
        if (kb == nk - 1)
            for (int z = nk; z < 4 * a.steps; ++z) mx4_put(a, part, frag, row, z, 0u, make_uint4(0u, 0u, 0u, 0u));
    };
    const int row = tid & 15;
    for (int b = tid >> 4; b < cols / 32; b += 16) {
        const unsigned char *p = smem + row * pitch + b * 32 * E;
        const int g = (c0 + 32 * b) / a.bi, kb = (c0 + 32 * b - g * a.bi) >> 5;
        uint32_t sb;
        uint4 c;
        if constexpr (E == 2) {
            uint32_t x[16];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint4 v = *reinterpret_cast<const uint4 *>(p + 16 * q);
                x[4 * q] = v.x; x[4 * q + 1] = v.y; x[4 * q + 2] = v.z; x[4 * q + 3] = v.w;
            }
            c = mx4_encode(x, sb);
        } else {
            float x[32];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float4 v = *reinterpret_cast<const float4 *>(p + 16 * q);
                x[4 * q] = v.x; x[4 * q + 1] = v.y; x[4 * q + 2] = v.z; x[4 * q + 3] = v.w;
            }
            c = mx4_encode(x, sb);
        }
        put(g, row, kb, sb, c);
    }
    if constexpr (RW > 0) {
        const int D = a.D, nb = cols / (32 * D), kb0 = tile * (a.span / (32 * D));
        for (int it = tid >> 4; it < nb * (D / RW); it += 16) {
            const int bl = it % nb, g = it / nb * RW;
            const unsigned char *p = smem + row * pitch + (bl * 32 * D + g) * E;
            if constexpr (E == 2) {
                constexpr int kW = RW > 1 ? RW / 2 : 1;
                uint32_t v[32][kW];
#pragma unroll
                for (int t = 0; t < 32; ++t) {
                    const unsigned char *q = p + t * D * E;
                    if constexpr (RW == 4) {
                        const uint2 u = *reinterpret_cast<const uint2 *>(q);
                        v[t][0] = u.x;
                        v[t][1] = u.y;
                    } else if constexpr (RW == 2) {
                        v[t][0] = *reinterpret_cast<const uint32_t *>(q);
                    } else {
                        v[t][0] = *reinterpret_cast<const uint16_t *>(q);
                    }
                }
#pragma unroll
                for (int r = 0; r < RW; ++r) {
                    uint32_t x[16], sb;
#pragma unroll
                    for (int t = 0; t < 16; ++t)
                        x[t] = __builtin_amdgcn_perm(v[2 * t + 1][r / 2], v[2 * t][r / 2], (r & 1) ? perm_sel(2, 6) : perm_sel(0, 4));
                    const uint4 c = mx4_encode(x, sb);
                    put(D + g + r, row, kb0 + bl, sb, c);
                }
            } else {
                float v[RW][32];
#pragma unroll
                for (int t = 0; t < 32; ++t) {
                    const unsigned char *q = p + t * D * E;
                    if constexpr (RW == 2) {
                        const float2 u = *reinterpret_cast<const float2 *>(q);
                        v[0][t] = u.x;
                        v[1][t] = u.y;
                    } else {
                        v[0][t] = *reinterpret_cast<const float *>(q);
                    }
                }
#pragma unroll
                for (int r = 0; r < RW; ++r) {
                    uint32_t sb;
                    const uint4 c = mx4_encode(v[r], sb);
                    put(D + g + r, row, kb0 + bl, sb, c);
                }
            }
        }
    }
}

// Input of any blocks whose rows fit LDS sixteen at a time: a workgroup stages
// 16 tokens whole and takes `per` of the parts from them.
template <typename T>
__global__ void __launch_bounds__(256) mx4_rows_kernel(Mx4PackArgs a, int per) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    constexpr int E = sizeof(T);
    const int tid = threadIdx.x, n = (int)a.n_in, pieces = n * E / 16, pitch = (n * E + 15) / 16 * 16 + 16;
    const int64_t frag = blockIdx.x / a.tiles, m0 = frag * 16;
    const int p0 = blockIdx.x % a.tiles * per, p1 = p0 + per < a.parts ? p0 + per : a.parts;
    const int real = (int)(a.M - m0 < 16 ? a.M - m0 : 16);
    const T *src = static_cast<const T *>(a.X) + m0 * n;
    for (int i = tid; i < real * pieces; i += 256) {
        const int row = i / pieces, q = i - row * pieces;
        *reinterpret_cast<uint4 *>(smem + row * pitch + 16 * q) = load_any<uint4>(src + (int64_t)row * n + q * (16 / E));
    }
    const int first = pieces * (16 / E), rest = n - first;
    for (int i = tid; i < real * rest; i += 256) {
        const int row = i / rest, c = first + i - row * rest;
        *reinterpret_cast<T *>(smem + row * pitch + c * E) = src[(int64_t)row * n + c];
    }
    __syncthreads();
    const int row = tid & 15, kbs = 4 * a.steps;
    for (int i = tid >> 4; i < (p1 - p0) * kbs; i += 16) {
        const int part = p0 + i / kbs, kb = i % kbs;
        const bool second = part >= a.D;
        const int g = second ? part - a.D : part;
        const bool strided = second && a.in_t;
        const int col0 = strided ? kb * 32 * a.D + g : g * a.bi + kb * 32, step = strided ? a.D : 1;
        float x[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            const int col = col0 + e * step;
            x[e] = row < real && kb * 32 + e < a.bi && col < n
                       ? load_f32<T>(reinterpret_cast<const T *>(smem + row * pitch), col) : 0.f;
        }
        uint32_t sb;
        const uint4 c = mx4_encode(x, sb);
        mx4_put(a, part, frag, row, kb, sb, c);
    }
}

hipError_t layout_args(Mx4PackArgs &a, const Mx4Layout &l) {
    if (l.frags >= ((int64_t)1 << 31) || l.parts >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
    a.parts = (int)l.parts; a.frags = (int)l.frags; a.steps = (int)l.steps; a.groups = (int)l.groups();
    a.scales = a.codes + l.code_bytes();
    a.items = l.parts * l.frags * l.steps;
    return (a.items + 3) / 4 < ((int64_t)1 << 31) ? hipSuccess : hipErrorInvalidValue;
}

template <typename T>
hipError_t run_input(Mx4PackArgs &a, hipStream_t s) {
    constexpr int E = sizeof(T);
    const int D = a.D;
    // whole steps of every residue where 64 KB hold them and the GPU has enough
    // workgroups, else fewer blocks; without residues any columns do
    int span = a.in_t ? 0 : (int64_t)a.frags * ((a.n_in + 511) / 512) >= 512 ? 512 : 128;
    if (a.in_t)
        for (int kb = 4; kb >= 1 && !span; kb /= 2)
            if ((int64_t)16 * 32 * kb * D * E <= 65536 &&
                (kb == 1 || a.frags * ((a.n_in + 32 * kb * D - 1) / (32 * kb * D)) >= 256))
                span = 32 * kb * D;
    // residues a lane takes: one where there are fewer than lanes otherwise
    const int64_t lanes = span / 32 * 16;
    const int rw = !a.in_t ? 0 : E == 2 && D % 4 == 0 && lanes >= 1024 ? 4 : D % 2 == 0 && lanes >= 512 ? 2 : 1;
    const int64_t tiles = span ? (a.n_in + span - 1) / span : 0;
    if (a.bi % 32 != 0 || a.n_in != (int64_t)D * a.bi || !span || tiles * a.frags >= ((int64_t)1 << 31)) {
        const size_t rows = 16 * ((size_t)(a.n_in * E + 15) / 16 * 16 + 16);
        if (rows <= 65536 + 256) {
            // as many workgroups to 16 tokens as fill the GPU
            const int64_t want = (512 + a.frags - 1) / a.frags, most = want < a.parts ? want : a.parts;
            const int per = (int)((a.parts + most - 1) / most);
            a.tiles = (a.parts + per - 1) / per;
            if ((int64_t)a.tiles * a.frags < ((int64_t)1 << 31)) {
                mx4_rows_kernel<T><<<(unsigned)(a.tiles * a.frags), 256, rows, s>>>(a, per);
                return hipGetLastError();
            }
        }
        mx4_pack_kernel<false, T><<<(unsigned)((a.items + 3) / 4), 256, 0, s>>>(a);
        return hipGetLastError();
    }
    a.span = span;
    a.tiles = (int)tiles;
    const unsigned grid = (unsigned)(tiles * a.frags);
    const size_t lds = (size_t)16 * (size_t)(span * E + 16);
    switch (rw) {
    case 0: mx4_input_kernel<0, T><<<grid, 256, lds, s>>>(a); break;
    case 1: mx4_input_kernel<1, T><<<grid, 256, lds, s>>>(a); break;
    case 2: mx4_input_kernel<2, T><<<grid, 256, lds, s>>>(a); break;
    default:
        if constexpr (E == 2) mx4_input_kernel<4, T><<<grid, 256, lds, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_pack(int64_t n_in, int64_t n_out, int64_t D, bool in_t, bool out_t, int dtype, const void *W1,
                           const void *W2, void *packed, hipStream_t s) {
    Mx4PackArgs a{};
    a.n_in = n_in; a.n_out = n_out; a.D = (int)D;
    a.bi = (int)((n_in + D - 1) / D); a.bo = (int)((n_out + D - 1) / D);
    a.in_t = in_t; a.out_t = out_t; a.by_residue = mx4_by_residue(D, a.bo, out_t);
    a.W1 = W1; a.W2 = W2;
    a.codes = static_cast<uint8_t *>(packed);
    const hipError_t e = layout_args(a, mx4_weights_layout(D, a.bi, a.bo));
    if (e != hipSuccess) return e;
    const unsigned grid = (unsigned)((a.items + 3) / 4);
    if (dtype == kBF16) mx4_pack_kernel<true, uint16_t><<<grid, 256, 0, s>>>(a);
    else mx4_pack_kernel<true, float><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_mx4_input(const Mx4Pass &p, hipStream_t s) {
    Mx4PackArgs a{};
    a.M = p.M; a.n_in = p.n_in; a.n_out = p.n_out; a.D = (int)p.D; a.bi = (int)p.bi; a.bo = (int)p.bo;
    a.in_t = p.in_t && p.D > 1; a.out_t = p.out_t;
    a.X = p.X;
    a.codes = static_cast<uint8_t *>(p.ws);
    const hipError_t e = layout_args(a, mx4_input_layout(p.D, p.bi, p.M, a.in_t));
    if (e != hipSuccess) return e;
    return p.dtype == kBF16 ? run_input<uint16_t>(a, s) : run_input<float>(a, s);
}

}  // namespace dyad
