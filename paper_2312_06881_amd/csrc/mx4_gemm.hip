// The fp4 product of a Dyad layer: Y = act(W Q(X) + b), W's blocks and X kept as
// fp4 codes with a scale byte for each 32 reduction indices of a row.
//
// Per output column f and token m, with the scales s and codes c of the
// operands' blocks B of 32:
//   sum over both components, over B:  2^(sw - 127) 2^(sx - 127) sum_k cw cx
// which one v_mfma_scale_f32_16x16x128_f8f6f4 does for four blocks of 16 x 16
// outputs, summing in fp32.
//
// Operands.  Weights and input lie in fragment order (mx_internal.h), so every
// fragment is one 16-byte load a lane of 1 KB in a row, with no staging, no
// swizzle and no edge: rows and steps past the real ones hold zeros.  The
// input's copy under an input transpose holds each residue's columns k*D + g
// as a block of its own, so the permutation costs the quantising pass alone.
//
// Output transpose.  Component 2's block g makes columns j*D + g, component 1's
// block i columns i*bo + r.  A workgroup owns 16 * CF * D consecutive columns:
// every residue's CF fragments of 16 j for component 2, whose sums meet their
// columns in LDS, and the fragments of component 1 over the same columns, which
// add to them as they finish.
#include "mx_common.h"

namespace dyad {

namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8_t;

struct Mx4Args {
    int64_t M, n_in, n_out;
    int D, bi, bo;
    const uint8_t *wc, *ws, *xc, *xs;    // codes and scales of weights and input
    int w_frags, x_frags, steps, words;
    const void *bias;
    void *Y;
    int gelu, in_t;
    int tiles_n, tiles;
};

// acc[c][t] += W fragment row c (codes at wc + wo[c], scales at ws + wso[c]) times
// X fragment t over all steps.  The weights are the first operand: a lane
// ends up with four consecutive outputs 4 * (lane / 16) + v of token lane % 16.
template <int CF, int TM>
struct Mx4Frags {
    int64_t w[CF], x[TM];   // fragment numbers (part * frags + fragment), wave-uniform
};

template <int CF, int TM>
__device__ __forceinline__ void mx4_span(const Mx4Args &a, const Mx4Frags<CF, TM> &f, int lane, f32x4_t (&acc)[CF][TM]) {
    const int steps = a.steps, words = a.words;
    auto step = [&](auto byte, const uint32_t (&sw)[CF], const uint32_t (&sx)[TM], int s) {
        constexpr int B = decltype(byte)::value;
        uint4 w[CF], x[TM];
#pragma unroll
        for (int c = 0; c < CF; ++c) w[c] = reinterpret_cast<const uint4 *>(a.wc + (f.w[c] * steps + s) * 1024)[lane];
#pragma unroll
        for (int t = 0; t < TM; ++t) x[t] = reinterpret_cast<const uint4 *>(a.xc + (f.x[t] * steps + s) * 1024)[lane];
#pragma unroll
        for (int c = 0; c < CF; ++c)
#pragma unroll
            for (int t = 0; t < TM; ++t) {
                const i32x8_t wv = {(int)w[c].x, (int)w[c].y, (int)w[c].z, (int)w[c].w, 0, 0, 0, 0};
                const i32x8_t xv = {(int)x[t].x, (int)x[t].y, (int)x[t].z, (int)x[t].w, 0, 0, 0, 0};
                acc[c][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, xv, acc[c][t], 4, 4, B, (int)sw[c], B,
                                                                             (int)sx[t]);
            }
    };
    for (int q = 0; q < words; ++q) {
        uint32_t sw[CF], sx[TM];
#pragma unroll
        for (int c = 0; c < CF; ++c) sw[c] = reinterpret_cast<const uint32_t *>(a.ws + (f.w[c] * words + q) * 256)[lane];
#pragma unroll
        for (int t = 0; t < TM; ++t) sx[t] = reinterpret_cast<const uint32_t *>(a.xs + (f.x[t] * words + q) * 256)[lane];
        const int s = 4 * q;
        step(std::integral_constant<int, 0>{}, sw, sx, s);
        if (s + 4 <= steps) {
            step(std::integral_constant<int, 1>{}, sw, sx, s + 1);
            step(std::integral_constant<int, 2>{}, sw, sx, s + 2);
            step(std::integral_constant<int, 3>{}, sw, sx, s + 3);
        } else {
            if (s + 1 < steps) step(std::integral_constant<int, 1>{}, sw, sx, s + 1);
            if (s + 2 < steps) step(std::integral_constant<int, 2>{}, sw, sx, s + 2);
        }
    }
}

template <int CF, int TM>
__device__ __forceinline__ void mx4_zero(f32x4_t (&acc)[CF][TM]) {
#pragma unroll
    for (int c = 0; c < CF; ++c)
#pragma unroll
        for (int t = 0; t < TM; ++t) acc[c][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
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
    if (a.gelu) {
#pragma unroll
        for (int v = 0; v < 4; ++v) x[v] = sizeof(T) == 2 ? gelu(x[v]) : gelu_f32(x[v]);
    }
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

// No output transpose: block i's columns take block i of both components; a
// wave owns CF x TM fragments of one block, a workgroup 2 x 2 waves.
template <int CF, int TM, typename T>
__global__ void __launch_bounds__(256) mx4_gemm_kernel(Mx4Args a) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = xcd_tile(blockIdx.x, a.tiles);
    const int per_block = a.tiles_n / a.D;
    const int tn = tile % a.tiles_n, g = tn / per_block;
    const int c0 = (tn - g * per_block) * 2 * CF + (wave & 1) * CF;
    const int t0 = (tile / a.tiles_n) * 2 * TM + (wave >> 1) * TM;
    if (c0 >= a.w_frags || t0 >= a.x_frags) return;
    f32x4_t acc[CF][TM];
    mx4_zero(acc);
#pragma unroll 1
    for (int comp = 0; comp < 2; ++comp) {
        Mx4Frags<CF, TM> f;
        const int64_t wp = (int64_t)(comp * a.D + g) * a.w_frags, xp = (int64_t)(comp && a.in_t ? a.D + g : g) * a.x_frags;
#pragma unroll
        for (int c = 0; c < CF; ++c) f.w[c] = wp + (c0 + c < a.w_frags ? c0 + c : a.w_frags - 1);
#pragma unroll
        for (int t = 0; t < TM; ++t) f.x[t] = xp + (t0 + t < a.x_frags ? t0 + t : a.x_frags - 1);
        mx4_span<CF, TM>(a, f, lane, acc);
    }
#pragma unroll
    for (int c = 0; c < CF; ++c) {
        const int r = (c0 + c) * 16 + 4 * (lane >> 4);
        const int64_t col = (int64_t)g * a.bo + r;
        const int64_t left = a.bo - r < a.n_out - col ? a.bo - r : a.n_out - col;
#pragma unroll
        for (int t = 0; t < TM; ++t)
            if (c0 + c < a.w_frags) mx4_store<T>(a, (int64_t)(t0 + t) * 16 + (lane & 15), col, left < 4 ? (int)left : 4, acc[c][t]);
    }
}

// Output transpose (see the top): 16 * TM tokens x 16 * CF * D columns.
template <int CF, int TM, typename T>
__global__ void __launch_bounds__(TM == 4 ? 512 : 1024) mx4_gemm_ot_kernel(Mx4Args a) {
    extern __shared__ __attribute__((aligned(16))) float sums[];
    const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = xcd_tile(blockIdx.x, a.tiles);
    const int D = a.D, bo = a.bo, N = 16 * CF * D, pitch = N + 4;
    const int64_t f0 = (int64_t)(tile % a.tiles_n) * N;
    const int jf0 = (tile % a.tiles_n) * CF, t0 = (tile / a.tiles_n) * TM;
    const int row = lane & 15, quad = 4 * (lane >> 4);
    Mx4Frags<CF, TM> f;
    f32x4_t acc[CF][TM];

    for (int g = wave; g < D; g += waves) {
        mx4_zero(acc);
        const int64_t wp = (int64_t)(D + g) * a.w_frags, xp = (int64_t)(a.in_t ? D + g : g) * a.x_frags;
#pragma unroll
        for (int c = 0; c < CF; ++c) f.w[c] = wp + (jf0 + c < a.w_frags ? jf0 + c : a.w_frags - 1);
#pragma unroll
        for (int t = 0; t < TM; ++t) f.x[t] = xp + (t0 + t < a.x_frags ? t0 + t : a.x_frags - 1);
        mx4_span<CF, TM>(a, f, lane, acc);
#pragma unroll
        for (int c = 0; c < CF; ++c)
#pragma unroll
            for (int t = 0; t < TM; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) sums[(t * 16 + row) * pitch + (16 * c + quad + v) * D + g] = acc[c][t][v];
    }
    __syncthreads();

    // component 1: the fragments of each block that reach into the columns, CF at a time
    const int64_t f1 = f0 + N < a.n_out ? f0 + N : a.n_out;
    int unit = 0;
    for (int i = (int)(f0 / bo); (int64_t)i * bo < f1; ++i) {
        const int64_t base = (int64_t)i * bo;
        const int lo = f0 > base ? (int)((f0 - base) / 16) : 0;
        const int hi = (int)(((f1 < base + bo ? f1 : base + bo) - base + 15) / 16);
        for (int r0 = lo; r0 < hi; r0 += CF, ++unit) {
            if (unit % waves != wave) continue;
            mx4_zero(acc);
            const int64_t wp = (int64_t)i * a.w_frags, xp = (int64_t)i * a.x_frags;
#pragma unroll
            for (int c = 0; c < CF; ++c) f.w[c] = wp + (r0 + c < hi ? r0 + c : hi - 1);
#pragma unroll
            for (int t = 0; t < TM; ++t) f.x[t] = xp + (t0 + t < a.x_frags ? t0 + t : a.x_frags - 1);
            mx4_span<CF, TM>(a, f, lane, acc);
#pragma unroll
            for (int c = 0; c < CF; ++c) {
                const int r = (r0 + c) * 16 + quad;
                const int64_t col = base + r;
                int64_t end = base + bo < f1 ? base + bo : f1;
                if (r0 + c >= hi) end = 0;
#pragma unroll
                for (int t = 0; t < TM; ++t) {
                    const int64_t m = (int64_t)(t0 + t) * 16 + row;
                    const float *src = sums + (t * 16 + row) * pitch + (col - f0);
                    if (col >= f0 && col + 4 <= end) {
                        f32x4_t x;
#pragma unroll
                        for (int v = 0; v < 4; ++v) x[v] = acc[c][t][v] + src[v];
                        mx4_store<T>(a, m, col, 4, x);
                    } else {
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (col + v >= f0 && col + v < end)
                                mx4_store<T>(a, m, col + v, 1, f32x4_t{acc[c][t][v] + src[v], 0.f, 0.f, 0.f});
                    }
                }
            }
        }
    }
}

// ---- fragment order ------------------------------------------------------------

// 32 values of a row into codes and a scale byte of fragment order: lane's
// place in fragment `frag` (numbered part * frags + fragment), step s.
__device__ __forceinline__ void mx4_put(uint8_t *codes, uint8_t *scales, int64_t frag, int steps, int words, int s, int lane,
                                        const float (&x)[4][8]) {
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, mag_bits(x[q][e]));
    const uint32_t sb = mx_scale<kMxFp4>(top);
    uint4 c = make_uint4(0u, 0u, 0u, 0u);
    if (sb != 255u) {
        const float pow = mx_pow(sb);
        c = make_uint4(mx_fp4x8(x[0], pow), mx_fp4x8(x[1], pow), mx_fp4x8(x[2], pow), mx_fp4x8(x[3], pow));
    }
    reinterpret_cast<uint4 *>(codes + (frag * steps + s) * 1024)[lane] = c;
    scales[(frag * words + s / 4) * 256 + lane * 4 + s % 4] = (uint8_t)sb;
}

struct Mx4PackArgs {
    int64_t M, n_in, n_out;
    int D, bi, bo, in_t, out_t;
    const void *W1, *W2, *X;
    uint8_t *codes, *scales;
    int parts, frags, steps, words;
    int64_t items;      // fragments times steps
};

// A wave a fragment and step; WEIGHTS: part = component * D + block of W1 / W2,
// else block (or, from D on, residue) of the input.
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
    const int64_t row = fr * 16 + (lane & 15);
    const int k0 = s * 128 + (lane >> 4) * 32;
    const int64_t n = a.n_in;
    float x[4][8];
    const T *src;
    int64_t step;
    bool real;
    if constexpr (WEIGHTS) {
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
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int k = k0 + 8 * q + e;
            const int64_t col = strided ? (int64_t)k * a.D + g : (int64_t)g * a.bi + k;
            x[q][e] = real && k < a.bi && col < n ? load_f32<T>(src, k * step) : 0.f;
        }
    mx4_put(a.codes, a.scales, part * (int64_t)a.frags + fr, a.steps, a.words, s, lane, x);
}

template <bool WEIGHTS>
hipError_t run_pack(Mx4PackArgs &a, const Mx4Layout &l, int dtype, hipStream_t s) {
    if (l.frags >= ((int64_t)1 << 31) || l.parts >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
    a.parts = (int)l.parts; a.frags = (int)l.frags; a.steps = (int)l.steps; a.words = (int)l.words();
    a.scales = a.codes + l.code_bytes();
    a.items = l.parts * l.frags * l.steps;
    const int64_t grid = (a.items + 3) / 4;
    if (grid >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
    if (dtype == kBF16) mx4_pack_kernel<WEIGHTS, uint16_t><<<(unsigned)grid, 256, 0, s>>>(a);
    else mx4_pack_kernel<WEIGHTS, float><<<(unsigned)grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_pack(int64_t n_in, int64_t n_out, int64_t D, bool in_t, bool out_t, int dtype, const void *W1,
                           const void *W2, void *packed, hipStream_t s) {
    Mx4PackArgs a{};
    a.n_in = n_in; a.n_out = n_out; a.D = (int)D;
    a.bi = (int)((n_in + D - 1) / D); a.bo = (int)((n_out + D - 1) / D);
    a.in_t = in_t; a.out_t = out_t;
    a.W1 = W1; a.W2 = W2;
    a.codes = static_cast<uint8_t *>(packed);
    return run_pack<true>(a, mx4_weights_layout(D, a.bi, a.bo), dtype, s);
}

hipError_t launch_mx4_forward(const Mx4Pass &p, hipStream_t s) {
    const Mx4Layout wl = mx4_weights_layout(p.D, p.bi, p.bo), xl = mx4_input_layout(p.D, p.bi, p.M, p.in_t);
    Mx4PackArgs q{};
    q.M = p.M; q.n_in = p.n_in; q.n_out = p.n_out; q.D = (int)p.D; q.bi = (int)p.bi; q.bo = (int)p.bo;
    q.in_t = p.in_t; q.out_t = p.out_t;
    q.X = p.X;
    q.codes = static_cast<uint8_t *>(p.ws);
    hipError_t e = run_pack<false>(q, xl, p.dtype, s);
    if (e != hipSuccess) return e;

    Mx4Args a{};
    a.M = p.M; a.n_in = p.n_in; a.n_out = p.n_out; a.D = (int)p.D; a.bi = (int)p.bi; a.bo = (int)p.bo;
    a.wc = static_cast<const uint8_t *>(p.packed);
    a.ws = a.wc + wl.code_bytes();
    a.xc = static_cast<const uint8_t *>(p.ws);
    a.xs = a.xc + xl.code_bytes();
    a.w_frags = (int)wl.frags; a.x_frags = (int)xl.frags; a.steps = (int)wl.steps; a.words = (int)wl.words();
    a.bias = p.bias; a.Y = p.Y; a.gelu = p.gelu; a.in_t = p.in_t;
    auto tiles = [&](int64_t n, int64_t m) -> bool {
        if (n * m >= ((int64_t)1 << 31)) return false;
        a.tiles_n = (int)n;
        a.tiles = (int)(n * m);
        return true;
    };
    auto by_type = [&](auto go) {
        if (p.dtype == kBF16) go(uint16_t{});
        else go(float{});
    };
    const int64_t xf = xl.frags, wf = wl.frags;
    if (!p.out_t || p.D == 1) {
        const bool small = xf <= 2;
        if (!tiles(p.D * ((wf + (small ? 1 : 7)) / (small ? 2 : 8)), small ? (xf + 1) / 2 : (xf + 7) / 8)) return hipErrorInvalidValue;
        by_type([&](auto t) {
            using T = decltype(t);
            if (small) mx4_gemm_kernel<1, 1, T><<<(unsigned)a.tiles, 256, 0, s>>>(a);
            else mx4_gemm_kernel<4, 4, T><<<(unsigned)a.tiles, 256, 0, s>>>(a);
        });
        return hipGetLastError();
    }
    const int64_t D = p.D, waves = D < 16 ? D : 16;
    auto ot = [&](auto cf, auto tm) -> hipError_t {
        constexpr int CF = decltype(cf)::value, TM = decltype(tm)::value;
        const int64_t N = 16 * CF * D;
        if (!tiles((p.n_out + N - 1) / N, (xf + TM - 1) / TM)) return hipErrorInvalidValue;
        const size_t lds = (size_t)(16 * TM) * (size_t)(N + 4) * sizeof(float);
        by_type([&](auto t) { mx4_gemm_ot_kernel<CF, TM, decltype(t)><<<(unsigned)a.tiles, (unsigned)(64 * waves), lds, s>>>(a); });
        return hipGetLastError();
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    using Four = std::integral_constant<int, 4>;
    if (xf <= 1) return ot(One{}, One{});
    if (D <= 8) return ot(Four{}, Four{});
    if (D <= 16) return ot(Four{}, Two{});
    return ot(Four{}, One{});
}

}  // namespace dyad
