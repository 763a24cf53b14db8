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
// Both components run in one loop over 2 * steps, the loads of the next steps
// in flight over a step's multiplies.
//
// Output transpose.  A wave owns a residue: its outputs j*D + g take block g of
// component 2, and component 1's rows kept by residue (mx4_by_residue), into the
// same accumulators.  The D waves of a workgroup make 16 * SN * D consecutive
// columns, which meet in LDS on the way out.  Shapes whose residues do not fit a
// block so run a form that adds component 1 to component 2's sums in LDS.
#include "mx4_gemm.h"

namespace dyad {

namespace {

// Where a wave's fragments start for each component.
struct Mx4Wave {
    int wp[2], wf[2];      // weights: part and first fragment
    int xp[2];             // input: part
    int xf;                // first token fragment
};

// acc += both components, PF steps of loads in flight.  Fragments past the last
// load the last again (their results are not stored).
template <int SN, int SM, int PF>
__device__ __forceinline__ void mx4_loop(const Mx4Args &a, const Mx4Wave &v, int lane, f32x4_t (&acc)[SN][SM]) {
    constexpr int GN = (SN + 3) / 4, GM = (SM + 3) / 4;
    uint4 w[PF][SN], x[PF][SM];
    uint32_t sw[PF][GN], sx[PF][GM];
    const int steps = a.steps, total = 2 * steps;
    const uint32_t l16 = 16u * (uint32_t)lane, l4 = 4u * (uint32_t)lane;
    auto load = [&](auto slot, int t) {
        constexpr int P = decltype(slot)::value;
        const int c = t >= steps ? 1 : 0, s = t - c * steps;
        const uint8_t *wb = a.wc + (int64_t)v.wp[c] * a.w_frags * steps * 1024 + (int64_t)s * 1024;
        const uint8_t *xb = a.xc + (int64_t)v.xp[c] * a.x_frags * steps * 1024 + (int64_t)s * 1024;
#pragma unroll
        for (int j = 0; j < SN; ++j) {
            const int f = v.wf[c] + j < a.w_frags ? v.wf[c] + j : a.w_frags - 1;
            w[P][j] = *reinterpret_cast<const uint4 *>(wb + (int64_t)f * steps * 1024 + l16);
        }
#pragma unroll
        for (int i = 0; i < SM; ++i) {
            const int f = v.xf + i < a.x_frags ? v.xf + i : a.x_frags - 1;
            x[P][i] = *reinterpret_cast<const uint4 *>(xb + (int64_t)f * steps * 1024 + l16);
        }
        const uint8_t *wsb = a.ws + ((int64_t)v.wp[c] * a.w_groups * steps + s) * 256;
        const uint8_t *xsb = a.xs + ((int64_t)v.xp[c] * a.x_groups * steps + s) * 256;
#pragma unroll
        for (int q = 0; q < GN; ++q) {
            const int f = (v.wf[c] >> 2) + q < a.w_groups ? (v.wf[c] >> 2) + q : a.w_groups - 1;
            sw[P][q] = *reinterpret_cast<const uint32_t *>(wsb + (int64_t)f * steps * 256 + l4);
            if constexpr (SN < 4) sw[P][q] >>= 8 * (v.wf[c] & 3);
        }
#pragma unroll
        for (int q = 0; q < GM; ++q) {
            const int f = (v.xf >> 2) + q < a.x_groups ? (v.xf >> 2) + q : a.x_groups - 1;
            sx[P][q] = *reinterpret_cast<const uint32_t *>(xsb + (int64_t)f * steps * 256 + l4);
            if constexpr (SM < 4) sx[P][q] >>= 8 * (v.xf & 3);
        }
    };
    auto multiply = [&](auto slot) {
        constexpr int P = decltype(slot)::value;
        mx4_multiply<0, 0, SN, SM>(w[P], x[P], sw[P], sx[P], acc);
    };
    using S0 = std::integral_constant<int, 0>;
    using S1 = std::integral_constant<int, 1>;
    load(S0{}, 0);
    load(S1{}, 1);
    if constexpr (PF == 2) {
        for (int t = 2; t < total; t += 2) {
            multiply(S0{});
            load(S0{}, t);
            multiply(S1{});
            load(S1{}, t + 1);
        }
        multiply(S0{});
        multiply(S1{});
    } else {
        // four steps at a time, the last two of an odd pair on their own
        using S2 = std::integral_constant<int, 2>;
        using S3 = std::integral_constant<int, 3>;
        int t = 2;
        for (; t + 4 <= total; t += 4) {
            load(S2{}, t);
            load(S3{}, t + 1);
            multiply(S0{});
            multiply(S1{});
            load(S0{}, t + 2);
            load(S1{}, t + 3);
            multiply(S2{});
            multiply(S3{});
        }
        if (t < total) {
            load(S2{}, t);
            load(S3{}, t + 1);
            multiply(S0{});
            multiply(S1{});
            multiply(S2{});
            multiply(S3{});
        } else {
            multiply(S0{});
            multiply(S1{});
        }
    }
}

// No output transpose: a wave owns SN x SM fragments of one block.
template <int SN, int SM, int PF, typename T>
__global__ void __launch_bounds__(256, 2) mx4_gemm_kernel(Mx4Args a) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = xcd_tile(blockIdx.x, a.tiles);
    const int per_block = a.tiles_n / a.D, wm = 4 / a.wave_n;
    const int tn = tile % a.tiles_n, g = tn / per_block;
    const int c0 = ((tn - g * per_block) * a.wave_n + wave % a.wave_n) * SN;
    const int t0 = (tile / a.tiles_n * wm + wave / a.wave_n) * SM;
    if (c0 >= a.w_frags || t0 >= a.x_frags) return;
    const Mx4Wave v{{g, a.D + g}, {c0, c0}, {g, a.in_t ? a.D + g : g}, t0};
    f32x4_t acc[SN][SM];
    mx4_zero(acc);
    mx4_loop<SN, SM, PF>(a, v, lane, acc);
    mx4_epilogue<SN, SM, T>(a, g, c0, t0, lane, acc);
}

// Output transpose by residue: wave g of D makes the SN fragments jl0.. of
// residue g in a block.  out: rows of 16 * SN * D columns for 16 tokens.
template <int SN, int SM, int PF, typename T>
__global__ void __launch_bounds__(SN * SM >= 16 ? 512 : 1024) mx4_gemm_res_kernel(Mx4Args a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    T *out = reinterpret_cast<T *>(smem);
    const int lane = threadIdx.x & 63;
    const int g = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = xcd_tile(blockIdx.x, a.tiles);
    const int D = a.D, per = a.bo / (16 * D);             // fragments of a residue in a block
    const int tn = tile % a.tiles_n, jf0 = tn * SN, i1 = jf0 / per;
    const int t0 = tile / a.tiles_n * SM;
    const Mx4Wave v{{i1, D + g}, {g * per + jf0 - i1 * per, jf0}, {i1, a.in_t ? D + g : g}, t0};
    f32x4_t acc[SN][SM];
    mx4_zero(acc);
    mx4_loop<SN, SM, PF>(a, v, lane, acc);

    constexpr int E = sizeof(T);
    const int N = 16 * SN * D, pitch = N + 16 / E;
    const int64_t f0 = (int64_t)tn * N;
    const int row = lane & 15, quad = 4 * (lane >> 4);
    const T *bias = static_cast<const T *>(a.bias);
    float b[SN][4];
#pragma unroll
    for (int j = 0; j < SN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t f = f0 + (16 * j + quad + q) * D + g;
            b[j][q] = bias && f < a.n_out ? load_f32<T>(bias, f) : 0.f;
        }
#pragma unroll
    for (int i = 0; i < SM; ++i) {
        if (i) __syncthreads();
#pragma unroll
        for (int j = 0; j < SN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                store_f32<T>(out, row * pitch + (16 * j + quad + q) * D + g, mx4_act<T>(a, acc[j][i][q] + b[j][q]));
        __syncthreads();
        const int64_t m0 = (int64_t)(t0 + i) * 16;
        const int real = (int)(a.M - m0 < 16 ? a.M - m0 : 16), cols = (int)(a.n_out - f0 < N ? a.n_out - f0 : N);
        T *dst = static_cast<T *>(a.Y) + m0 * a.n_out + f0;
        if (a.n_out * E % 16 == 0) {
            // pieces of 16 bytes, a power of two or a few to a row: N * E / 16 = 2 * SN * D * E / 2
            const int per_row = cols * E / 16;
            for (int p = threadIdx.x; p < real * per_row; p += blockDim.x) {
                const int r = p / per_row, q = p - r * per_row;
                *reinterpret_cast<uint4 *>(reinterpret_cast<unsigned char *>(dst + r * a.n_out) + 16 * q) =
                    *reinterpret_cast<const uint4 *>(smem + (r * pitch) * E + 16 * q);
            }
        } else {
            for (int p = threadIdx.x; p < real * cols; p += blockDim.x) {
                const int r = p / cols, q = p - r * cols;
                dst[r * a.n_out + q] = out[r * pitch + q];
            }
        }
    }
}

// ---- output transpose, any block size ---------------------------------------------

template <int CF, int TM>
struct Mx4Frags {
    int wp, w[CF], xp, x[TM];   // parts, and fragments in them
};

template <int CF, int TM>
__device__ __forceinline__ void mx4_span(const Mx4Args &a, const Mx4Frags<CF, TM> &f, int lane, f32x4_t (&acc)[CF][TM]) {
    const int steps = a.steps;
    for (int s = 0; s < steps; ++s) {
        uint4 w[CF], x[TM];
        uint32_t sw[CF], sx[TM];
        auto code = [&](const uint8_t *c, int part, int frags, int n) {
            return reinterpret_cast<const uint4 *>(c + (((int64_t)part * frags + n) * steps + s) * 1024)[lane];
        };
        auto scale = [&](const uint8_t *c, int part, int groups, int n) {
            return reinterpret_cast<const uint32_t *>(c + (((int64_t)part * groups + (n >> 2)) * steps + s) * 256)[lane] >> (8 * (n & 3));
        };
#pragma unroll
        for (int c = 0; c < CF; ++c) {
            w[c] = code(a.wc, f.wp, a.w_frags, f.w[c]);
            sw[c] = scale(a.ws, f.wp, a.w_groups, f.w[c]);
        }
#pragma unroll
        for (int t = 0; t < TM; ++t) {
            x[t] = code(a.xc, f.xp, a.x_frags, f.x[t]);
            sx[t] = scale(a.xs, f.xp, a.x_groups, f.x[t]);
        }
#pragma unroll
        for (int c = 0; c < CF; ++c)
#pragma unroll
            for (int t = 0; t < TM; ++t) acc[c][t] = mx4_mfma<0, 0>(w[c], x[t], acc[c][t], sw[c], sx[t]);
    }
}

// 16 * TM tokens x 16 * CF * D columns: component 2's sums go to their columns
// in LDS, component 1's fragments over the same columns add to them.
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
#pragma unroll
    for (int t = 0; t < TM; ++t) f.x[t] = t0 + t < a.x_frags ? t0 + t : a.x_frags - 1;

    for (int g = wave; g < D; g += waves) {
        mx4_zero(acc);
        f.wp = D + g;
        f.xp = a.in_t ? D + g : g;
#pragma unroll
        for (int c = 0; c < CF; ++c) f.w[c] = jf0 + c < a.w_frags ? jf0 + c : a.w_frags - 1;
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
            f.wp = f.xp = i;
#pragma unroll
            for (int c = 0; c < CF; ++c) f.w[c] = r0 + c < hi ? r0 + c : hi - 1;
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

template <int N>
using Int = std::integral_constant<int, N>;

}  // namespace

hipError_t launch_mx4_forward(const Mx4Pass &p, hipStream_t s) {
    hipError_t e = launch_mx4_input(p, s);
    if (e != hipSuccess) return e;
    const bool in_t = p.in_t && p.D > 1, out_t = p.out_t && p.D > 1;
    const Mx4Layout wl = mx4_weights_layout(p.D, p.bi, p.bo), xl = mx4_input_layout(p.D, p.bi, p.M, in_t);
    Mx4Args a{};
    a.M = p.M; a.n_in = p.n_in; a.n_out = p.n_out; a.D = (int)p.D; a.bi = (int)p.bi; a.bo = (int)p.bo;
    a.wc = static_cast<const uint8_t *>(p.packed);
    a.ws = a.wc + wl.code_bytes();
    a.xc = static_cast<const uint8_t *>(p.ws);
    a.xs = a.xc + xl.code_bytes();
    a.w_frags = (int)wl.frags; a.w_groups = (int)wl.groups();
    a.x_frags = (int)xl.frags; a.x_groups = (int)xl.groups();
    a.steps = (int)wl.steps;
    a.bias = p.bias; a.Y = p.Y; a.gelu = p.gelu; a.in_t = in_t;
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
    const int64_t xf = xl.frags, wf = wl.frags, D = p.D;
    if (!out_t) {
        if (const hipError_t pp = launch_mx4_tiles(a, p.dtype == kBF16, s); pp != hipErrorNotSupported) return pp;
        auto plain = [&](auto sn, auto sm, auto pf, int wave_n) -> hipError_t {
            constexpr int SN = decltype(sn)::value, SM = decltype(sm)::value, PF = decltype(pf)::value;
            const int64_t bn = (int64_t)SN * wave_n, bm = (int64_t)SM * (4 / wave_n);
            a.wave_n = wave_n;
            if (!tiles(D * ((wf + bn - 1) / bn), (xf + bm - 1) / bm)) return hipErrorInvalidValue;
            by_type([&](auto t) { mx4_gemm_kernel<SN, SM, PF, decltype(t)><<<(unsigned)a.tiles, 256, 0, s>>>(a); });
            return hipGetLastError();
        };
        // the largest wave tile that still gives every SIMD two waves
        auto waves = [&](int sn, int sm) { return D * ((wf + sn - 1) / sn) * ((xf + sm - 1) / sm); };
        if (xf >= 4 && waves(4, 4) >= 2048) return plain(Int<4>{}, Int<4>{}, Int<2>{}, 2);
        if (xf >= 2 && waves(2, 2) >= 2048) return plain(Int<2>{}, Int<2>{}, Int<2>{}, 2);
        return plain(Int<1>{}, Int<1>{}, Int<4>{}, xf >= 2 ? 2 : 4);
    }
    if (mx4_by_residue(D, p.bo, out_t)) {
        const int64_t per = p.bo / (16 * D), all = (p.n_out + 16 * D - 1) / (16 * D);
        auto res = [&](auto sn, auto sm, auto pf) -> hipError_t {
            constexpr int SN = decltype(sn)::value, SM = decltype(sm)::value, PF = decltype(pf)::value;
            if (!tiles((all + SN - 1) / SN, (xf + SM - 1) / SM)) return hipErrorInvalidValue;
            by_type([&](auto t) {
                using T = decltype(t);
                const size_t lds = 16 * ((size_t)(16 * SN * D) * sizeof(T) + 16);
                mx4_gemm_res_kernel<SN, SM, PF, T><<<(unsigned)a.tiles, (unsigned)(64 * D), lds, s>>>(a);
            });
            return hipGetLastError();
        };
        auto waves = [&](int sn, int sm) { return D * ((all + sn - 1) / sn) * ((xf + sm - 1) / sm); };
        if (per % 4 == 0 && xf >= 4 && waves(4, 4) >= 2048 && D <= 8) return res(Int<4>{}, Int<4>{}, Int<2>{});
        if (per % 2 == 0 && xf >= 4 && waves(2, 4) >= 2048) return res(Int<2>{}, Int<4>{}, Int<2>{});
        if (xf >= 4 && waves(1, 4) >= 2048) return res(Int<1>{}, Int<4>{}, Int<2>{});
        if (xf >= 2) return res(Int<1>{}, Int<2>{}, Int<2>{});
        return res(Int<1>{}, Int<1>{}, Int<4>{});
    }
    const int64_t waves = D < 16 ? D : 16;
    auto ot = [&](auto cf, auto tm) -> hipError_t {
        constexpr int CF = decltype(cf)::value, TM = decltype(tm)::value;
        const int64_t N = 16 * CF * D;
        if (!tiles((p.n_out + N - 1) / N, (xf + TM - 1) / TM)) return hipErrorInvalidValue;
        const size_t lds = (size_t)(16 * TM) * (size_t)(N + 4) * sizeof(float);
        by_type([&](auto t) { mx4_gemm_ot_kernel<CF, TM, decltype(t)><<<(unsigned)a.tiles, (unsigned)(64 * waves), lds, s>>>(a); });
        return hipGetLastError();
    };
    if (xf <= 1) return ot(Int<1>{}, Int<1>{});
    if (D <= 8) return ot(Int<4>{}, Int<4>{});
    if (D <= 16) return ot(Int<4>{}, Int<2>{});
    return ot(Int<4>{}, Int<1>{});
}

}  // namespace dyad
