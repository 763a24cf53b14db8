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

// acc += both components, PF steps of loads in flight (PF divides 2 * steps).
// Fragments past the last
// load the last again (their results are not stored).
template <int SN, int SM, int PF>
__device__ __forceinline__ void mx4_loop(const Mx4Args &a, const Mx4Wave &v, int lane, f32x4_t (&acc)[SN][SM]) {
    constexpr int GN = (SN + 3) / 4, GM = (SM + 3) / 4;
    uint4 w[PF][SN], x[PF][SM];
    uint32_t sw[PF][GN], sx[PF][GM];
    const int steps = a.steps, total = 2 * steps;
    const uint32_t l16 = 16u * (uint32_t)lane, l4 = 4u * (uint32_t)lane;
    auto load = [&](int P, int t) __attribute__((always_inline)) {
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
    auto multiply = [&](int P) __attribute__((always_inline)) {
        mx4_multiply<0, 0, SN, SM>(w[P], x[P], sw[P], sx[P], acc);
    };
#pragma unroll
    for (int p = 0; p < PF; ++p) load(p, p);
    for (int t = PF; t < total; t += PF) {
#pragma unroll
        for (int p = 0; p < PF; ++p) {
            multiply(p);
            load(p, t + p);
        }
    }
#pragma unroll
    for (int p = 0; p < PF; ++p) multiply(p);
}

// Small tiles: the tile of a workgroup.  Consecutive tiles share an XCD, whose L2
// then reads either the input or the weights once: the larger of the two (256
// tokens of 32768 -> 8192, n_dyad 16, Dyad-OT, 18 MB of weights over 4 of input:
// 33 -> 31 us).
__device__ __forceinline__ void mx4_tile(const Mx4Args &a, int &tn, int &tm) {
    const int tile = xcd_tile(blockIdx.x, a.tiles);
    tn = a.m_fast ? tile / a.tiles_m : tile % a.tiles_n;
    tm = a.m_fast ? tile % a.tiles_m : tile / a.tiles_n;
}

// No output transpose: a wave owns SN x SM fragments of one block.
template <int SN, int SM, int PF, typename T>
__global__ void __launch_bounds__(256, 2) mx4_gemm_kernel(Mx4Args a) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tn, tm;
    mx4_tile(a, tn, tm);
    const int per_block = a.tiles_n / a.D, g = tn / per_block;
    const int c0 = ((tn - g * per_block) * a.wave_n + wave % a.wave_n) * SN;
    const int t0 = (tm * (4 / a.wave_n) + wave / a.wave_n) * SM;
    if (c0 >= a.w_frags || t0 >= a.x_frags) return;
    const Mx4Wave v{{g, a.D + g}, {c0, c0}, {g, a.in_t ? a.D + g : g}, t0};
    f32x4_t acc[SN][SM];
    mx4_zero(acc);
    mx4_loop<SN, SM, PF>(a, v, lane, acc);
    mx4_epilogue<SN, SM, T>(a, g, c0, t0, lane, acc);
}

// A wave's biases: outputs f0 + (16 j + 4 (lane / 16) + q) * D + g of the
// workgroup's columns f0 = 16 * SN * D * tn.
template <int SN, typename T>
__device__ __forceinline__ void mx4_bias_res(const Mx4Args &a, int tn, int g, int lane, float (&b)[SN][4]) {
    const T *bias = static_cast<const T *>(a.bias);
    const int64_t f0 = (int64_t)tn * 16 * SN * a.D;
#pragma unroll
    for (int j = 0; j < SN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t f = f0 + (16 * j + 4 * (lane >> 4) + q) * a.D + g;
            b[j][q] = bias && f < a.n_out ? load_f32<T>(bias, f) : 0.f;
        }
}

// The residues' outputs meet in LDS (16 * SM rows of 16 * SN * D columns) and
// leave in rows.
template <int SN, int SM, typename T>
__device__ __forceinline__ void mx4_store_res(const Mx4Args &a, unsigned char *smem, int tn, int t0, int g, int lane,
                                              const float (&b)[SN][4], const f32x4_t (&acc)[SN][SM]) {
    constexpr int E = sizeof(T);
    const int D = a.D, N = 16 * SN * D, pitch = N * E + 16;
    const int64_t f0 = (int64_t)tn * N, m0 = (int64_t)t0 * 16;
#pragma unroll
    for (int i = 0; i < SM; ++i) {
        unsigned char *row = smem + (16 * i + (lane & 15)) * pitch + (4 * (lane >> 4) * D + g) * E;
#pragma unroll
        for (int j = 0; j < SN; ++j) {
            unsigned char *at = row + 16 * j * D * E;
            float x[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = mx4_act<T>(a, acc[j][i][q] + b[j][q]);
            if constexpr (E == 2) {
#pragma unroll
                for (int q = 0; q < 4; q += 2) {
                    const uint32_t w = pack_bf16(x[q], x[q + 1]);
                    *reinterpret_cast<uint16_t *>(at + q * D * E) = (uint16_t)w;
                    *reinterpret_cast<uint16_t *>(at + (q + 1) * D * E) = (uint16_t)(w >> 16);
                }
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) *reinterpret_cast<float *>(at + q * D * E) = x[q];
            }
        }
    }
    __syncthreads();
    const int real = (int)(a.M - m0 < 16 * SM ? a.M - m0 : 16 * SM), cols = (int)(a.n_out - f0 < N ? a.n_out - f0 : N);
    unsigned char *dst = static_cast<unsigned char *>(a.Y) + (m0 * a.n_out + f0) * E;
    if (a.n_out * E % 16 == 0) {
        const int per_row = cols * E / 16;
        for (int p = threadIdx.x; p < real * per_row; p += blockDim.x) {
            const int r = p / per_row, q = p - r * per_row;
            *reinterpret_cast<uint4 *>(dst + r * a.n_out * E + 16 * q) = *reinterpret_cast<const uint4 *>(smem + r * pitch + 16 * q);
        }
    } else {
        for (int p = threadIdx.x; p < real * cols; p += blockDim.x) {
            const int r = p / cols, q = p - r * cols;
            reinterpret_cast<T *>(dst)[r * a.n_out + q] = reinterpret_cast<const T *>(smem + r * pitch)[q];
        }
    }
}

// Output transpose by residue: wave g of D makes SN fragments of residue g in a
// block, the workgroup 16 * SM tokens x 16 * SN * D columns.
template <int SN, int SM, int PF, typename T>
__global__ void __launch_bounds__(SN * SM >= 8 ? 512 : 1024) mx4_gemm_res_kernel(Mx4Args a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int g = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int tn, tm;
    mx4_tile(a, tn, tm);
    const int D = a.D, per = a.bo / (16 * D);             // fragments of a residue in a block
    const int jf0 = tn * SN, i1 = jf0 / per, t0 = tm * SM;
    const Mx4Wave v{{i1, D + g}, {g * per + jf0 - i1 * per, jf0}, {i1, a.in_t ? D + g : g}, t0};
    float b[SN][4];
    mx4_bias_res<SN, T>(a, tn, g, lane, b);
    f32x4_t acc[SN][SM];
    mx4_zero(acc);
    mx4_loop<SN, SM, PF>(a, v, lane, acc);
    mx4_store_res<SN, SM, T>(a, smem, tn, t0, g, lane, b, acc);
}

// ---- up to 16 tokens of a narrow input: quantised where it is multiplied ---------

// A step's 32 values of the lane's row (token) and block, as pairs of bf16 or floats.
template <typename T>
struct Mx4Raw {
    static constexpr int kWords = sizeof(T) == 2 ? 16 : 32;
    typename std::conditional<sizeof(T) == 2, uint32_t, float>::type v[kWords];
};

// part: block or, strided, residue (columns k*D + g).  Blocks of a multiple of 8.
template <typename T>
__device__ __forceinline__ void mx4_raw(const Mx4Args &a, int g, bool strided, int s, int lane, Mx4Raw<T> &r) {
    const int row = lane & 15, k0 = s * 128 + (lane >> 4) * 32;
    constexpr int W = Mx4Raw<T>::kWords;
#pragma unroll
    for (int e = 0; e < W; ++e) r.v[e] = 0;
    if (row >= a.M) return;
    const T *x = static_cast<const T *>(a.X) + (int64_t)row * a.n_in;
    if (!strided) {
        const T *p = x + (int64_t)g * a.bi + k0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (k0 + 8 * q >= a.bi) continue;
            if constexpr (sizeof(T) == 2) {
                const uint4 v = *reinterpret_cast<const uint4 *>(p + 8 * q);
                r.v[4 * q] = v.x; r.v[4 * q + 1] = v.y; r.v[4 * q + 2] = v.z; r.v[4 * q + 3] = v.w;
            } else {
                const f32x4_t lo = *reinterpret_cast<const f32x4_t *>(p + 8 * q), hi = *reinterpret_cast<const f32x4_t *>(p + 8 * q + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    r.v[8 * q + e] = lo[e];
                    r.v[8 * q + 4 + e] = hi[e];
                }
            }
        }
    } else {
        const T *p = x + (int64_t)k0 * a.D + g;
        T t[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) t[e] = k0 + e < a.bi ? p[e * a.D] : (T)0;
#pragma unroll
        for (int e = 0; e < W; ++e) {
            if constexpr (sizeof(T) == 2) r.v[e] = (uint32_t)t[2 * e] | (uint32_t)t[2 * e + 1] << 16;
            else r.v[e] = t[e];
        }
    }
}

// A wave a fragment of 16 outputs; the workgroup's waves are its residues under an
// output transpose (OT), else neighbouring fragments.
template <bool OT, typename T>
__global__ void __launch_bounds__(OT ? 1024 : 256) mx4_few_kernel(Mx4Args a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tn = blockIdx.x, D = a.D;
    int g, c0;                                     // block (or residue) and its fragment
    int wp[2], wf[2], xp[2];
    float b[1][4];
    if constexpr (OT) {
        const int per = a.bo / (16 * D), i1 = tn / per;
        g = wave;
        c0 = 0;
        wp[0] = i1; wp[1] = D + g;
        wf[0] = g * per + tn - i1 * per; wf[1] = tn;
        xp[0] = i1; xp[1] = g;
        mx4_bias_res<1, T>(a, tn, g, lane, b);
    } else {
        const int per_block = a.tiles_n / D;
        g = tn / per_block;
        c0 = (tn - g * per_block) * 4 + wave;
        if (c0 >= a.w_frags) return;
        wp[0] = g; wp[1] = D + g;
        wf[0] = wf[1] = c0;
        xp[0] = xp[1] = g;
    }
    f32x4_t acc[1][1];
    mx4_zero(acc);
    const int steps = a.steps, total = 2 * steps;
    uint4 w[2];
    uint32_t sw[2];
    Mx4Raw<T> raw[2];
    auto load = [&](auto slot, int t) {
        constexpr int P = decltype(slot)::value;
        const int c = t >= steps ? 1 : 0, s = t - c * steps;
        w[P] = reinterpret_cast<const uint4 *>(a.wc + (((int64_t)wp[c] * a.w_frags + wf[c]) * steps + s) * 1024)[lane];
        sw[P] = reinterpret_cast<const uint32_t *>(a.ws + (((int64_t)wp[c] * a.w_groups + (wf[c] >> 2)) * steps + s) * 256)[lane] >> (8 * (wf[c] & 3));
        mx4_raw<T>(a, xp[c], c && a.in_t, s, lane, raw[P]);
    };
    auto multiply = [&](auto slot) {
        constexpr int P = decltype(slot)::value;
        uint32_t sx;
        const uint4 x = mx4_encode(raw[P].v, sx);
        acc[0][0] = mx4_mfma<0, 0>(w[P], x, acc[0][0], sw[P], sx);
    };
    using S0 = std::integral_constant<int, 0>;
    using S1 = std::integral_constant<int, 1>;
    load(S0{}, 0);
    load(S1{}, 1);
    for (int t = 2; t < total; t += 2) {
        multiply(S0{});
        load(S0{}, t);
        multiply(S1{});
        load(S1{}, t + 1);
    }
    multiply(S0{});
    multiply(S1{});
    if constexpr (OT) mx4_store_res<1, 1, T>(a, smem, tn, 0, g, lane, b, acc);
    else mx4_epilogue<1, 1, T>(a, g, c0, 0, lane, acc);
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
    int tn, tm;
    mx4_tile(a, tn, tm);
    const int D = a.D, bo = a.bo, N = 16 * CF * D, pitch = N + 4;
    const int64_t f0 = (int64_t)tn * N;
    const int jf0 = tn * CF, t0 = tm * TM;
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

// Up to 16 tokens over blocks of at most two steps: each wave quantises what it
// multiplies, in place of a pass in front (a launch, 3 us at one token of 768).
// All fragments of a block's outputs repeat it, and residues are gathered value
// by value.  A call of 1 / 4 / 16 tokens, against the two launches: 768 -> 3072,
// n_dyad 4, Dyad-IT 10.6 / 10.2 / 10.9 us (11.8 / 11.7 / 11.2), -OT 10.9 / 10.0 / 9.8
// (11.8 / 11.4 / 11.1); 2048 -> 8192, n_dyad 8, -IT 10.1 / 11.2 / 12.7 (11.6 / 11.7 /
// 11.0), -OT 10.2 / 9.7 / 10.3 (11.6 / 11.4 / 10.9); blocks of 768 (3072 -> 768), -IT
// 20 / 21 / 29 (11.8 / 11.7 / 11.7), -OT 11.5 / 10.9 / 10.8 (11.4 / 11.5 / 11.4).
bool mx4_in_place(int64_t n_in, int64_t D, int64_t bi, int64_t bo, int64_t M, bool in_t, bool out_t) {
    return M <= (in_t && D > 1 ? 4 : 16) && bi <= 256 && bi % 8 == 0 && n_in == D * bi &&
           (!out_t || D == 1 || mx4_by_residue(D, bo, out_t));
}

hipError_t launch_mx4_forward(const Mx4Pass &p, hipStream_t s) {
    const bool in_t = p.in_t && p.D > 1, out_t = p.out_t && p.D > 1;
    const Mx4Layout wl = mx4_weights_layout(p.D, p.bi, p.bo), xl = mx4_input_layout(p.D, p.bi, p.M, in_t);
    const int64_t xf = xl.frags, wf = wl.frags, D = p.D;
    Mx4Args a{};
    a.M = p.M; a.n_in = p.n_in; a.n_out = p.n_out; a.D = (int)p.D; a.bi = (int)p.bi; a.bo = (int)p.bo;
    a.X = p.X;
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
        a.tiles_m = (int)m;
        a.tiles = (int)(n * m);
        a.m_fast = wl.bytes() > xl.bytes();
        return true;
    };
    auto by_type = [&](auto go) {
        if (p.dtype == kBF16) go(uint16_t{});
        else go(float{});
    };
    if (mx4_in_place(p.n_in, D, p.bi, p.bo, p.M, in_t, out_t)) {
        if (!tiles(out_t ? (p.n_out + 16 * D - 1) / (16 * D) : D * ((wf + 3) / 4), 1)) return hipErrorInvalidValue;
        by_type([&](auto t) {
            using T = decltype(t);
            if (out_t) mx4_few_kernel<true, T><<<(unsigned)a.tiles, (unsigned)(64 * D), 16 * ((size_t)(16 * D) * sizeof(T) + 16), s>>>(a);
            else mx4_few_kernel<false, T><<<(unsigned)a.tiles, 256, 0, s>>>(a);
        });
        return hipGetLastError();
    }
    const hipError_t e = launch_mx4_input(p, s);
    if (e != hipSuccess) return e;

    // Steps of loads in flight: as many as divide the steps, up to `most` for the
    // small wave tiles, two for the others (registers).
    auto ahead = [&](auto sn, auto sm, auto most, auto go) {
        constexpr int kMost = decltype(sn)::value * decltype(sm)::value <= 2 ? decltype(most)::value : decltype(sn)::value * decltype(sm)::value <= 4 ? 4 : 2;
        if constexpr (kMost >= 8)
            if (a.steps % 4 == 0) return go(Int<8>{});
        if constexpr (kMost >= 4)
            if (a.steps % 2 == 0) return go(Int<4>{});
        go(Int<2>{});
    };
    // A tile's time on a CU, in cycles: its waves' fragments at 64 bytes a cycle
    // over all steps, and its outputs; times the rounds that the tiles take.
    auto cost = [&](int64_t count, int64_t waves, int sn, int sm) {
        return (count + 255) / 256 * waves * ((sn + sm) * 16 * 2 * (int64_t)a.steps + sn * sm * (p.gelu ? 150 : 60));
    };
    if (!out_t) {
        if (const hipError_t t = launch_mx4_tiles(a, p.dtype == kBF16, s); t != hipErrorNotSupported) return t;
        auto count = [&](int sn, int sm, int wave_n) {
            return D * ((wf + sn * wave_n - 1) / (sn * wave_n)) * ((xf + sm * (4 / wave_n) - 1) / (sm * (4 / wave_n)));
        };
        auto plain = [&](auto sn, auto sm, int wave_n) -> hipError_t {
            constexpr int SN = decltype(sn)::value, SM = decltype(sm)::value;
            const int64_t bn = (int64_t)SN * wave_n, bm = (int64_t)SM * (4 / wave_n);
            a.wave_n = wave_n;
            if (!tiles(D * ((wf + bn - 1) / bn), (xf + bm - 1) / bm)) return hipErrorInvalidValue;
            by_type([&](auto t) {
                ahead(sn, sm, Int<8>{}, [&](auto pf) {
                    mx4_gemm_kernel<SN, SM, decltype(pf)::value, decltype(t)><<<(unsigned)a.tiles, 256, 0, s>>>(a);
                });
            });
            return hipGetLastError();
        };
        const int64_t c44 = cost(count(4, 4, 2), 4, 4, 4), c22 = cost(count(2, 2, 2), 4, 2, 2);
        const int wide = xf >= 2 ? 2 : 4;
        const int64_t c11 = cost(count(1, 1, wide), 4, 1, 1);
        if (xf >= 4 && c44 <= c22 && c44 <= c11) return plain(Int<4>{}, Int<4>{}, 2);
        if (xf >= 2 && c22 <= c11) return plain(Int<2>{}, Int<2>{}, 2);
        return plain(Int<1>{}, Int<1>{}, wide);
    }
    if (mx4_by_residue(D, p.bo, out_t)) {
        if (p.dtype == kBF16)
            if (const hipError_t t = launch_mx4_res_tiles(a, s); t != hipErrorNotSupported) return t;
        const int64_t per = p.bo / (16 * D), all = (p.n_out + 16 * D - 1) / (16 * D);
        auto res = [&](auto sn, auto sm) -> hipError_t {
            constexpr int SN = decltype(sn)::value, SM = decltype(sm)::value;
            if (!tiles((all + SN - 1) / SN, (xf + SM - 1) / SM)) return hipErrorInvalidValue;
            by_type([&](auto t) {
                using T = decltype(t);
                const size_t lds = 16 * SM * ((size_t)(16 * SN * D) * sizeof(T) + 16);
                ahead(sn, sm, Int<SM == 1 ? 8 : 4>{}, [&](auto pf) {
                    mx4_gemm_res_kernel<SN, SM, decltype(pf)::value, T><<<(unsigned)a.tiles, (unsigned)(64 * D), lds, s>>>(a);
                });
            });
            return hipGetLastError();
        };
        int sn = 1, sm = 1;
        int64_t best = 0;
        // the widest wave tiles keep to eight waves (registers), and rows of a
        // workgroup's columns to 80 KB of LDS
        auto consider = [&](int n, int m) {
            const int64_t lds = 16 * m * (16 * n * D * (p.dtype == kBF16 ? 2 : 4) + 16);
            if (per % n != 0 || xf < m || lds > 80 * 1024 || (n * m >= 8 && D > 8)) return;
            const int64_t c = cost((all + n - 1) / n * ((xf + m - 1) / m), D, n, m);
            if (!best || c < best) {
                best = c;
                sn = n;
                sm = m;
            }
        };
        consider(4, 4);
        consider(2, 4);
        consider(1, 4);
        consider(1, 2);
        consider(1, 1);
        if (sn == 4) return res(Int<4>{}, Int<4>{});
        if (sn == 2) return res(Int<2>{}, Int<4>{});
        if (sm == 4) return res(Int<1>{}, Int<4>{});
        if (sm == 2) return res(Int<1>{}, Int<2>{});
        return res(Int<1>{}, Int<1>{});
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
    // as many tokens to a workgroup as LDS holds sums of and still fill the GPU
    const int64_t cols = (p.n_out + 64 * D - 1) / (64 * D);
    if (xf <= 1 || cols * xf < 256) return ot(Int<1>{}, Int<1>{});
    if (D <= 8 && cols * ((xf + 3) / 4) >= 512) return ot(Int<4>{}, Int<4>{});
    if (D <= 16 && cols * ((xf + 1) / 2) >= 512) return ot(Int<4>{}, Int<2>{});
    return ot(Int<4>{}, Int<1>{});
}

}  // namespace dyad
