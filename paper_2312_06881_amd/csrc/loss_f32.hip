// The loss's matrix products in fp32, on the fp32 matrix instructions
// (v_mfma_f32_16x16x4_f32, 32 cycles each), which bound them.  One kernel serves the three
// layouts: C[i][j] = sum_k A(i, k) B(j, k) with each side's k contiguous in memory or its rows.
// Four waves take a tile of 128 x 128 or 64 x 64, 16 k a stage, double-buffered.
// LDS rows of 16 k are 20 floats apart: the sixteen rows and four k of a fragment read fall on
// all 64 banks.  The sum over k has no order of its own, so lane group g takes k = 4g .. 4g + 3
// of the stage as one 16-byte read and feeds four instructions with it.
#include "lm_internal.h"
#include "mfma_common.h"

namespace dyad {

namespace {

constexpr int kThreads = 256, kStage = 16, kPitch = 20;
enum Kind { kStats, kGrad, kStore, kAdd };

struct Gemm {
    const float *A, *B;
    int64_t lda, ldb, I, J, K;
    int tiles_i;
    LossEpi e;
    int64_t v0;       // first vocabulary column (kStats: 0)
    float *out;
    int64_t ldo;
};

// Four consecutive values of a side at (row, k), along k or along the rows; zero outside.
template <bool KC>
__device__ __forceinline__ f32x4_t load4(const float *p, int64_t ld, int64_t row, int64_t k, int64_t rows, int64_t K) {
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    if (KC ? row < rows && k + 4 <= K : k < K && row + 4 <= rows) {
        __builtin_memcpy(&v, p + (KC ? row * ld + k : k * ld + row), 16);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (KC ? row < rows && k + e < K : k < K && row + e < rows) v[e] = p[KC ? row * ld + k + e : k * ld + row + e];
    }
    return v;
}

template <int BT, bool AK, bool BK, Kind KIND>
__global__ void __launch_bounds__(kThreads) loss_f32_kernel(Gemm g) {
    constexpr int S = BT / 32, kLoads = BT * kStage / 4 / kThreads;   // 2 x 2 waves of BT / 2
    // a token without a gradient leaves none, whatever it (side B of dW) and the weights (dX) hold: 0 times NaN is NaN
    constexpr bool kDw = !AK && !BK, kDx = AK && !BK;
    __shared__ float lds[2][2][BT * kPitch];
    __shared__ float2 red[KIND == kStats ? BT * 2 : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, lg = lane >> 4;
    const int64_t i0 = (int64_t)(blockIdx.x % g.tiles_i) * BT, j0 = (int64_t)(blockIdx.x / g.tiles_i) * BT;
    const int wm0 = (wave >> 1) * (BT / 2), wn0 = (wave & 1) * (BT / 2);
    f32x4_t acc[S][S];
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
        for (int j = 0; j < S; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    f32x4_t ra[kLoads], rb[kLoads];
    const auto row_of = [&](bool kc, int v) { return kc ? v / 4 : v % (BT / 4) * 4; };
    const auto k_of = [&](bool kc, int v) { return kc ? v % 4 * 4 : v / (BT / 4); };
    const auto fetch = [&](int64_t k0) {
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int v = tid + q * kThreads;
            ra[q] = load4<AK>(g.A, g.lda, i0 + row_of(AK, v), k0 + k_of(AK, v), g.I, g.K);
            rb[q] = load4<BK>(g.B, g.ldb, j0 + row_of(BK, v), k0 + k_of(BK, v), g.J, g.K);
            if constexpr (kDw) {
                const int64_t m = k0 + k_of(BK, v);
                if (m < g.K && loss_scale(g.e, m, g.e.targets[m]) == 0.f) rb[q] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
        }
    };
    const auto put = [&](bool kc, float *dst, int v, const f32x4_t &r) {
        float *d = dst + row_of(kc, v) * kPitch + k_of(kc, v);
        if (kc) *reinterpret_cast<f32x4_t *>(d) = r;
        else
#pragma unroll
            for (int e = 0; e < 4; ++e) d[e * kPitch] = r[e];
    };
    const auto stash = [&](int b) {
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            put(AK, lds[b][0], tid + q * kThreads, ra[q]);
            put(BK, lds[b][1], tid + q * kThreads, rb[q]);
        }
    };
    fetch(0);
    stash(0);
    __syncthreads();
    int b = 0;
    for (int64_t k0 = 0; k0 < g.K; k0 += kStage, b ^= 1) {
        const bool more = k0 + kStage < g.K;
        if (more) fetch(k0 + kStage);
        f32x4_t a[S], c[S];
#pragma unroll
        for (int i = 0; i < S; ++i) {
            a[i] = *reinterpret_cast<const f32x4_t *>(&lds[b][0][(wm0 + 16 * i + lr) * kPitch + 4 * lg]);
            c[i] = *reinterpret_cast<const f32x4_t *>(&lds[b][1][(wn0 + 16 * i + lr) * kPitch + 4 * lg]);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int i = 0; i < S; ++i)
#pragma unroll
                for (int j = 0; j < S; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(c[j][s], a[i][s], acc[i][j], 0, 0, 0);
        if (more) stash(b ^ 1);
        __syncthreads();
    }
    if constexpr (KIND == kStats) {
        loss_stats<S, S, BT, 2>(g.e, acc, i0, g.I, j0, (int)(j0 / BT), wm0, wn0, wave & 1, red);
        return;
    }
#pragma unroll
    for (int i = 0; i < S; ++i) {
        const int64_t row = i0 + wm0 + 16 * i + lr;
        if (row >= g.I) continue;
        float dl = 0.f, lse = 0.f;
        int64_t t = -1;
        if constexpr (KIND == kGrad || kDx) {
            t = g.e.targets[row];
            dl = loss_scale(g.e, row, t);
        }
        if constexpr (KIND == kGrad) {
            lse = g.e.lse[row];
            t -= g.v0;
        }
#pragma unroll
        for (int j = 0; j < S; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int64_t col = j0 + wn0 + 16 * j + 4 * lg + v;
                if (col >= g.J) continue;
                float x = acc[i][j][v];
                float *o = g.out + row * g.ldo + col;
                if constexpr (KIND == kGrad)
                    x = dl != 0.f ? dl * (__builtin_amdgcn_exp2f((x - lse) * kLog2e) - (col == t ? 1.f : 0.f)) : 0.f;
                if constexpr (KIND == kAdd) x += *o;
                if constexpr (kDx) x = dl != 0.f ? x : 0.f;
                *o = x;
            }
    }
}

// 128 x 128 where that gives every CU a tile.
bool wide_tiles(int64_t I, int64_t J) { return ((I + 127) / 128) * ((J + 127) / 128) >= 256; }

template <bool AK, bool BK, Kind KIND>
hipError_t launch(Gemm g, hipStream_t s) {
    const int bt = wide_tiles(g.I, g.J) ? 128 : 64;
    g.tiles_i = (int)((g.I + bt - 1) / bt);
    const int64_t tiles = g.tiles_i * ((g.J + bt - 1) / bt);
    if (tiles >= (int64_t)1 << 31) return hipErrorNotSupported;
    if (bt == 128) loss_f32_kernel<128, AK, BK, KIND><<<(unsigned)tiles, kThreads, 0, s>>>(g);
    else loss_f32_kernel<64, AK, BK, KIND><<<(unsigned)tiles, kThreads, 0, s>>>(g);
    return hipGetLastError();
}

}  // namespace

int loss_f32_tiles(int64_t M, int64_t V) {
    const int bt = wide_tiles(M, V) ? 128 : 64;
    return (int)((V + bt - 1) / bt);
}

hipError_t launch_loss_f32_stats(const LossPass &p, const LossEpi &e, hipStream_t s) {
    Gemm g{};
    g.A = static_cast<const float *>(p.X);
    g.B = static_cast<const float *>(p.W);
    g.lda = g.ldb = g.K = p.n;
    g.I = p.M;
    g.J = p.V;
    g.e = e;
    return launch<true, true, kStats>(g, s);
}

hipError_t launch_loss_f32_piece(const LossPass &p, const LossEpi &e, int64_t v0, int64_t vp, float *G, bool first,
                                 hipStream_t s) {
    const float *W = static_cast<const float *>(p.W) + v0 * p.n;
    Gemm g{};
    g.e = e;
    g.v0 = v0;
    g.A = static_cast<const float *>(p.X);
    g.B = W;
    g.lda = g.ldb = g.K = p.n;
    g.I = p.M;
    g.J = vp;
    g.out = G;
    g.ldo = vp;
    hipError_t err = launch<true, true, kGrad>(g, s);
    if (err == hipSuccess && p.dX) {
        g.A = G;
        g.lda = g.K = vp;
        g.B = W;
        g.ldb = g.J = g.ldo = p.n;
        g.out = static_cast<float *>(p.dX);
        err = first ? launch<true, false, kStore>(g, s) : launch<true, false, kAdd>(g, s);
    }
    if (err == hipSuccess && p.dW) {
        g.A = G;
        g.lda = g.I = vp;
        g.B = static_cast<const float *>(p.X);
        g.ldb = g.J = g.ldo = p.n;
        g.K = p.M;
        g.out = static_cast<float *>(p.dW) + v0 * p.n;
        err = launch<false, false, kStore>(g, s);
    }
    return err;
}

}  // namespace dyad
