// The loss's matrix products in bf16, on the pipelined eight-wave tiles of pp_core.h:
//   kStats  Z = X W^T, tokens by vocabulary: per token (largest, sum of exponentials) of the tile
//   kGrad   Z^T = W X^T of a piece of the vocabulary, as G^T = exp(Z^T - lse) - onehot
//   kDw     dW = G^T (dloss X) of the piece
//   kDx     dX^T += W^T G of the piece, in fp32; times dloss at the end
// Side A's rows run along the reduction, side B's do (W, X) or are its indices (X, G^T read
// transposed out of LDS), so one copy of G serves both products.  What they need laid out
// otherwise is laid out once a call: W^T, and X and W with rows of whole 64s where n is not.
// Padded reduction indices are zero on one side and finite on the other.
//
// G, dloss X and W^T are fp16 there: G's values lie in [-1, 1], and in bf16 their rounding would
// put as much error into the gradients as the gradients' own (2.4e-3 to 2.7e-3 off 64 bits in
// place of 1.7e-3), where eleven bits put an eighth of that.  fp16's range is met by powers of two:
// 2^15 for G (values from 2^-29 on keep all bits), and one a column for the other two, which
// takes the column's largest magnitude to 2^14 .. 2^15 and goes out again with the sums.
//
// Tokens that do not count take no part: from kCompactFrom tokens the others are gathered, in
// order, and the kernels take their number from device memory (prompts and padding are often half
// of a batch: 3001 tokens of 1000 over 50021, half of them counting, 1.87 -> 0.75 ms a step).
#include "lm_internal.h"
#include "pp_core.h"
#include "row_io.h"

namespace dyad {

namespace {

enum Kind { kStats, kGrad, kDw, kDx };

// What the gradient's epilogue needs of a token, tokens past the last too.
struct Token {
    float *scale, *lse2;   // 0 where the token does not count; lse log2(e)
    int *target;           // -1 where it does not
};

constexpr int kGExp = 15;                       // G is held as G 2^15

// What a column is multiplied by, as an exponent, from the bits of its largest finite magnitude.
__device__ __forceinline__ int column_exp(uint32_t top) {
    if (top == 0u) return 0;
    const int e = 14 + 127 - (int)(top >> 23);
    return e < -100 ? -100 : e > 120 ? 120 : e;
}

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;
    const f32x2_t v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2_t));
}

struct Args {
    const uint16_t *A, *B;
    int64_t lda, ldb, I, J, K;   // K: a multiple of 64
    int64_t rows_b;              // side B's rows where they are the reduction's indices
    int group;
    int splits;                  // kDx: of the reduction, each into an acc of its own
    const int *count;            // tokens, in place of the side that runs over them; null: as given
    LossEpi e;
    Token tok;
    const uint32_t *col_top;     // kDw: of the columns of dloss X
    int64_t v0;
    uint16_t *out;
    float *acc;
    int64_t ldo;
    bool first;
};

template <int BM, int BN, int WGM, int WGN, bool TB>
struct Cfg {
    static constexpr int WM = BM / WGM, WN = BN / WGN, kSubM = WM / 16, kSubN = WN / 16;
    using A = PPSide<BM, false>;
    using B = PPSide<BN, TB>;
    static constexpr bool kTwo = BM * BN <= 128 * 128;   // two workgroups share a CU
    static constexpr int kSlotA = kTwo ? 2 : 3, kSlotB = 2;
    static constexpr int kOffB = kSlotA * A::kBytes, kLds = kOffB + kSlotB * B::kBytes;
    static_assert(WGM * WGN == kPPWaves && kLds <= 160 * 1024, "eight waves, LDS budget");
};

// Swaps the odd 16-lane rows of a with the even ones of b.
__device__ __forceinline__ void swap_lane_rows(uint32_t &a, uint32_t &b) {
    typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
    const u32x2_t r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r.x;
    b = r.y;
}

// x: a lane's four sums of column block 2 jp and of the next.  After the swap it holds 8
// consecutive columns, from lane_piece() of the pair on.
template <class Pack>
__device__ __forceinline__ uint4 pack_pair(const float (&x)[8], Pack pack) {
    uint32_t d0 = pack(x[0], x[1]), d1 = pack(x[2], x[3]), s0 = pack(x[4], x[5]), s1 = pack(x[6], x[7]);
    swap_lane_rows(d0, s0);
    swap_lane_rows(d1, s1);
    return make_uint4(d0, d1, s0, s1);
}
__device__ __forceinline__ int lane_piece(int lg) { return (lg & 1) * 16 + (lg >> 1) * 8; }

template <int BM, int BN, int WGM, int WGN, bool TB, Kind KIND>
__global__ void __launch_bounds__(kPPThreads, 1) loss_pp_kernel(Args g) {
    using C = Cfg<BM, BN, WGM, WGN, TB>;
    using SA = typename C::A;
    using SB = typename C::B;
    constexpr int SM = C::kSubM, SN = C::kSubN;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[C::kLds];
    lds_u8 *lds = (lds_u8 *)smem;
    const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (g.count) {
        const int64_t tokens = *g.count;
        if (KIND == kStats) g.I = tokens;
        if (KIND == kGrad || KIND == kDx) g.J = tokens;
        if (KIND == kDw) {
            g.K = (tokens + kPPK - 1) / kPPK * kPPK;
            g.rows_b = tokens;
        }
    }
    const int tiles_i = (int)((g.I + BM - 1) / BM), tiles_j = (int)((g.J + BN - 1) / BN), tiles = tiles_i * tiles_j;
    if ((int)blockIdx.x >= tiles * g.splits) return;
    // runs of `group` panels of side A, side A fastest: the workgroups that run together on an
    // XCD share both sides
    int item = xcd_tile(blockIdx.x, tiles * g.splits);
    const int split = KIND == kDx ? item / tiles : 0;
    item -= split * tiles;
    const int run = g.group * tiles_j, first = item / run * g.group;
    const int gm = tiles_i - first < g.group ? tiles_i - first : g.group;
    const int64_t i0 = (int64_t)(first + item % run % gm) * BM;
    const int tile_j = item % run / gm;
    const int64_t j0 = (int64_t)tile_j * BN;
    const int64_t left_i = g.I - i0 < BM ? g.I - i0 : BM, left_j = g.J - j0 < BN ? g.J - j0 : BN;
    const int all = (int)(g.K / kPPK);
    const int u0 = KIND == kDx ? (int)((int64_t)all * split / g.splits) : 0;
    const int units = (KIND == kDx ? (int)((int64_t)all * (split + 1) / g.splits) : all) - u0;

    const __amdgpu_buffer_rsrc_t rA = buffer_rsrc(g.A + i0 * g.lda, (uint32_t)(left_i * g.lda * 2));
    const __amdgpu_buffer_rsrc_t rB0 = buffer_rsrc(g.B + j0 * g.ldb, TB ? 0u : (uint32_t)(left_j * g.ldb * 2));
    uint32_t voA[SA::kPer], voB[SB::kPer], loA[SA::kPer], loB[SB::kPer];
#pragma unroll
    for (int q = 0; q < SA::kPer; ++q) {
        int row, byte;
        const int i = pp_instr(wave, q);
        pp_source<BM, false>(i, lane, row, byte);
        voA[q] = (uint32_t)row * (uint32_t)g.lda * 2u + (uint32_t)byte;
        loA[q] = 1024u * (uint32_t)i;
    }
#pragma unroll
    for (int q = 0; q < SB::kPer; ++q) {
        int row, byte;
        const int i = pp_instr(wave, q);
        pp_source<BN, TB>(i, lane, row, byte);
        voB[q] = (uint32_t)row * (uint32_t)g.ldb * 2u + (uint32_t)byte;
        loB[q] = (uint32_t)C::kOffB + 1024u * (uint32_t)i;
    }
    const auto clamp = [&](int d) { return u0 + (d < units ? d : units - 1); };
    auto issue_a = [&](int d) {
        lds_u8 *slot = lds + d % C::kSlotA * SA::kBytes;
        const uint32_t so = (uint32_t)clamp(d) * (uint32_t)(2 * kPPK);
#pragma unroll
        for (int q = 0; q < SA::kPer; ++q) dma16(rA, slot + loA[q], voA[q], so);
    };
    auto issue_b = [&](int d) {
        lds_u8 *slot = lds + d % C::kSlotB * SB::kBytes;
        __amdgpu_buffer_rsrc_t r = rB0;
        uint32_t so = 0;
        if constexpr (TB) {
            // the rows of this unit: their offsets pass 32 bits over the reduction, and those
            // past the last read zero
            const int64_t k0 = (int64_t)clamp(d) * kPPK;
            const int64_t rows = g.rows_b - k0 < kPPK ? g.rows_b - k0 : kPPK;
            r = buffer_rsrc(g.B + k0 * g.ldb + j0, rows > 0 ? (uint32_t)((rows * g.ldb - j0) * 2) : 0u);
        } else {
            so = (uint32_t)clamp(d) * (uint32_t)(2 * kPPK);
        }
#pragma unroll
        for (int q = 0; q < SB::kPer; ++q) dma16(r, slot + loB[q], voB[q], so);
    };
    const int wm0 = (wave / WGN) * C::WM, wn0 = (wave % WGN) * C::WN;
    const uint32_t base = (uint32_t)(uintptr_t)lds;
    const uint32_t fa = base + pp_frag<BM, false>(wm0, 0, lane);
    uint32_t fb[TB ? SN : 1];
#pragma unroll
    for (int j = 0; j < (TB ? SN : 1); ++j) fb[j] = base + (uint32_t)C::kOffB + pp_frag<BN, TB>(wn0, j, lane);
    auto addr = [&](int d, int h, uint32_t &pa, uint32_t (&pb)[TB ? SN : 1]) {
        pa = pp_step<BM, false>(fa + (uint32_t)(d % C::kSlotA * SA::kBytes), h);
#pragma unroll
        for (int j = 0; j < (TB ? SN : 1); ++j) pb[j] = pp_step<BN, TB>(fb[j] + (uint32_t)(d % C::kSlotB * SB::kBytes), h);
    };
    f32x4_t acc[SM][SN];
#pragma unroll
    for (int i = 0; i < SM; ++i)
#pragma unroll
        for (int j = 0; j < SN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (units > 0)
        pp_loop<SM, SN, TB, 4 * SB::kPitch, SA::kPer, SB::kPer, C::kSlotA, C::kSlotB, KIND == kDw || KIND == kDx>(
            units, wave, acc, issue_a, issue_b, addr, [](int) { return true; });
    // acc[i][j][v]: side A's row wm0 + 16 i + lr, side B's wn0 + 16 j + 4 lg + v
    if constexpr (KIND == kStats) {
        loss_stats<SM, SN, BM, WGN>(g.e, acc, i0, g.I, j0, tile_j, wm0, wn0, wave % WGN, reinterpret_cast<float2 *>(smem));
    } else if constexpr (KIND == kGrad) {
        const int v_lane = (int)(g.v0 + i0) + wm0 + lr;
#pragma unroll
        for (int jp = 0; jp < SN / 2; ++jp) {
            float scale[8], lse2[8];
            int target[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t t = j0 + wn0 + 32 * jp + 16 * h + 4 * lg;   // tokens are laid out for whole tiles
                __builtin_memcpy(scale + 4 * h, __builtin_assume_aligned(g.tok.scale + t, 16), 16);
                __builtin_memcpy(lse2 + 4 * h, __builtin_assume_aligned(g.tok.lse2 + t, 16), 16);
                __builtin_memcpy(target + 4 * h, __builtin_assume_aligned(g.tok.target + t, 16), 16);
            }
            const int64_t col = j0 + wn0 + 32 * jp + lane_piece(lg);
            uint16_t *o = g.out + (i0 + wm0 + lr) * g.ldo + col;
#pragma unroll
            for (int i = 0; i < SM; ++i) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float z = acc[i][2 * jp + (e >> 2)][e & 3];
                    const float p = __builtin_amdgcn_exp2f(fmaf(z, kLog2e, -lse2[e])) - (target[e] == v_lane + 16 * i ? 1.f : 0.f);
                    x[e] = scale[e] != 0.f ? p * (float)(1 << kGExp) : 0.f;   // zero whatever p is
                }
                const uint4 w = pack_pair(x, pack_f16);
                if (col < g.ldo && i0 + wm0 + 16 * i + lr < g.I) *reinterpret_cast<uint4 *>(o + (int64_t)(16 * i) * g.ldo) = w;
            }
        }
    } else if constexpr (KIND == kDw) {
#pragma unroll
        for (int jp = 0; jp < SN / 2; ++jp) {
            int back[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t top[4];                               // laid out for whole tiles
                __builtin_memcpy(top, __builtin_assume_aligned(g.col_top + j0 + wn0 + 32 * jp + 16 * h + 4 * lg, 16), 16);
#pragma unroll
                for (int v = 0; v < 4; ++v) back[4 * h + v] = -(column_exp(top[v]) + kGExp);
            }
            const int64_t col = j0 + wn0 + 32 * jp + lane_piece(lg);
#pragma unroll
            for (int i = 0; i < SM; ++i) {
                const int64_t row = i0 + wm0 + 16 * i + lr;
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = ldexpf(acc[i][2 * jp + (e >> 2)][e & 3], back[e]);
                const uint4 w = pack_pair(x, pack_bf16);
                if (row >= g.I) continue;
                uint16_t *o = g.out + row * g.ldo + col;
                if (col + 8 <= g.J) {
                    __builtin_memcpy(o, &w, 16);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (col + e < g.J) o[e] = (uint16_t)(word_of(w, e >> 1) >> (16 * (e & 1)));
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < SM; ++i) {
            const int64_t row = i0 + wm0 + 16 * i + lr;
#pragma unroll
            for (int j = 0; j < SN; ++j) {
                const int64_t col = j0 + wn0 + 16 * j + 4 * lg;
                if (row >= g.I || col >= g.ldo) continue;
                f32x4_t *o = reinterpret_cast<f32x4_t *>(g.acc + ((int64_t)split * g.I + row) * g.ldo + col);
                f32x4_t s = acc[i][j];
                if (!g.first) {
                    const f32x4_t t = *o;
#pragma unroll
                    for (int v = 0; v < 4; ++v) s[v] += t[v];
                }
                *o = s;
            }
        }
    }
}

// The tokens that count, in order: their places idx, their targets and how many; the others'
// loss and lse are zero (forward).  One workgroup, a run of tokens a thread.
__global__ void __launch_bounds__(1024) compact_kernel(LossEpi e, int64_t M, int *idx, int64_t *targets, int *count,
                                                       float *loss, float *lse) {
    __shared__ int sums[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t per = (M + 1023) / 1024, m0 = tid * per, m1 = m0 + per < M ? m0 + per : M;
    int n = 0;
    for (int64_t m = m0; m < m1; ++m) n += loss_counts(e, e.targets[m]) ? 1 : 0;
    int before = n;
#pragma unroll
    for (int w = 1; w < 64; w <<= 1) {
        const int t = __shfl_up(before, w);
        if (lane >= w) before += t;
    }
    if (lane == 63) sums[wave] = before;
    __syncthreads();
    before -= n;
    for (int w = 0; w < wave; ++w) before += sums[w];
    if (tid == 1023) *count = before + n;
    for (int64_t m = m0; m < m1; ++m) {
        const int64_t t = e.targets[m];
        if (loss_counts(e, t)) {
            idx[before] = (int)m;
            targets[before++] = t;
        } else if (loss) {
            loss[m] = 0.f;
            lse[m] = 0.f;
        }
    }
}

// dst[r][c] = src[idx[r]][c] for c < n, else 0, c < np (a multiple of 64).  idx null: row r;
// count null: all rows.
__global__ void __launch_bounds__(256) gather_kernel(const uint16_t *src, uint16_t *dst, int64_t rows, int n, int np,
                                                     const int *idx, const int *count) {
    if (count) rows = *count;
    const int64_t total = rows * (np / 8);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / (np / 8);
        const int c = (int)(i - r * (np / 8)) * 8;
        float v[8];
        load_cols<true>(src + (idx ? idx[r] : r) * n, c, n, v);
        store8(dst + r * np + c, v);
    }
}

// Rows of tokens that do not count: their gradient is zero.
__global__ void __launch_bounds__(256) zero_rows_kernel(LossEpi e, uint16_t *dx, int64_t M, int n) {
    for (int64_t m = blockIdx.x; m < M; m += gridDim.x) {
        if (loss_counts(e, e.targets[m])) continue;
        for (int c = threadIdx.x; c < n; c += 256) dx[m * n + c] = 0;
    }
}

// The largest finite magnitude of each column of src (times each row's scale), as bits, into
// top, which starts at zero.  256 columns by eight rows a workgroup, a stretch of rows.
__global__ void __launch_bounds__(256) column_top_kernel(const uint16_t *src, const float *scale, int64_t rows, int n, int ld,
                                                         const int *count, uint32_t *top) {
    __shared__ uint32_t t[8][256 + 8];
    if (count) rows = *count;
    const int c = blockIdx.y * 256 + (threadIdx.x & 31) * 8, r = threadIdx.x >> 5;
    uint32_t best[8] = {};
    if (c < n) {
        for (int64_t m = (int64_t)blockIdx.x * 8 + r; m < rows; m += (int64_t)gridDim.x * 8) {
            float v[8];
            load_cols<true>(src + m * ld, c, n, v);
            const float s = scale ? scale[m] : 1.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t b = __float_as_uint(v[e] * s) & 0x7fffffffu;
                best[e] = b < 0x7f800000u && b > best[e] ? b : best[e];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) t[r][(threadIdx.x & 31) * 8 + e] = best[e];
    __syncthreads();
    uint32_t b = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) b = t[k][threadIdx.x] > b ? t[k][threadIdx.x] : b;
    // the order of these does not matter
    if (blockIdx.y * 256 + threadIdx.x < n && b) atomicMax(top + blockIdx.y * 256 + threadIdx.x, b);
}

// dst[m][c] = src[m][c] scale[m] in fp16 at the column's scale, rows of np columns.
__global__ void __launch_bounds__(256) scale_kernel(const uint16_t *src, const float *scale, const uint32_t *top,
                                                    uint16_t *dst, int64_t rows, int np, const int *count) {
    if (count) rows = *count;
    const int64_t total = rows * (np / 8);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / (np / 8);
        const int c = (int)(i - m * (np / 8)) * 8;
        float v[8];
        load8(src + m * np + c, v);
        const float s = scale[m];
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = s != 0.f ? ldexpf(v[e] * s, column_exp(top[c + e])) : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_f16(v[2 * e], v[2 * e + 1]);
        __builtin_memcpy(__builtin_assume_aligned(dst + m * np + c, 16), w, 16);
    }
}

// dst[c][r] = src[r][c] for r < rows, else 0, r < ld (a multiple of 64), in fp16 at the column's
// scale: 64 x 64 tiles.
__global__ void __launch_bounds__(256) transpose_kernel(const uint16_t *src, const uint32_t *top, uint16_t *dst, int64_t rows,
                                                        int n, int64_t ld) {
    __shared__ uint16_t t[64][66];
    const int64_t r0 = (int64_t)blockIdx.x * 64;
    const int c0 = blockIdx.y * 64, tid = threadIdx.x;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int r = (tid + 256 * q) / 8, c = (tid + 256 * q) % 8 * 8;
        uint16_t v[8];
        if (r0 + r < rows && c0 + c + 8 <= n) {
            __builtin_memcpy(v, src + (r0 + r) * n + c0 + c, 16);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = r0 + r < rows && c0 + c + e < n ? src[(r0 + r) * n + c0 + c + e] : (uint16_t)0;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) t[c + e][r] = v[e];
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int c = (tid + 256 * q) / 8, r = (tid + 256 * q) % 8 * 8;
        if (c0 + c >= n) continue;
        const int up = column_exp(top[c0 + c]);
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = pack_f16(ldexpf(bf16_to_f32(t[c][r + 2 * e]), up), ldexpf(bf16_to_f32(t[c][r + 2 * e + 1]), up));
        __builtin_memcpy(__builtin_assume_aligned(dst + (int64_t)(c0 + c) * ld + r0 + r, 16), w, 16);
    }
}

// dX[idx[m]][c] = scale[m] times the fp32 sums acc[split][c][m], added in order, rounded: 64 x 64 tiles.
__global__ void __launch_bounds__(256) round_transpose_kernel(const float *acc, int splits, const float *scale,
                                                              const uint32_t *top, uint16_t *dst, int64_t M, int n,
                                                              int64_t ld, const int *idx, const int *count) {
    __shared__ float t[64][65];
    if (count) M = *count;
    const int64_t m0 = (int64_t)blockIdx.x * 64;
    const int c0 = blockIdx.y * 64, tid = threadIdx.x;
    if (m0 >= M) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int c = (tid + 256 * q) / 16, m = (tid + 256 * q) % 16 * 4;
        f32x4_t v = {0.f, 0.f, 0.f, 0.f};
        if (c0 + c < n) {
            const float *src = acc + (int64_t)(c0 + c) * ld + m0 + m;
            v = *reinterpret_cast<const f32x4_t *>(src);
            for (int s = 1; s < splits; ++s) {
                const f32x4_t u = *reinterpret_cast<const f32x4_t *>(src + (int64_t)s * n * ld);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += u[e];
            }
        }
        const int back = c0 + c < n ? -(column_exp(top[c0 + c]) + kGExp) : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[m + e][c] = ldexpf(v[e], back);
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int m = (tid + 256 * q) / 8, c = (tid + 256 * q) % 8 * 8;
        if (m0 + m >= M) continue;
        const float by = scale[m0 + m];
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = by != 0.f ? t[m][c + e] * by : 0.f;
        store_cols<true>(dst + (idx ? idx[m0 + m] : m0 + m) * n, c0 + c, n, v);
    }
}

// The tokens' part of the gradient, and zeros to start the columns' largest magnitudes from.
__global__ void __launch_bounds__(256) token_kernel(LossEpi e, Token t, int64_t M, int64_t padded, const int *idx,
                                                    const int *count, uint32_t *top, int64_t tops) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    for (int64_t k = c; k < tops; k += (int64_t)gridDim.x * 256) top[k] = 0u;
    if (c >= padded) return;
    if (count) M = *count;
    float scale = 0.f, lse = 0.f;
    int target = -1;
    if (c < M) {
        const int64_t m = idx ? idx[c] : c, v = e.targets[m];
        if (loss_counts(e, v)) {
            scale = loss_scale(e, m, v);
            lse = e.lse[m];
            target = (int)v;
        }
    }
    t.scale[c] = scale;
    t.lse2[c] = lse * kLog2e;
    t.target[c] = target;
}

// Tiles: rows of side A and B, and the time of a round of them next to 256 x 256's, with one, two
// or three workgroups on every CU (measured at 768, 1000 and 4096 wide; the wide ones fill a CU).
struct Tile {
    int bm, bn, per_cu;
    double time[3];
};
constexpr Tile kTiles[] = {
    {256, 256, 1, {1.0}}, {192, 256, 1, {0.85}}, {128, 128, 2, {0.36, 0.62}}, {64, 128, 3, {0.22, 0.38, 0.54}}};

struct Choice {
    int tile, splits;
};
// The tile of least time over 256 CUs, and with `most_splits` above 1 the reduction's splits,
// where the tiles alone leave CUs idle.
Choice choose(int64_t I, int64_t J, int64_t most_splits = 1) {
    Choice best{0, 1};
    double least = 0;
    for (int t = 0; t < 4; ++t) {
        const Tile &k = kTiles[t];
        const int64_t tiles = ((I + k.bm - 1) / k.bm) * ((J + k.bn - 1) / k.bn);
        int64_t splits = 256 / tiles;
        splits = splits > most_splits ? most_splits : splits < 1 ? 1 : splits;
        const int64_t count = tiles * splits, round = 256 * k.per_cu, rest = (count % round + 255) / 256;
        const double time = ((double)(count / round) * k.time[k.per_cu - 1] + (rest ? k.time[rest - 1] : 0.0)) / (double)splits;
        if (t == 0 || time < least) {
            best = {t, (int)splits};
            least = time;
        }
    }
    return best;
}

template <int BM, int BN, int WGM, int WGN, bool TB, Kind KIND>
hipError_t launch_tile(Args &g, hipStream_t s) {
    const int64_t tiles = ((g.I + BM - 1) / BM) * ((g.J + BN - 1) / BN) * g.splits;
    if (tiles >= (int64_t)1 << 31) return hipErrorNotSupported;
    g.group = 8;
    loss_pp_kernel<BM, BN, WGM, WGN, TB, KIND><<<(unsigned)tiles, kPPThreads, 0, s>>>(g);
    return hipGetLastError();
}

template <bool TB, Kind KIND>
hipError_t launch(Args g, const Choice &c, hipStream_t s) {
    g.splits = c.splits;
    switch (c.tile) {
    case 0: return launch_tile<256, 256, 2, 4, TB, KIND>(g, s);
    case 1: return launch_tile<192, 256, 2, 4, TB, KIND>(g, s);
    case 2: return launch_tile<128, 128, 2, 4, TB, KIND>(g, s);
    default: return launch_tile<64, 128, 2, 4, TB, KIND>(g, s);
    }
}

// Below this the launches that gather would take longer than what they save.
constexpr int64_t kCompactFrom = 257;

int64_t up(int64_t v, int64_t q) { return (v + q - 1) / q * q; }
size_t part(size_t bytes) { return (bytes + 255) / 256 * 256; }

hipError_t gather(const void *src, uint16_t *dst, int64_t rows, int64_t n, int64_t np, const int *idx, const int *count,
                  hipStream_t s) {
    const int64_t blocks = (rows * (np / 8) + 255) / 256;
    gather_kernel<<<(unsigned)(blocks < 16384 ? blocks : 16384), 256, 0, s>>>(static_cast<const uint16_t *>(src), dst, rows,
                                                                              (int)n, (int)np, idx, count);
    return hipGetLastError();
}

// Where things lie in the workspace; a size of 0 for what a call does not need.
struct Space {
    size_t total = 0;
    size_t take(size_t bytes) {
        const size_t at = total;
        total += (bytes + 255) / 256 * 256;
        return at;
    }
};

// The tokens that count and the operands as the kernels read them.
struct Operands {
    int64_t np;                  // columns
    bool compact;
    size_t idx, targets, count, x, w;
};
Operands operands_of(Space &space, int64_t M, int64_t n, int64_t V) {
    Operands o;
    o.np = up(n, kPPK);
    o.compact = M >= kCompactFrom;
    o.idx = space.take(o.compact ? (size_t)M * 4 : 0);
    o.targets = space.take(o.compact ? (size_t)M * 8 : 0);
    o.count = space.take(o.compact ? 4 : 0);
    o.x = space.take(o.compact || o.np != n ? (size_t)(M * o.np) * 2 : 0);
    o.w = space.take(o.np != n ? (size_t)(V * o.np) * 2 : 0);
    return o;
}

// What the launches take of them.
struct Prepared {
    const uint16_t *X, *W;
    const int *idx, *count;
    const int64_t *targets;
};
hipError_t prepare(const Operands &o, const LossPass &p, const LossEpi &e, char *ws, float *loss, float *lse, Prepared &r,
                   hipStream_t s) {
    r = {static_cast<const uint16_t *>(p.X), static_cast<const uint16_t *>(p.W), nullptr, nullptr, e.targets};
    hipError_t err = hipSuccess;
    if (o.compact) {
        int *idx = reinterpret_cast<int *>(ws + o.idx), *count = reinterpret_cast<int *>(ws + o.count);
        int64_t *targets = reinterpret_cast<int64_t *>(ws + o.targets);
        compact_kernel<<<1, 1024, 0, s>>>(e, p.M, idx, targets, count, loss, lse);
        err = hipGetLastError();
        r.idx = idx;
        r.count = count;
        r.targets = targets;
    }
    if (err == hipSuccess && (o.compact || o.np != p.n)) {
        uint16_t *x = reinterpret_cast<uint16_t *>(ws + o.x);
        err = gather(p.X, x, p.M, p.n, o.np, r.idx, r.count, s);
        r.X = x;
    }
    if (err == hipSuccess && o.np != p.n) {
        uint16_t *w = reinterpret_cast<uint16_t *>(ws + o.w);
        err = gather(p.W, w, p.V, p.n, o.np, nullptr, nullptr, s);
        r.W = w;
    }
    return err;
}

// Vocabulary columns of a piece, and the workspace of a backward pass.
struct Layout {
    Operands ops;
    int64_t Mp, Mq, Vp, vp;
    Choice dx;
    size_t tokens, tops, xs, wt, gt, acc, total;
    int64_t nq;
};
Layout layout_of(int64_t M, int64_t n, int64_t V) {
    Layout l;
    Space space;
    l.ops = operands_of(space, M, n, V);
    l.Mp = up(M, kPPK);
    l.Mq = up(M, 256) + 256;     // the last tile's tokens, whatever its width
    l.Vp = up(V, kPPK);
    // G^T of a piece within 512 MB, but for very many tokens; pieces of one size, whole tiles
    int64_t most = ((int64_t)512 << 20) / (2 * l.Mp) / 256 * 256;
    if (most < 2048) most = 2048;
    const int64_t pieces = (V + most - 1) / most;
    l.vp = up((V + pieces - 1) / pieces, 256);
    // at least 16 units a split, and the splits' sums within the weights' gradient's size
    int64_t splits = l.vp / kPPK / 16;
    const int64_t room = l.vp / (2 * l.Mp);
    splits = splits < room ? splits : room;
    l.dx = choose(n, M, splits < 1 ? 1 : splits);
    l.tokens = space.take((size_t)l.Mq * 12);
    l.nq = up(n, 256) + 256;
    l.tops = space.take((size_t)l.nq * 8);
    l.xs = space.take((size_t)(M * l.ops.np) * 2);
    l.wt = space.take((size_t)(n * l.Vp) * 2);
    l.gt = space.take((size_t)(l.vp * l.Mp) * 2);
    l.acc = space.take((size_t)(l.dx.splits * n * l.Mp) * 4);
    l.total = space.total;
    return l;
}

}  // namespace

int loss_mfma_tiles(int64_t M, int64_t V) {
    const int bn = kTiles[choose(M, V).tile].bn;
    return (int)((V + bn - 1) / bn);
}

size_t loss_mfma_forward_bytes(int64_t M, int64_t n, int64_t V) {
    Space space;
    operands_of(space, M, n, V);
    return space.total;
}

size_t loss_mfma_backward_bytes(int64_t M, int64_t n, int64_t V) { return layout_of(M, n, V).total; }

hipError_t launch_loss_mfma_stats(const LossPass &p, const LossEpi &e, void *ws, float *each, LossTokens &tokens,
                                  hipStream_t s) {
    Space space;
    const Operands o = operands_of(space, p.M, p.n, p.V);
    Prepared r;
    hipError_t err = prepare(o, p, e, static_cast<char *>(ws), each, p.lse, r, s);
    if (err != hipSuccess) return err;
    tokens = {r.idx, r.count};
    Args g{};
    g.e = e;
    g.e.targets = r.targets;
    g.count = r.count;
    g.A = r.X;
    g.B = r.W;
    g.I = p.M;
    g.J = p.V;
    g.K = g.lda = g.ldb = o.np;
    return launch<false, kStats>(g, choose(p.M, p.V), s);
}

hipError_t launch_loss_mfma_grad(const LossPass &p, const LossEpi &e, hipStream_t s) {
    const Layout l = layout_of(p.M, p.n, p.V);
    char *ws = static_cast<char *>(p.ws);
    const auto at = [&](size_t o) { return reinterpret_cast<uint16_t *>(ws + o); };
    Prepared r;
    hipError_t err = prepare(l.ops, p, e, ws, nullptr, nullptr, r, s);
    if (err != hipSuccess) return err;
    Token tok;
    tok.scale = reinterpret_cast<float *>(ws + l.tokens);
    tok.lse2 = tok.scale + l.Mq;
    tok.target = reinterpret_cast<int *>(tok.lse2 + l.Mq);
    uint32_t *const x_top = reinterpret_cast<uint32_t *>(ws + l.tops), *const w_top = x_top + l.nq;
    token_kernel<<<(unsigned)(l.Mq / 256), 256, 0, s>>>(e, tok, p.M, l.Mq, r.idx, r.count, x_top, 2 * l.nq);
    err = hipGetLastError();
    const int np = (int)l.ops.np, n = (int)p.n;
    const auto top_grid = [&](int64_t rows) {
        const int64_t blocks = (rows + 63) / 64;
        return dim3((unsigned)(blocks < 1024 ? blocks : 1024), (unsigned)((n + 255) / 256));
    };
    if (err == hipSuccess && p.dW) {
        const int64_t blocks = (p.M * (np / 8) + 255) / 256;
        column_top_kernel<<<top_grid(p.M), 256, 0, s>>>(r.X, tok.scale, p.M, n, np, r.count, x_top);
        scale_kernel<<<(unsigned)(blocks < 16384 ? blocks : 16384), 256, 0, s>>>(r.X, tok.scale, x_top, at(l.xs), p.M, np,
                                                                                 r.count);
        err = hipGetLastError();
    }
    if (err == hipSuccess && p.dX) {
        const uint16_t *W = static_cast<const uint16_t *>(p.W);
        column_top_kernel<<<top_grid(p.V), 256, 0, s>>>(W, nullptr, p.V, n, n, nullptr, w_top);
        transpose_kernel<<<dim3((unsigned)(l.Vp / 64), (unsigned)(np / 64)), 256, 0, s>>>(W, w_top, at(l.wt), p.V, n, l.Vp);
        if (r.count)
            zero_rows_kernel<<<(unsigned)(p.M < 8192 ? p.M : 8192), 256, 0, s>>>(e, static_cast<uint16_t *>(p.dX), p.M, n);
        err = hipGetLastError();
    }
    float *acc = reinterpret_cast<float *>(ws + l.acc);
    for (int64_t v0 = 0; v0 < p.V && err == hipSuccess; v0 += l.vp) {
        const int64_t vn = p.V - v0 < l.vp ? p.V - v0 : l.vp;
        Args g{};
        g.e = e;
        g.count = r.count;
        g.tok = tok;
        g.v0 = v0;
        g.A = r.W + v0 * l.ops.np;
        g.B = r.X;
        g.lda = g.ldb = g.K = l.ops.np;
        g.I = vn;
        g.J = p.M;
        g.out = at(l.gt);
        g.ldo = l.Mp;
        err = launch<false, kGrad>(g, choose(g.I, g.J), s);
        if (err == hipSuccess && p.dW) {
            g.A = at(l.gt);
            g.lda = g.K = l.Mp;
            g.B = at(l.xs);
            g.rows_b = p.M;
            g.J = g.ldo = p.n;
            g.col_top = x_top;
            g.out = static_cast<uint16_t *>(p.dW) + v0 * p.n;
            err = launch<true, kDw>(g, choose(g.I, g.J), s);
        }
        if (err == hipSuccess && p.dX) {
            g.A = at(l.wt) + v0;
            g.lda = l.Vp;
            g.B = at(l.gt);
            g.ldb = g.ldo = l.Mp;
            g.I = p.n;
            g.J = p.M;
            g.K = up(vn, kPPK);
            g.rows_b = vn;
            g.acc = acc;
            g.first = v0 == 0;
            err = launch<true, kDx>(g, l.dx, s);
        }
    }
    if (err == hipSuccess && p.dX) {
        round_transpose_kernel<<<dim3((unsigned)(l.Mp / 64), (unsigned)(l.ops.np / 64)), 256, 0, s>>>(
            acc, l.dx.splits, tok.scale, w_top, static_cast<uint16_t *>(p.dX), p.M, (int)p.n, l.Mp, r.idx, r.count);
        err = hipGetLastError();
    }
    return err;
}

}  // namespace dyad
