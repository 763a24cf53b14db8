// The loss's matrix products on the pipelined eight-wave bf16 tiles of pp_core.h:
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
// An entry that every token finds improbable has a row of G, and of dW, below that range.  Rows whose
// largest |G| is under 2^-24 are formed again, gathered, each at a power of two of its own (kGrad and kDw with
// RARE).  From 2^-24 on fp16's smallest step, 2^-39, is at most 2^-15 of the row's largest value.  A step
// without such rows takes up to 3 % longer for it, one where half of them are 9 to 30 % (512 and 16384
// tokens of 768 over 50000).
//
// fp32 operands (from kSplitFrom tokens) are split in three bf16 values, x = h + m + l with 8 bits
// each, exact to 2^-27, and six of the nine products h h, h m, m h, h l, l h, m m are summed in
// fp32; the others are below 2^-26 of the whole.  The reduction is six times as long at eight
// times the rate of the fp32 matrix instructions (157 TFLOP/s, of which plain tiles get half).
// G is split as it is formed, and holds dloss.
//
// Tokens that do not count take no part: from kCompactFrom tokens the others are gathered, in
// order, and the kernels take their number from device memory (prompts and padding are often half
// of a batch: 3001 tokens of 1000 over 50021, half of them counting, 1.87 -> 0.90 ms a step, with
// the splits of dX's reduction).
#include "lm_internal.h"
#include "pp_core.h"
#include "row_io.h"

namespace dyad {

namespace {

enum Kind { kStats, kGrad, kDw, kDx };

// What the gradient's epilogue needs of a token, tokens past the last too.
struct Token {
    float *scale, *lse;    // dloss, 0 where the token does not count; lse, in bf16 times log2(e)
    int *target;           // -1 where it does not
};

constexpr int kGExp = 15;                       // G is held as G 2^15

// What a column is multiplied by, as an exponent, from the bits of its largest finite magnitude:
// -113 for magnitudes of 2^127 and more, and at most 120 (2^-106 and less are held below 2^14).
__device__ __forceinline__ int column_exp(uint32_t top) {
    if (top == 0u) return 0;
    const int e = 14 + 127 - (int)(top >> 23);
    return e > 120 ? 120 : e;
}

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;
    const f32x2_t v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2_t));
}

// The planes (h 0, m 1, l 2) of the product that unit d of a split reduction multiplies.
constexpr int kProducts = 6;
__device__ __forceinline__ int plane_a(int d) { return 0x120100 >> (4 * (d % kProducts)) & 15; }
__device__ __forceinline__ int plane_b(int d) { return 0x102010 >> (4 * (d % kProducts)) & 15; }

// Eight values as three planes of eight bf16; an infinity or NaN stays in the first alone.
__device__ __forceinline__ void split8(const float (&v)[8], uint4 (&p)[3]) {
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = v[e];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const uint32_t w[4] = {pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3]), pack_bf16(r[4], r[5]), pack_bf16(r[6], r[7])};
        p[k] = make_uint4(w[0], w[1], w[2], w[3]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float h = unpack_bf16(w[e >> 1], e & 1);
            r[e] = (__float_as_uint(h) & 0x7f800000u) != 0x7f800000u ? r[e] - h : 0.f;
        }
    }
}

struct Args {
    const uint16_t *A, *B;
    int64_t plane_a, plane_b, plane_out;   // values from one plane to the next (fp32)
    int64_t lda, ldb, I, J, K;   // K: a multiple of 64
    int64_t rows_b;              // side B's rows where they are the reduction's indices
    int group;
    int splits;                  // kDx: of the reduction, each into an acc of its own
    const int *count;            // tokens, in place of the side that runs over them; null: as given
    LossEpi e;
    Token tok;
    const uint32_t *col_top;     // kDw: of the columns of dloss X
    float *row_top;              // kGrad: each row's largest |G| 2^15 of a tile's tokens, [tiles][ldt]; null: not wanted
    int64_t ldt;
    // RARE: how many rows, and for each its vocabulary entry in the piece and its exponent beside kGExp
    const int *rare, *rare_row, *rare_exp;
    int64_t v0;                  // the piece's first vocabulary column
    void *out;
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

// x: a lane's four sums of column block 2 jp and of the next.  After the swap it holds 8
// consecutive columns, from lane_piece() of the pair on.
template <class Pack>
__device__ __forceinline__ uint4 pack_pair(const float (&x)[8], Pack pack) {
    uint32_t d0 = pack(x[0], x[1]), d1 = pack(x[2], x[3]), s0 = pack(x[4], x[5]), s1 = pack(x[6], x[7]);
    swap_rows(d0, s0);
    swap_rows(d1, s1);
    return make_uint4(d0, d1, s0, s1);
}
__device__ __forceinline__ int lane_piece(int lg) { return (lg & 1) * 16 + (lg >> 1) * 8; }

// One tile of one split.
template <int BM, int BN, int WGM, int WGN, bool TB, Kind KIND, bool F32, bool RARE>
__device__ __forceinline__ void loss_tile(const Args &g, int block, int tiles_i, int tiles_j) {
    using C = Cfg<BM, BN, WGM, WGN, TB>;
    using SA = typename C::A;
    using SB = typename C::B;
    constexpr int SM = C::kSubM, SN = C::kSubN;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[C::kLds];
    lds_u8 *lds = (lds_u8 *)smem;
    const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles = tiles_i * tiles_j;
    // runs of `group` panels of side A, side A fastest: the workgroups that run together on an
    // XCD share both sides
    int item = RARE ? block : xcd_tile(block, tiles * g.splits);
    const int split = KIND == kDx ? item / tiles : 0;
    item -= split * tiles;
    const int run = g.group * tiles_j, first = item / run * g.group;
    const int gm = tiles_i - first < g.group ? tiles_i - first : g.group;
    const int64_t i0 = (int64_t)(first + item % run % gm) * BM;
    const int tile_j = item % run / gm;
    const int64_t j0 = (int64_t)tile_j * BN;
    const int64_t left_i = g.I - i0 < BM ? g.I - i0 : BM, left_j = g.J - j0 < BN ? g.J - j0 : BN;
    const int all = (int)(g.K / kPPK) * (F32 ? kProducts : 1);
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
        const int u = clamp(d), k = F32 ? u / kProducts : u;
        const uint32_t so = (uint32_t)k * (uint32_t)(2 * kPPK);
        __amdgpu_buffer_rsrc_t r = rA;
        if constexpr (F32) r = buffer_rsrc(g.A + plane_a(u) * g.plane_a + i0 * g.lda, (uint32_t)(left_i * g.lda * 2));
#pragma unroll
        for (int q = 0; q < SA::kPer; ++q) dma16(r, slot + loA[q], voA[q], so);
    };
    auto issue_b = [&](int d) {
        lds_u8 *slot = lds + d % C::kSlotB * SB::kBytes;
        const int u = clamp(d), k = F32 ? u / kProducts : u;
        const uint16_t *plane = g.B;
        if constexpr (F32) plane += plane_b(u) * g.plane_b;
        __amdgpu_buffer_rsrc_t r = rB0;
        uint32_t so = 0;
        if constexpr (TB) {
            // the rows of this unit: their offsets pass 32 bits over the reduction, and those
            // past the last read zero
            const int64_t k0 = (int64_t)k * kPPK;
            const int64_t rows = g.rows_b - k0 < kPPK ? g.rows_b - k0 : kPPK;
            r = buffer_rsrc(plane + k0 * g.ldb + j0, rows > 0 ? (uint32_t)((rows * g.ldb - j0) * 2) : 0u);
        } else {
            so = (uint32_t)k * (uint32_t)(2 * kPPK);
            if constexpr (F32) r = buffer_rsrc(plane + j0 * g.ldb, (uint32_t)(left_j * g.ldb * 2));
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
        pp_loop<SM, SN, TB, 4 * SB::kPitch, SA::kPer, SB::kPer, C::kSlotA, C::kSlotB, !F32 && (KIND == kDw || KIND == kDx)>(
            units, wave, acc, issue_a, issue_b, addr, [](int) { return true; });
    // acc[i][j][v]: side A's row wm0 + 16 i + lr, side B's wn0 + 16 j + 4 lg + v
    if constexpr (KIND == kStats) {
        loss_stats<SM, SN, BM, WGN>(g.e, acc, i0, g.I, g.v0 + j0, (int)(g.v0 / BN) + tile_j, wm0, wn0, wave % WGN, reinterpret_cast<float2 *>(smem));
    } else if constexpr (KIND == kGrad) {
        int v_of[SM], up_by[SM];     // the lane's rows: their vocabulary entries, and exponents
        float top[SM];               // of what the lane has of them, the largest
#pragma unroll
        for (int i = 0; i < SM; ++i) {
            int row = (int)i0 + wm0 + 16 * i + lr;
            if constexpr (RARE) row = row < g.I ? row : 0;
            v_of[i] = (int)g.v0 + (RARE ? g.rare_row[row] : row);
            up_by[i] = kGExp + (RARE ? g.rare_exp[row] : 0);
            top[i] = 0.f;
        }
#pragma unroll
        for (int jp = 0; jp < SN / 2; ++jp) {
            float scale[8], lse[8];
            int target[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t t = j0 + wn0 + 32 * jp + 16 * h + 4 * lg;   // tokens are laid out for whole tiles
                __builtin_memcpy(scale + 4 * h, __builtin_assume_aligned(g.tok.scale + t, 16), 16);
                __builtin_memcpy(lse + 4 * h, __builtin_assume_aligned(g.tok.lse + t, 16), 16);
                __builtin_memcpy(target + 4 * h, __builtin_assume_aligned(g.tok.target + t, 16), 16);
            }
            const int64_t col = j0 + wn0 + 32 * jp + lane_piece(lg);
            uint16_t *o = static_cast<uint16_t *>(g.out) + (i0 + wm0 + lr) * g.ldo + col;
#pragma unroll
            for (int i = 0; i < SM; ++i) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float z = acc[i][2 * jp + (e >> 2)][e & 3];
                    const float p = __builtin_amdgcn_exp2f(F32 ? (z - lse[e]) * kLog2e : fmaf(z, kLog2e, -lse[e])) - (target[e] == v_of[i] ? 1.f : 0.f);
                    x[e] = scale[e] != 0.f ? F32 ? p * scale[e] : RARE ? ldexpf(p, up_by[i]) : p * (float)(1 << kGExp) : 0.f;   // zero whatever p is
                    if constexpr (!F32 && !RARE) top[i] = fmaxf(top[i], fabsf(x[e]));
                }
                const bool in = col < g.ldo && i0 + wm0 + 16 * i + lr < g.I;
                if constexpr (F32) {
                    uint4 p[3];
                    split8(x, p);
#pragma unroll
                    for (int k = 0; k < 3; ++k) {
                        swap_rows(p[k].x, p[k].z);
                        swap_rows(p[k].y, p[k].w);
                        if (in) *reinterpret_cast<uint4 *>(o + k * g.plane_out + (int64_t)(16 * i) * g.ldo) = p[k];
                    }
                } else {
                    const uint4 w = pack_pair(x, pack_f16);
                    if (in) *reinterpret_cast<uint4 *>(o + (int64_t)(16 * i) * g.ldo) = w;
                }
            }
        }
        if constexpr (!F32 && !RARE) {
            if (g.row_top) {
                float *red = reinterpret_cast<float *>(smem);      // [WGN][BM]
#pragma unroll
                for (int i = 0; i < SM; ++i) {
                    top[i] = fmaxf(top[i], __shfl_xor(top[i], 16));
                    top[i] = fmaxf(top[i], __shfl_xor(top[i], 32));
                    if (lg == 0) red[(wave % WGN) * BM + wm0 + 16 * i + lr] = top[i];
                }
                __syncthreads();
                for (int r = threadIdx.x; r < left_i; r += kPPThreads) {
                    float t = red[r];
#pragma unroll
                    for (int w = 1; w < WGN; ++w) t = fmaxf(t, red[w * BM + r]);
                    g.row_top[(int64_t)tile_j * g.ldt + i0 + r] = t;
                }
            }
        }
    } else if constexpr (KIND == kDw && F32) {
#pragma unroll
        for (int i = 0; i < SM; ++i) {
            const int64_t row = i0 + wm0 + 16 * i + lr;
#pragma unroll
            for (int j = 0; j < SN; ++j) {
                const int64_t col = j0 + wn0 + 16 * j + 4 * lg;
                if (row >= g.I) continue;
                float *o = static_cast<float *>(g.out) + row * g.ldo + col;
                if (col + 4 <= g.J) {
                    __builtin_memcpy(o, &acc[i][j], 16);
                } else {
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        if (col + v < g.J) o[v] = acc[i][j][v];
                }
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
                const int64_t own = row < g.I ? row : 0;
                const int down = RARE ? g.rare_exp[own] : 0;
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = ldexpf(acc[i][2 * jp + (e >> 2)][e & 3], back[e] - down);
                const uint4 w = pack_pair(x, pack_bf16);
                if (row >= g.I) continue;
                uint16_t *o = static_cast<uint16_t *>(g.out) + (RARE ? g.rare_row[own] : row) * g.ldo + col;
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

// RARE: the grid is smaller than the tiles may be many, and a workgroup takes several.
template <int BM, int BN, int WGM, int WGN, bool TB, Kind KIND, bool F32, bool RARE = false>
__global__ void __launch_bounds__(kPPThreads, 1) loss_pp_kernel(Args g) {
    if (g.count) {
        const int64_t tokens = *g.count;
        if (KIND == kStats) g.I = tokens;
        if (KIND == kGrad || KIND == kDx) g.J = tokens;
        if (KIND == kDw) {
            g.K = (tokens + kPPK - 1) / kPPK * kPPK;
            g.rows_b = tokens;
        }
    }
    if constexpr (RARE) g.I = *g.rare;
    const int tiles_i = (int)((g.I + BM - 1) / BM), tiles_j = (int)((g.J + BN - 1) / BN), items = tiles_i * tiles_j * g.splits;
    if constexpr (RARE) {
        for (int block = blockIdx.x; block < items; block += gridDim.x)
            loss_tile<BM, BN, WGM, WGN, TB, KIND, F32, RARE>(g, block, tiles_i, tiles_j);
    } else if ((int)blockIdx.x < items) {
        loss_tile<BM, BN, WGM, WGN, TB, KIND, F32, RARE>(g, blockIdx.x, tiles_i, tiles_j);
    }
}

// The tokens that count, in order: their places idx, their targets and how many; the others'
// loss and lse are zero (forward).  One workgroup, eight tokens a thread at a time (16384 tokens
// 20 us; a run of tokens a thread, read twice, took 39).
__global__ void __launch_bounds__(1024) compact_kernel(LossEpi e, int64_t M, int *idx, int64_t *targets, int *count,
                                                       float *loss, float *lse) {
    __shared__ int sums[2][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int total = 0, parity = 0;
    for (int64_t base = 0; base < M; base += 8192, parity ^= 1) {
        const int64_t m0 = base + 8 * tid;
        int64_t t[8];
        uint32_t in = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = m0 + k < M ? e.targets[m0 + k] : -1;
#pragma unroll
        for (int k = 0; k < 8; ++k) in |= loss_counts(e, t[k]) ? 1u << k : 0u;
        const int n = __popc(in);
        int before = n;
#pragma unroll
        for (int w = 1; w < 64; w <<= 1) {
            const int up = __shfl_up(before, w);
            if (lane >= w) before += up;
        }
        if (lane == 63) sums[parity][wave] = before;
        __syncthreads();
        before += total - n;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            const int c = sums[parity][w];
            before += w < wave ? c : 0;
            total += c;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (in >> k & 1u) {
                idx[before] = (int)(m0 + k);
                targets[before++] = t[k];
            } else if (loss && m0 + k < M) {
                loss[m0 + k] = 0.f;
                lse[m0 + k] = 0.f;
            }
        }
    }
    if (tid == 0) *count = total;
}

// Row and first column of octet i of rows of np columns.
__device__ __forceinline__ void octet_at(int64_t i, int64_t total, int np, int64_t &r, int &c) {
    const uint32_t per = (uint32_t)np / 8;
    r = total >> 32 ? i / per : (int64_t)((uint32_t)i / per);   // the 64-bit division takes longer than the copy
    c = (int)(i - r * per) * 8;
}

// dst[r][c] = src[idx[r]][c] for c < n, else 0, c < np (a multiple of 64).  idx null: row r;
// count null: all rows.
__global__ void __launch_bounds__(256) gather_kernel(const uint16_t *src, uint16_t *dst, int64_t rows, int n, int np,
                                                     const int *idx, const int *count) {
    if (count) rows = *count;
    const int64_t total = rows * (np / 8);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        int64_t r;
        int c;
        octet_at(i, total, np, r, c);
        float v[8];
        load_cols(src + (idx ? idx[r] : r) * n, c, n, v);
        store8(dst + r * np + c, v);
    }
}

// The same of fp32 rows, as three planes.  e's targets, where given, are the rows': those that do not count become
// zero, as dW multiplies them as they are, by a G of zero, which leaves a NaN (with bf16 operands scale_kernel does it).
__global__ void __launch_bounds__(256) gather_split_kernel(const float *src, uint16_t *dst, int64_t plane, int64_t rows, int n,
                                                           int np, const int *idx, const int *count, LossEpi e) {
    if (count) rows = *count;
    const int64_t total = rows * (np / 8);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        int64_t r;
        int c;
        octet_at(i, total, np, r, c);
        float v[8];
        load_cols(src + (idx ? idx[r] : r) * n, c, n, v);
        if (e.targets && !loss_counts(e, e.targets[r]))
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 0.f;
        uint4 p[3];
        split8(v, p);
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4 *>(dst + k * plane + r * np + c) = p[k];
    }
}

// dst[c][r] = src[r][c] of fp32 rows for r < rows, else 0, r < ld, as three planes: 64 x 64 tiles.
__global__ void __launch_bounds__(256) transpose_split_kernel(const float *src, uint16_t *dst, int64_t plane, int64_t rows,
                                                              int n, int64_t ld) {
    __shared__ float t[64][65];
    const int64_t r0 = (int64_t)blockIdx.x * 64;
    const int c0 = blockIdx.y * 64, tid = threadIdx.x;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int r = (tid + 256 * q) / 8, c = (tid + 256 * q) % 8 * 8;
        float v[8] = {};
        if (r0 + r < rows) load_cols(src + (r0 + r) * n, c0 + c, n, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) t[c + e][r] = v[e];
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int c = (tid + 256 * q) / 8, r = (tid + 256 * q) % 8 * 8;
        if (c0 + c >= n) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = t[c][r + e];
        uint4 p[3];
        split8(v, p);
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4 *>(dst + k * plane + (int64_t)(c0 + c) * ld + r0 + r) = p[k];
    }
}

// Rows of tokens that do not count: their gradient is zero.
template <class T>
__global__ void __launch_bounds__(256) zero_rows_kernel(LossEpi e, T *dx, int64_t M, int n) {
    for (int64_t m = blockIdx.x; m < M; m += gridDim.x) {
        if (loss_counts(e, e.targets[m])) continue;
        for (int c = threadIdx.x; c < n; c += 256) dx[m * n + c] = T(0);
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
            load_cols(src + m * ld, c, n, v);
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

// The rows of G, held times 2^15, whose largest value over the tiles of the tokens is under 2^-24: how
// many, which, the exponents that take them to 2^14 .. 2^15, and their rows of W, in any order,
// which the results do not depend on.  *rare starts at zero.
__global__ void __launch_bounds__(256) rare_kernel(const float *row_top, int64_t ldt, int64_t M, const int *count, int bn,
                                                   int64_t rows, const uint16_t *W, int n, int np, int *rare, int *rare_row,
                                                   int *rare_exp, uint16_t *dst) {
    __shared__ float tops[4][64];
    __shared__ int found[64], first, many;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t v = (int64_t)blockIdx.x * 64 + lane;
    if (count) M = *count;
    const int tiles = (int)((M + bn - 1) / bn);
    float top = 0.f;
    if (v < rows)
#pragma unroll 8
        for (int j = wave; j < tiles; j += 4) top = fmaxf(top, row_top[j * ldt + v]);
    tops[wave][lane] = top;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int w = 1; w < 4; ++w) top = fmaxf(top, tops[w][lane]);
        const bool is = top > 0.f && top < 0x1p-9f;
        const uint64_t all = __ballot(is);
        int at = 0;
        if (lane == 0 && all) at = atomicAdd(rare, __popcll(all));
        at = __shfl(at, 0);
        const int place = __popcll(all & (((uint64_t)1 << lane) - 1));
        if (is) {
            found[place] = (int)v;
            rare_row[at + place] = (int)v;
            rare_exp[at + place] = 14 + 127 - (int)(__float_as_uint(top) >> 23);
        }
        if (lane == 0) {
            first = at;
            many = __popcll(all);
        }
    }
    __syncthreads();
    for (int k = wave; k < many; k += 4)
        for (int c = lane * 8; c < np; c += 512) {
            float w[8];
            load_cols(W + (int64_t)found[k] * n, c, n, w);
            store8(dst + (int64_t)(first + k) * np + c, w);
        }
}

// dst[m][c] = src[m][c] scale[m] in fp16 at the column's scale, rows of np columns.
__global__ void __launch_bounds__(256) scale_kernel(const uint16_t *src, const float *scale, const uint32_t *top,
                                                    uint16_t *dst, int64_t rows, int np, const int *count) {
    if (count) rows = *count;
    const int64_t total = rows * (np / 8);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        int64_t m;
        int c;
        octet_at(i, total, np, m, c);
        float v[8];
        load8(src + m * np + c, v);
        const float s = scale[m];
        uint32_t w[4], b[8];
        __builtin_memcpy(b, __builtin_assume_aligned(top + c, 16), 32);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = s != 0.f ? ldexpf(v[e] * s, column_exp(b[e])) : 0.f;
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

// dX[idx[m]][c] = the fp32 sums acc[split][c][m] added in order, in bf16 times scale[m] at the
// column's scale: 64 x 64 tiles.
template <class T>
__global__ void __launch_bounds__(256) round_transpose_kernel(const float *acc, int splits, const float *scale,
                                                              const uint32_t *top, T *dst, int64_t M, int n,
                                                              int64_t ld, const int *idx, const int *count) {
    constexpr bool kBf16 = sizeof(T) == 2;
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
        const int back = kBf16 && c0 + c < n ? -(column_exp(top[c0 + c]) + kGExp) : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[m + e][c] = ldexpf(v[e], back);
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int m = (tid + 256 * q) / 8, c = (tid + 256 * q) % 8 * 8;
        if (m0 + m >= M) continue;
        const float own = scale[m0 + m], by = kBf16 || own == 0.f ? own : 1.f;   // fp32 sums hold it already
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = by != 0.f ? t[m][c + e] * by : 0.f;
        store_cols<true>(dst + (idx ? idx[m0 + m] : m0 + m) * n, c0 + c, n, v);
    }
}

// The tokens' part of the gradient, and zeros to start the columns' largest magnitudes from.
__global__ void __launch_bounds__(256) token_kernel(LossEpi e, Token t, int64_t M, int64_t padded, const int *idx,
                                                    const int *count, float lse_by, uint32_t *top, int64_t tops) {
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
    t.lse[c] = lse * lse_by;
    t.target[c] = target;
}

// Tiles: rows of side A and B, workgroups to a CU, the time of a round of them on all 256 CUs next
// to 256 x 256's (measured at 4096 wide: 800, 903, 1129 and 1386 us for the same logits), and
// that of a tile where they are few, when clocks are higher and less is shared.
struct Tile {
    int bm, bn, per_cu;
    double round, alone;
};
constexpr Tile kTiles[] = {{256, 256, 1, 1.0, 0.77}, {192, 256, 1, 0.79, 0.74}, {128, 128, 2, 0.694, 0.33}, {64, 128, 3, 0.66, 0.2}};

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
        for (int w = 1; w <= k.per_cu; ++w) {
            int64_t splits = 256 * w / tiles;
            splits = splits > most_splits ? most_splits : splits < 1 ? 1 : splits;
            const int64_t count = tiles * splits, round = 256 * k.per_cu;
            const double rest = k.round * (double)(count % round) / (double)round;
            const double last = count % round == 0 ? 0.0 : rest > k.alone ? rest : k.alone;
            const double time = (k.round * (double)(count / round) + last) / (double)splits;
            if (least == 0 || time < least) {
                best = {t, (int)splits};
                least = time;
            }
        }
    }
    return best;
}

template <int BM, int BN, int WGM, int WGN, bool TB, Kind KIND, bool F32>
hipError_t launch_tile(Args &g, hipStream_t s) {
    const int64_t tiles = ((g.I + BM - 1) / BM) * ((g.J + BN - 1) / BN) * g.splits;
    if (tiles >= (int64_t)1 << 31) return hipErrorNotSupported;
    g.group = 4;   // of 1 to 32, at 768, 1000 and 4096 wide: 8 took G of 768 columns 368 us, 4 326
    loss_pp_kernel<BM, BN, WGM, WGN, TB, KIND, F32><<<(unsigned)tiles, kPPThreads, 0, s>>>(g);
    return hipGetLastError();
}

template <bool TB, Kind KIND, bool F32>
hipError_t launch_as(Args &g, const Choice &c, hipStream_t s) {
    switch (c.tile) {
    case 0: return launch_tile<256, 256, 2, 4, TB, KIND, F32>(g, s);
    case 1: return launch_tile<192, 256, 2, 4, TB, KIND, F32>(g, s);
    case 2: return launch_tile<128, 128, 2, 4, TB, KIND, F32>(g, s);
    default: return launch_tile<64, 128, 2, 4, TB, KIND, F32>(g, s);
    }
}

template <bool TB, Kind KIND>
hipError_t launch(Args g, const Choice &c, bool f32, hipStream_t s) {
    g.splits = c.splits;
    return f32 ? launch_as<TB, KIND, true>(g, c, s) : launch_as<TB, KIND, false>(g, c, s);
}

// The rare rows' products, of at most `rows`: two workgroups a CU of tiles that two share, as many
// rounds as the rows then are.
template <bool TB, Kind KIND>
hipError_t launch_rare(Args g, int64_t rows, hipStream_t s) {
    const int64_t tiles = ((rows + 127) / 128) * ((g.J + 127) / 128);
    if (tiles >= (int64_t)1 << 31) return hipErrorNotSupported;
    g.group = 4;
    g.splits = 1;
    loss_pp_kernel<128, 128, 2, 4, TB, KIND, false, true><<<(unsigned)(tiles < 512 ? tiles : 512), kPPThreads, 0, s>>>(g);
    return hipGetLastError();
}

// Below this the launches that gather would take longer than what they save.
constexpr int64_t kCompactFrom = 257;

// Where things lie in the workspace; a size of 0 for what a call does not need.
struct Space {
    size_t total = 0;
    size_t take(size_t bytes) {
        const size_t at = total;
        total += (bytes + 255) / 256 * 256;
        return at;
    }
};

// The tokens that count and the operands as the kernels read them, W a piece at a time; in fp32
// three planes each.
struct Operands {
    int64_t np;                  // columns
    bool compact, f32;
    size_t idx, targets, count, x, w;
};
bool lays_out_w(int64_t n, bool f32) { return f32 || n % kPPK != 0; }
Operands operands_of(Space &space, int64_t M, int64_t n, int64_t piece, bool f32) {
    Operands o;
    o.np = up(n, kPPK);
    o.compact = M >= kCompactFrom;
    o.f32 = f32;
    o.idx = space.take(o.compact ? (size_t)M * 4 : 0);
    o.targets = space.take(o.compact ? (size_t)M * 8 : 0);
    o.count = space.take(o.compact ? 4 : 0);
    o.x = space.take(f32 ? (size_t)(M * o.np) * 6 : o.compact || o.np != n ? (size_t)(M * o.np) * 2 : 0);
    o.w = space.take(lays_out_w(n, f32) ? (size_t)(piece * o.np) * (f32 ? 6 : 2) : 0);
    return o;
}

// What the launches take of them.
struct Prepared {
    const uint16_t *X;
    const int *idx, *count;
    const int64_t *targets;
};
hipError_t gather(const void *src, uint16_t *dst, int64_t rows, int64_t n, int64_t np, bool f32, const int *idx,
                  const int *count, const LossEpi &e, hipStream_t s) {
    const int64_t blocks = (rows * (np / 8) + 255) / 256;
    const unsigned grid = (unsigned)(blocks < 16384 ? blocks : 16384);
    if (f32)
        gather_split_kernel<<<grid, 256, 0, s>>>(static_cast<const float *>(src), dst, rows * np, rows, (int)n, (int)np, idx, count, e);
    else
        gather_kernel<<<grid, 256, 0, s>>>(static_cast<const uint16_t *>(src), dst, rows, (int)n, (int)np, idx, count);
    return hipGetLastError();
}
hipError_t prepare(const Operands &o, const LossPass &p, const LossEpi &e, char *ws, float *loss, float *lse, Prepared &r,
                   hipStream_t s) {
    r = {static_cast<const uint16_t *>(p.X), nullptr, nullptr, e.targets};
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
    if (err == hipSuccess && (o.compact || o.np != p.n || o.f32)) {
        uint16_t *x = reinterpret_cast<uint16_t *>(ws + o.x);
        err = gather(p.X, x, p.M, p.n, o.np, o.f32, r.idx, r.count, o.compact ? LossEpi{} : e, s);
        r.X = x;
    }
    return err;
}
// Rows v0 .. v0 + vn - 1 of W.
hipError_t prepare_w(const Operands &o, const LossPass &p, int64_t v0, int64_t vn, char *ws, const uint16_t *&W, hipStream_t s) {
    const char *rows = static_cast<const char *>(p.W) + v0 * p.n * (o.f32 ? 4 : 2);
    W = reinterpret_cast<const uint16_t *>(rows);
    if (!lays_out_w(p.n, o.f32)) return hipSuccess;
    uint16_t *w = reinterpret_cast<uint16_t *>(ws + o.w);
    W = w;
    return gather(rows, w, vn, p.n, o.np, o.f32, nullptr, nullptr, LossEpi{}, s);
}

// The vocabulary in pieces of one size, whole tiles, of at most `most` columns or 2048 (which of
// very long rows are more than the bytes that `most` is from).
int64_t piece_of(int64_t V, int64_t most) {
    most = most / 256 * 256;
    if (most < 2048) most = 2048;
    const int64_t pieces = (V + most - 1) / most;
    return up((V + pieces - 1) / pieces, 256);
}
// What a piece of G may take, and one of W laid out otherwise; of W as many columns all the same as
// give each of 256 CUs a tile (129 tokens of 4096 over 50000 in fp32: forward 1532 us in three
// pieces, 798 in one; the step 5005 in five).
constexpr int64_t kGradBytes = (int64_t)512 << 20, kWeightBytes = (int64_t)768 << 20;
int64_t weight_columns(int64_t M, int64_t n, bool f32) {
    const int64_t by_bytes = kWeightBytes / ((f32 ? 6 : 2) * up(n, kPPK)), by_tiles = up(65536 / ((M + 255) / 256), 256);
    return by_bytes > by_tiles ? by_bytes : by_tiles;
}
int64_t forward_piece(int64_t M, int64_t n, int64_t V, bool f32) {
    return lays_out_w(n, f32) ? piece_of(V, weight_columns(M, n, f32)) : V;
}
// The tile that every piece of a forward pass takes.
Choice forward_tile(int64_t M, int64_t n, int64_t V, bool f32) {
    const int64_t piece = forward_piece(M, n, V, f32);
    return choose(M, piece < V ? piece : V);
}

// dX's reduction units in one accumulator at most (split fp32: 16384 vocabulary columns; bf16: 98304).  Each unit is two
// additions, and each may lose half of the last bit of a sum that a target's term has made as large as the whole
// gradient: 1e-4 of it at worst.  (fp32, 43520 columns of small terms of one sign: 1.2e-5 of dX, in one sum 3.6e-5.)
constexpr int64_t kMostUnits = 1536;

// Vocabulary columns of a piece, and the workspace of a backward pass.
struct Layout {
    Operands ops;
    int64_t Mp, Mq, nq, vp;
    Choice dx;
    size_t tokens, tops, xs, wt, gt, row_top, rare_row, rare_exp, acc, total;
    int64_t pieces;
};
Layout layout_of(int64_t M, int64_t n, int64_t V, bool f32) {
    Layout l;
    Space space;
    const size_t value = f32 ? 6 : 2;    // bytes
    l.Mp = up(M, kPPK);
    l.Mq = up(M, 256) + 256;     // the last tile's tokens, whatever its width
    l.nq = up(n, 256) + 256;
    const int64_t np = up(n, kPPK), most = kGradBytes / ((int64_t)value * l.Mp), columns = weight_columns(M, n, f32);
    l.vp = piece_of(V, most < columns ? most : columns);
    // at least 16 units a split, and the splits' sums within 256 MB
    int64_t splits = l.vp / kPPK * (f32 ? kProducts : 1) / 16;
    const int64_t room = ((int64_t)64 << 20) / (n * l.Mp);
    splits = splits < room ? splits : room;
    l.dx = choose(n, M, splits < 1 ? 1 : splits);
    const int64_t longest = l.dx.splits * kMostUnits / (f32 ? kProducts : 1) * kPPK;
    if (l.vp > longest) l.vp = piece_of(V, longest);
    l.ops = operands_of(space, M, n, 0, f32);
    l.tokens = space.take((size_t)l.Mq * 12);
    l.pieces = (V + l.vp - 1) / l.vp;
    l.tops = space.take(f32 ? 0 : (size_t)(2 * l.nq + l.pieces) * 4);   // and a piece's number of rare rows
    l.xs = space.take(f32 ? 0 : (size_t)(M * l.ops.np) * 2);
    // W of a piece for its logits, then W^T of it, then its rare rows
    l.wt = l.ops.w = space.take((size_t)(np * l.vp) * value);
    l.gt = space.take((size_t)(l.vp * l.Mp) * value);
    l.row_top = space.take(f32 ? 0 : (size_t)(up(M, 128) / 128 * l.vp) * 4);
    l.rare_row = space.take(f32 ? 0 : (size_t)l.vp * 4);
    l.rare_exp = space.take(f32 ? 0 : (size_t)l.vp * 4);
    l.acc = space.take((size_t)(l.dx.splits * n * l.Mp) * 4);
    l.total = space.total;
    return l;
}

}  // namespace

int loss_mfma_tiles(int64_t M, int64_t n, int64_t V, bool f32) {
    const int bn = kTiles[forward_tile(M, n, V, f32).tile].bn;
    return (int)((V + bn - 1) / bn);
}

size_t loss_mfma_forward_bytes(int64_t M, int64_t n, int64_t V, bool f32) {
    Space space;
    operands_of(space, M, n, forward_piece(M, n, V, f32), f32);
    return space.total;
}

size_t loss_mfma_backward_bytes(int64_t M, int64_t n, int64_t V, bool f32) { return layout_of(M, n, V, f32).total; }

hipError_t launch_loss_mfma_stats(const LossPass &p, const LossEpi &e, void *ws, float *each, LossTokens &tokens,
                                  hipStream_t s) {
    Space space;
    const bool f32 = p.dtype == kF32;
    const int64_t piece = forward_piece(p.M, p.n, p.V, f32);
    const Operands o = operands_of(space, p.M, p.n, piece, f32);
    const Choice tile = forward_tile(p.M, p.n, p.V, f32);
    Prepared r;
    hipError_t err = prepare(o, p, e, static_cast<char *>(ws), each, p.lse, r, s);
    if (err != hipSuccess) return err;
    tokens = {r.idx, r.count};
    Args g{};
    g.e = e;
    g.e.targets = r.targets;
    g.count = r.count;
    g.A = r.X;
    g.plane_a = p.M * o.np;
    g.I = p.M;
    g.K = g.lda = g.ldb = o.np;
    for (int64_t v0 = 0; v0 < p.V && err == hipSuccess; v0 += piece) {
        g.v0 = v0;
        g.J = p.V - v0 < piece ? p.V - v0 : piece;
        g.plane_b = g.J * o.np;
        err = prepare_w(o, p, v0, g.J, static_cast<char *>(ws), g.B, s);
        if (err == hipSuccess) err = launch<false, kStats>(g, tile, f32, s);
    }
    return err;
}

hipError_t launch_loss_mfma_grad(const LossPass &p, const LossEpi &e, hipStream_t s) {
    const bool f32 = p.dtype == kF32;
    const Layout l = layout_of(p.M, p.n, p.V, f32);
    char *ws = static_cast<char *>(p.ws);
    const auto at = [&](size_t o) { return reinterpret_cast<uint16_t *>(ws + o); };
    Prepared r;
    hipError_t err = prepare(l.ops, p, e, ws, nullptr, nullptr, r, s);
    if (err != hipSuccess) return err;
    Token tok;
    tok.scale = reinterpret_cast<float *>(ws + l.tokens);
    tok.lse = tok.scale + l.Mq;
    tok.target = reinterpret_cast<int *>(tok.lse + l.Mq);
    uint32_t *const x_top = reinterpret_cast<uint32_t *>(ws + l.tops), *const w_top = x_top + l.nq;
    token_kernel<<<(unsigned)(l.Mq / 256), 256, 0, s>>>(e, tok, p.M, l.Mq, r.idx, r.count, f32 ? 1.f : kLog2e, x_top,
                                                        f32 ? 0 : 2 * l.nq + l.pieces);
    err = hipGetLastError();
    const int np = (int)l.ops.np, n = (int)p.n;
    const auto top_grid = [&](int64_t rows) {
        const int64_t blocks = (rows + 63) / 64;
        return dim3((unsigned)(blocks < 1024 ? blocks : 1024), (unsigned)((n + 255) / 256));
    };
    const int64_t plane_x = p.M * l.ops.np, plane_wt = p.n * l.vp, plane_gt = l.vp * l.Mp;
    if (err == hipSuccess && p.dW && !f32) {
        const int64_t blocks = (p.M * (np / 8) + 255) / 256;
        column_top_kernel<<<top_grid(p.M), 256, 0, s>>>(r.X, tok.scale, p.M, n, np, r.count, x_top);
        scale_kernel<<<(unsigned)(blocks < 16384 ? blocks : 16384), 256, 0, s>>>(r.X, tok.scale, x_top, at(l.xs), p.M, np,
                                                                                 r.count);
        err = hipGetLastError();
    }
    if (err == hipSuccess && p.dX) {
        const unsigned rows = (unsigned)(p.M < 8192 ? p.M : 8192);
        if (!f32)
            column_top_kernel<<<top_grid(p.V), 256, 0, s>>>(static_cast<const uint16_t *>(p.W), nullptr, p.V, n, n, nullptr, w_top);
        if (r.count && f32) zero_rows_kernel<<<rows, 256, 0, s>>>(e, static_cast<float *>(p.dX), p.M, n);
        if (r.count && !f32) zero_rows_kernel<<<rows, 256, 0, s>>>(e, static_cast<uint16_t *>(p.dX), p.M, n);
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
        err = prepare_w(l.ops, p, v0, vn, ws, g.A, s);
        if (err != hipSuccess) break;
        g.B = r.X;
        g.plane_a = vn * l.ops.np;
        g.plane_b = plane_x;
        g.lda = g.ldb = g.K = l.ops.np;
        g.I = vn;
        g.J = p.M;
        g.out = at(l.gt);
        g.plane_out = plane_gt;
        g.ldo = l.Mp;
        const Choice tile = choose(g.I, g.J);
        if (p.dW && !f32) {
            g.row_top = reinterpret_cast<float *>(ws + l.row_top);
            g.ldt = l.vp;
        }
        Args grad = g;
        err = launch<false, kGrad>(g, tile, f32, s);
        if (err == hipSuccess && p.dW) {
            g.A = at(l.gt);
            g.plane_a = plane_gt;
            g.lda = g.K = l.Mp;
            if (!f32) g.B = at(l.xs);
            g.rows_b = p.M;
            g.J = g.ldo = p.n;
            g.col_top = x_top;
            g.out = static_cast<char *>(p.dW) + v0 * p.n * (f32 ? 4 : 2);
            err = launch<true, kDw>(g, choose(g.I, g.J), f32, s);
        }
        Args dw = g;
        if (err == hipSuccess && p.dX) {
            const dim3 grid((unsigned)((vn + 63) / 64), (unsigned)(np / 64));
            if (f32)
                transpose_split_kernel<<<grid, 256, 0, s>>>(static_cast<const float *>(p.W) + v0 * n, at(l.wt), plane_wt, vn, n, l.vp);
            else
                transpose_kernel<<<grid, 256, 0, s>>>(static_cast<const uint16_t *>(p.W) + v0 * n, w_top, at(l.wt), vn, n, l.vp);
            err = hipGetLastError();
        }
        if (err == hipSuccess && p.dX) {
            g.A = at(l.wt);
            g.plane_a = plane_wt;
            g.lda = l.vp;
            g.B = at(l.gt);
            g.plane_b = plane_gt;
            g.ldb = g.ldo = l.Mp;
            g.I = p.n;
            g.J = p.M;
            g.K = up(vn, kPPK);
            g.rows_b = vn;
            g.acc = acc;
            g.first = v0 == 0;
            err = launch<true, kDx>(g, l.dx, f32, s);
        }
        if (err == hipSuccess && p.dW && !f32) {
            int *rare = reinterpret_cast<int *>(w_top + l.nq) + v0 / l.vp, *rare_row = reinterpret_cast<int *>(ws + l.rare_row),
                *rare_exp = reinterpret_cast<int *>(ws + l.rare_exp);
            rare_kernel<<<(unsigned)((vn + 63) / 64), 256, 0, s>>>(grad.row_top, l.vp, p.M, r.count, kTiles[tile.tile].bn, vn,
                                                                  static_cast<const uint16_t *>(p.W) + v0 * n, n, np, rare,
                                                                  rare_row, rare_exp, at(l.wt));
            err = hipGetLastError();
            for (Args *again : {&grad, &dw}) {
                again->rare = rare;
                again->rare_row = rare_row;
                again->rare_exp = rare_exp;
            }
            grad.A = at(l.wt);
            if (err == hipSuccess) err = launch_rare<false, kGrad>(grad, vn, s);
            if (err == hipSuccess) err = launch_rare<true, kDw>(dw, vn, s);
        }
    }
    if (err == hipSuccess && p.dX) {
        const dim3 grid((unsigned)(l.Mp / 64), (unsigned)(np / 64));
        if (f32)
            round_transpose_kernel<<<grid, 256, 0, s>>>(acc, l.dx.splits, tok.scale, w_top, static_cast<float *>(p.dX), p.M, n,
                                                        l.Mp, r.idx, r.count);
        else
            round_transpose_kernel<<<grid, 256, 0, s>>>(acc, l.dx.splits, tok.scale, w_top, static_cast<uint16_t *>(p.dX), p.M,
                                                        n, l.Mp, r.idx, r.count);
        err = hipGetLastError();
    }
    return err;
}

}  // namespace dyad
