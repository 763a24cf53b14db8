// The fp4 product on large tiles under an output transpose, bf16, shapes that
// keep component 1's rows by residue (mx4_by_residue).
//
// A workgroup makes 16 * SM tokens x RG residues of 16 * SN * SUB outputs each, SUB waves
// to a residue.  Component 1's block of the input serves every wave and goes through
// a shared LDS ring, loaded ahead; in component 2 each wave reads a block of its
// own, through a private pair of slots that needs no barrier (the wave's own
// wait says when its loads have arrived, and it loads a slot again once it has
// read it).  Weights and scale words go to registers, two sets by turns.  The
// alternative, one workgroup of all residues loading fragments straight to
// registers (mx4_gemm_res_kernel), repeats component 1's input in every wave.
//
// Outputs leave through LDS: a token's columns (or, with RG < D, runs of RG) in a row.
#include "mx4_gemm.h"
#include "mx4_lds.h"

namespace dyad {

namespace {

template <int SM, int SN, int RG, int SUB>
struct Mx4ResTile {
    static constexpr int kWaves = RG * SUB;
    static constexpr int kSlot = SM * 1024;
    // two workgroups to a CU where their rings fit twice
    static constexpr int kSlots =
        kWaves * 2 * kSlot + 2 * kSlot <= 80 * 1024 && kWaves * 2 * kSlot + 3 * kSlot > 80 * 1024 ? 2 : 3;
    static constexpr int kPrivate = kSlots * kSlot;                        // first private slot
    static constexpr int kRings = kPrivate + kWaves * 2 * kSlot;
    static constexpr int kRun = RG * 2;                                    // bytes of a column j's residues
    static constexpr int kPitch = 16 * SN * SUB * kRun + 16;
    static constexpr int kLds = kRings > 16 * SM * kPitch ? kRings : 16 * SM * kPitch;
    static constexpr int kGroups = 2 * kLds <= 160 * 1024 ? 2 : 1;         // workgroups to a CU
    static_assert(kLds <= 160 * 1024, "LDS");
};

template <int SM, int SN, int RG, int SUB>
__global__ void __launch_bounds__(64 * RG * SUB, (RG * SUB / 4 * Mx4ResTile<SM, SN, RG, SUB>::kGroups))
mx4_res_tile_kernel(Mx4Args a) {
    using C = Mx4ResTile<SM, SN, RG, SUB>;
    constexpr int W = C::kWaves, GM = SM / 4, GN = (SN + 3) / 4, kPer = SM >= W ? SM / W : 1, kSet = SN + GM + GN;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[C::kLds];
    lds_u8 *lds = (lds_u8 *)smem;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // tiles: the D / RG residue groups of the same columns next to each other, then
    // group_m token panels, then the columns
    const int item = xcd_tile(blockIdx.x, a.tiles), D = a.D, halves = D / RG;
    const int pair = item / halves, cols_n = a.tiles_n / halves;
    const int run = a.group_m * cols_n, first = pair / run * a.group_m;
    const int gm = a.tiles_m - first < a.group_m ? a.tiles_m - first : a.group_m;
    const int t0 = (first + pair % run % gm) * SM;
    const int tn = pair % run / gm, g0 = item % halves * RG, gw = wave % RG, g = g0 + gw;
    const int per = a.bo / (16 * D), jf0 = tn * SN * SUB, i1 = jf0 / per, jf = jf0 + SN * (wave / RG);
    const int steps = a.steps, total = 2 * steps;

    // fragments past the tokens read as zeros; a block's SN fragments all exist
    const uint32_t xn = (uint32_t)(a.x_frags - t0 < SM ? a.x_frags - t0 : SM);
    auto x_rsrc = [&](int part) {
        return buffer_rsrc(a.xc + ((int64_t)part * a.x_frags + t0) * steps * 1024, xn * (uint32_t)steps * 1024u);
    };
    auto xs_rsrc = [&](int part) {
        return buffer_rsrc(a.xs + ((int64_t)part * a.x_groups + t0 / 4) * steps * 256, (xn + 3) / 4 * (uint32_t)steps * 256u);
    };
    auto w_rsrc = [&](int part, int frag) {
        return buffer_rsrc(a.wc + ((int64_t)part * a.w_frags + frag) * steps * 1024, (uint32_t)SN * (uint32_t)steps * 1024u);
    };
    auto ws_rsrc = [&](int part, int frag) {
        return buffer_rsrc(a.ws + ((int64_t)part * a.w_groups + frag / 4) * steps * 256, (uint32_t)GN * (uint32_t)steps * 256u);
    };
    const int wf1 = g * per + jf - i1 * per, x2 = a.in_t ? D + g : g;
    const __amdgpu_buffer_rsrc_t rX1 = x_rsrc(i1), rX2 = x_rsrc(x2), sX1 = xs_rsrc(i1), sX2 = xs_rsrc(x2);
    const __amdgpu_buffer_rsrc_t rW1 = w_rsrc(i1, wf1), rW2 = w_rsrc(D + g, jf), sW1 = ws_rsrc(i1, wf1), sW2 = ws_rsrc(D + g, jf);

    const uint32_t row = (uint32_t)steps * 1024u, srow = (uint32_t)steps * 256u, l16 = 16u * lane, l4 = 4u * lane;
    // component 1's step s into ring slot `slot`: wave w takes fragments w, w + W ..
    auto issue1 = [&](int s, int slot) {
        s = s < steps ? s : steps - 1;
#pragma unroll
        for (int q = 0; q < kPer; ++q)
            if (SM >= W || wave < SM)
                dma16(rX1, lds + slot * C::kSlot + 1024 * (wave + W * q), (uint32_t)(wave + W * q) * row + l16, (uint32_t)s * 1024u);
    };
    // component 2's step s into the wave's slot s % 2
    auto issue2 = [&](int s) {
        const int t = s < steps ? s : steps - 1;
#pragma unroll
        for (int i = 0; i < SM; ++i)
            dma16(rX2, lds + C::kPrivate + (2 * wave + (s & 1)) * C::kSlot + 1024 * i, (uint32_t)i * row + l16, (uint32_t)t * 1024u);
    };
    struct Set {
        uint4 w[SN];
        uint32_t sw[GN], sx[GM];
    };
    auto fetch = [&](int t, Set &f) {
        t = t < total ? t : total - 1;
        const bool c = t >= steps;
        const uint32_t s = (uint32_t)(c ? t - steps : t);
#pragma unroll
        for (int q = 0; q < GM; ++q)
            f.sx[q] = __builtin_amdgcn_raw_buffer_load_b32(c ? sX2 : sX1, (int)(l4 + (uint32_t)q * srow), (int)(s * 256u), 0);
#pragma unroll
        for (int q = 0; q < GN; ++q)
            f.sw[q] = __builtin_amdgcn_raw_buffer_load_b32(c ? sW2 : sW1, (int)(l4 + (uint32_t)q * srow), (int)(s * 256u), 0);
#pragma unroll
        for (int j = 0; j < SN; ++j) f.w[j] = bload16(c ? rW2 : rW1, (uint32_t)j * row + l16, s * 1024u);
    };
    const uint32_t base = (uint32_t)(uintptr_t)lds + l16;
    f32x4_t acc[SN][SM];
    mx4_zero(acc);
    auto multiply = [&](const Set &f, const uint4 (&x)[SM], int wf) {
        uint32_t sw[GN];
        // fewer than four fragments start anywhere in a word
#pragma unroll
        for (int q = 0; q < GN; ++q) sw[q] = SN < 4 ? f.sw[q] >> (8 * (wf & 3)) : f.sw[q];
        mx4_multiply<0, 0, SN, SM>(f.w, x, sw, f.sx, acc);
        // kept in this step: the compiler would sink them to where their sums are next used
#pragma unroll
        for (int j = 0; j < SN; ++j)
#pragma unroll
            for (int i = 0; i < SM; ++i) asm volatile("" : "+v"(acc[j][i]));
    };

    Set f0, f1;
    issue2(0);
    issue2(1);
#pragma unroll
    for (int s = 0; s + 1 < C::kSlots; ++s) issue1(s, s);
    fetch(0, f0);
    fetch(1, f1);
    int slot = 0;
    // After step s's input come kSlots - 2 later steps' and at least a set of
    // weights and scales; the barrier also says that every wave has read the
    // step before, whose slot is loaded next.
    auto one = [&](int s, Set &f) {
        wait_vm<(C::kSlots - 2) * kPer + kSet>();
        pp_barrier();
        const int next = slot == 0 ? C::kSlots - 1 : slot - 1;
        issue1(s + C::kSlots - 1, next);
        uint4 x[SM];
        mx4_read<SM>(base + (uint32_t)(slot * C::kSlot), x);
        multiply(f, x, wf1);
        fetch(s + 2, f);
        slot = slot == C::kSlots - 1 ? 0 : slot + 1;
    };
    // After step s's input come the next step's and at least a set.
    auto two = [&](int t, Set &f) {
        const int s = t - steps;
        wait_vm<SM + kSet>();
        uint4 x[SM];
        mx4_read<SM>(base + (uint32_t)(C::kPrivate + (2 * wave + (s & 1)) * C::kSlot), x);
        issue2(s + 2);
        multiply(f, x, jf);
        fetch(t + 2, f);
    };
    int t = 0;
    for (; t + 1 < steps; t += 2) {
        one(t, f0);
        one(t + 1, f1);
    }
    if (t < steps) {
        one(t, f0);
        const Set later = f0;
        f0 = f1;
        f1 = later;
        ++t;
    }
    for (; t + 1 < total; t += 2) {
        two(t, f0);
        two(t + 1, f1);
    }
    if (t < total) two(t, f0);
    wait_vm<0>();                                  // no load into LDS outlives the loop
    pp_barrier();

    const int row16 = lane & 15, quad = 4 * (lane >> 4);
    const uint16_t *bias = static_cast<const uint16_t *>(a.bias);
    const int64_t f00 = (int64_t)jf0 * 16 * D + g0;        // the tile's first column
    const int c0 = 16 * (jf - jf0) + quad;
#pragma unroll
    for (int j = 0; j < SN; ++j) {
        float b[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t f = f00 + (int64_t)(c0 + 16 * j + q) * D + gw;
            b[q] = bias && f < a.n_out ? bf16_to_f32(bias[f]) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < SM; ++i) {
            unsigned char *at = smem + (16 * i + row16) * C::kPitch + (c0 + 16 * j) * C::kRun + 2 * gw;
            float x[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = mx4_act<uint16_t>(a, acc[j][i][q] + b[q]);
#pragma unroll
            for (int q = 0; q < 4; q += 2) {
                const uint32_t v = pack_bf16(x[q], x[q + 1]);
                *reinterpret_cast<uint16_t *>(at + q * C::kRun) = (uint16_t)v;
                *reinterpret_cast<uint16_t *>(at + (q + 1) * C::kRun) = (uint16_t)(v >> 16);
            }
        }
    }
    __syncthreads();
    // 16-byte pieces: with RG = 8 a column j's eight residues, else 8 / RG columns of all
    constexpr int kRow = 16 * SN * SUB * C::kRun / 16, kCols = 8 / RG;
    const int64_t m0 = (int64_t)t0 * 16;
    uint16_t *dst = static_cast<uint16_t *>(a.Y) + m0 * a.n_out;
#pragma unroll 4
    for (int q = 0; q < 16 * SM * kRow / (64 * W); ++q) {
        const int p = threadIdx.x + q * 64 * W, r = p / kRow, at = p % kRow;
        const int64_t f = f00 + (int64_t)(at * kCols) * D;
        if (m0 + r < a.M && f + 8 <= a.n_out)
            *reinterpret_cast<uint4 *>(dst + r * a.n_out + f) = *reinterpret_cast<const uint4 *>(smem + r * C::kPitch + 16 * at);
    }
}

}  // namespace

template <int SM, int SN, int RG, int SUB = 1>
static hipError_t launch(Mx4Args a, hipStream_t s) {
    const int64_t tiles_n = a.n_out / (16 * SN * SUB * a.D) * (a.D / RG), tiles_m = (a.x_frags + SM - 1) / SM;
    if (tiles_n * tiles_m >= ((int64_t)1 << 31)) return hipErrorNotSupported;
    a.tiles_n = (int)tiles_n;
    a.tiles_m = (int)tiles_m;
    a.tiles = (int)(tiles_n * tiles_m);
    a.group_m = 8;
    mx4_res_tile_kernel<SM, SN, RG, SUB><<<(unsigned)a.tiles, 64 * RG * SUB, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_mx4_res_tiles(const Mx4Args &a, hipStream_t s) {
    const int D = a.D, per = a.bo / (16 * D);
    // whole rows of outputs in 16-byte pieces, 32-bit offsets inside a tile
    if ((D != 2 && D != 4 && D != 8 && D != 16) || a.n_out != (int64_t)D * a.bo || a.x_frags < 4 || (int64_t)8 * a.steps * 1024 >= ((int64_t)1 << 31))
        return hipErrorNotSupported;
    // short reductions are mostly epilogue, which smaller workgroups overlap better
    // (8192 tokens of 768 -> 3072, n_dyad 4, two steps: 35 us against 31; 2048 -> 8192,
    // n_dyad 8, two steps, 75 against 89)
    if (a.steps < 4 && D == 4) return hipErrorNotSupported;
    const int rg = D == 4 ? 4 : 8, sn = per % 4 == 0 ? 4 : per % 2 == 0 ? 2 : 1;
    auto tiles = [&](int sm, int n) { return (int64_t)(a.n_out / (16 * n * D)) * (D / rg) * ((a.x_frags + sm - 1) / sm); };
    // n_dyad 2: two waves to a residue.  Against the small tiles, 4096 -> 4096, 7561
    // tokens (960 tiles of 16 steps) 106 us against 153; 16384 -> 4096, 1402 tokens
    // (176 of 64) 93 against 150; 1024 -> 4096, 2048 tokens (256 of 4) 22 against 20
    if (D == 2) {
        if (per % 8 != 0 || a.n_out / 256 * ((a.x_frags + 7) / 8) < (a.steps >= 16 ? 128 : 512)) return hipErrorNotSupported;
        return launch<8, 4, 2, 2>(a, s);
    }
    if (rg == 4) {
        // long reductions from half a tile a CU: 16384 -> 4096, 1100 tokens (144 tiles)
        // 59 us against 71; 8192 -> 8192, 512 tokens (128 of 16 steps) 34 and 33
        if (sn == 4 && tiles(8, 4) >= (a.steps >= 16 ? 128 : 512)) return launch<8, 4, 4>(a, s);
        if (sn >= 2 && tiles(8, 2) >= 512) return launch<8, 2, 4>(a, s);
        return hipErrorNotSupported;
    }
    // two workgroups to a CU, one storing while the other multiplies, where the
    // reduction is short: 2048 -> 8192, two steps, 66 us against 76 on the tile of
    // twice the tokens; 4096 -> 16384, four, 210 against 233; 32768 -> 8192, 32, 135
    // against 124
    if (sn == 4 && a.steps <= 4 && tiles(4, 4) >= 512) return launch<4, 4, 8>(a, s);
    if (sn == 4 && tiles(8, 4) >= 256) return launch<8, 4, 8>(a, s);
    if (sn >= 2 && tiles(4, 2) >= 512) return launch<4, 2, 8>(a, s);
    if (tiles(4, 1) >= 256) return launch<4, 1, 8>(a, s);
    return hipErrorNotSupported;
}

}  // namespace dyad
