// The fp4 product on large tiles: four waves side by side multiply 16 * SM
// tokens x 64 * SN columns.
//
// A step is 128 reduction indices; the steps of both components form one
// sequence.  The input's fragments, which all waves read, go through an LDS ring
// that global-to-LDS loads fill two steps ahead (a fragment's kilobyte lies in
// a row in memory and in LDS: no swizzle).  A wave's weights are its own: they
// and the scale words go straight to registers, two sets by turns, so LDS
// carries 40 KB a step instead of 72.  Two workgroups share a CU: the reductions
// are short (16 steps for blocks of 1024), so one multiplies while the other
// fills its ring or stores its outputs.
//
// Whole bf16 tiles leave through LDS as whole rows of the tile, streamed: straight
// from the accumulators, in half lines, the product below took 44 us more.
//
// Measured at 8192 tokens of 4096 -> 16384, n_dyad 4 (550 GFLOP, 340 MB): 170-178 us,
// 3.1 PFLOP/s; 145 of it without the outputs, 100 with an input and weights of
// zeros (the clock gives way to the matrix cores' power).  Eight waves in two
// halves a phase apart, one workgroup to a CU, took 240.
#include "mx4_gemm.h"
#include "mx4_lds.h"

namespace dyad {

namespace {

constexpr int kMx4Threads = 256, kMx4Waves = 4;

template <int SM, int SN, typename T>
__global__ void __launch_bounds__(kMx4Threads, 2) mx4_tile_kernel(Mx4Args a) {
    constexpr int BM = 16 * SM, BN = 64 * SN, GM = (SM + 3) / 4, GN = (SN + 3) / 4;
    constexpr int kSlots = 3, kSlot = SM * 1024, kPer = SM / kMx4Waves;      // ring, wave loads of a step
    constexpr int kPitch = 2 * BN + 16;                                     // bytes of a token's columns on the way out
    constexpr int kLds = kSlots * kSlot > BM * kPitch ? kSlots * kSlot : BM * kPitch;
    static_assert(2 * kLds <= 160 * 1024 && SM % kMx4Waves == 0, "two workgroups to a CU");
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kLds];
    lds_u8 *lds = (lds_u8 *)smem;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // tiles in runs of group_m token panels, panels fastest
    const int item = xcd_tile(blockIdx.x, a.tiles);
    const int tiles_m = a.tiles / a.tiles_n, run = a.group_m * a.tiles_n;
    const int first = item / run * a.group_m;
    const int gm = tiles_m - first < a.group_m ? tiles_m - first : a.group_m;
    const int t0 = (first + item % run % gm) * SM;
    const int tn = item % run / gm, per_block = a.tiles_n / a.D;
    const int g = tn / per_block, c0 = (tn - g * per_block) * (BN / 16);

    const int steps = a.steps, total = 2 * steps;
    auto w_part = [&](int c) { return c ? a.D + g : g; };
    auto x_part = [&](int c) { return c && a.in_t ? a.D + g : g; };
    // a tile's fragments as buffers: those past a part's last read as zeros
    const uint32_t xn = (uint32_t)(a.x_frags - t0 < SM ? a.x_frags - t0 : SM);
    const uint32_t wn = (uint32_t)(a.w_frags - c0 < BN / 16 ? a.w_frags - c0 : BN / 16);
    auto x_rsrc = [&](int c) {
        return buffer_rsrc(a.xc + ((int64_t)x_part(c) * a.x_frags + t0) * steps * 1024, xn * (uint32_t)steps * 1024u);
    };
    auto w_rsrc = [&](int c) {
        return buffer_rsrc(a.wc + ((int64_t)w_part(c) * a.w_frags + c0) * steps * 1024, wn * (uint32_t)steps * 1024u);
    };
    // scale words of a step: fragments in fours
    auto xs_rsrc = [&](int c) {
        return buffer_rsrc(a.xs + ((int64_t)x_part(c) * a.x_groups + t0 / 4) * steps * 256, (xn + 3) / 4 * (uint32_t)steps * 256u);
    };
    auto ws_rsrc = [&](int c) {
        return buffer_rsrc(a.ws + ((int64_t)w_part(c) * a.w_groups + c0 / 4) * steps * 256, (wn + 3) / 4 * (uint32_t)steps * 256u);
    };
    const __amdgpu_buffer_rsrc_t rX1 = x_rsrc(0), rX2 = x_rsrc(1), rW1 = w_rsrc(0), rW2 = w_rsrc(1);
    const __amdgpu_buffer_rsrc_t sX1 = xs_rsrc(0), sX2 = xs_rsrc(1), sW1 = ws_rsrc(0), sW2 = ws_rsrc(1);

    const int wn0 = wave * SN;                                   // the wave's first column fragment
    const uint32_t row = (uint32_t)steps * 1024u, vX = (uint32_t)wave * row + 16u * lane, vW = (uint32_t)wn0 * row + 16u * lane;
    const uint32_t srow = (uint32_t)steps * 256u, vsX = 4u * lane, vsW = (uint32_t)(wn0 / 4) * srow + 4u * lane;
    // steps past the last load the last again: nothing reads them
    auto issue = [&](int t, int slot) {
        t = t < total ? t : total - 1;
        const bool c = t >= steps;
#pragma unroll
        for (int q = 0; q < kPer; ++q)
            dma16(c ? rX2 : rX1, lds + slot * kSlot + 1024 * (wave + kMx4Waves * q), vX + (uint32_t)(kMx4Waves * q) * row,
                  (uint32_t)(c ? t - steps : t) * 1024u);
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
            f.sx[q] = __builtin_amdgcn_raw_buffer_load_b32(c ? sX2 : sX1, (int)(vsX + (uint32_t)q * srow), (int)(s * 256u), 0);
#pragma unroll
        for (int q = 0; q < GN; ++q)
            f.sw[q] = __builtin_amdgcn_raw_buffer_load_b32(c ? sW2 : sW1, (int)(vsW + (uint32_t)q * srow), (int)(s * 256u), 0);
#pragma unroll
        for (int j = 0; j < SN; ++j) f.w[j] = bload16(c ? rW2 : rW1, vW + (uint32_t)j * row, s * 1024u);
    };
    const uint32_t base = (uint32_t)(uintptr_t)lds + 16u * lane;

    f32x4_t acc[SN][SM];
    mx4_zero(acc);
    Set f0, f1;
    issue(0, 0);
    issue(1, 1);
    fetch(0, f0);
    fetch(1, f1);
    int slot = 0;
    // After step t's input come a later step's (kPer loads) and at least two sets
    // of weights and scales but one; the barrier also says that every wave has
    // read step t - 1, whose slot step t + 2 takes.
    constexpr int kSet = SN + GM + GN;
    auto step = [&](int t, Set &f) {
        wait_vm<kPer + kSet>();
        pp_barrier();
        issue(t + 2, slot == 0 ? 2 : slot - 1);
        uint4 x[SM];
        mx4_read<SM>(base + (uint32_t)(slot * kSlot), x);
        uint32_t sw[GN];
#pragma unroll
        for (int q = 0; q < GN; ++q) sw[q] = SN < 4 ? f.sw[q] >> (8 * (wn0 & 3)) : f.sw[q];
        mx4_multiply<0, 0, SN, SM>(f.w, x, sw, f.sx, acc);
        // kept in this step: the compiler would sink them to where their sums are next used
#pragma unroll
        for (int j = 0; j < SN; ++j)
#pragma unroll
            for (int i = 0; i < SM; ++i) asm volatile("" : "+v"(acc[j][i]));
        fetch(t + 2, f);
        slot = slot == 2 ? 0 : slot + 1;
    };
    for (int t = 0; t < total; t += 2) {
        step(t, f0);
        step(t + 1, f1);
    }
    wait_vm<0>();                                  // no load into LDS outlives the loop
    const int64_t col = (int64_t)g * a.bo + c0 * 16, end = (int64_t)(g + 1) * a.bo < a.n_out ? (int64_t)(g + 1) * a.bo : a.n_out;
    if constexpr (sizeof(T) == 2) {
        // whole tiles in bf16 leave through LDS, a token's columns in a row
        if (col + BN <= end && a.n_out % 8 == 0 && a.bo % 8 == 0) {
            pp_barrier();
            const uint16_t *bias = static_cast<const uint16_t *>(a.bias);
            const int quad = 4 * (lane >> 4);
#pragma unroll
            for (int j = 0; j < SN; ++j) {
                const int c = (wn0 + j) * 16 + quad;
                float b[4];
#pragma unroll
                for (int v = 0; v < 4; ++v) b[v] = bias ? bf16_to_f32(bias[col + c + v]) : 0.f;
#pragma unroll
                for (int i = 0; i < SM; ++i) {
                    float x[4];
#pragma unroll
                    for (int v = 0; v < 4; ++v) x[v] = mx4_act<T>(a, acc[j][i][v] + b[v]);
                    *reinterpret_cast<uint2 *>(smem + (i * 16 + (lane & 15)) * kPitch + 2 * c) =
                        make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
                }
            }
            __syncthreads();
            const int64_t m0 = (int64_t)t0 * 16;
            const __amdgpu_buffer_rsrc_t out = buffer_rsrc(static_cast<uint16_t *>(a.Y) + m0 * a.n_out + col,
                                                           (uint32_t)((a.M - m0 < BM ? a.M - m0 : BM) * a.n_out * 2));
            constexpr int kRow = BN / 8;             // pieces of 16 bytes
#pragma unroll
            for (int q = 0; q < BM * kRow / kMx4Threads; ++q) {
                const int p = threadIdx.x + q * kMx4Threads, r = p / kRow, at = p % kRow * 16;
                bstore16(out, (uint32_t)r * (uint32_t)a.n_out * 2u + (uint32_t)at,
                         *reinterpret_cast<const uint4 *>(smem + r * kPitch + at));
            }
            return;
        }
    }
    mx4_epilogue<SN, SM, T>(a, g, c0 + wn0, t0, lane, acc);
}

}  // namespace

template <int SM, int SN>
static hipError_t launch(Mx4Args a, bool bf16, hipStream_t s) {
    const int64_t tiles_n = (int64_t)a.D * ((a.w_frags + 4 * SN - 1) / (4 * SN)), tiles_m = (a.x_frags + SM - 1) / SM;
    if (tiles_n * tiles_m >= ((int64_t)1 << 31)) return hipErrorNotSupported;
    a.tiles_n = (int)tiles_n;
    a.tiles = (int)(tiles_n * tiles_m);
    a.group_m = 8;
    if (bf16) mx4_tile_kernel<SM, SN, uint16_t><<<(unsigned)a.tiles, kMx4Threads, 0, s>>>(a);
    else mx4_tile_kernel<SM, SN, float><<<(unsigned)a.tiles, kMx4Threads, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_mx4_tiles(const Mx4Args &a, bool bf16, hipStream_t s) {
    // 32-bit offsets inside a tile
    if ((int64_t)16 * a.steps * 1024 >= ((int64_t)1 << 31) || (int64_t)128 * a.n_out * 2 >= ((int64_t)1 << 31))
        return hipErrorNotSupported;
    auto tiles = [&](int sm, int sn) {
        return (int64_t)a.D * ((a.w_frags + 4 * sn - 1) / (4 * sn)) * ((a.x_frags + sm - 1) / sm);
    };
    // tiles of 128 tokens, not for a few of them
    if (a.x_frags < 8) return hipErrorNotSupported;
    if (tiles(8, 4) >= 512) return launch<8, 4>(a, bf16, s);
    if (tiles(8, 2) >= 256) return launch<8, 2>(a, bf16, s);
    return hipErrorNotSupported;
}

}  // namespace dyad
