// Internal interface of the microscaled operators (mx_*.hip) to the C entry
// points in mx_abi.hip.
#pragma once

#include "dyad_internal.h"

namespace dyad {

enum MxFormat { kMxInt8 = 0, kMxFp4 = 1 };
constexpr int kMxBlock = 32;   // values that share a scale

// Row-major quantisation of X [rows][cols] and back.  gelu: the values read
// back are GELU of the ones stored (fp32, rounded once to the output type).
hipError_t launch_mx_quantize(int fmt, int64_t rows, int64_t cols, int dtype, const void *X, void *codes, void *scales,
                              hipStream_t s);
hipError_t launch_mx_dequantize(int fmt, int64_t rows, int64_t cols, int dtype, const void *codes, const void *scales,
                                bool gelu, void *Y, hipStream_t s);

// ---- the fp4 product ----------------------------------------------------------
//
// Both operands of v_mfma_scale_f32_16x16x128_f8f6f4 are kept in the order in
// which its lanes take them, so that a fragment (16 rows x 128 reduction
// indices) is 1 KB read with one 16-byte load a lane: lane 16 * b + r holds row
// r's block b of 32 codes.  The scale bytes of a lane in four neighbouring
// fragments share a word (the instruction picks the byte), so that a wave's
// fragments need a word or two a step.
//   codes  [part][fragment][step]      of 64 lanes x 16 bytes
//   scales [part][fragment / 4][step]  of 64 lanes x 4 bytes
// step: 128 reduction indices; indices past a block's width hold zeros.
// Weights: part = component * D + block, rows = the block's bo outputs.
// Input: part = block (the contiguous blocks), then D more of the residues
// under an input transpose; rows = tokens.
struct Mx4Layout {
    int64_t parts, frags, steps;
    int64_t groups() const { return (frags + 3) / 4; }
    int64_t code_bytes() const { return parts * frags * steps * 1024; }
    int64_t scale_bytes() const { return parts * groups() * steps * 256; }
    int64_t bytes() const { return code_bytes() + scale_bytes(); }
};
inline Mx4Layout mx4_weights_layout(int64_t D, int64_t bi, int64_t bo) { return {2 * D, (bo + 15) / 16, (bi + 127) / 128}; }
inline Mx4Layout mx4_input_layout(int64_t D, int64_t bi, int64_t M, bool in_t) {
    return {in_t ? 2 * D : D, (M + 15) / 16, (bi + 127) / 128};
}

// Under an output transpose whose 16 * D columns j*D + g never leave a block,
// component 1's rows are kept residue by residue: row l of a block is its
// output l % (bo / D) * D + l / (bo / D).  A fragment of either component then
// holds the same 16 outputs, and both add into one accumulator.
inline bool mx4_by_residue(int64_t D, int64_t bo, bool out_t) { return out_t && D > 1 && D <= 16 && bo % (16 * D) == 0; }

struct Mx4Pass {
    int64_t M, n_in, n_out, D, bi, bo;
    bool in_t, out_t, gelu;
    int dtype;
    const void *X, *packed, *bias;
    void *Y, *ws;
};

// Whether a call multiplies its input without a pass that quantises it in front
// (and needs no workspace).
bool mx4_in_place(int64_t n_in, int64_t D, int64_t bi, int64_t bo, int64_t M, bool in_t, bool out_t);

constexpr int64_t kMx4MaxOutResidues = 32;   // n_dyad under an output transpose

// W1, W2 [D][bo][bi] into `packed`; entries past n_in / n_out are stored as zero.
hipError_t launch_mx4_pack(int64_t n_in, int64_t n_out, int64_t D, bool in_t, bool out_t, int dtype, const void *W1,
                           const void *W2, void *packed, hipStream_t s);
// The input in fragment order, into p.ws (mx4_input_layout; its residues only with n_dyad > 1).
hipError_t launch_mx4_input(const Mx4Pass &p, hipStream_t s);
hipError_t launch_mx4_forward(const Mx4Pass &p, hipStream_t s);

}  // namespace dyad
