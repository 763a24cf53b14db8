// C entry points of the microscaled operators (include/dyad.h).  Every check
// runs before the first HIP call.
#include "dyad.h"

#include "abi_checks.h"
#include "mx_internal.h"

using namespace dyad::abi;
using dyad::GemmPass;

static size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }

static int check_matrix(int fmt, int64_t rows, int64_t cols, int dtype) {
    if (fmt != DYAD_MX_INT8 && fmt != DYAD_MX_FP4) return DYAD_ERR_INVALID_ARG;
    if (dtype != DYAD_F32 && dtype != DYAD_BF16) return DYAD_ERR_DTYPE;
    if (rows < 0 || cols <= 0 || rows >= kMaxDim || cols >= kMaxDim || rows * cols >= kMaxElems) return DYAD_ERR_INVALID_ARG;
    return DYAD_OK;
}

static size_t elem(int dtype) { return dtype == DYAD_BF16 ? 2 : 4; }

// The matrix-core tiles write and read an 8-bit pre-activation in their
// epilogues.  Other shapes (zero-padded blocks, fp32, n_dyad without tiles) run
// the plain pass beside a copy of it in the layer's type, a chunk of tokens of at
// most kChunkBytes at a time, in the workspace.  The weight gradient always reads
// a copy: staged from 8 bits tile by tile it was slower (OPT-125m fc1 73 us
// against 66 + 8 for the copy, OPT-350m 157 against 95 + 11; with GELU, which
// every tile then repeats, OPT-125m fc2 186 against 67 + 41).
constexpr size_t kChunkBytes = (size_t)64 << 20;

static int64_t chunk_tokens(int64_t n, int64_t M, int dtype) {
    int64_t c = (int64_t)(kChunkBytes / ((size_t)n * elem(dtype))) / 256 * 256;
    if (c < 1024) c = 1024;
    return M < c ? M : c;
}

// A pass whose pre-activation is kept in 8 bits, but for its operands.
static GemmPass h8_pass(int pass, int variant, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M, int dtype) {
    const bool fwd = pass == DYAD_MX8_FORWARD;
    GemmPass p{};
    p.M = M; p.D = n_dyad; p.dtype = dtype;
    p.Kin = fwd ? n_in : n_out; p.Nout = fwd ? n_out : n_in;
    p.bk = block(p.Kin, n_dyad); p.bn = block(p.Nout, n_dyad);
    p.in_t = fwd ? in_transposed(variant) : out_transposed(variant);
    p.out_t = fwd ? out_transposed(variant) : in_transposed(variant);
    p.w_t = !fwd;
    p.epilogue = fwd ? dyad::kEpiBiasGelu : dyad::kEpiGeluGrad;
    return p;
}

// A pass on the kernels that take its pre-activation in 8 bits.
static hipError_t run_h8(const GemmPass &p, hipStream_t s) {
    if (p.dtype != DYAD_BF16 || p.Nout % 32 != 0 || p.Nout != p.D * p.bn) return hipErrorNotSupported;
    const dyad::WorkspaceHold hold;
    hipError_t e = !p.plan && dyad::skinny_ok(p) ? dyad::launch_skinny_gemm(p, s) : hipErrorNotSupported;
    if (e == hipErrorNotSupported) e = dyad::launch_mfma_gemm(p, s);
    return e;
}

// Bytes of the copy in front of the inner call's own workspace: none where an
// epilogue does its work whatever else there is no memory for (so also while a
// graph is captured on a stream that no call has warmed up).
static size_t kept_bytes(int pass, int variant, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M, int dtype) {
    if (pass == DYAD_MX8_DW) return round256((size_t)M * (size_t)n_in * elem(dtype));
    GemmPass p = h8_pass(pass, variant, n_in, n_out, n_dyad, M, dtype);
    p.plan = true;
    if (M == 0 || run_h8(p, nullptr) == hipSuccess) return 0;
    return round256((size_t)chunk_tokens(p.Nout, M, dtype) * (size_t)p.Nout * elem(dtype));
}

static const void *rows(const void *p, int64_t m, int64_t n, size_t e) { return static_cast<const char *>(p) + (size_t)m * (size_t)n * e; }
static void *rows(void *p, int64_t m, int64_t n, size_t e) { return static_cast<char *>(p) + (size_t)m * (size_t)n * e; }

extern "C" {

int dyad_mx_quantize(dyad_mx_format format, int64_t rows, int64_t cols, dyad_dtype dtype_arg, const void *X,
                     void *codes, void *scales, hipStream_t stream) {
    const int fmt = enum_value(format), dtype = enum_value(dtype_arg);
    const int rc = check_matrix(fmt, rows, cols, dtype);
    if (rc) return rc;
    if (rows > 0 && (!X || !codes || !scales)) return DYAD_ERR_INVALID_ARG;
    if (!aligned16(X) || !aligned16(codes) || !aligned16(scales)) return DYAD_ERR_ALIGN;
    if (rows == 0) return DYAD_OK;
    return launch_status(dyad::launch_mx_quantize(fmt, rows, cols, dtype, X, codes, scales, stream));
}

int dyad_mx_dequantize(dyad_mx_format format, int64_t rows, int64_t cols, dyad_dtype dtype_arg, const void *codes,
                       const void *scales, void *Y, hipStream_t stream) {
    const int fmt = enum_value(format), dtype = enum_value(dtype_arg);
    const int rc = check_matrix(fmt, rows, cols, dtype);
    if (rc) return rc;
    if (rows > 0 && (!Y || !codes || !scales)) return DYAD_ERR_INVALID_ARG;
    if (!aligned16(Y) || !aligned16(codes) || !aligned16(scales)) return DYAD_ERR_ALIGN;
    if (rows == 0) return DYAD_OK;
    return launch_status(dyad::launch_mx_dequantize(fmt, rows, cols, dtype, codes, scales, false, Y, stream));
}

size_t dyad_mx4_weight_bytes(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad) {
    if (check_sizes(enum_value(variant), n_in, n_out, n_dyad, 0, DYAD_BF16)) return 0;
    return (size_t)dyad::mx4_weights_layout(n_dyad, block(n_in, n_dyad), block(n_out, n_dyad)).bytes();
}

int dyad_mx4_quantize_weights(dyad_variant variant_arg, int64_t n_in, int64_t n_out, int64_t n_dyad,
                              dyad_dtype dtype_arg, const void *W1, const void *W2, void *packed, size_t packed_bytes,
                              hipStream_t stream) {
    const int variant = enum_value(variant_arg), dtype = enum_value(dtype_arg);
    const int rc = check_sizes(variant, n_in, n_out, n_dyad, 0, dtype);
    if (rc) return rc;
    if (!W1 || !W2) return DYAD_ERR_INVALID_ARG;
    if (!aligned16(W1) || !aligned16(W2) || !aligned16(packed)) return DYAD_ERR_ALIGN;
    if (!packed || packed_bytes < dyad_mx4_weight_bytes(variant_arg, n_in, n_out, n_dyad)) return DYAD_ERR_WORKSPACE;
    return launch_status(dyad::launch_mx4_pack(n_in, n_out, n_dyad, in_transposed(variant), out_transposed(variant), dtype,
                                               W1, W2, packed, stream));
}

size_t dyad_mx4_workspace_bytes(dyad_variant variant_arg, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M) {
    const int variant = enum_value(variant_arg);
    if (check_sizes(variant, n_in, n_out, n_dyad, M, DYAD_BF16)) return 0;
    if (dyad::mx4_in_place(n_in, n_dyad, block(n_in, n_dyad), block(n_out, n_dyad), M, in_transposed(variant),
                           out_transposed(variant)))
        return 0;
    return (size_t)dyad::mx4_input_layout(n_dyad, block(n_in, n_dyad), M, in_transposed(variant)).bytes();
}

int dyad_mx4_forward(dyad_variant variant_arg, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M,
                     dyad_dtype dtype_arg, const void *X, const void *packed, size_t packed_bytes, const void *bias,
                     dyad_act act_arg, void *Y, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const int variant = enum_value(variant_arg), dtype = enum_value(dtype_arg), act = enum_value(act_arg);
    const int rc = check_sizes(variant, n_in, n_out, n_dyad, M, dtype);
    if (rc) return rc;
    if (act != DYAD_ACT_NONE && act != DYAD_ACT_GELU) return DYAD_ERR_INVALID_ARG;
    if (M > 0 && (!X || !Y)) return DYAD_ERR_INVALID_ARG;
    if (!aligned16(X) || !aligned16(packed) || !aligned16(bias) || !aligned16(Y) || !aligned16(workspace))
        return DYAD_ERR_ALIGN;
    if (!packed || packed_bytes < dyad_mx4_weight_bytes(variant_arg, n_in, n_out, n_dyad)) return DYAD_ERR_WORKSPACE;
    if (out_transposed(variant) && n_dyad > dyad::kMx4MaxOutResidues) return DYAD_ERR_SHAPE;
    if (M == 0) return DYAD_OK;
    const size_t need = dyad_mx4_workspace_bytes(variant_arg, n_in, n_out, n_dyad, M);
    if (need > 0 && (!workspace || workspace_bytes < need)) return DYAD_ERR_WORKSPACE;
    dyad::Mx4Pass p{};
    p.M = M; p.n_in = n_in; p.n_out = n_out; p.D = n_dyad; p.bi = block(n_in, n_dyad); p.bo = block(n_out, n_dyad);
    p.in_t = in_transposed(variant); p.out_t = out_transposed(variant); p.gelu = act == DYAD_ACT_GELU;
    p.dtype = dtype; p.X = X; p.packed = packed; p.bias = bias; p.Y = Y; p.ws = workspace;
    return launch_status(dyad::launch_mx4_forward(p, stream));
}

size_t dyad_mx8_workspace_bytes(dyad_mx8_pass pass_arg, dyad_variant variant, int64_t n_in, int64_t n_out,
                                int64_t n_dyad, int64_t M, dyad_dtype dtype_arg, dyad_act act_in) {
    const int pass = enum_value(pass_arg), dtype = enum_value(dtype_arg), act = enum_value(act_in);
    if (check_sizes(enum_value(variant), n_in, n_out, n_dyad, M, dtype)) return 0;
    if (pass != DYAD_MX8_FORWARD && pass != DYAD_MX8_DX && pass != DYAD_MX8_DW) return 0;
    if (act != DYAD_ACT_NONE && act != DYAD_ACT_GELU) return 0;
    const size_t kept = kept_bytes(pass, enum_value(variant), n_in, n_out, n_dyad, M, dtype);
    if (pass != DYAD_MX8_DW) return kept;
    return kept + dyad_dw_workspace_bytes(variant, n_in, n_out, n_dyad, M, dtype_arg);
}

int dyad_forward_mx8(dyad_variant variant_arg, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M,
                     dyad_dtype dtype_arg, const void *X, const void *W1, const void *W2, const void *bias, void *Y,
                     void *H8, void *Hs, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const int variant = enum_value(variant_arg), dtype = enum_value(dtype_arg);
    int rc = check_sizes(variant, n_in, n_out, n_dyad, M, dtype);
    if (rc) return rc;
    if (!W1 || !W2 || (M > 0 && (!X || !Y || !H8 || !Hs))) return DYAD_ERR_INVALID_ARG;
    if (!aligned16(X) || !aligned16(W1) || !aligned16(W2) || !aligned16(bias) || !aligned16(Y) || !aligned16(H8) ||
        !aligned16(Hs) || !aligned16(workspace))
        return DYAD_ERR_ALIGN;
    if (M == 0) return DYAD_OK;
    const size_t need = dyad_mx8_workspace_bytes(DYAD_MX8_FORWARD, variant_arg, n_in, n_out, n_dyad, M, dtype_arg, DYAD_ACT_NONE);
    if (need > 0 && (!workspace || workspace_bytes < need)) return DYAD_ERR_WORKSPACE;
    GemmPass p = h8_pass(DYAD_MX8_FORWARD, variant, n_in, n_out, n_dyad, M, dtype);
    p.in = X; p.W1 = W1; p.W2 = W2; p.bias = bias; p.out = Y;
    p.h8 = static_cast<uint8_t *>(H8); p.hs = static_cast<uint8_t *>(Hs);
    const hipError_t e = run_h8(p, stream);
    if (e != hipErrorNotSupported || need == 0) return launch_status(e);
    const int64_t chunk = chunk_tokens(n_out, M, dtype);
    for (int64_t m = 0; m < M; m += chunk) {
        const int64_t c = M - m < chunk ? M - m : chunk;
        if (dtype == DYAD_F32) {
            p.M = c; p.in = rows(X, m, n_in, 4); p.out = rows(Y, m, n_out, 4); p.h_out = workspace;
            p.h8 = p.hs = nullptr;
            p.wide_sums = true;
            rc = launch_status(dyad::launch_simt_gemm(p, stream));
        } else {
            rc = dyad_forward(variant_arg, n_in, n_out, n_dyad, c, dtype_arg, rows(X, m, n_in, 2), W1, W2, bias,
                              DYAD_ACT_GELU, rows(Y, m, n_out, 2), workspace, stream);
        }
        if (rc) return rc;
        rc = launch_status(dyad::launch_mx_quantize(DYAD_MX_INT8, c, n_out, dtype, workspace, rows(H8, m, n_out, 1),
                                                    rows(Hs, m, (n_out + 31) / 32, 1), stream));
        if (rc) return rc;
    }
    return DYAD_OK;
}

int dyad_backward_dx_mx8(dyad_variant variant_arg, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M,
                         dyad_dtype dtype_arg, const void *dZ, const void *W1, const void *W2, const void *H8,
                         const void *Hs, void *dX, void *A, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const int variant = enum_value(variant_arg), dtype = enum_value(dtype_arg);
    int rc = check_sizes(variant, n_in, n_out, n_dyad, M, dtype);
    if (rc) return rc;
    if (!W1 || !W2 || (M > 0 && (!dZ || !dX || !H8 || !Hs))) return DYAD_ERR_INVALID_ARG;
    if (!aligned16(dZ) || !aligned16(W1) || !aligned16(W2) || !aligned16(H8) || !aligned16(Hs) || !aligned16(dX) ||
        !aligned16(A) || !aligned16(workspace))
        return DYAD_ERR_ALIGN;
    if (M == 0) return DYAD_OK;
    const size_t need = dyad_mx8_workspace_bytes(DYAD_MX8_DX, variant_arg, n_in, n_out, n_dyad, M, dtype_arg, DYAD_ACT_NONE);
    if (need > 0 && (!workspace || workspace_bytes < need)) return DYAD_ERR_WORKSPACE;
    GemmPass p = h8_pass(DYAD_MX8_DX, variant, n_in, n_out, n_dyad, M, dtype);
    p.in = dZ; p.W1 = W1; p.W2 = W2; p.out = dX;
    p.h8 = static_cast<uint8_t *>(const_cast<void *>(H8)); p.hs = static_cast<uint8_t *>(const_cast<void *>(Hs));
    p.a_out = A;
    const hipError_t e = run_h8(p, stream);
    if (e != hipErrorNotSupported || need == 0) return launch_status(e);
    const int64_t chunk = chunk_tokens(n_in, M, dtype);
    for (int64_t m = 0; m < M; m += chunk) {
        const int64_t c = M - m < chunk ? M - m : chunk;
        rc = launch_status(dyad::launch_mx_dequantize(DYAD_MX_INT8, c, n_in, dtype, rows(H8, m, n_in, 1),
                                                      rows(Hs, m, (n_in + 31) / 32, 1), false, workspace, stream));
        if (!rc && A)
            rc = launch_status(dyad::launch_mx_dequantize(DYAD_MX_INT8, c, n_in, dtype, rows(H8, m, n_in, 1),
                                                          rows(Hs, m, (n_in + 31) / 32, 1), true,
                                                          rows(A, m, n_in, elem(dtype)), stream));
        if (rc) return rc;
        rc = dyad_backward_dx(variant_arg, n_in, n_out, n_dyad, c, dtype_arg, rows(dZ, m, n_out, elem(dtype)), W1, W2,
                              DYAD_ACT_GELU, workspace, rows(dX, m, n_in, elem(dtype)), stream);
        if (rc) return rc;
    }
    return DYAD_OK;
}

int dyad_backward_dw_mx8(dyad_variant variant_arg, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M,
                         dyad_dtype dtype_arg, dyad_act act_in_arg, const void *dZ, const void *X8, const void *Xs,
                         void *dW1, void *dW2, void *dbias, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const int variant = enum_value(variant_arg), dtype = enum_value(dtype_arg), act_in = enum_value(act_in_arg);
    const int rc = check_sizes(variant, n_in, n_out, n_dyad, M, dtype);
    if (rc) return rc;
    if (act_in != DYAD_ACT_NONE && act_in != DYAD_ACT_GELU) return DYAD_ERR_INVALID_ARG;
    if (!dW1 || !dW2 || (M > 0 && (!dZ || !X8 || !Xs))) return DYAD_ERR_INVALID_ARG;
    if (!aligned16(dZ) || !aligned16(X8) || !aligned16(Xs) || !aligned16(dW1) || !aligned16(dW2) || !aligned16(dbias) ||
        !aligned16(workspace))
        return DYAD_ERR_ALIGN;
    const size_t need = dyad_mx8_workspace_bytes(DYAD_MX8_DW, variant_arg, n_in, n_out, n_dyad, M, dtype_arg, act_in_arg);
    if (need > 0 && (!workspace || workspace_bytes < need)) return DYAD_ERR_WORKSPACE;
    const size_t kept = kept_bytes(DYAD_MX8_DW, variant, n_in, n_out, n_dyad, M, dtype);
    if (M > 0) {
        const hipError_t e =
            dyad::launch_mx_dequantize(DYAD_MX_INT8, M, n_in, dtype, X8, Xs, act_in == DYAD_ACT_GELU, workspace, stream);
        if (e != hipSuccess) return launch_status(e);
    }
    const size_t left = need - kept;
    void *inner = left > 0 ? static_cast<unsigned char *>(workspace) + kept : nullptr;
    return dyad_backward_dw(variant_arg, n_in, n_out, n_dyad, M, dtype_arg, dZ, M > 0 ? workspace : nullptr, dW1, dW2, dbias,
                            inner, left, stream);
}

}  // extern "C"
