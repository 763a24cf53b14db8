// Host-only check of the microscaled C entry points (mx_abi.hip, over
// dyad_abi.hip) under AddressSanitizer and UndefinedBehaviorSanitizer.  Every
// launcher is a mock that touches the first and last byte of each operand that
// its kernel would read or write, and every buffer is a heap block of exactly
// the documented size: a chunk, an offset or a workspace that is wrong is a
// fault here.
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <memory>
#include <vector>

#include "dyad.h"
#include "mx_internal.h"

namespace {

int failures = 0;

#define EXPECT(cond)                                                             \
    do {                                                                         \
        if (!(cond)) {                                                           \
            fprintf(stderr, "FAILED line %d: %s\n", __LINE__, #cond);            \
            ++failures;                                                          \
        }                                                                        \
    } while (0)

volatile uint8_t sink;

void reads(const void *p, size_t n) {
    if (n == 0) return;
    const uint8_t *b = static_cast<const uint8_t *>(p);
    sink = b[0];
    sink = b[n - 1];
}
void writes(void *p, size_t n) {
    if (n == 0) return;
    uint8_t *b = static_cast<uint8_t *>(p);
    b[0] = 1;
    b[n - 1] = 1;
}

}  // namespace

namespace dyad {

hipError_t g_result = hipSuccess;     // of every mock launcher
bool g_epilogue = false;              // whether a matrix-core kernel takes 8-bit pre-activations
int g_launches = 0;
int64_t g_tokens = 0;                 // that mock GEMMs have made
size_t g_dw_ws = 0;

static size_t esize(int dtype) { return dtype == kBF16 ? 2 : 4; }

static hipError_t gemm(const GemmPass &p) {
    ++g_launches;
    const size_t e = esize(p.dtype), out = (size_t)(p.M * p.Nout);
    reads(p.in, (size_t)(p.M * p.Kin) * e);
    reads(p.W1, (size_t)(p.D * p.bk * p.bn) * e);
    reads(p.W2, (size_t)(p.D * p.bk * p.bn) * e);
    if (p.bias) reads(p.bias, (size_t)p.Nout * e);
    if (p.h_in) reads(p.h_in, out * e);
    writes(p.out, out * e);
    if (p.h_out) writes(p.h_out, out * e);
    if (p.h8) {
        EXPECT(p.Nout % 32 == 0 && p.dtype == kBF16);
        writes(p.h8, out);
        writes(p.hs, out / 32);
        if (p.a_out) writes(p.a_out, out * e);
    }
    g_tokens += p.M;
    return g_result;
}

bool skinny_ok(const GemmPass &) { return false; }
hipError_t launch_skinny_gemm(const GemmPass &, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_mfma_gemm(const GemmPass &p, hipStream_t) {
    if (p.dtype != kBF16 || p.Kin != p.D * p.bk || p.Nout != p.D * p.bn || !g_epilogue) return hipErrorNotSupported;
    return p.plan ? hipSuccess : gemm(p);
}
hipError_t launch_padded_gemm(const GemmPass &, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_general_mfma_gemm(const GemmPass &p, hipStream_t) { return p.dtype == kBF16 ? gemm(p) : hipErrorNotSupported; }
hipError_t launch_simt_gemm(const GemmPass &p, hipStream_t) {
    EXPECT(p.wide_sums == (p.epilogue == kEpiBiasGelu && p.dtype == kF32));
    return gemm(p);
}
bool mfma_dw_ok(const DwPass &) { return true; }
size_t mfma_dw_workspace(const DwPass &) { return g_dw_ws; }
bool general_dw_ok(const DwPass &) { return false; }
size_t general_dw_workspace(const DwPass &) { return 0; }
size_t simt_dw_workspace(const DwPass &) { return 0; }
hipError_t launch_mfma_dw(const DwPass &p, hipStream_t) {
    ++g_launches;
    const size_t e = esize(p.dtype);
    reads(p.dZ, (size_t)(p.M * p.n_out) * e);
    reads(p.X, (size_t)(p.M * p.n_in) * e);
    writes(p.dW1, (size_t)(p.D * p.bi * p.bo) * e);
    writes(p.dW2, (size_t)(p.D * p.bi * p.bo) * e);
    if (p.db) writes(p.db, (size_t)p.n_out * e);
    EXPECT(p.ws_bytes == g_dw_ws && (p.ws != nullptr) == (g_dw_ws > 0));
    writes(p.ws, p.ws_bytes);
    return g_result;
}
hipError_t launch_general_mfma_dw(const DwPass &, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_simt_dw(const DwPass &, hipStream_t) { return hipErrorNotSupported; }
ScratchScope::ScratchScope(void *p, size_t b) : ptr(p), bytes(b), prev(nullptr) {}
ScratchScope::~ScratchScope() {}
const ScratchScope *current_scratch() { return nullptr; }
hipError_t noalloc_scratch(void **out) { *out = nullptr; return hipErrorNotSupported; }

static void quantised(int fmt, int64_t rows, int64_t cols, size_t *codes, size_t *scales) {
    *codes = (size_t)rows * (size_t)(fmt == kMxInt8 ? cols : (cols + 1) / 2);
    *scales = (size_t)rows * (size_t)((cols + 31) / 32);
}
hipError_t launch_mx_quantize(int fmt, int64_t rows, int64_t cols, int dtype, const void *X, void *codes, void *scales, hipStream_t) {
    ++g_launches;
    size_t c, s;
    quantised(fmt, rows, cols, &c, &s);
    reads(X, (size_t)(rows * cols) * esize(dtype));
    writes(codes, c);
    writes(scales, s);
    return g_result;
}
hipError_t launch_mx_dequantize(int fmt, int64_t rows, int64_t cols, int dtype, const void *codes, const void *scales, bool,
                                void *Y, hipStream_t) {
    ++g_launches;
    size_t c, s;
    quantised(fmt, rows, cols, &c, &s);
    reads(codes, c);
    reads(scales, s);
    writes(Y, (size_t)(rows * cols) * esize(dtype));
    return g_result;
}
bool mx4_in_place(int64_t, int64_t, int64_t, int64_t, int64_t M, bool, bool) { return M <= 2; }
hipError_t launch_mx4_pack(int64_t n_in, int64_t n_out, int64_t D, bool, bool, int dtype, const void *W1, const void *W2,
                           void *packed, hipStream_t) {
    ++g_launches;
    const int64_t bi = (n_in + D - 1) / D, bo = (n_out + D - 1) / D;
    reads(W1, (size_t)(D * bi * bo) * esize(dtype));
    reads(W2, (size_t)(D * bi * bo) * esize(dtype));
    writes(packed, (size_t)mx4_weights_layout(D, bi, bo).bytes());
    return g_result;
}
hipError_t launch_mx4_forward(const Mx4Pass &p, hipStream_t) {
    ++g_launches;
    const size_t e = esize(p.dtype);
    reads(p.X, (size_t)(p.M * p.n_in) * e);
    reads(p.packed, (size_t)mx4_weights_layout(p.D, p.bi, p.bo).bytes());
    if (p.bias) reads(p.bias, (size_t)p.n_out * e);
    writes(p.Y, (size_t)(p.M * p.n_out) * e);
    if (p.M > 2) writes(p.ws, (size_t)mx4_input_layout(p.D, p.bi, p.M, p.in_t).bytes());
    return g_result;
}

}  // namespace dyad

using namespace dyad;

// A block of exactly n bytes (16-byte aligned, as the heap's are); null for none.
struct Block {
    std::unique_ptr<uint8_t[]> p;
    explicit Block(size_t n) : p(n ? new uint8_t[n] : nullptr) {
        if (n) p[0] = p[n - 1] = 0;
    }
    operator void *() const { return p.get(); }
};

static void check(int variant, int64_t n_in, int64_t n_out, int64_t D, int64_t M, int dtype) {
    const dyad_variant v = (dyad_variant)variant;
    const dyad_dtype t = (dyad_dtype)dtype;
    const size_t e = esize(dtype), in = (size_t)(M * n_in), out = (size_t)(M * n_out);
    const int64_t bi = (n_in + D - 1) / D, bo = (n_out + D - 1) / D, nb_in = (n_in + 31) / 32, nb_out = (n_out + 31) / 32;
    const size_t w = (size_t)(D * bi * bo) * e;
    const Block X(in * e), Y(out * e), W1(w), W2(w), bias((size_t)n_out * e), dbias((size_t)n_out * e), dZ(out * e), dX(in * e),
        A(in * e);
    const Block H8(out), Hs((size_t)(M * nb_out)), X8(in), Xs((size_t)(M * nb_in)), dW1(w), dW2(w);
    auto workspace = [&](dyad_mx8_pass p, dyad_act a = DYAD_ACT_NONE) {
        return dyad_mx8_workspace_bytes(p, v, n_in, n_out, D, M, t, a);
    };
    const bool takes = g_epilogue && dtype == DYAD_BF16 && n_in % D == 0 && n_out % D == 0;
    {
        const size_t n = workspace(DYAD_MX8_FORWARD);
        const Block ws(n);
        EXPECT((n == 0) == (M == 0 || (takes && n_out % 32 == 0)));
        g_tokens = 0;
        EXPECT(dyad_forward_mx8(v, n_in, n_out, D, M, t, X, W1, W2, bias, Y, H8, Hs, ws, n, nullptr) == DYAD_OK);
        EXPECT(g_tokens == M);
        if (n) EXPECT(dyad_forward_mx8(v, n_in, n_out, D, M, t, X, W1, W2, bias, Y, H8, Hs, ws, n - 1, nullptr) == DYAD_ERR_WORKSPACE);
    }
    for (const bool with_act : {false, true}) {
        const size_t n = workspace(DYAD_MX8_DX);
        const Block ws(n);
        EXPECT((n == 0) == (M == 0 || (takes && n_in % 32 == 0)));
        g_tokens = 0;
        EXPECT(dyad_backward_dx_mx8(v, n_in, n_out, D, M, t, dZ, W1, W2, X8, Xs, dX, with_act ? (void *)A : nullptr, ws, n,
                                    nullptr) == DYAD_OK);
        EXPECT(g_tokens == M);
    }
    for (const size_t extra : {(size_t)0, (size_t)1000}) {
        g_dw_ws = extra;
        const size_t n = workspace(DYAD_MX8_DW, DYAD_ACT_GELU);
        const Block ws(n);
        EXPECT(dyad_backward_dw_mx8(v, n_in, n_out, D, M, t, DYAD_ACT_GELU, dZ, X8, Xs, dW1, dW2, dbias, ws, n, nullptr) == DYAD_OK);
    }
    for (const dyad_mx_format f : {DYAD_MX_INT8, DYAD_MX_FP4}) {
        const Block codes((size_t)M * (size_t)(f == DYAD_MX_INT8 ? n_in : (n_in + 1) / 2));
        EXPECT(dyad_mx_quantize(f, M, n_in, t, X, codes, Xs, nullptr) == DYAD_OK);
        EXPECT(dyad_mx_dequantize(f, M, n_in, t, codes, Xs, X, nullptr) == DYAD_OK);
    }
    const size_t pn = dyad_mx4_weight_bytes(v, n_in, n_out, D), wn = dyad_mx4_workspace_bytes(v, n_in, n_out, D, M);
    const Block packed(pn), ws(wn);
    EXPECT(pn > 0 && (wn == 0) == (M <= 2));
    EXPECT(dyad_mx4_quantize_weights(v, n_in, n_out, D, t, W1, W2, packed, pn, nullptr) == DYAD_OK);
    EXPECT(dyad_mx4_forward(v, n_in, n_out, D, M, t, X, packed, pn, bias, DYAD_ACT_GELU, Y, ws, wn, nullptr) ==
           (variant != DYAD_IT && D > kMx4MaxOutResidues ? DYAD_ERR_SHAPE : DYAD_OK));
    if (wn && D <= kMx4MaxOutResidues)
        EXPECT(dyad_mx4_forward(v, n_in, n_out, D, M, t, X, packed, pn, bias, DYAD_ACT_GELU, Y, ws, wn - 1, nullptr) == DYAD_ERR_WORKSPACE);
}

int main() {
    const int64_t shapes[][4] = {   // n_in, n_out, n_dyad, tokens
        {64, 256, 4, 8}, {64, 256, 4, 0}, {768, 96, 4, 1}, {7, 6, 2, 5}, {250, 154, 4, 65}, {8, 8, 16, 5}, {160, 64, 40, 3},
        {33, 1, 1, 2},
        // several chunks of tokens, the last one short
        {5, 20001, 5, 2100}, {20001, 5, 5, 2100}, {64, 20480, 4, 2300},
    };
    for (const bool epilogue : {false, true}) {
        g_epilogue = epilogue;
        for (const auto &s : shapes)
            for (int variant = 0; variant < 3; ++variant)
                for (int dtype = 0; dtype < 2; ++dtype) {
                    if (s[3] > 1000 && variant == 1) continue;
                    check(variant, s[0], s[1], s[2], s[3], dtype);
                }
    }
    // a launch the runtime refuses is DYAD_ERR_LAUNCH, at whichever step it comes
    const Block big(1 << 20);
    for (const bool epilogue : {false, true})
        for (int dtype = 0; dtype < 2; ++dtype) {
            g_epilogue = epilogue;
            g_result = hipErrorLaunchFailure;
            g_dw_ws = 0;
            const dyad_dtype t = (dyad_dtype)dtype;
            EXPECT(dyad_forward_mx8(DYAD_IT, 64, 256, 4, 8, t, big, big, big, nullptr, big, big, big, big, 1 << 20, nullptr) == DYAD_ERR_LAUNCH);
            EXPECT(dyad_backward_dx_mx8(DYAD_IT, 64, 256, 4, 8, t, big, big, big, big, big, big, big, big, 1 << 20, nullptr) == DYAD_ERR_LAUNCH);
            EXPECT(dyad_backward_dw_mx8(DYAD_IT, 64, 256, 4, 8, t, DYAD_ACT_NONE, big, big, big, big, big, big, big, 1 << 20, nullptr) ==
                   DYAD_ERR_LAUNCH);
            EXPECT(dyad_mx_quantize(DYAD_MX_FP4, 4, 40, t, big, big, big, nullptr) == DYAD_ERR_LAUNCH);
            EXPECT(dyad_mx_dequantize(DYAD_MX_FP4, 4, 40, t, big, big, big, nullptr) == DYAD_ERR_LAUNCH);
            EXPECT(dyad_mx4_quantize_weights(DYAD_OT, 64, 256, 4, t, big, big, big, 1 << 20, nullptr) == DYAD_ERR_LAUNCH);
            EXPECT(dyad_mx4_forward(DYAD_OT, 64, 256, 4, 8, t, big, big, 1 << 20, big, DYAD_ACT_NONE, big, big, 1 << 20, nullptr) ==
                   DYAD_ERR_LAUNCH);
            g_result = hipSuccess;
        }
    // sizes are checked before any launch, the largest too
    g_launches = 0;
    const int64_t huge = INT64_MAX;
    for (const int64_t s : {huge, (int64_t)1 << 40, (int64_t)-1}) {
        EXPECT(dyad_mx_quantize(DYAD_MX_INT8, s, 64, DYAD_F32, big, big, big, nullptr) == DYAD_ERR_INVALID_ARG);
        EXPECT(dyad_mx_dequantize(DYAD_MX_FP4, 4, s, DYAD_F32, big, big, big, nullptr) == DYAD_ERR_INVALID_ARG);
        EXPECT(dyad_mx4_weight_bytes(DYAD_IT, s, 64, 4) == 0 && dyad_mx4_workspace_bytes(DYAD_IT, 64, 64, 4, s) == 0);
        EXPECT(dyad_mx8_workspace_bytes(DYAD_MX8_DW, DYAD_IT, 64, 64, 4, s, DYAD_F32, DYAD_ACT_NONE) == 0);
        EXPECT(dyad_forward_mx8(DYAD_IT, 64, 256, 4, s, DYAD_F32, big, big, big, nullptr, big, big, big, big, 1 << 20, nullptr) ==
               DYAD_ERR_INVALID_ARG);
        EXPECT(dyad_mx4_forward(DYAD_IT, s, 256, 4, 8, DYAD_F32, big, big, 1 << 20, big, DYAD_ACT_NONE, big, big, 1 << 20, nullptr) ==
               DYAD_ERR_INVALID_ARG);
    }
    EXPECT(g_launches == 0);
    if (failures) return 1;
    printf("mx mock ok\n");
    return 0;
}
