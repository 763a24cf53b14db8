// C entry points of dropout, the residual stream's norms and the loss (include/dyad.h):
// argument checks, each before the first HIP call, and launches.
#include "abi_checks.h"
#include "lm_internal.h"
#include "philox.h"

namespace {

using namespace dyad::abi;

bool known_dtype(int d) { return d == DYAD_F32 || d == DYAD_BF16; }
bool probability(double p) { return p >= 0.0 && p <= 1.0; }   // false for NaN

bool aligned8(const void *p) { return ((uintptr_t)p & 7u) == 0; }

bool small(int64_t rows, int64_t cols) {
    return rows >= 0 && rows < kMaxDim && cols > 0 && cols < kMaxDim && rows * cols < kMaxElems;
}

int norm_pass(const dyad_add_norm_args *a, const dyad_add_norm_grads *g, dyad::AddNormPass &p) {
    if (!a) return DYAD_ERR_INVALID_ARG;
    p = dyad::AddNormPass{};
    p.M = a->M; p.n = a->n; p.groups = a->groups;
    p.stream_dtype = enum_value(a->stream_dtype); p.dtype = enum_value(a->dtype);
    p.param_dtype = enum_value(a->param_dtype);
    p.norm = enum_value(a->norm); p.post = enum_value(a->post);
    p.x_scale = a->x_scale; p.y_scale = a->y_scale; p.eps = a->eps;
    p.x = a->x; p.y = a->y; p.w = a->weight; p.b = a->bias; p.pw = a->post_weight; p.pb = a->post_bias;
    p.gate = a->gate; p.h = a->h; p.out = a->out; p.stats = a->stats; p.post_stats = a->post_stats;
    if (!known_dtype(p.stream_dtype) || !known_dtype(p.dtype) || !known_dtype(p.param_dtype)) return DYAD_ERR_DTYPE;
    if ((p.stream_dtype == DYAD_BF16 && p.dtype == DYAD_F32) || (p.dtype == DYAD_F32 && p.param_dtype == DYAD_BF16))
        return DYAD_ERR_DTYPE;
    for (const int kind : {p.norm, p.post})
        if (kind != DYAD_NORM_NONE && kind != DYAD_NORM_LAYER && kind != DYAD_NORM_RMS) return DYAD_ERR_INVALID_ARG;
    if (!small(p.M, p.n) || p.groups <= 0 || p.M % p.groups != 0 || !probability(a->p) || !(p.eps >= 0.f))
        return DYAD_ERR_INVALID_ARG;
    if (p.n < 8 || p.n > dyad::kNormMaxWidth) return DYAD_ERR_SHAPE;
    if (!p.y && p.M == 0) p.y = a;   // never read: an empty tensor need not have an address
    if (!p.y) { p.post = DYAD_NORM_NONE; p.gate = nullptr; }
    if (!p.gate) p.groups = 1;
    if (p.norm == DYAD_NORM_NONE) { p.w = p.b = nullptr; }
    if (p.post == DYAD_NORM_NONE) { p.pw = p.pb = nullptr; }
    for (const void *q : {p.x, a->y, p.w, p.b, p.pw, p.pb, p.gate, (const void *)p.h, (const void *)p.out,
                          (const void *)p.stats, (const void *)p.post_stats})
        if (!aligned16(q)) return DYAD_ERR_ALIGN;
    if (!aligned8(a->offset_dev)) return DYAD_ERR_ALIGN;
    if (!g) return DYAD_OK;
    p.dh = g->dh; p.dout = g->dout; p.dx = g->dx; p.dy = g->dy; p.dw = g->dweight; p.db = g->dbias;
    p.dpw = g->dpost_weight; p.dpb = g->dpost_bias; p.dgate = g->dgate;
    for (const void *q : {p.dh, p.dout, (const void *)p.dx, (const void *)p.dy, (const void *)p.dw, (const void *)p.db,
                          (const void *)p.dpw, (const void *)p.dpb, (const void *)p.dgate})
        if (!aligned16(q)) return DYAD_ERR_ALIGN;
    // a gradient of what the call does not have
    if ((p.dw || p.db || p.dout) && p.norm == DYAD_NORM_NONE) return DYAD_ERR_INVALID_ARG;
    if ((p.dpw || p.dpb) && p.post == DYAD_NORM_NONE) return DYAD_ERR_INVALID_ARG;
    if ((p.dy && !p.y) || (p.dgate && !p.gate)) return DYAD_ERR_INVALID_ARG;
    return DYAD_OK;
}

int loss_sizes(int64_t M, int64_t n, int64_t V, int dtype) {
    if (!known_dtype(dtype)) return DYAD_ERR_DTYPE;
    if (!small(M, n) || !small(V, n) || V <= 0) return DYAD_ERR_INVALID_ARG;
    if (M > dyad::kLossMaxRows || V > dyad::kLossMaxRows || n > dyad::kLossMaxWidth || M * V > dyad::kLossMaxLogits)
        return DYAD_ERR_SHAPE;
    return DYAD_OK;
}

}  // namespace

extern "C" {

int dyad_dropout(int64_t rows, int64_t cols, dyad_dtype dtype_arg, const void *X, double p, uint64_t seed,
                 uint64_t offset, const uint64_t *offset_dev, void *Y, hipStream_t stream) {
    const int dtype = enum_value(dtype_arg);
    if (!known_dtype(dtype)) return DYAD_ERR_DTYPE;
    // a row's columns are counted in 32 bits, eight at a time
    if (!small(rows, cols) || cols > kMaxDim - 16 || !probability(p) || (rows > 0 && (!X || !Y))) return DYAD_ERR_INVALID_ARG;
    if (!aligned16(X) || !aligned16(Y) || !aligned8(offset_dev)) return DYAD_ERR_ALIGN;
    if (rows == 0) return DYAD_OK;
    return launch_status(dyad::launch_dropout(rows, cols, dtype, X, dyad::drop_args(p, seed, offset, offset_dev), Y, stream));
}

int dyad_add_norm_forward(const dyad_add_norm_args *args, hipStream_t stream) {
    dyad::AddNormPass p;
    const int rc = norm_pass(args, nullptr, p);
    if (rc) return rc;
    if (p.M == 0) return DYAD_OK;
    if (!p.x || (p.norm != DYAD_NORM_NONE && !p.out) || (p.norm == DYAD_NORM_NONE && !p.h)) return DYAD_ERR_INVALID_ARG;
    return launch_status(dyad::launch_add_norm(p, dyad::drop_args(args->p, args->seed, args->offset, args->offset_dev), stream));
}

size_t dyad_add_norm_workspace_bytes(const dyad_add_norm_args *args, const dyad_add_norm_grads *grads) {
    dyad::AddNormPass p;
    if (!grads || norm_pass(args, grads, p)) return 0;
    return dyad::add_norm_workspace(p);
}

int dyad_add_norm_backward(const dyad_add_norm_args *args, const dyad_add_norm_grads *grads, void *workspace,
                           size_t workspace_bytes, hipStream_t stream) {
    if (!grads) return DYAD_ERR_INVALID_ARG;
    dyad::AddNormPass p;
    const int rc = norm_pass(args, grads, p);
    if (rc) return rc;
    if (p.M > 0) {
        if (p.dout && ((!p.h && !p.x) || !p.stats)) return DYAD_ERR_INVALID_ARG;
        if (p.post != DYAD_NORM_NONE && !p.post_stats) return DYAD_ERR_INVALID_ARG;
    }
    if (!aligned16(workspace)) return DYAD_ERR_ALIGN;
    const size_t need = dyad::add_norm_workspace(p);
    if (need > 0 && (!workspace || workspace_bytes < need)) return DYAD_ERR_WORKSPACE;
    p.ws = workspace;
    return launch_status(dyad::launch_add_norm_grad(p, dyad::drop_args(args->p, args->seed, args->offset, args->offset_dev), stream));
}

size_t dyad_linear_ce_workspace_bytes(dyad_ce_pass pass_arg, int64_t M, int64_t n, int64_t V, dyad_dtype dtype_arg) {
    const int pass = enum_value(pass_arg), dtype = enum_value(dtype_arg);
    if (loss_sizes(M, n, V, dtype) || (pass != DYAD_CE_FORWARD && pass != DYAD_CE_BACKWARD)) return 0;
    return dyad::loss_workspace(pass == DYAD_CE_BACKWARD, M, n, V, dtype);
}

static int loss_call(bool backward, dyad::LossPass &p, size_t workspace_bytes, hipStream_t stream) {
    const int rc = loss_sizes(p.M, p.n, p.V, p.dtype);
    if (rc) return rc;
    if (p.reduction != DYAD_REDUCE_NONE && p.reduction != DYAD_REDUCE_SUM && p.reduction != DYAD_REDUCE_MEAN)
        return DYAD_ERR_INVALID_ARG;
    const bool one = p.reduction != DYAD_REDUCE_NONE, mean = p.reduction == DYAD_REDUCE_MEAN;
    if (!p.W || (p.M > 0 && (!p.X || !p.targets || !p.lse)) || (mean && !p.count)) return DYAD_ERR_INVALID_ARG;
    if (backward ? p.M > 0 && !p.dloss : (p.M > 0 || one) && !p.loss) return DYAD_ERR_INVALID_ARG;
    for (const void *q : {p.X, p.W, (const void *)p.targets, (const void *)p.loss, (const void *)p.lse,
                          (const void *)p.count, (const void *)p.dloss, (const void *)p.dX, (const void *)p.dW,
                          (const void *)p.ws})
        if (!aligned16(q)) return DYAD_ERR_ALIGN;
    if (backward && !p.dX && !p.dW) return DYAD_OK;
    const size_t need = dyad::loss_workspace(backward, p.M, p.n, p.V, p.dtype);
    if (need > 0 && (!p.ws || workspace_bytes < need)) return DYAD_ERR_WORKSPACE;
    return launch_status(backward ? dyad::launch_loss_backward(p, stream) : dyad::launch_loss_forward(p, stream));
}

int dyad_linear_ce_forward(int64_t M, int64_t n, int64_t V, dyad_dtype dtype, const void *X, const void *W,
                           const int64_t *targets, int64_t ignore_index, dyad_reduction reduction, float *loss,
                           float *lse, float *count, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    dyad::LossPass p{};
    p.M = M; p.n = n; p.V = V; p.dtype = enum_value(dtype); p.reduction = enum_value(reduction);
    p.X = X; p.W = W; p.targets = targets; p.ignore = ignore_index; p.loss = loss; p.lse = lse; p.count = count;
    p.ws = workspace;
    return loss_call(false, p, workspace_bytes, stream);
}

int dyad_linear_ce_backward(int64_t M, int64_t n, int64_t V, dyad_dtype dtype, const void *X, const void *W,
                            const int64_t *targets, int64_t ignore_index, dyad_reduction reduction, const float *lse,
                            const float *count, const float *dloss, void *dX, void *dW, void *workspace,
                            size_t workspace_bytes, hipStream_t stream) {
    dyad::LossPass p{};
    p.M = M; p.n = n; p.V = V; p.dtype = enum_value(dtype); p.reduction = enum_value(reduction);
    p.X = X; p.W = W; p.targets = targets; p.ignore = ignore_index;
    p.lse = const_cast<float *>(lse); p.count = const_cast<float *>(count); p.dloss = dloss; p.dX = dX; p.dW = dW;
    p.ws = workspace;
    return loss_call(true, p, workspace_bytes, stream);
}

}  // extern "C"
