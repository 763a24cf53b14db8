// Softmax cross entropy of z = X W^T against targets, z never kept: loss = lse(z) - z_target.
// Forward: tiles of logits leave (largest, sum of exponentials) per token, joined here.
// Backward, a piece of the vocabulary at a time: the tiles' logits again, as
// G = dloss (exp(z - lse) - onehot), then dX += G W and dW = G^T X of the piece.  Forming z
// twice is 8 M n V operations for the four products where 6 M n V would do with z kept.  That
// takes the memory for M V values, and writing and reading them at 4 bytes: 1.5 ps each at a large
// copy's rate, where forming one takes 1.1 ps at 768 columns and 6 at 4096.
#include "lm_internal.h"

namespace dyad {

namespace {

// A wave a token: joins the tiles' statistics.
__global__ void __launch_bounds__(256) loss_join_kernel(LossEpi e, int64_t M, LossTokens tokens, float *loss, float *lse) {
    const int lane = threadIdx.x & 63;
    if (tokens.count) M = *tokens.count;
    for (int64_t c = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); c < M; c += (int64_t)gridDim.x * 4) {
        const int64_t m = tokens.idx ? tokens.idx[c] : c;
        float2 s = make_float2(-INFINITY, 0.f);
        for (int t = lane; t < e.tiles; t += 64) s = join_stats(s, e.part[c * e.tiles + t]);
#pragma unroll
        for (int w = 32; w > 0; w >>= 1) s = join_stats(s, make_float2(__shfl_xor(s.x, w), __shfl_xor(s.y, w)));
        if (lane == 0) {
            const float l = s.x + logf(s.y);
            lse[m] = l;
            loss[m] = loss_counts(e, e.targets[m]) ? l - e.at_target[c] : 0.f;
        }
    }
}

// Sum over the tokens, in 64 bits and a fixed order, and how many count; the mean of none is 0.
__global__ void __launch_bounds__(1024) loss_sum_kernel(LossEpi e, int64_t M, const float *each, bool mean, float *loss,
                                                        float *count) {
    __shared__ double sums[16];
    __shared__ int64_t counts[16];
    double s = 0.0;
    int64_t c = 0;
    for (int64_t m = threadIdx.x; m < M; m += 1024) {
        s += (double)each[m];
        c += loss_counts(e, e.targets[m]) ? 1 : 0;
    }
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) {
        s += __shfl_xor(s, w);
        c += __shfl_xor(c, w);
    }
    if ((threadIdx.x & 63) == 0) {
        sums[threadIdx.x >> 6] = s;
        counts[threadIdx.x >> 6] = c;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        c = 0;
        for (int w = 0; w < 16; ++w) {
            s += sums[w];
            c += counts[w];
        }
        *loss = (float)(mean && c > 0 ? s / (double)c : s);
        if (count) *count = (float)c;
    }
}

__global__ void __launch_bounds__(256) zero_kernel(uint16_t *p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = 0;
}

// Which fp32 calls run on fp32 matrix instructions.
bool plain_f32(int64_t M, int dtype) { return dtype == kF32 && M < kSplitFrom; }

// Vocabulary columns of a piece on fp32 matrix instructions: dX's sums in one accumulator are no
// longer than that.  (Over 524288 columns, beside a target's term of the whole gradient's size, the
// terms below half of the sum's last bit were lost, 1e-3 of dX.)
int64_t f32_piece(int64_t V) { return V < 16384 ? V : 16384; }

// Every token's loss, its target's logit and the tiles' statistics.
size_t stats_bytes(int64_t M, int64_t tiles) { return (size_t)up(2 * up(M, 4) * 4 + M * tiles * 8, 256); }

LossEpi epi_of(const LossPass &p) {
    LossEpi e{};
    e.targets = p.targets;
    e.ignore = p.ignore;
    e.V = p.V;
    e.lse = p.lse;
    e.dloss = p.dloss;
    e.count = p.count;
    e.reduction = p.reduction;
    return e;
}

}  // namespace

size_t loss_workspace(bool backward, int64_t M, int64_t n, int64_t V, int dtype) {
    if (M == 0) return 0;
    const bool f32 = dtype == kF32, plain = plain_f32(M, dtype);
    if (backward) return plain ? (size_t)(M * f32_piece(V)) * 4 : loss_mfma_backward_bytes(M, n, V, f32);
    return plain ? stats_bytes(M, loss_f32_tiles(M, V))
                 : stats_bytes(M, loss_mfma_tiles(M, n, V, f32)) + loss_mfma_forward_bytes(M, n, V, f32);
}

hipError_t launch_loss_forward(const LossPass &p, hipStream_t s) {
    LossEpi e = epi_of(p);
    float *each = static_cast<float *>(p.ws);
    if (p.M > 0) {
        e.at_target = each + up(p.M, 4);
        e.part = reinterpret_cast<float2 *>(e.at_target + up(p.M, 4));
        if (p.reduction == kReduceNone) each = p.loss;
        const bool plain = plain_f32(p.M, p.dtype);
        e.tiles = plain ? loss_f32_tiles(p.M, p.V) : loss_mfma_tiles(p.M, p.n, p.V, p.dtype == kF32);
        LossTokens tokens{};
        const hipError_t err = plain ? launch_loss_f32_stats(p, e, s)
                                     : launch_loss_mfma_stats(p, e, static_cast<char *>(p.ws) + stats_bytes(p.M, e.tiles),
                                                              each, tokens, s);
        if (err != hipSuccess) return err;
        const int64_t blocks = (p.M + 3) / 4;
        loss_join_kernel<<<(unsigned)(blocks < 8192 ? blocks : 8192), 256, 0, s>>>(e, p.M, tokens, each, p.lse);
    }
    if (p.reduction != kReduceNone)
        loss_sum_kernel<<<1, 1024, 0, s>>>(e, p.M, each, p.reduction == kReduceMean, p.loss, p.count);
    return hipGetLastError();
}

hipError_t launch_loss_backward(const LossPass &p, hipStream_t s) {
    if (p.M == 0) {
        if (!p.dW) return hipSuccess;
        zero_kernel<<<1024, 256, 0, s>>>(static_cast<uint16_t *>(p.dW), p.n * p.V * (p.dtype == kF32 ? 2 : 1));
        return hipGetLastError();
    }
    const LossEpi e = epi_of(p);
    if (!plain_f32(p.M, p.dtype)) return launch_loss_mfma_grad(p, e, s);
    const int64_t piece = f32_piece(p.V);
    for (int64_t v0 = 0; v0 < p.V; v0 += piece) {
        const hipError_t err = launch_loss_f32_piece(p, e, v0, p.V - v0 < piece ? p.V - v0 : piece,
                                                     static_cast<float *>(p.ws), v0 == 0, s);
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

}  // namespace dyad
