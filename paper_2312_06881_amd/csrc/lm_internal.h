// Internal interface of the operators around the Dyad layers of a language model:
// dropout, norms with gate and residual, the loss over a vocabulary.
#pragma once

#include "dyad_internal.h"

namespace dyad {

struct DropArgs;   // philox.h

inline int64_t up(int64_t v, int64_t q) { return (v + q - 1) / q * q; }   // to a multiple of q

hipError_t launch_dropout(int64_t rows, int64_t cols, int dtype, const void *x, const DropArgs &d, void *y, hipStream_t s);

// ---- h = x_scale x + y_scale gate * drop(post(y)),  out = norm(h) -------------------

constexpr int kNormNone = 0, kNormLayer = 1, kNormRms = 2;
constexpr int64_t kNormMaxWidth = 16384;   // a row stays in the registers of one workgroup

struct AddNormPass {
    int64_t M, n;
    int64_t groups;              // rows of the gate; row m takes gate row m / (M / groups)
    int stream_dtype, dtype, param_dtype;
    int norm, post;
    float x_scale, y_scale, eps;
    const void *x, *y, *w, *b, *pw, *pb, *gate;
    void *h, *out;               // in the backward pass h is read
    float *stats, *post_stats;   // [M][2]: mean and 1 / deviation
    // backward
    const void *dh, *dout;
    void *dx, *dy, *dw, *db, *dpw, *dpb, *dgate;
    void *ws;
};

hipError_t launch_add_norm(const AddNormPass &p, const DropArgs &d, hipStream_t s);
size_t add_norm_workspace(const AddNormPass &p);
hipError_t launch_add_norm_grad(const AddNormPass &p, const DropArgs &d, hipStream_t s);

// ---- softmax cross entropy of X W^T, the vocabulary in pieces ------------------------

constexpr int kReduceNone = 0, kReduceSum = 1, kReduceMean = 2;
// Tokens and vocabulary of a call: offsets within a tile's operand rows are 32-bit.
constexpr int64_t kLossMaxRows = (int64_t)1 << 22;
constexpr int64_t kLossMaxWidth = (int64_t)1 << 20;
constexpr int64_t kLossMaxLogits = (int64_t)1 << 38;   // a launch has fewer than 2^32 threads, 512 to 2^16 logits

struct LossPass {
    int64_t M, n, V;
    int dtype, reduction;
    const void *X, *W;
    const int64_t *targets;
    int64_t ignore;
    float *loss, *lse, *count;   // count: counted tokens; read by the backward pass of a mean
    const float *dloss;
    void *dX, *dW;
    void *ws;
};

constexpr float kLog2e = 1.44269504088896341f;

// What the logits of a tile turn into.
struct LossEpi {
    const int64_t *targets;
    int64_t ignore, V;
    // forward: per token and vocabulary tile the largest logit and the sum of
    // exp(logit - it), [M][tiles]; and the target's logit
    float2 *part;
    float *at_target;
    int tiles;
    // backward: lse, and the loss's gradient
    const float *lse, *dloss, *count;
    int reduction;
};

// A target that counts: in the vocabulary, and not the one to ignore.
__device__ __forceinline__ bool loss_counts(const LossEpi &e, int64_t t) { return t >= 0 && t < e.V && t != e.ignore; }

// The gradient that reaches token m's loss; 0 where it does not count.
__device__ __forceinline__ float loss_scale(const LossEpi &e, int64_t m, int64_t t) {
    if (!loss_counts(e, t)) return 0.f;
    const float g = e.dloss[e.reduction == kReduceNone ? m : 0];
    return e.reduction == kReduceMean ? g / *e.count : g;
}

// (largest logit, sum of exp(logit - it)) of two sets of columns together; (-inf, 0) is the empty set.
__device__ __forceinline__ float2 join_stats(float2 s, float2 t) {
    const float top = fmaxf(s.x, t.x), base = top == -INFINITY ? 0.f : top;
    return make_float2(top, s.y * __builtin_amdgcn_exp2f((s.x - base) * kLog2e) + t.y * __builtin_amdgcn_exp2f((t.x - base) * kLog2e));
}

// Of tile columns v0 .. v0 + BN - 1 in the vocabulary: a wave's WM x WN block of logits,
// acc[i][j][v] that of token 16 i + l % 16 and column 16 j + 4 (l / 16) + v, into the tile's
// statistics.  red: [BM][WGN] float2.  Columns past the vocabulary count for nothing.
template <int SM, int SN, int BM, int WGN, class Acc>
__device__ __forceinline__ void loss_stats(const LossEpi &e, const Acc (&acc)[SM][SN], int64_t m0, int64_t M, int64_t v0,
                                           int tile, int wm0, int wn0, int wave_n, float2 *red) {
    const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
    const int left = (int)(e.V - v0 < ((int64_t)1 << 30) ? e.V - v0 : (int64_t)1 << 30) - wn0 - 4 * lg;   // columns left from this lane's first
#pragma unroll
    for (int i = 0; i < SM; ++i) {
        const int row = wm0 + 16 * i + lr;
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < SN; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (16 * j + v < left) top = fmaxf(top, acc[i][j][v]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < SN; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (16 * j + v < left) sum += __builtin_amdgcn_exp2f((acc[i][j][v] - base) * kLog2e);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (lg == 0) red[row * WGN + wave_n] = make_float2(top, sum);
        if (m0 + row < M) {
            const int64_t t = e.targets[m0 + row] - v0 - wn0 - 4 * lg;
            if (t >= 0 && t < left && t < 16 * SN) {
#pragma unroll
                for (int j = 0; j < SN; ++j)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        if (t == 16 * j + v) e.at_target[m0 + row] = acc[i][j][v];
            }
        }
    }
    __syncthreads();
    for (int row = threadIdx.x; row < BM; row += blockDim.x) {
        if (m0 + row >= M) break;
        float2 s = red[row * WGN];
#pragma unroll
        for (int w = 1; w < WGN; ++w) s = join_stats(s, red[row * WGN + w]);
        e.part[(m0 + row) * e.tiles + tile] = s;
    }
}

hipError_t launch_loss_forward(const LossPass &p, hipStream_t s);
hipError_t launch_loss_backward(const LossPass &p, hipStream_t s);
size_t loss_workspace(bool backward, int64_t M, int64_t n, int64_t V, int dtype);

// Splitting fp32 operands takes a pass over the weights, which fewer tokens do not pay for in the
// forward pass (768 x 50000: 127 us for 128 tokens, 171 split for 129).  With gradients they would
// (2.3 ms against 0.72): the unsplit dX has few workgroups.
constexpr int64_t kSplitFrom = 129;

// fp32 up to there (loss_f32.hip).  Forward: the statistics.  Backward: a piece of the vocabulary,
// columns v0 .. v0 + vp - 1: the logits' gradient G [M][vp], then dX (added to, but for the
// first piece) and dW of the piece; either may be null.
int loss_f32_tiles(int64_t M, int64_t V);
hipError_t launch_loss_f32_stats(const LossPass &p, const LossEpi &e, hipStream_t s);
hipError_t launch_loss_f32_piece(const LossPass &p, const LossEpi &e, int64_t v0, int64_t vp, float *G, bool first,
                                 hipStream_t s);


// bf16, and fp32 from kSplitFrom tokens (loss_mfma.hip).  The statistics (ws: forward_bytes), and the whole backward pass (the
// call's workspace: backward_bytes).
int loss_mfma_tiles(int64_t M, int64_t n, int64_t V, bool f32);
size_t loss_mfma_forward_bytes(int64_t M, int64_t n, int64_t V, bool f32);
size_t loss_mfma_backward_bytes(int64_t M, int64_t n, int64_t V, bool f32);
// Which token row c of the statistics is, and how many rows there are; null: c, and all.
struct LossTokens {
    const int *idx, *count;
};
hipError_t launch_loss_mfma_stats(const LossPass &p, const LossEpi &e, void *ws, float *each, LossTokens &tokens,
                                  hipStream_t s);
hipError_t launch_loss_mfma_grad(const LossPass &p, const LossEpi &e, hipStream_t s);

}  // namespace dyad
