/*
 * libdyad -- the Dyad layer (arXiv 2312.06881) on AMD Instinct MI355X (gfx950).
 *
 * A Dyad layer replaces the dense weight W (n_out x n_in) of y = W x + b
 * (Sec. 2.1) by the sum of two sparse components (Sec. 2.2, Eq. 1), each stored
 * as a 3-D tensor of n_dyad blocks:
 *   W1 = BlockDiag  [n_dyad][bo][bi]   (Sec. 2.2.1, Eq. 2)
 *   W2 = BlockTrans [n_dyad][bo][bi]   (Sec. 2.2.2, Eq. 5-10)
 * With D = n_dyad, bi = ceil(n_in/D), bo = ceil(n_out/D), entry W_c[i][j][k]
 * sits in the dense W at (row, col):
 *   W1, every variant:  (i*bo + j, i*bi + k)
 *   W2, DYAD_IT:        (i*bo + j, k*D  + i)   input transposed   (Eq. 9-10)
 *   W2, DYAD_OT:        (j*D  + i, i*bi + k)   output transposed  (Sec. 2.4.1, Eq. 11-13)
 *   W2, DYAD_DT:        (j*D  + i, k*D  + i)   both               (Sec. 2.4.2, Eq. 14-16)
 * (The paper's n_in/n_out are per-block sizes; here n_in/n_out are the full
 * layer widths, and bi/bo the per-block ones.)
 * Widths that n_dyad does not divide are zero-padded up to D*bi and D*bo
 * (appendix, caveat on rectangular W): the layer acts as the one of widths
 * D*bi -> D*bo on X with zero columns appended, and only its first n_out
 * outputs exist.  Entries whose row is >= n_out or whose column is >= n_in
 * have no effect, and their gradients are zero.  Such widths run on
 * zero-padded copies of the blocks or on the general kernels.
 *
 * Layouts: every activation is token-major and row-major: X[M][n_in],
 * Y, H, dZ [M][n_out], dX, H_in [M][n_in]; W1, W2, dW1, dW2 as above; bias and
 * db [n_out].  All tensors are contiguous device memory of the call's dtype,
 * every non-NULL pointer 16-byte aligned.  Arithmetic accumulates in fp32;
 * bf16 results are rounded to nearest even.
 *
 * Ownership and ordering: the caller allocates and owns every buffer, the
 * dW workspace included; dyad_backward_dw allocates nothing (its fp32 partial
 * sums, the de-interleaved copies of dZ and / or X at n_dyad 3, 6, 8 and 16
 * with large batches, and for shapes the fused tiles refuse the zero-padded
 * block copies of dZ and X and the padded gradients all live in the
 * workspace the caller passes).
 * dyad_forward and dyad_backward_dx are the one bounded departure from
 * "caller owns everything": they may keep intermediates in a library-owned
 * device buffer, one per (device, stream), taken in stream order from a
 * per-device memory pool the first time that stream needs it, regrown in
 * stream order when a later call needs more, and kept until the process
 * ends.  It holds the fp32 partial sums of a split reduction (small batches,
 * few output tiles; a few slices of M x n_out fp32, at most 2 GiB); with large
 * batches at n_dyad 2, 3, 4, 6, 8 and 16, by the token chunk, a de-interleaved
 * copy of the input, fp32 slices of the output or its bf16 results before
 * they are interleaved, and for an input gradient a copy of W1; for shapes
 * the fused tiles refuse (from 512 tokens), zero-padded block copies of the
 * input and the weights and one fp32 slice (each form within 2 GiB; the
 * tokens are taken in chunks beyond that).  Calls on one stream share it in
 * stream order, from several host threads too: a call holds the buffer until
 * its last launch is enqueued.  Calls on different streams never share it,
 * but for hipStreamPerThread: its buffer is one for all threads, and a call of
 * another thread than the last waits on the GPU for that one's work.
 * While the stream is being captured into a graph the buffer is never
 * allocated or regrown; when it cannot be had (capture, or the pool fails),
 * the call runs a plan that needs none, with the same results up to the order
 * of the fp32 sums.  A call captured while its stream has a buffer uses that buffer at every replay (it
 * is kept for the graph if the stream's is regrown later), so replays and
 * other calls on the stream the graph was captured from must be ordered with
 * each other; where they are not, capture on a stream that no other call uses.
 * Every call only enqueues work on `stream`
 * (NULL = the null stream) and returns without synchronising; results are
 * valid once that work completes.  Outputs are overwritten, never accumulated
 * into.
 *
 * Errors: each call returns DYAD_OK (0) or a negative dyad_status.  All
 * argument checks run before any HIP call, so a rejected call touches no
 * device state.  M == 0 is a valid, empty batch.
 */
#ifndef DYAD_H
#define DYAD_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { DYAD_IT = 0, DYAD_OT = 1, DYAD_DT = 2 } dyad_variant; /* Sec. 2.2, 2.4 */
typedef enum { DYAD_F32 = 0, DYAD_BF16 = 1 } dyad_dtype;
typedef enum { DYAD_ACT_NONE = 0, DYAD_ACT_GELU = 1 } dyad_act; /* GELU(x) = x * Phi(x), erf form */

typedef enum {
    DYAD_OK = 0,
    DYAD_ERR_INVALID_ARG = -1, /* unknown enum, size < 0 (M) or <= 0 (n_in, n_out, n_dyad), size overflow, NULL required pointer */
    DYAD_ERR_SHAPE = -2,       /* the _ex calls with an input activation, dyad_mx4_forward, dyad_add_norm_* and dyad_linear_ce_*: no kernel for this shape */
    DYAD_ERR_ALIGN = -3,       /* a non-NULL pointer is not 16-byte aligned */
    DYAD_ERR_DTYPE = -4,       /* unknown dtype */
    DYAD_ERR_WORKSPACE = -5,   /* a workspace (or the packed weights) NULL or smaller than its _bytes() call says */
    DYAD_ERR_LAUNCH = -6,      /* the HIP runtime rejected a kernel launch */
} dyad_status;

/*
 * Forward pass, Sec. 2.2 Eq. 1: Y[m] = W X[m] + bias for every token m, with W
 * assembled from W1, W2 by the variant's maps.  bias may be NULL (no bias).
 * act == DYAD_ACT_GELU returns Y = GELU(W X + bias); then, when H is not NULL,
 * H receives the pre-activation W X + bias (what dyad_backward_dx needs as
 * H_in for the next layer).  H is ignored when act == DYAD_ACT_NONE.
 * X, Y may be NULL when M == 0.
 */
int dyad_forward(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M,
                 dyad_dtype dtype, const void *X, const void *W1, const void *W2,
                 const void *bias, dyad_act act, void *Y, void *H, hipStream_t stream);

/*
 * dyad_forward for callers that cannot allocate device memory: code under HIP
 * graph capture, tight serving loops, harnesses that forbid allocation.
 * Same arguments, checks and results as dyad_forward (outputs within the
 * same tolerance; the same plan, hence the same bits, whenever that plan's
 * scratch fits).  It calls no hipMalloc, hipFree or allocating routine: where
 * dyad_forward would take a split-reduction or large-batch buffer from its
 * per-stream pool, this call takes it from a fixed static device array of
 * 64 MiB (one per GPU the library runs on, held until the process ends; its
 * address is looked up once per device).  A plan that would need more than
 * 64 MiB of scratch is refused by the scratch array, and the call runs a plan
 * that needs none.  No part of the array needs to start at zero: every plan
 * writes each partial-sum slice in full before reading it.  All calls on one
 * GPU share the one array: two calls whose work overlaps in time on that GPU
 * (different streams, or different host threads without ordering) race and
 * give undefined results; calls ordered on one stream are safe.
 */
int dyad_forward_noalloc(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M,
                         dyad_dtype dtype, const void *X, const void *W1, const void *W2,
                         const void *bias, dyad_act act, void *Y, void *H, hipStream_t stream);

/*
 * dyad_forward for a layer whose input is an activation of X: with
 * act_in == DYAD_ACT_GELU it computes Y = W GELU(X) + bias (then act and H as
 * in dyad_forward), where X is the stashed pre-activation of the layer before
 * (the H that dyad_forward wrote for it) -- the second layer of a feed-forward
 * block fc1 -> GELU -> fc2 whose activation is never written to memory
 * (the paper times that block as one unit, Sec. 3.3; the concatenated-component
 * idea of Sec. 3.4.3 is carried further by fusing the activation too).  GELU
 * is applied to the input operand as it is staged, in fp32, rounded once to
 * bf16.  act_in == DYAD_ACT_NONE is exactly dyad_forward.  With GELU it runs
 * on the matrix-core tiles only: bf16 (else DYAD_ERR_DTYPE), n_dyad in
 * {1, 2, 4, 8, 16} dividing both widths, input blocks a multiple of 32, output
 * blocks a multiple of 64, and no output transpose (Dyad-OT / -DT) above
 * n_dyad 4; any other shape returns DYAD_ERR_SHAPE before any launch.
 */
int dyad_forward_ex(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M,
                    dyad_dtype dtype, dyad_act act_in, const void *X, const void *W1, const void *W2,
                    const void *bias, dyad_act act, void *Y, void *H, hipStream_t stream);

/*
 * Input gradient of y = W x + b (the paper gives no backward pass; this is the
 * gradient of Eq. 1): dX[m] = W^T dZ[m], where dZ is the gradient w.r.t. this
 * layer's linear output.  If this layer's input was X = GELU(H_in)
 * (act_in == DYAD_ACT_GELU), dX is returned already multiplied by GELU'(H_in),
 * i.e. it is the gradient w.r.t. H_in; H_in [M][n_in] is then required.
 * dZ, dX may be NULL when M == 0.
 */
int dyad_backward_dx(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M,
                     dyad_dtype dtype, const void *dZ, const void *W1, const void *W2,
                     dyad_act act_in, const void *H_in, void *dX, hipStream_t stream);

/*
 * Weight and bias gradients of Eq. 1: dW_c[i][j][k] = sum_m dZ[m][row] X[m][col]
 * over the (row, col) the entry occupies, db[f] = sum_m dZ[m][f].  dbias may be
 * NULL.  The sums over m are taken in a fixed order, so results are bitwise
 * reproducible run to run.  workspace must hold dyad_dw_workspace_bytes() bytes
 * (it may be NULL when that is 0); its contents on entry do not matter.
 * With M == 0 the gradients are zero.
 */
int dyad_backward_dw(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M,
                     dyad_dtype dtype, const void *dZ, const void *X, void *dW1, void *dW2,
                     void *dbias, void *workspace, size_t workspace_bytes, hipStream_t stream);

/* Workspace bytes dyad_backward_dw needs for these arguments (0 if none, or if they are invalid). */
size_t dyad_dw_workspace_bytes(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad,
                               int64_t M, dyad_dtype dtype);

/*
 * Weight and bias gradients of the layer of dyad_forward_ex: with
 * act_in == DYAD_ACT_GELU the layer's input is GELU(X), X the stashed
 * pre-activation, formed as X is staged (dW_c[i][j][k] = sum_m dZ[m][row]
 * GELU(X[m][col])); db as in dyad_backward_dw.  act_in == DYAD_ACT_NONE is
 * exactly dyad_backward_dw.  With GELU: bf16 (else DYAD_ERR_DTYPE), n_dyad in
 * {1, 2, 4, 8, 16} dividing both widths into blocks of multiples of 64, else
 * DYAD_ERR_SHAPE before any launch.  workspace must hold
 * dyad_dw_workspace_bytes_ex() bytes for the same arguments.
 */
int dyad_backward_dw_ex(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M,
                        dyad_dtype dtype, dyad_act act_in, const void *dZ, const void *X, void *dW1, void *dW2,
                        void *dbias, void *workspace, size_t workspace_bytes, hipStream_t stream);

/* Workspace bytes dyad_backward_dw_ex needs (0 if none, or if the arguments are invalid or unsupported). */
size_t dyad_dw_workspace_bytes_ex(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad,
                                  int64_t M, dyad_dtype dtype, dyad_act act_in);

/*
 * ---- Microscaled formats -------------------------------------------------------
 *
 * OCP microscaling (MX): 32 consecutive values of a row share a scale byte s,
 * the power of two 2^(s - 127), and each keeps an 8- or 4-bit element:
 *   DYAD_MX_INT8  two's complement k, the value k / 64 * 2^(s - 127), |k| <= 127
 *   DYAD_MX_FP4   sign and one of 0, .5, 1, 1.5, 2, 3, 4, 6, times 2^(s - 127)
 * s - 127 is floor(log2) of the block's largest magnitude, less 2 for fp4;
 * elements are rounded to nearest even and saturate.  A block of zeros reads
 * back as zeros.  A block that holds an infinity or a NaN gets s = 255 and reads
 * back as NaN throughout.  A row's last block may be short.
 *
 * The calls below take the same kinds of arguments and give the same
 * guarantees as those above: they only enqueue work on `stream`, allocate
 * nothing (every buffer, the workspaces too, is the caller's; a workspace's
 * contents on entry do not matter), overwrite their outputs, and check every
 * argument before any HIP call.  Only dyad_forward_mx8 and
 * dyad_backward_dx_mx8 may use the per-stream buffer of dyad_forward.
 */
typedef enum { DYAD_MX_INT8 = 0, DYAD_MX_FP4 = 1 } dyad_mx_format;

/*
 * X [rows][cols] of dtype, row-major, into codes and scales [rows][ceil(cols/32)]
 * (one byte each), and back.  int8 codes are [rows][cols]; fp4 codes
 * [rows][ceil(cols/2)] bytes, an even column in the low nibble.  Reading back
 * is exact in fp32, and in bf16 but for fp4 and int8 steps below bf16's
 * smallest subnormal.  rows == 0 is valid.
 */
int dyad_mx_quantize(dyad_mx_format format, int64_t rows, int64_t cols, dyad_dtype dtype, const void *X, void *codes,
                     void *scales, hipStream_t stream);
int dyad_mx_dequantize(dyad_mx_format format, int64_t rows, int64_t cols, dyad_dtype dtype, const void *codes,
                       const void *scales, void *Y, hipStream_t stream);

/*
 * Weights of one layer for dyad_mx4_forward: W1, W2 [n_dyad][bo][bi] of dtype
 * quantised to fp4 along the reduction (each row of a block on its own; entries
 * of padded rows or columns are zero), into dyad_mx4_weight_bytes() bytes whose
 * layout is the library's own.  The variant is part of the result.
 * dyad_mx4_weight_bytes is 0 for invalid arguments.
 */
size_t dyad_mx4_weight_bytes(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad);
int dyad_mx4_quantize_weights(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad, dyad_dtype dtype,
                              const void *W1, const void *W2, void *packed, size_t packed_bytes, hipStream_t stream);

/*
 * Forward pass on fp4 operands: Y[m] = act(W Q(X)[m] + bias), summed in fp32 and
 * rounded once to dtype, where W holds the quantised entries and each component
 * sees X quantised to fp4 in its own block order: component 1 the blocks
 * X[m][i*bi + k], component 2 the same or, under an input transpose, the
 * residues X[m][k*n_dyad + i], 32 consecutive k to a scale.  X is quantised within
 * the call, each token on its own, into the workspace of
 * dyad_mx4_workspace_bytes() bytes (0 for a few tokens of a narrow layer).  With Dyad-OT / -DT, n_dyad above 32 returns
 * DYAD_ERR_SHAPE.
 */
size_t dyad_mx4_workspace_bytes(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M);
int dyad_mx4_forward(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M, dyad_dtype dtype,
                     const void *X, const void *packed, size_t packed_bytes, const void *bias, dyad_act act, void *Y,
                     void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Training with activations checkpointed in DYAD_MX_INT8 (codes and scales as
 * dyad_mx_quantize writes them, along each token's row):
 *   dyad_forward_mx8      dyad_forward with GELU, whose pre-activation H is kept as
 *                         H8 / Hs, the quantised value of what H would hold (in
 *                         fp32: of H summed in 64 bits and rounded once)
 *   dyad_backward_dx_mx8  dyad_backward_dx with act_in GELU at the kept H:
 *                         dX = (W^T dZ) * GELU'(H8).  A, when not NULL, receives
 *                         GELU(H8) [M][n_in], this layer's input, for the weight
 *                         gradient (dyad_backward_dw)
 *   dyad_backward_dw_mx8  dyad_backward_dw with X read from X8 / Xs; with act_in
 *                         GELU the layer's input is GELU(X8)
 * H8 [M][n_out] for the forward pass, [M][n_in] for the input gradient; X8 [M][n_in].
 * The workspace holds dyad_mx8_workspace_bytes() bytes for the pass (act_in
 * counts for the weight gradient only): none for forward passes and input
 * gradients whose kernels keep and read 8 bits themselves (most bf16 layers
 * without padding), at most 64 MB or 1024 tokens of them for the others.
 */
typedef enum { DYAD_MX8_FORWARD = 0, DYAD_MX8_DX = 1, DYAD_MX8_DW = 2 } dyad_mx8_pass;
size_t dyad_mx8_workspace_bytes(dyad_mx8_pass pass, dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad,
                                int64_t M, dyad_dtype dtype, dyad_act act_in);
int dyad_forward_mx8(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M, dyad_dtype dtype,
                     const void *X, const void *W1, const void *W2, const void *bias, void *Y, void *H8, void *Hs,
                     void *workspace, size_t workspace_bytes, hipStream_t stream);
int dyad_backward_dx_mx8(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M,
                         dyad_dtype dtype, const void *dZ, const void *W1, const void *W2, const void *H8,
                         const void *Hs, void *dX, void *A, void *workspace, size_t workspace_bytes, hipStream_t stream);
int dyad_backward_dw_mx8(dyad_variant variant, int64_t n_in, int64_t n_out, int64_t n_dyad, int64_t M,
                         dyad_dtype dtype, dyad_act act_in, const void *dZ, const void *X8, const void *Xs, void *dW1,
                         void *dW2, void *dbias, void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * ---- Around the Dyad layers of a language model --------------------------------
 *
 * Dropout, the residual stream with its norms, and the loss over a vocabulary.  The
 * calls only enqueue work on `stream`, allocate nothing, overwrite their outputs, and
 * check every argument before any HIP call; every non-NULL pointer is 16-byte
 * aligned (offset_dev: 8); sums are fp32 and results are rounded once, and repeat bit by bit.
 *
 * Dropout draws its mask from a counter, so that none is stored: of a matrix of
 * `cols` columns, value j of octet o = row * ceil(cols / 8) + col / 8 (j = col % 8)
 * has bits 16 (j % 2) .. + 15 of word j / 2 of Philox-4x32-10 at the counter
 * (o, offset) and the key seed, 64 bits each, low words first.  It is dropped where
 * they are below t = rint(65536 p); the others are scaled by 65536 / (65536 - t).
 * (p is so a multiple of 2^-16, and the scale goes with what is dropped; p == 1
 * drops everything.)  What is dropped becomes 0 whatever it was.  offset_dev, when
 * not NULL, is a value in device memory that is added to offset: a captured call
 * draws another mask at every replay if the program changes it in between.
 */

/* Y = X dropped and scaled; the gradient is the same call on dY.  Y may be X.  cols <= 2^31 - 16. */
int dyad_dropout(int64_t rows, int64_t cols, dyad_dtype dtype, const void *X, double p, uint64_t seed, uint64_t offset,
                 const uint64_t *offset_dev, void *Y, hipStream_t stream);

/*
 *   h   = x_scale x + y_scale gate * drop(post(y))
 *   out = norm(h)
 * x is the residual stream [M][n], y a block's output; out is the next block's input.
 * LAYER: norm(v) = (v - mean) / sqrt(mean((v - mean)^2) + eps) weight + bias over a
 * row, RMS: v / sqrt(mean(v^2) + eps) weight + bias.  8 <= n <= 16384, else
 * DYAD_ERR_SHAPE.
 *
 * x and h have stream_dtype, y and out dtype: both bf16, both fp32, or an fp32 stream
 * with bf16 blocks (else DYAD_ERR_DTYPE).  The parameters (weights, biases, gate) have
 * param_dtype, fp32 or, with bf16 blocks, bf16.  out is the norm of h before it is
 * rounded.
 *
 * May be NULL: y (then h = x_scale x, and post, gate and p have no effect); h; weight,
 * bias, post_weight, post_bias (1 and 0); gate (1); stats and post_stats, which a
 * backward pass needs.  gate is [groups][n]: row m takes gate row m / (M / groups), and
 * groups divides M.  norm == NONE: out is not written.  h may be x, and out y where
 * their types agree.
 */
typedef enum { DYAD_NORM_NONE = 0, DYAD_NORM_LAYER = 1, DYAD_NORM_RMS = 2 } dyad_norm;
typedef struct {
    int64_t M, n, groups;
    dyad_dtype stream_dtype, dtype, param_dtype;
    dyad_norm norm, post;
    float x_scale, y_scale, eps;
    double p;                    /* dropout of post(y); 0: none */
    uint64_t seed, offset;
    const uint64_t *offset_dev;
    const void *x, *y, *weight, *bias, *post_weight, *post_bias, *gate;
    void *h, *out;
    float *stats, *post_stats;   /* [M][2]: mean and 1 / sqrt(...) of h's rows, and of y's */
} dyad_add_norm_args;
int dyad_add_norm_forward(const dyad_add_norm_args *args, hipStream_t stream);

/*
 * The gradients.  args is the forward call's, with stats (with a norm) and post_stats
 * (with a post norm) as it wrote them.  h is formed again from x and y, or with x NULL
 * read as the forward pass wrote it: a bf16 stream's rounding of h is then in the
 * gradients of the norm's weights.  y's values are read where h is formed again, with a
 * post norm, and for dgate.  out is not read.  dh is the gradient that reaches h, dout that which reaches
 * out; either may be NULL (none).  Of the results any may be NULL: dx [M][n] of
 * stream_dtype, dy [M][n] of dtype, those of the parameters (of param_dtype), dgate
 * [groups][n].  dx may be dh, and dy dout where their types agree.  The workspace holds
 * dyad_add_norm_workspace_bytes() bytes for the same arguments (0 for invalid ones).
 * M == 0 gives zero gradients of the parameters.
 */
typedef struct {
    const void *dh, *dout;
    void *dx, *dy, *dweight, *dbias, *dpost_weight, *dpost_bias, *dgate;
} dyad_add_norm_grads;
size_t dyad_add_norm_workspace_bytes(const dyad_add_norm_args *args, const dyad_add_norm_grads *grads);
int dyad_add_norm_backward(const dyad_add_norm_args *args, const dyad_add_norm_grads *grads, void *workspace,
                           size_t workspace_bytes, hipStream_t stream);

/*
 * Softmax cross entropy of the logits Z = X W^T, which are never kept: X [M][n] the
 * tokens, W [V][n] the vocabulary's rows.  A token's loss is log(sum_v exp Z[m][v]) -
 * Z[m][target]; a target that is ignore_index, or lies outside 0 .. V - 1, counts for
 * nothing: loss 0, no gradient.  reduction NONE: loss [M]; SUM, MEAN over the tokens
 * that count (0 where none does): loss [1].  lse [M] and, for MEAN, count [1] (the
 * tokens that count) are what the backward pass needs of the forward one; lse of a
 * token that does not count has no meaning.
 *
 * Backward: dloss, of loss's length, is the gradient that reaches it; dX [M][n] and
 * dW [V][n], either of which may be NULL, are the gradients.  The logits are formed
 * again, a piece of the vocabulary at a time.  With bf16 operands their gradient G, W
 * and X times dloss enter the products in fp16 at powers of two: one a column for W and for
 * X times dloss, whose values below 2^-39 of the column's largest become zero; 2^15 for G,
 * whose values below 2^-39 become zero in dX, and in dW only beside larger ones in their row
 * (a row whose largest is under 2^-24 has a power of its own).  The sums are fp32.
 *
 * M, V <= 2^22, M V <= 2^38 and n <= 2^20, else DYAD_ERR_SHAPE.  The workspace holds
 * dyad_linear_ce_workspace_bytes() bytes for the pass (0 for invalid arguments): about
 * M n values twice, and for the pieces up to 512 MB of G, 256 MB of sums and 768 MB of W
 * laid out otherwise (or 65536 / ceil(M / 256) rows of W, at 2 bytes a value in bf16 and 6 in
 * fp32, where that is more).  For few tokens that is more than their logits would take.
 */
typedef enum { DYAD_REDUCE_NONE = 0, DYAD_REDUCE_SUM = 1, DYAD_REDUCE_MEAN = 2 } dyad_reduction;
typedef enum { DYAD_CE_FORWARD = 0, DYAD_CE_BACKWARD = 1 } dyad_ce_pass;
size_t dyad_linear_ce_workspace_bytes(dyad_ce_pass pass, int64_t M, int64_t n, int64_t V, dyad_dtype dtype);
int dyad_linear_ce_forward(int64_t M, int64_t n, int64_t V, dyad_dtype dtype, const void *X, const void *W,
                           const int64_t *targets, int64_t ignore_index, dyad_reduction reduction, float *loss,
                           float *lse, float *count, void *workspace, size_t workspace_bytes, hipStream_t stream);
int dyad_linear_ce_backward(int64_t M, int64_t n, int64_t V, dyad_dtype dtype, const void *X, const void *W,
                            const int64_t *targets, int64_t ignore_index, dyad_reduction reduction, const float *lse,
                            const float *count, const float *dloss, void *dX, void *dW, void *workspace,
                            size_t workspace_bytes, hipStream_t stream);

/* Static, human-readable text for a dyad_status value. */
const char *dyad_strerror(int status);

#ifdef __cplusplus
}
#endif

#endif /* DYAD_H */
