/*
 * mlkv_dense.h -- C ABI of the dense operators beside the embedding store.
 *
 * A training step over the store (mlkv_gpu.h) is Get -> dense network -> loss
 * -> gradients -> the gradient apply.  MLKV leaves the part in between to the
 * application (arXiv 2504.01506, Section 2.1: N(w_nn; E(w_emb; x)); Figure 2,
 * lines 10-16).  These calls are that part's operators: the layer norm of
 * looked-up rows, the matrix product with bias, activation and residual, the
 * log probabilities of given tokens with their entropy and the likeliest
 * alternatives, and the gradients of all three.
 *
 * Conventions shared by every call (as mlkv_gpu.h's where it has them)
 *   - Pointers named d_* are DEVICE pointers owned by the caller.  Buffers must
 *     stay valid until the stream has executed the call.
 *   - A matrix has unit stride along its rows; its row stride is given in
 *     elements, at least the row's length.  Any alignment that the element type
 *     allows is taken.  Inputs may overlap inputs; an output may overlap nothing
 *     else, except where a call says so.
 *   - Element types are MLKV_TYPE_*.  Sums, means, softmax statistics and
 *     accumulators are held in 32 bits; an output is rounded once, to nearest.
 *   - Calls are asynchronous on `stream` (a cudaStream_t; NULL = legacy default
 *     stream), allocate nothing, keep nothing between calls and may be captured
 *     into a CUDA graph.  Calls on different streams or host threads share no
 *     memory but their arguments (and a device's count of waits that ran out, which
 *     mlkv_dense_sync reads).  The stream's device must be current.
 *   - A call that needs working memory has a function that says how many bytes;
 *     the caller gives that much device memory, 256-byte aligned, which the call
 *     uses until it is done on the stream.  It goes by the device that is current.
 *     (-1: the arguments are not valid, or there is no device.)
 *   - Errors a host check finds are returned at once (MLKV_ERR_INVALID,
 *     MLKV_ERR_UNSUPPORTED, MLKV_ERR_CUDA) and nothing is enqueued.
 *   - Results do not change from run to run: no sum's order depends on timing.
 *   - Each call that enqueues work is an NVTX range named after the call.
 */
#ifndef MLKV_DENSE_H
#define MLKV_DENSE_H

#include <stdint.h>

#include "mlkv_gpu.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define MLKV_TYPE_FLOAT 0  /* IEEE fp32 */
#define MLKV_TYPE_BFLOAT 1 /* bfloat16 */
#define MLKV_TYPE_HALF 2   /* IEEE fp16 */

/* Activations of mlkv_linear. */
#define MLKV_ACT_NONE 0
#define MLKV_ACT_RELU 1
#define MLKV_ACT_GELU_TANH 2 /* z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) / 2 */
#define MLKV_ACT_SILU 3      /* z / (1 + exp(-z)) */

/* Most alternatives mlkv_token_logprobs returns per row. */
#define MLKV_MAX_TOP 32

/* Layer norm of `rows` rows of `dim` values: with mu and v the mean and the
 * (biased) variance of a row,
 *     y = (x - mu) / sqrt(v + eps) * weight + bias.
 * x_type: any; y_type: x_type, or any when x_type is MLKV_TYPE_FLOAT (the
 * store's rows enter 16-bit arithmetic here).  d_weight, d_bias: [dim] of
 * w_type, either may be null (1, 0).  d_stats: null, or fp32 [rows][2], which
 * takes each row's (mu, 1 / sqrt(v + eps)) for the backward pass.  0 <= rows < 2^30,
 * 1 <= dim < 2^20, eps >= 0.  d_y may be d_x where types and strides agree. */
int mlkv_layer_norm(const void* d_x, int64_t x_stride, int32_t x_type, int64_t rows, int64_t dim,
                    const void* d_weight, const void* d_bias, int32_t w_type, float eps, void* d_y,
                    int64_t y_stride, int32_t y_type, float* d_stats, void* stream);

/* Its gradients: d_dy of dy_type (the forward's y_type) gives d_dx of x_type
 * and, where not null, d_dweight and d_dbias, [dim] of w_type.  With rows == 0
 * these two are zero.  d_weight null: 1.  d_dx may be d_dy where types and
 * strides agree, or null (not wanted). */
int64_t mlkv_layer_norm_backward_workspace(int64_t rows, int64_t dim);
int mlkv_layer_norm_backward(const void* d_dy, int64_t dy_stride, int32_t dy_type, const void* d_x,
                             int64_t x_stride, int32_t x_type, int64_t rows, int64_t dim, const void* d_weight,
                             int32_t w_type, const float* d_stats, void* d_dx, int64_t dx_stride,
                             void* d_dweight, void* d_dbias, void* d_workspace, int64_t workspace_bytes,
                             void* stream);

/* A matrix product with its epilogue, and its gradients.  All matrices are of
 * `type` (MLKV_TYPE_BFLOAT or MLKV_TYPE_HALF).
 *   forward:   z = x weight^T + bias;  y = act(z) + residual
 *   backward:  p = dy * act'(z);  dx = p weight;  dweight = p^T x;  dbias = sum of p's rows
 *              (the residual's gradient is dy itself)
 * x: [m][k]; weight: [n][k]; bias: [n] or null; residual: [m][n] or null; y:
 * [m][n]; pre: [m][n], z rounded to `type`: an output of the forward pass where
 * not null, an input of the backward pass with an activation (null without).
 * dy: [m][n]; dx: [m][k]; dweight: [n][k]; dbias: [n]; each of the three may be
 * null (not wanted).  m, n, k >= 0, each < 2^30; k == 0 gives z = bias, m == 0
 * gives zero dweight and dbias.  p is rounded to `type` where act is not NONE.
 * With MLKV_ACT_RELU, whose slope jumps there, sums next to 0 are computed again
 * in 64 bits (of more than 64 rows, where a tile's k is not shared out; the
 * smallest of 32 columns at most).  A sum of exactly 0 is such a sum unless all 32
 * are 0: weight rows of zeros, without a bias, cost every row a product in 64 bits for
 * each 32 columns that hold one (65,536 x 416 to 512: 37 us, 304 with one such
 * row, 2,800 with one in each 32). */
typedef struct mlkv_linear_args {
    int64_t m, n, k;
    const void* d_x;
    int64_t x_stride;
    const void* d_weight;
    int64_t weight_stride;
    const void* d_bias;
    const void* d_residual;
    int64_t residual_stride;
    void* d_y;
    int64_t y_stride;
    void* d_pre;
    int64_t pre_stride;
    const void* d_dy;
    int64_t dy_stride;
    void* d_dx;
    int64_t dx_stride;
    void* d_dweight;
    int64_t dweight_stride;
    void* d_dbias;
    void* d_workspace;
    int64_t workspace_bytes;
    int32_t type;
    int32_t activation;
} mlkv_linear_args;

/* The working memory of the two calls below with these arguments (their
 * d_workspace and workspace_bytes are not looked at). */
int64_t mlkv_linear_workspace(const mlkv_linear_args* args);
int64_t mlkv_linear_backward_workspace(const mlkv_linear_args* args);
int mlkv_linear(const mlkv_linear_args* args, void* stream);
int mlkv_linear_backward(const mlkv_linear_args* args, void* stream);

/* Waits for the stream.  MLKV_ERR_TIMEOUT when a bounded wait inside a product's
 * kernel has run out since this was last told (its outputs are then not valid;
 * the product's own call returned before), else MLKV_OK.  What is told is the
 * current device's, of whichever stream, and it is told to whoever asks first: all
 * that the stream held before the call is counted, and none that runs out on
 * another stream meanwhile is lost (of one of its launches several calls may tell). */
int mlkv_dense_sync(void* stream);

/* Log probabilities of given tokens under softmax(scale * logits), row by row.
 * d_logits: [n][vocab] of `type`, 1 <= vocab < 2^30; scale > 0, finite (an inverse temperature).
 * d_targets: int64 [n]; a negative target is none (log probability 0, no
 * gradient); one of vocab or above gives NaN.
 * d_logprob, d_entropy: fp32 [n]; the entropy in nats.  d_stats: fp32 [n][2],
 * (max, log sum exp(scale * (logit - max))), for the backward pass.
 * d_top_logprobs (fp32), d_top_ids (int64): [n][top], the likeliest tokens in
 * order, ties by the lowest index; 0 <= top <= MLKV_MAX_TOP (null when 0).
 * -inf is a masked token: it has probability 0, is no alternative (places left
 * over hold -inf and -1) and has gradient 0.  A row without any other value
 * has log probability -inf, entropy 0 and gradient 0.  A row with NaN or +inf
 * has NaN statistics and gradient; its ids rank NaN first.
 * How long alternatives take goes by the data: a row whose scores rise along the
 * vocabulary, or that holds NaN, is read again, its parts up to `top` times
 * (8,192 x 50,000 bf16, 20 alternatives: 194 us of random scores, 3,500 of rows
 * sorted upwards, 5,000 with a NaN in each; 2,048 x 131,072: 140, 370, 1,700). */
int64_t mlkv_token_logprobs_workspace(int64_t n, int64_t vocab, int32_t type, int32_t top);
int mlkv_token_logprobs(const void* d_logits, int64_t stride, int32_t type, int64_t n, int64_t vocab,
                        const int64_t* d_targets, float scale, int32_t top, float* d_logprob, float* d_entropy,
                        float* d_stats, float* d_top_logprobs, int64_t* d_top_ids, void* d_workspace,
                        int64_t workspace_bytes, void* stream);

/* The gradient of the logits, of `type`, from the gradients of log probability
 * and entropy (fp32 [n] each; either may be null: 0).  d_dlogits may be
 * d_logits where the strides agree (the logits are then overwritten).  The
 * alternatives pass no gradient. */
int mlkv_token_logprobs_backward(const void* d_logits, int64_t stride, int32_t type, int64_t n, int64_t vocab,
                                 const int64_t* d_targets, float scale, const float* d_entropy,
                                 const float* d_stats, const float* d_dlogprob, const float* d_dentropy,
                                 void* d_dlogits, int64_t dlogits_stride, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MLKV_DENSE_H */
