/*
 * gasloc_layers.h -- the layers of a decoder that hold parameters, for all
 * worker replicas of a context at once: embedding lookup, layer norm and
 * linear layers, forward and backward.  They turn the workers' rows into
 * activations and write parameter gradients into the rows [n, grad_ld] that
 * gasloc_local_step and gasloc_local_step_gossip_round read.
 *
 * Conventions, beside those of gasloc.h:
 *   - Token rows.  A call takes the token rows of all workers, packed: worker
 *     i has rows row_ptr[i] .. row_ptr[i+1] - 1 of every activation.  row_ptr:
 *     host int64[n+1], row_ptr[0] = 0, non-decreasing, row_ptr[n] <= 2^27.  A
 *     worker may have none.  Rows from row_ptr[n] on are neither read nor
 *     written.  The counts go with the launch: a call recorded in a HIP graph
 *     keeps them.
 *   - Weights.  `begin` is the column of every worker's row at which a weight
 *     starts (row-major, packed: a linear layer's weight [out_features,
 *     in_features] takes out_features * in_features columns).  Worker i's
 *     weights are read from its live iterate: row i of y if it took a local
 *     step since the last round, else row i of x.  Which of the two is decided
 *     when the call is made, also for a call that is recorded in a graph: a
 *     replay reads the rows that were live at the recording.  It gives what an
 *     eager call would while the same workers have stepped since the last round
 *     as then, so a program with several local steps per round records its step
 *     twice, once before and once after the first of them.
 *   - Activations: device memory, row t at offset t * ld elements (ld >= the
 *     row's length, < 2^21), dtype GASLOC_F32 or GASLOC_BF16, aligned to the
 *     element.  Types go together as (parameters, activations) = (F32, F32),
 *     (F32, BF16), (BF16, BF16); EINVAL for F32 activations with BF16
 *     parameters.
 *   - Gradients: device fp32 [n, grad_ld], 16-byte aligned, grad_ld >= P and a
 *     multiple of 4, as for gasloc_local_step.  accumulate = 0 writes the
 *     weight's columns of every worker (zeros for a worker without rows),
 *     accumulate = 1 adds to them.  Other columns are left as they are.
 *   - Sums, means and products are taken in fp32 (never in fewer bits), and
 *     rounded once, to nearest even, where the result is BF16.  Every sum has
 *     an order that depends on the sizes, the types, the alignment of rows and
 *     weights and the GPU alone: the same call gives the same bits again.
 *   - All work is enqueued on the context's stream; no call waits, allocates or
 *     copies, so each may be recorded in a graph (of a context whose stream is not
 *     the default one).  Workspaces are the caller's
 *     (device, 256-byte aligned; calls that may overlap in time, or graphs whose
 *     replays may, need one each); what one holds before or after a call does
 *     not matter.
 *   - Buffers of a call must not overlap, except where a call says so.
 *   - Dead workers (gasloc_set_alive) are computed like any other: what they
 *     get for a gradient is not used by their skipped steps.
 *   - Vector accesses are taken where rows and weights begin on 16-byte
 *     boundaries and row lengths are a multiple of 8 (BF16) or 4 (F32)
 *     elements (features of linear layers: of 8 in either type); anything else
 *     is served too, at half to three quarters of the rate in linear layers.
 *   - Errors: EINVAL (checked before any device work; also for what one launch of
 *     fewer than 2^32 threads cannot hold), ENOMEM (host memory), EDEVICE, ESTATE.
 */
#ifndef GASLOC_LAYERS_H
#define GASLOC_LAYERS_H

#include <stddef.h>
#include <stdint.h>

#include "gasloc.h"

#ifdef __cplusplus
extern "C" {
#endif

/* out[t, :] = scale * E_i[tokens[t], :] for every row t of worker i; E_i:
 * [vocab, width] at column `begin`, vocab <= 2^24.  tokens: device int32, row_ptr[n] of
 * them.  A token outside [0, vocab) is padding: its row of out is zero.
 * Enqueues one kernel. */
gasloc_status gasloc_embedding(gasloc_ctx *ctx, int64_t begin, int32_t vocab, int32_t width, float scale,
                               const int64_t *row_ptr, const int32_t *tokens, int32_t dtype, void *out,
                               int64_t out_ld);

/* The gradient of gasloc_embedding: for every worker i and table row k,
 *   grads_i[begin + k * width ..] (+)= scale * sum over t with tokens[t] = k of dout[t, :].
 * The tokens are sorted first (stable), so that every table row is written
 * once, by sums that go over its tokens in order.  Padding tokens contribute
 * nothing.  Enqueues three kernels (fewer with few rows), and one more for each factor of 8 by which
 * the longest worker exceeds 8192 rows.  workspace: at least
 * gasloc_embedding_grad_workspace bytes. */
gasloc_status gasloc_embedding_grad(gasloc_ctx *ctx, int64_t begin, int32_t vocab, int32_t width, float scale,
                                    const int64_t *row_ptr, const int32_t *tokens, int32_t dtype, const void *dout,
                                    int64_t dout_ld, float *grads, int64_t grad_ld, int32_t accumulate,
                                    void *workspace, size_t workspace_bytes);

/* Bytes of workspace for gasloc_embedding_grad with these rows.  Host only. */
gasloc_status gasloc_embedding_grad_workspace(const gasloc_ctx *ctx, int32_t width, const int64_t *row_ptr,
                                              size_t *bytes);

/* Layer norm: with mean = sum_c x[t, c] / width and rstd = 1 / sqrt(sum_c
 * (x[t, c] - mean)^2 / width + eps),
 *   out[t, c] = (x[t, c] - mean) * rstd * gain_i[c] + bias_i[c].
 * gain, bias: the columns at which the two vectors start; bias < 0: none.
 * width in [1, 16384]; eps finite and > 0.  x and out have the same dtype;
 * out may be x (with the same row length).  stats: device fp32 [row_ptr[n], 2], 8-byte aligned, receives
 * (mean, rstd) of every row for the backward pass; NULL: not kept.  Enqueues
 * one kernel. */
gasloc_status gasloc_layer_norm(gasloc_ctx *ctx, int64_t gain, int64_t bias, int32_t width, float eps,
                                const int64_t *row_ptr, const void *x, int64_t x_ld, int32_t dtype, void *out,
                                int64_t out_ld, float *stats);

/* The gradients of gasloc_layer_norm.  With h = dout * gain_i and xh = (x -
 * mean) * rstd,
 *   dx[t, :] = rstd * (h - mean_c(h) - xh * mean_c(h * xh))
 *   grads_i[gain + c] (+)= sum_t dout[t, c] * xh[t, c]
 *   grads_i[bias + c] (+)= sum_t dout[t, c]              (bias >= 0)
 * stats: what the forward pass kept.  dx may be dout or x (with the same row length).  Enqueues two
 * kernels.  workspace: at least gasloc_layer_norm_grad_workspace bytes. */
gasloc_status gasloc_layer_norm_grad(gasloc_ctx *ctx, int64_t gain, int64_t bias, int32_t width,
                                     const int64_t *row_ptr, const void *x, int64_t x_ld, const float *stats,
                                     const void *dout, int64_t dout_ld, int32_t dtype, void *dx, int64_t dx_ld,
                                     float *grads, int64_t grad_ld, int32_t accumulate, void *workspace,
                                     size_t workspace_bytes);

/* Bytes of workspace for gasloc_layer_norm_grad with these rows.  Host only. */
gasloc_status gasloc_layer_norm_grad_workspace(const gasloc_ctx *ctx, int32_t width, const int64_t *row_ptr,
                                               size_t *bytes);

/* Linear layer without bias: out[t, :] = W_i x[t, :] for every row t of worker
 * i; W_i: [out_features, in_features] at column `weight`.  F32 weights meet
 * BF16 activations rounded to BF16 (nearest even), as in a mixed-precision
 * step.  Features in [1, 2^20].  Enqueues one kernel, and one more where a
 * product with few rows is split along its sums.  workspace: at least
 * gasloc_linear_workspace bytes (may be NULL if that is 0). */
gasloc_status gasloc_linear(gasloc_ctx *ctx, int64_t weight, int32_t out_features, int32_t in_features,
                            const int64_t *row_ptr, const void *x, int64_t x_ld, int32_t dtype, void *out,
                            int64_t out_ld, void *workspace, size_t workspace_bytes);

/* Its gradient of the input, dx[t, :] = W_i^T dout[t, :]; weights rounded, kernels
 * and workspace as in the forward pass. */
gasloc_status gasloc_linear_grad_input(gasloc_ctx *ctx, int64_t weight, int32_t out_features, int32_t in_features,
                                       const int64_t *row_ptr, const void *dout, int64_t dout_ld, int32_t dtype,
                                       void *dx, int64_t dx_ld, void *workspace, size_t workspace_bytes);

/* Its gradient of the weight, grads_i[weight + o * in_features + c] (+)= sum_t
 * dout[t, o] * x[t, c] over the rows of worker i.  Kernels and workspace as
 * in the forward pass. */
gasloc_status gasloc_linear_grad_weight(gasloc_ctx *ctx, int64_t weight, int32_t out_features, int32_t in_features,
                                        const int64_t *row_ptr, const void *x, int64_t x_ld, const void *dout,
                                        int64_t dout_ld, int32_t dtype, float *grads, int64_t grad_ld,
                                        int32_t accumulate, void *workspace, size_t workspace_bytes);

/* Bytes of workspace with which each of the three calls can be made for a
 * layer of these sizes with these rows.  Host only. */
gasloc_status gasloc_linear_workspace(const gasloc_ctx *ctx, int32_t out_features, int32_t in_features,
                                      const int64_t *row_ptr, int32_t dtype, size_t *bytes);

#ifdef __cplusplus
}
#endif

#endif /* GASLOC_LAYERS_H */
