/*
 * maestro_train.h -- what a length predictor is scored and trained with.
 *
 * Stages that have run come back with their observed output lengths (the paper's post-execution
 * profiling, which calibrates the predictor). maestro_predict keeps hidden layers and logits on
 * chip; these calls keep them, and take the gradient of the observed lengths back:
 *
 *   maestro_layer            one Linear layer of a predictor, its activations stored
 *   maestro_logprobs         log probability of given tokens (length bins, or tokens of a served
 *                            model's vocabulary), entropy, and the likeliest tokens
 *   maestro_logprobs_grad    its gradient with respect to the logits
 *   maestro_layer_grad       a layer's gradients: weights, biases, and its input's
 *   maestro_clip_gradients   the global norm over many gradient tensors, and clipping by it
 *
 * The conventions of maestro.h hold: device pointers, caller-owned arrays and workspaces
 * (16-byte aligned, contents on entry do not matter), asynchronous on `stream`, host-side checks
 * before anything is enqueued, no allocation and no synchronisation in a call, empty inputs are valid.
 * Results do not depend on timing: equal calls give equal bits.
 */
#ifndef MAESTRO_TRAIN_H
#define MAESTRO_TRAIN_H

#include "maestro.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The most alternatives maestro_logprobs lists, and the widest layer that is built. */
#define MAESTRO_MAX_ALTERNATIVES 16
#define MAESTRO_MAX_LAYER_WIDTH 16384

/* Row i holds v logits at logits + i * row_stride (elements of `dtype`, row_stride >= v, aligned to an
 * element; what lies between rows is not read). With m the row's largest logit, d_j = x_j - m and
 * S = sum_j e^(d_j), all in float32:
 *   logprob     (out) [n] float32: d_t - ln S for token t = token[i]; 0 for a token outside [0, v) (none given)
 *   entropy     (out) [n] float32: ln S - (sum_j e^(d_j) d_j) / S; NULL: not wanted
 *   top_id      (out) [n][k] int32, top_logprob (out) [n][k] float32: the k largest logits, largest first,
 *               equal ones in ascending index, and their log probabilities; 0 <= k <= MAESTRO_MAX_ALTERNATIVES
 *               (both may be NULL for k = 0)
 *   stats       (out) [n][2] float32: m and ln S, for maestro_logprobs_grad; NULL: not wanted
 * token and logprob may be NULL together. A logit of -inf is masked: it has probability 0 and is not
 * listed; lists are filled up with id -1 and -inf. A row masked throughout has log probability -inf
 * (0 without a token), entropy 0 and stats (-inf, -inf). A row with a NaN or +inf has no
 * distribution: NaN in its outputs (log probability 0 without a token), ids -1.
 * Workspace: maestro_logprobs_workspace() bytes (0 for most sizes: NULL is then allowed). */
MAESTRO_API size_t maestro_logprobs_workspace(int64_t n, int32_t v, int32_t k, int32_t dtype);
MAESTRO_API maestro_status maestro_logprobs(int64_t n, int32_t v, const void* logits, int64_t row_stride,
                             int32_t dtype, const int32_t* token, int32_t k, float* logprob, float* entropy,
                             int32_t* top_id, float* top_logprob, float* stats, void* workspace,
                             size_t workspace_bytes, void* stream);

/* Gradient with respect to the logits of sum_i g_logprob[i] logprob[i] + g_entropy[i] entropy[i]:
 *   grad[i][j] = g_logprob[i] ([j = token[i]] - p_j) - g_entropy[i] p_j (ln p_j + entropy[i]),
 * p_j = e^(x_j - m - ln S) from `stats`, computed in float32 and rounded once to `dtype`. token and
 * g_logprob may be NULL together, g_entropy may be NULL (entropy is then not read), not all three. A row without a
 * token takes no part in g_logprob. Rows whose two coefficients are zero, and rows masked
 * throughout, get zeros, whatever they hold; masked logits get 0 (the token's own apart: its
 * derivative is g_logprob), for all finite coefficients. A p_j below float32's least normal number may count as 0. grad may be the logits themselves with the same stride, and must not
 * overlap them otherwise. */
MAESTRO_API maestro_status maestro_logprobs_grad(int64_t n, int32_t v, const void* logits, int64_t row_stride,
                             int32_t dtype, const int32_t* token, const float* stats, const float* entropy,
                             const float* g_logprob, const float* g_entropy, void* grad, int64_t grad_stride,
                             void* stream);

/* y [n][d_out] = x [n][d_in] * weight^T + bias, then max(., 0) where relu is not 0; x, weight
 * [d_out][d_in] and y in `dtype` (16-byte aligned, rows contiguous), bias [d_out] float32. Products
 * accumulate in float32; one rounding to `dtype` at the end. Widths are multiples of 16 up to
 * MAESTRO_MAX_LAYER_WIDTH (MAESTRO_ERR_UNSUPPORTED otherwise); n is any. y overlaps no input. */
MAESTRO_API maestro_status maestro_layer(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* x,
                             const void* weight, const float* bias, int32_t relu, void* y, void* stream);

/* Gradients of a layer z = x * weight^T + bias given g_z [n][d_out] (of z, in `dtype`):
 *   g_weight (out) [d_out][d_in] float32: g_z^T * x      g_bias (out) [d_out] float32: sum of g_z over rows
 *   g_x      (out) [n][d_in] in `dtype`, or NULL where it is not wanted: g_z * weight, and 0 wherever
 *            x is not positive if relu_input is not 0 (x is a rectified layer's output, g_x the gradient of that layer's z)
 * Sums are float32; g_x is rounded once. Sizes, alignment and errors as maestro_layer; outputs overlap no
 * input. n = 0 writes zeros. Workspace: maestro_layer_grad_workspace() bytes. */
MAESTRO_API size_t maestro_layer_grad_workspace(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype);
MAESTRO_API maestro_status maestro_layer_grad(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* x,
                             const void* weight, const void* g_z, int32_t relu_input, void* g_x, float* g_weight,
                             float* g_bias, void* workspace, size_t workspace_bytes, void* stream);

/* The norm of all values of n_tensors tensors together, and clipping: norm[0] (out, float32) is the root
 * of the sum of squares, accumulated in float64; where it exceeds max_norm, every tensor is scaled by
 * max_norm / norm. max_norm = INFINITY computes the norm alone (out must be NULL).
 *   tensors, sizes, dtypes  HOST arrays [n_tensors], read during the call: device pointers (aligned to an
 *                           element, NULL allowed for size 0), element counts (up to 2^39 bytes), maestro_dtype
 *   out                     HOST array [n_tensors] of device pointers the result is written to, scaled
 *                           or not, each of its tensor's type and size; NULL: in place, where nothing is
 *                           written unless the norm exceeds max_norm. out[i] is tensors[i] itself or overlaps none;
 *                           no two tensors overlap
 * A norm that is not finite in float64 (an input is NaN or infinite) scales nothing; one past float32 is
 * written as infinity and scales all the same. Workspace: maestro_clip_gradients_workspace() bytes. */
MAESTRO_API size_t maestro_clip_gradients_workspace(int32_t n_tensors);
MAESTRO_API maestro_status maestro_clip_gradients(int32_t n_tensors, void* const* tensors, void* const* out,
                             const int64_t* sizes, const int32_t* dtypes, float max_norm, float* norm,
                             void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MAESTRO_TRAIN_H */
