/*
 * maestro_layers.h -- a length predictor's layers by role, in 8-bit integers, and from 8-bit checkpoints.
 *
 * Next to maestro_layer and maestro_layer_grad (maestro_train.h):
 *
 *   maestro_layer_grouped       a layer whose rows belong to groups with weights of their own (the paper's per-role
 *                               regressors, Sec. III-B: a role's stages lie one after the other), as many as there are
 *   maestro_layer_grouped_grad  its gradients
 *   maestro_quantize_rows       rows as signed bytes with a scale each (stages, or a layer's output channels)
 *   maestro_layer_int8          a layer of rows and weights so quantised, its products in whole numbers
 *   maestro_pack_activations    activations kept in 8 bits between the forward and the backward pass
 *   maestro_unpack_activations  their values
 *   maestro_layer_grad_packed   a layer's gradients from an input so kept
 *
 * The conventions of maestro_train.h hold: device pointers aligned to 16 bytes where nothing else is said, rows
 * contiguous, caller-owned arrays and workspaces, asynchronous on `stream`, host-side checks before anything is
 * enqueued, no allocation and no synchronisation in a call, empty inputs are valid, equal calls give equal bits.
 * Widths (d, d_in, d_out) are multiples of 16 up to MAESTRO_MAX_LAYER_WIDTH (MAESTRO_ERR_UNSUPPORTED otherwise).
 * Outputs overlap no input and no other output.
 */
#ifndef MAESTRO_LAYERS_H
#define MAESTRO_LAYERS_H

#include "maestro_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The most groups of a grouped layer. */
#define MAESTRO_MAX_LAYER_GROUPS 256

/* For group g of n_groups (1 .. MAESTRO_MAX_LAYER_GROUPS) and its rows r, offsets[g] <= r < offsets[g + 1]:
 *   y[r] = x[r] * weight[g]^T + bias[g], then max(., 0) where relu is not 0
 * x [n][d_in], weight [n_groups][d_out][d_in] and y [n][d_out] in `dtype`, bias [n_groups][d_out] float32, offsets
 * [n_groups + 1] int64 (DEVICE, aligned to 8). Sums and rounding as maestro_layer. Groups may be empty. Rows of no group
 * (before offsets[0], from offsets[n_groups] on) are not read, and theirs of y are left as they are. An offset below an
 * earlier one counts as that one, one outside 0 .. n as the nearer bound. n is below 2^31 - 2^16, and n * d_in and n * d_out
 * below about 2^43 (MAESTRO_ERR_UNSUPPORTED otherwise). */
MAESTRO_API maestro_status maestro_layer_grouped(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, int32_t dtype,
                             const void* x, const void* weight, const float* bias, const int64_t* offsets, int32_t relu,
                             void* y, void* stream);

/* Gradients of a grouped layer z given g_z [n][d_out] (of z, in `dtype`), as maestro_layer_grad's for every group:
 *   g_weight (out) [n_groups][d_out][d_in] float32, g_bias (out) [n_groups][d_out] float32: of empty groups zeros
 *   g_x      (out) [n][d_in] in `dtype`, or NULL where it is not wanted; rows of no group are left as they are
 * Workspace: maestro_layer_grouped_grad_workspace() bytes (0 for few rows: NULL is then allowed). */
MAESTRO_API size_t maestro_layer_grouped_grad_workspace(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, int32_t dtype);
MAESTRO_API maestro_status maestro_layer_grouped_grad(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, int32_t dtype,
                             const void* x, const void* weight, const void* g_z, const int64_t* offsets, int32_t relu_input,
                             void* g_x, float* g_weight, float* g_bias, void* workspace, size_t workspace_bytes, void* stream);

/* Rows of x [n][d] (`dtype`) as codes (out) [n][d], signed bytes, and scale (out) [n] float32 (aligned to 4):
 *   scale = max(largest magnitude / 127, 2^-126), the quotient rounded to float32
 *   code  = x / scale, the real quotient to the nearest whole number, ties to the even one: -127 .. 127
 * A row with a NaN or an infinite value has codes 0 and the scale NaN. */
MAESTRO_API maestro_status maestro_quantize_rows(int64_t n, int32_t d, int32_t dtype, const void* x, int8_t* codes, float* scale,
                             void* stream);

/* y [n][d_out] = x * weight^T + bias for x [n][d_in] and weight [d_out][d_in] in codes, x_scale [n] (aligned to 4) and
 * weight_scale [d_out] float32, then max(., 0) where relu is not 0; y in `dtype`, bias [d_out] float32. The products
 * are summed in 32-bit integers, exactly (codes -128 are valid); then in float32 fma(sum * x_scale, weight_scale, bias), the
 * sum and its product with x_scale rounded to float32, rounded once to `dtype`. */
MAESTRO_API maestro_status maestro_layer_int8(int64_t n, int32_t d_in, int32_t d_out, const int8_t* x, const float* x_scale,
                             const int8_t* weight, const float* weight_scale, const float* bias, int32_t relu, int32_t dtype,
                             void* y, void* stream);

/* x [n][d] (`dtype`) as codes (out) [n][d], a byte each, and exponents (out) [n][(d + 31) / 32] bytes (no alignment): every 32 values of
 * a row share the step 2^(exponent - 127), the least one (from 2^-126 on) that leaves all of them within the codes, at most 2^121
 * (2^120 where rectified): one more would make 2^128, an infinity, of finite values, which have the last code instead.
 *   rectified = 0: signed bytes, code = x / step to the nearest, ties to the even one: -127 .. 127
 *   rectified = 1: unsigned bytes 0 .. 255; values that are not positive have code 0, positive ones at least 1 (a
 *                  value below half a step counts as a step), so that code > 0 where x > 0
 * 32 values with a NaN or an infinite one among them have codes 0 and exponent 255: all of them count as NaN
 * (rectified = 1: a -inf among them counts as 0). */
MAESTRO_API maestro_status maestro_pack_activations(int64_t n, int32_t d, int32_t dtype, const void* x, int32_t rectified,
                             void* codes, uint8_t* exponents, void* stream);

/* x (out) [n][d] in `dtype`: the values code * 2^(exponent - 127), exactly. An exponent of 255 counts as an infinite step (0 times
 * it is NaN), one of 0, which packing never gives, as a step of 0. */
MAESTRO_API maestro_status maestro_unpack_activations(int64_t n, int32_t d, int32_t dtype, const void* codes,
                             const uint8_t* exponents, int32_t rectified, void* x, void* stream);

/* maestro_layer_grad for an input kept as codes and exponents: its g_weight, g_bias and g_x are those of the values that
 * maestro_unpack_activations gives. relu_input needs rectified codes (0 elsewhere is MAESTRO_ERR_INVALID_ARG) and
 * makes g_x 0 where the code is 0. Workspace: maestro_layer_grad_packed_workspace() bytes (0 for few rows). */
MAESTRO_API size_t maestro_layer_grad_packed_workspace(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype);
MAESTRO_API maestro_status maestro_layer_grad_packed(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* codes,
                             const uint8_t* exponents, int32_t rectified, const void* weight, const void* g_z,
                             int32_t relu_input, void* g_x, float* g_weight, float* g_bias, void* workspace,
                             size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MAESTRO_LAYERS_H */
