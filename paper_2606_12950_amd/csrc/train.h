// Internal launch interface of the training operators (include/maestro_train.h).
#pragma once

#include "internal.h"
#include "maestro_train.h"

namespace maestro {

size_t logprobs_workspace_bytes(int64_t n, int32_t v, int32_t k, int32_t dtype);
maestro_status launch_logprobs(int64_t n, int32_t v, const void* logits, int64_t row_stride, int32_t dtype,
                               const int32_t* token, int32_t k, float* logprob, float* entropy, int32_t* top_id,
                               float* top_logprob, float* stats, void* workspace, hipStream_t stream);
maestro_status launch_logprobs_grad(int64_t n, int32_t v, const void* logits, int64_t row_stride, int32_t dtype,
                                    const int32_t* token, const float* stats, const float* entropy,
                                    const float* g_logprob, const float* g_entropy, void* grad, int64_t grad_stride,
                                    hipStream_t stream);

maestro_status launch_layer(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* x, const void* weight,
                            const float* bias, bool relu, void* y, hipStream_t stream);
size_t layer_grad_workspace_bytes(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype);
maestro_status launch_layer_grad(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* x,
                                 const void* weight, const void* g_z, bool relu_input, void* g_x, float* g_weight,
                                 float* g_bias, void* workspace, hipStream_t stream);

// the bfloat16 layers, on the matrix cores
maestro_status launch_layer_bf16(int64_t n, int32_t d_in, int32_t d_out, const void* x, const void* weight,
                                 const float* bias, bool relu, void* y, hipStream_t stream);
size_t layer_grad_bf16_workspace_bytes(int64_t n, int32_t d_in, int32_t d_out);
maestro_status launch_layer_grad_bf16(int64_t n, int32_t d_in, int32_t d_out, const void* x, const void* weight,
                                      const void* g_z, bool relu_input, void* g_x, float* g_weight, float* g_bias,
                                      void* workspace, hipStream_t stream);

// g_w (size values; n_gw = 1: it is there already) and g_b from their shares, summed in order; no shares: zeros
maestro_status launch_join(const float* gw_parts, int32_t n_gw, float* gw, int64_t size, const float* gb_parts,
                           int32_t n_gb, float* gb, int32_t d_out, hipStream_t stream);

constexpr int64_t kClipMaxBytes = (int64_t)1 << 39;      // of a tensor to clip: 2^24 units of work
size_t clip_workspace_bytes(int32_t n_tensors);
maestro_status launch_clip(int32_t n_tensors, void* const* tensors, void* const* out, const int64_t* sizes,
                           const int32_t* dtypes, float max_norm, float* norm, void* workspace, hipStream_t stream);

}  // namespace maestro
