// C-ABI entry points of the training operators: host-side argument checks, then the launchers.
// Nothing here touches device memory; every check happens before the first launch.
#include <math.h>

#include "train.h"

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
bool optional(const void* p, size_t a) { return !p || aligned(p, a); }
bool typed(int32_t dtype) { return dtype == MAESTRO_F32 || dtype == MAESTRO_BF16; }
size_t element(int32_t dtype) { return dtype == MAESTRO_F32 ? 4 : 2; }
hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

constexpr int64_t kMaxRows = (int64_t)1 << 40;   // keeps rows * stride and byte offsets within 63 bits

maestro_status check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (!need) return MAESTRO_OK;
  if (!workspace || !aligned(workspace, 16)) return MAESTRO_ERR_INVALID_ARG;
  return bytes < need ? MAESTRO_ERR_WORKSPACE : MAESTRO_OK;
}

// whether [n][v] rows of a stride stay within the address arithmetic
bool rows_fit(int64_t n, int32_t v, int64_t stride) {
  return stride >= v && stride <= ((int64_t)1 << 40) && (n == 0 || stride <= (((int64_t)1 << 60) / n));
}

maestro_status check_layer(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype) {
  if (n < 0 || n > kMaxRows || d_in < 1 || d_out < 1 || !typed(dtype)) return MAESTRO_ERR_INVALID_ARG;
  if (d_in % 16 || d_out % 16 || d_in > MAESTRO_MAX_LAYER_WIDTH || d_out > MAESTRO_MAX_LAYER_WIDTH)
    return MAESTRO_ERR_UNSUPPORTED;
  return MAESTRO_OK;
}

}  // namespace

extern "C" {

size_t maestro_logprobs_workspace(int64_t n, int32_t v, int32_t k, int32_t dtype) {
  if (n < 0 || v < 1 || k < 0 || k > MAESTRO_MAX_ALTERNATIVES || !typed(dtype)) return 0;
  return maestro::logprobs_workspace_bytes(n, v, k, dtype);
}

maestro_status maestro_logprobs(int64_t n, int32_t v, const void* logits, int64_t row_stride, int32_t dtype,
                                const int32_t* token, int32_t k, float* logprob, float* entropy, int32_t* top_id,
                                float* top_logprob, float* stats, void* workspace, size_t workspace_bytes,
                                void* stream) {
  if (n < 0 || n > kMaxRows || v < 1 || k < 0 || k > MAESTRO_MAX_ALTERNATIVES || !typed(dtype))
    return MAESTRO_ERR_INVALID_ARG;
  if (!rows_fit(n, v, row_stride) || !token != !logprob) return MAESTRO_ERR_INVALID_ARG;
  if (!optional(token, 4) || !optional(logprob, 4) || !optional(entropy, 4) || !optional(top_id, 4) ||
      !optional(top_logprob, 4) || !optional(stats, 8))
    return MAESTRO_ERR_INVALID_ARG;
  if (n > 0 && (!logits || !aligned(logits, element(dtype)) || (k > 0 && (!top_id || !top_logprob))))
    return MAESTRO_ERR_INVALID_ARG;
  if (n == 0 || (!logprob && !entropy && !stats && k == 0)) return MAESTRO_OK;
  const maestro_status st = check_workspace(workspace, workspace_bytes, maestro::logprobs_workspace_bytes(n, v, k, dtype));
  if (st != MAESTRO_OK) return st;
  return maestro::launch_logprobs(n, v, logits, row_stride, dtype, token, k, logprob, entropy, top_id, top_logprob,
                                  stats, workspace, as_stream(stream));
}

maestro_status maestro_logprobs_grad(int64_t n, int32_t v, const void* logits, int64_t row_stride, int32_t dtype,
                                     const int32_t* token, const float* stats, const float* entropy,
                                     const float* g_logprob, const float* g_entropy, void* grad, int64_t grad_stride,
                                     void* stream) {
  if (n < 0 || n > kMaxRows || v < 1 || !typed(dtype)) return MAESTRO_ERR_INVALID_ARG;
  if (!rows_fit(n, v, row_stride) || !rows_fit(n, v, grad_stride)) return MAESTRO_ERR_INVALID_ARG;
  if (!token != !g_logprob || (!g_logprob && !g_entropy)) return MAESTRO_ERR_INVALID_ARG;
  if (!optional(token, 4) || !optional(stats, 8) || !optional(entropy, 4) || !optional(g_logprob, 4) ||
      !optional(g_entropy, 4))
    return MAESTRO_ERR_INVALID_ARG;
  if (n == 0) return MAESTRO_OK;
  if (!logits || !grad || !stats || (g_entropy && !entropy)) return MAESTRO_ERR_INVALID_ARG;
  if (!aligned(logits, element(dtype)) || !aligned(grad, element(dtype))) return MAESTRO_ERR_INVALID_ARG;
  if (grad == logits && grad_stride != row_stride) return MAESTRO_ERR_INVALID_ARG;
  return maestro::launch_logprobs_grad(n, v, logits, row_stride, dtype, token, stats, entropy, g_logprob, g_entropy,
                                       grad, grad_stride, as_stream(stream));
}

maestro_status maestro_layer(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* x, const void* weight,
                             const float* bias, int32_t relu, void* y, void* stream) {
  const maestro_status st = check_layer(n, d_in, d_out, dtype);
  if (st == MAESTRO_ERR_INVALID_ARG) return st;
  if (!weight || !bias || !aligned(weight, 16) || !aligned(bias, 16)) return MAESTRO_ERR_INVALID_ARG;
  if (n > 0 && (!x || !y || !aligned(x, 16) || !aligned(y, 16))) return MAESTRO_ERR_INVALID_ARG;
  if (st != MAESTRO_OK || n == 0) return st;
  return maestro::launch_layer(n, d_in, d_out, dtype, x, weight, bias, relu != 0, y, as_stream(stream));
}

size_t maestro_layer_grad_workspace(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype) {
  if (check_layer(n, d_in, d_out, dtype) != MAESTRO_OK) return 0;
  return maestro::layer_grad_workspace_bytes(n, d_in, d_out, dtype);
}

maestro_status maestro_layer_grad(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* x,
                                  const void* weight, const void* g_z, int32_t relu_input, void* g_x, float* g_weight,
                                  float* g_bias, void* workspace, size_t workspace_bytes, void* stream) {
  maestro_status st = check_layer(n, d_in, d_out, dtype);
  if (st == MAESTRO_ERR_INVALID_ARG) return st;
  if (!weight || !g_weight || !g_bias || !aligned(weight, 16) || !aligned(g_weight, 16) || !aligned(g_bias, 16))
    return MAESTRO_ERR_INVALID_ARG;
  if (n > 0 && (!x || !g_z || !aligned(x, 16) || !aligned(g_z, 16) || !optional(g_x, 16)))
    return MAESTRO_ERR_INVALID_ARG;
  if (st != MAESTRO_OK) return st;
  st = check_workspace(workspace, workspace_bytes, maestro::layer_grad_workspace_bytes(n, d_in, d_out, dtype));
  if (st != MAESTRO_OK) return st;
  return maestro::launch_layer_grad(n, d_in, d_out, dtype, x, weight, g_z, relu_input != 0, n > 0 ? g_x : nullptr,
                                    g_weight, g_bias, workspace, as_stream(stream));
}

size_t maestro_clip_gradients_workspace(int32_t n_tensors) {
  return n_tensors < 0 ? 0 : maestro::clip_workspace_bytes(n_tensors);
}

maestro_status maestro_clip_gradients(int32_t n_tensors, void* const* tensors, void* const* out, const int64_t* sizes,
                                      const int32_t* dtypes, float max_norm, float* norm, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  if (n_tensors < 0 || !(max_norm >= 0.0f) || !norm || !aligned(norm, 4)) return MAESTRO_ERR_INVALID_ARG;
  if (max_norm == INFINITY && out) return MAESTRO_ERR_INVALID_ARG;
  if (n_tensors > 0 && (!tensors || !sizes || !dtypes)) return MAESTRO_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n_tensors; ++i) {
    if (!typed(dtypes[i]) || sizes[i] < 0 || sizes[i] > maestro::kClipMaxBytes / (int64_t)element(dtypes[i]))
      return MAESTRO_ERR_INVALID_ARG;
    if (sizes[i] == 0) continue;
    if (!tensors[i] || !aligned(tensors[i], element(dtypes[i]))) return MAESTRO_ERR_INVALID_ARG;
    if (out && (!out[i] || !aligned(out[i], element(dtypes[i])))) return MAESTRO_ERR_INVALID_ARG;
  }
  const maestro_status st = check_workspace(workspace, workspace_bytes, maestro::clip_workspace_bytes(n_tensors));
  if (st != MAESTRO_OK) return st;
  return maestro::launch_clip(n_tensors, tensors, out, sizes, dtypes, max_norm, norm, workspace, as_stream(stream));
}

}  // extern "C"
