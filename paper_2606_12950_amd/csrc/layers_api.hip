// C-ABI entry points of include/maestro_layers.h: host-side argument checks, then the launchers.
// Nothing here touches device memory; every check happens before the first launch.
#include "groups.h"
#include "layers.h"

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
bool given(const void* p, size_t a) { return p && aligned(p, a); }
bool typed(int32_t dtype) { return dtype == MAESTRO_F32 || dtype == MAESTRO_BF16; }
hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

constexpr int64_t kMaxRows = (int64_t)1 << 40;   // keeps rows * width and byte offsets within 63 bits

maestro_status check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (!need) return MAESTRO_OK;
  if (!given(workspace, 16)) return MAESTRO_ERR_INVALID_ARG;
  return bytes < need ? MAESTRO_ERR_WORKSPACE : MAESTRO_OK;
}

maestro_status check_width(int32_t d) { return d % 16 || d > MAESTRO_MAX_LAYER_WIDTH ? MAESTRO_ERR_UNSUPPORTED : MAESTRO_OK; }

maestro_status check_layer(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype) {
  if (n < 0 || n > kMaxRows || d_in < 1 || d_out < 1 || !typed(dtype)) return MAESTRO_ERR_INVALID_ARG;
  return check_width(d_in) != MAESTRO_OK ? check_width(d_in) : check_width(d_out);
}

maestro_status check_grouped(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, int32_t dtype) {
  if (n_groups < 1) return MAESTRO_ERR_INVALID_ARG;
  const maestro_status st = check_layer(n, d_in, d_out, dtype);
  if (st != MAESTRO_OK) return st;
  // rows and tiles (64 x 64 at the least) are counted in 32 bits; 2^31 tiles are past any memory
  if (n_groups > MAESTRO_MAX_LAYER_GROUPS || n > maestro::kMaxGroupedRows ||
      (n / 64 + n_groups) * (((d_in > d_out ? d_in : d_out) + 63) / 64) >= (int64_t)1 << 31)
    return MAESTRO_ERR_UNSUPPORTED;
  return MAESTRO_OK;
}

}  // namespace

extern "C" {

maestro_status maestro_layer_grouped(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, int32_t dtype, const void* x,
                                     const void* weight, const float* bias, const int64_t* offsets, int32_t relu, void* y,
                                     void* stream) {
  const maestro_status st = check_grouped(n, n_groups, d_in, d_out, dtype);
  if (st == MAESTRO_ERR_INVALID_ARG) return st;
  if (!given(weight, 16) || !given(bias, 16) || !given(offsets, 8)) return MAESTRO_ERR_INVALID_ARG;
  if (n > 0 && (!given(x, 16) || !given(y, 16))) return MAESTRO_ERR_INVALID_ARG;
  if (st != MAESTRO_OK || n == 0) return st;
  if (dtype == MAESTRO_BF16)
    return maestro::launch_layer_grouped_bf16(n, n_groups, d_in, d_out, x, weight, bias, offsets, relu != 0, y, as_stream(stream));
  return maestro::launch_layer_grouped_f32(n, n_groups, d_in, d_out, static_cast<const float*>(x),
                                           static_cast<const float*>(weight), bias, offsets, relu != 0, static_cast<float*>(y),
                                           as_stream(stream));
}

size_t maestro_layer_grouped_grad_workspace(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, int32_t dtype) {
  if (check_grouped(n, n_groups, d_in, d_out, dtype) != MAESTRO_OK) return 0;
  return dtype == MAESTRO_BF16 ? maestro::grouped_grad_bf16_workspace_bytes(n, n_groups, d_in, d_out)
                               : maestro::grouped_grad_f32_workspace_bytes(n, n_groups, d_in, d_out);
}

maestro_status maestro_layer_grouped_grad(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, int32_t dtype,
                                          const void* x, const void* weight, const void* g_z, const int64_t* offsets,
                                          int32_t relu_input, void* g_x, float* g_weight, float* g_bias, void* workspace,
                                          size_t workspace_bytes, void* stream) {
  maestro_status st = check_grouped(n, n_groups, d_in, d_out, dtype);
  if (st == MAESTRO_ERR_INVALID_ARG) return st;
  if (!given(weight, 16) || !given(g_weight, 16) || !given(g_bias, 16) || !given(offsets, 8)) return MAESTRO_ERR_INVALID_ARG;
  if (n > 0 && (!given(x, 16) || !given(g_z, 16) || !aligned(g_x, 16))) return MAESTRO_ERR_INVALID_ARG;
  if (st != MAESTRO_OK) return st;
  st = check_workspace(workspace, workspace_bytes, maestro_layer_grouped_grad_workspace(n, n_groups, d_in, d_out, dtype));
  if (st != MAESTRO_OK) return st;
  if (dtype == MAESTRO_BF16)
    return maestro::launch_grouped_grad_bf16(n, n_groups, d_in, d_out, x, weight, g_z, offsets, relu_input != 0, g_x, g_weight,
                                             g_bias, workspace, as_stream(stream));
  return maestro::launch_grouped_grad_f32(n, n_groups, d_in, d_out, static_cast<const float*>(x),
                                          static_cast<const float*>(weight), static_cast<const float*>(g_z), offsets,
                                          relu_input != 0, static_cast<float*>(g_x), g_weight, g_bias, workspace,
                                          as_stream(stream));
}

maestro_status maestro_quantize_rows(int64_t n, int32_t d, int32_t dtype, const void* x, int8_t* codes, float* scale,
                                     void* stream) {
  if (n < 0 || n > kMaxRows || d < 1 || !typed(dtype)) return MAESTRO_ERR_INVALID_ARG;
  if (n > 0 && (!given(x, 16) || !given(codes, 16) || !given(scale, 4))) return MAESTRO_ERR_INVALID_ARG;
  if (check_width(d) != MAESTRO_OK || n == 0) return check_width(d);
  return maestro::launch_quantize_rows(n, d, dtype, x, codes, scale, as_stream(stream));
}

maestro_status maestro_layer_int8(int64_t n, int32_t d_in, int32_t d_out, const int8_t* x, const float* x_scale,
                                  const int8_t* weight, const float* weight_scale, const float* bias, int32_t relu,
                                  int32_t dtype, void* y, void* stream) {
  const maestro_status st = check_layer(n, d_in, d_out, dtype);
  if (st == MAESTRO_ERR_INVALID_ARG) return st;
  if (!given(weight, 16) || !given(weight_scale, 16) || !given(bias, 16)) return MAESTRO_ERR_INVALID_ARG;
  if (n > 0 && (!given(x, 16) || !given(x_scale, 4) || !given(y, 16))) return MAESTRO_ERR_INVALID_ARG;
  if (st != MAESTRO_OK || n == 0) return st;
  return maestro::launch_layer_int8(n, d_in, d_out, x, x_scale, weight, weight_scale, bias, relu != 0, dtype, y, as_stream(stream));
}

maestro_status maestro_pack_activations(int64_t n, int32_t d, int32_t dtype, const void* x, int32_t rectified, void* codes,
                                        uint8_t* exponents, void* stream) {
  if (n < 0 || n > kMaxRows || d < 1 || !typed(dtype)) return MAESTRO_ERR_INVALID_ARG;
  if (n > 0 && (!given(x, 16) || !given(codes, 16) || !exponents)) return MAESTRO_ERR_INVALID_ARG;
  if (check_width(d) != MAESTRO_OK || n == 0) return check_width(d);
  return maestro::launch_pack(n, d, dtype, x, rectified != 0, codes, exponents, as_stream(stream));
}

maestro_status maestro_unpack_activations(int64_t n, int32_t d, int32_t dtype, const void* codes, const uint8_t* exponents,
                                          int32_t rectified, void* x, void* stream) {
  if (n < 0 || n > kMaxRows || d < 1 || !typed(dtype)) return MAESTRO_ERR_INVALID_ARG;
  if (n > 0 && (!given(x, 16) || !given(codes, 16) || !exponents)) return MAESTRO_ERR_INVALID_ARG;
  if (check_width(d) != MAESTRO_OK || n == 0) return check_width(d);
  return maestro::launch_unpack(n, d, dtype, codes, exponents, rectified != 0, x, as_stream(stream));
}

size_t maestro_layer_grad_packed_workspace(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype) {
  if (check_layer(n, d_in, d_out, dtype) != MAESTRO_OK) return 0;
  return maestro::grad_packed_workspace_bytes(n, d_in, d_out, dtype);
}

maestro_status maestro_layer_grad_packed(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* codes,
                                         const uint8_t* exponents, int32_t rectified, const void* weight, const void* g_z,
                                         int32_t relu_input, void* g_x, float* g_weight, float* g_bias, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  maestro_status st = check_layer(n, d_in, d_out, dtype);
  if (st == MAESTRO_ERR_INVALID_ARG) return st;
  if (relu_input && !rectified) return MAESTRO_ERR_INVALID_ARG;
  if (!given(weight, 16) || !given(g_weight, 16) || !given(g_bias, 16)) return MAESTRO_ERR_INVALID_ARG;
  if (n > 0 && (!given(codes, 16) || !exponents || !given(g_z, 16) || !aligned(g_x, 16))) return MAESTRO_ERR_INVALID_ARG;
  if (st != MAESTRO_OK) return st;
  st = check_workspace(workspace, workspace_bytes, maestro::grad_packed_workspace_bytes(n, d_in, d_out, dtype));
  if (st != MAESTRO_OK) return st;
  return maestro::launch_grad_packed(n, d_in, d_out, dtype, codes, exponents, rectified != 0, weight, g_z, relu_input != 0,
                                     n > 0 ? g_x : nullptr, g_weight, g_bias, workspace, as_stream(stream));
}

}  // extern "C"
