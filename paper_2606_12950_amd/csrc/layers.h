// Internal launch interface of the layers by role, in 8-bit integers and from checkpoints (include/maestro_layers.h).
#pragma once

#include "maestro_layers.h"
#include "train.h"

namespace maestro {

maestro_status launch_layer_grouped_f32(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, const float* x,
                                        const float* weight, const float* bias, const int64_t* offsets, bool relu, float* y,
                                        hipStream_t stream);
maestro_status launch_layer_grouped_bf16(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, const void* x,
                                         const void* weight, const float* bias, const int64_t* offsets, bool relu, void* y,
                                         hipStream_t stream);
size_t grouped_grad_f32_workspace_bytes(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out);
size_t grouped_grad_bf16_workspace_bytes(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out);
maestro_status launch_grouped_grad_f32(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, const float* x,
                                       const float* weight, const float* g_z, const int64_t* offsets, bool relu_input,
                                       float* g_x, float* g_weight, float* g_bias, void* workspace, hipStream_t stream);
maestro_status launch_grouped_grad_bf16(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, const void* x,
                                        const void* weight, const void* g_z, const int64_t* offsets, bool relu_input,
                                        void* g_x, float* g_weight, float* g_bias, void* workspace, hipStream_t stream);
// every group's g_w and g_b from those of its units of k_split rows (by_group: kTiles, else kShares); a group of one unit has them already
maestro_status launch_join_groups(int64_t n, int32_t n_groups, const int64_t* offsets, int64_t k_split, bool by_group,
                                  const float* gw_parts, float* gw, int64_t size, const float* gb_parts, float* gb, int32_t d_out,
                                  hipStream_t stream);

maestro_status launch_quantize_rows(int64_t n, int32_t d, int32_t dtype, const void* x, int8_t* codes, float* scale,
                                    hipStream_t stream);
maestro_status launch_layer_int8(int64_t n, int32_t d_in, int32_t d_out, const int8_t* x, const float* x_scale,
                                 const int8_t* weight, const float* weight_scale, const float* bias, bool relu, int32_t dtype,
                                 void* y, hipStream_t stream);

maestro_status launch_pack(int64_t n, int32_t d, int32_t dtype, const void* x, bool rectified, void* codes, uint8_t* exponents,
                           hipStream_t stream);
maestro_status launch_unpack(int64_t n, int32_t d, int32_t dtype, const void* codes, const uint8_t* exponents, bool rectified,
                             void* x, hipStream_t stream);
size_t grad_packed_f32_workspace_bytes(int64_t n, int32_t d_in, int32_t d_out);
size_t grad_packed_bf16_workspace_bytes(int64_t n, int32_t d_in, int32_t d_out);
maestro_status launch_grad_packed_f32(int64_t n, int32_t d_in, int32_t d_out, const void* codes, const uint8_t* exponents,
                                      bool rectified, const float* weight, const float* g_z, bool relu_input, float* g_x,
                                      float* g_weight, float* g_bias, void* workspace, hipStream_t stream);
maestro_status launch_grad_packed_bf16(int64_t n, int32_t d_in, int32_t d_out, const void* codes, const uint8_t* exponents,
                                       bool rectified, const void* weight, const void* g_z, bool relu_input, void* g_x,
                                       float* g_weight, float* g_bias, void* workspace, hipStream_t stream);
size_t grad_packed_workspace_bytes(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype);
maestro_status launch_grad_packed(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* codes,
                                  const uint8_t* exponents, bool rectified, const void* weight, const void* g_z, bool relu_input,
                                  void* g_x, float* g_weight, float* g_bias, void* workspace, hipStream_t stream);

}  // namespace maestro
