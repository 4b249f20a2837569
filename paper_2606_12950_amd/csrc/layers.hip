// A predictor's Linear layer with its activations kept, and the layer's gradients.
#include "train.h"

namespace maestro {
namespace {

constexpr int kTile = 64, kDepth = 16, kThreads = 256;
constexpr int kSpan = 2048;   // terms of a sum in one chain; the chains' sums are added up apart, so long sums stay exact

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return (float)v; }

// 64 x 64 tiles of C = A B over a float32 accumulator: A(i, k) at a[i * ai + k * ak], B(k, j) at
// b[k * bk + j * bj]; `store` takes C(i, j).
template <typename T, typename Store>
__device__ __forceinline__ void tiles(int64_t rows, int64_t cols, int64_t depth, const T* a, int64_t ai, int64_t ak,
                                      const T* b, int64_t bk, int64_t bj, const Store& store) {
  __shared__ float as[kDepth][kTile + 4], bs[kDepth][kTile + 4];
  const int64_t across = (cols + kTile - 1) / kTile, all = (rows + kTile - 1) / kTile * across;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (int64_t tile = blockIdx.x; tile < all; tile += gridDim.x) {
    const int64_t i0 = tile / across * kTile, j0 = tile % across * kTile;
    float acc[4][4] = {}, sum[4][4] = {};
    for (int64_t k0 = 0; k0 < depth; k0 += kDepth) {
      if (k0 % kSpan == 0)
        for (int i = 0; i < 4; ++i)
          for (int j = 0; j < 4; ++j) sum[i][j] += acc[i][j], acc[i][j] = 0.0f;
      for (int e = threadIdx.x; e < kDepth * kTile; e += kThreads) {
        // the index that is contiguous in memory runs over neighbouring threads
        const int ka = ak == 1 ? e % kDepth : e / kTile, i = ak == 1 ? e / kDepth : e % kTile;
        const int kb = bk == 1 ? e % kDepth : e / kTile, j = bk == 1 ? e / kDepth : e % kTile;
        as[ka][i] = k0 + ka < depth && i0 + i < rows ? to_f32(a[(i0 + i) * ai + (k0 + ka) * ak]) : 0.0f;
        bs[kb][j] = k0 + kb < depth && j0 + j < cols ? to_f32(b[(k0 + kb) * bk + (j0 + j) * bj]) : 0.0f;
      }
      __syncthreads();
      for (int k = 0; k < kDepth; ++k)
        for (int i = 0; i < 4; ++i)
          for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(as[k][ty * 4 + i], bs[k][tx * 4 + j], acc[i][j]);
      __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j)
        if (i0 + ty * 4 + i < rows && j0 + tx * 4 + j < cols) store(i0 + ty * 4 + i, j0 + tx * 4 + j, sum[i][j] + acc[i][j]);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void forward_kernel(int64_t n, int32_t d_in, int32_t d_out, const T* x,
                                                           const T* w, const float* bias, bool relu, T* y) {
  tiles(n, d_out, d_in, x, d_in, 1, w, 1, d_in, [=](int64_t i, int64_t j, float c) {
    c += bias[j];
    y[i * d_out + j] = (T)(relu && c < 0.0f ? 0.0f : c);
  });
}

template <typename T>
__global__ __launch_bounds__(kThreads) void input_grad_kernel(int64_t n, int32_t d_in, int32_t d_out, const T* x,
                                                              const T* w, const T* gz, bool relu, T* gx) {
  tiles(n, d_in, d_out, gz, d_out, 1, w, d_in, 1, [=](int64_t i, int64_t j, float c) {
    gx[i * d_in + j] = (T)(relu && !(to_f32(x[i * d_in + j]) > 0.0f) ? 0.0f : c);
  });
}

template <typename T>
__global__ __launch_bounds__(kThreads) void weight_grad_kernel(int64_t n, int32_t d_in, int32_t d_out, const T* x,
                                                               const T* gz, float* gw) {
  tiles(d_out, d_in, n, gz, 1, d_out, x, d_in, 1, [=](int64_t i, int64_t j, float c) { gw[i * d_in + j] = c; });
}

// one workgroup sums 64 columns: four groups of lanes take every fourth row
template <typename T>
__global__ __launch_bounds__(kThreads) void bias_grad_kernel(int64_t n, int32_t d_out, const T* gz, float* gb) {
  __shared__ float part[4][64];
  const int c = threadIdx.x % 64, q = threadIdx.x / 64;
  const int64_t j = (int64_t)blockIdx.x * 64 + c;
  double s = 0.0;
  if (j < d_out)
    for (int64_t i = q; i < n; i += 4) s += to_f32(gz[i * d_out + j]);
  part[q][c] = (float)s;
  __syncthreads();
  if (q == 0 && j < d_out) gb[j] = (part[0][c] + part[1][c]) + (part[2][c] + part[3][c]);
}

unsigned grid_of(int64_t rows, int64_t cols) {
  const int64_t t = (rows + kTile - 1) / kTile * ((cols + kTile - 1) / kTile);
  return (unsigned)(t < (1 << 20) ? t : 1 << 20);
}

template <typename T>
maestro_status grads(int64_t n, int32_t d_in, int32_t d_out, const T* x, const T* w, const T* gz, bool relu, T* gx,
                     float* gw, float* gb, hipStream_t stream) {
  if (gx) input_grad_kernel<<<grid_of(n, d_in), kThreads, 0, stream>>>(n, d_in, d_out, x, w, gz, relu, gx);
  weight_grad_kernel<<<grid_of(d_out, d_in), kThreads, 0, stream>>>(n, d_in, d_out, x, gz, gw);
  bias_grad_kernel<<<(d_out + 63) / 64, kThreads, 0, stream>>>(n, d_out, gz, gb);
  return launch_status();
}

}  // namespace

maestro_status launch_layer(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* x, const void* weight,
                            const float* bias, bool relu, void* y, hipStream_t stream) {
  if (dtype == MAESTRO_BF16) return launch_layer_bf16(n, d_in, d_out, x, weight, bias, relu, y, stream);
  forward_kernel<<<grid_of(n, d_out), kThreads, 0, stream>>>(n, d_in, d_out, static_cast<const float*>(x),
                                                             static_cast<const float*>(weight), bias, relu,
                                                             static_cast<float*>(y));
  return launch_status();
}

size_t layer_grad_workspace_bytes(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype) {
  return dtype == MAESTRO_BF16 ? layer_grad_bf16_workspace_bytes(n, d_in, d_out) : 0;
}

maestro_status launch_layer_grad(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* x,
                                 const void* weight, const void* g_z, bool relu_input, void* g_x, float* g_weight,
                                 float* g_bias, void* workspace, hipStream_t stream) {
  if (dtype == MAESTRO_BF16)
    return launch_layer_grad_bf16(n, d_in, d_out, x, weight, g_z, relu_input, g_x, g_weight, g_bias, workspace, stream);
  return grads(n, d_in, d_out, static_cast<const float*>(x), static_cast<const float*>(weight),
               static_cast<const float*>(g_z), relu_input, static_cast<float*>(g_x), g_weight, g_bias, stream);
}

}  // namespace maestro
