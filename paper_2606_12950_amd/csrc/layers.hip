// A predictor's Linear layer with its activations kept, and the layer's gradients: the float32 products (products_f32.h), and the
// choice between them and the bfloat16 ones.
//
// Bound by the float32 matrix cores (64 operations a cycle and SIMD, 1/16 of bfloat16) on wide
// layers, by launches on the small ones it is for. Measured: 4,096 x 64 -> 128 5.5 us, 60,000 x 1024 -> 1024
// 1,061 (floor 833), 150,000 x 256 -> 256 195 (130): one 16-k stage ahead does not cover a load; see wide and cut_of for the rest.
#include "products_f32.h"

namespace maestro {
namespace {

template <int W, bool kPT, bool kQT, class Out>
__global__ __launch_bounds__(kThreads, 2) void product_kernel(Product g, Out out) {
  __shared__ __attribute__((aligned(16))) Lds<W> lds;
  product<W, kPT, kQT>(g, out, Dense<64 * W, Floats>(g), lds, blockIdx.x, gridDim.x);
}

// Both gradients in one launch, in 64 x 64 tiles: the first `blocks` workgroups make the input's, the others the weights'.
__global__ __launch_bounds__(kThreads, 2) void pair_kernel(Product gx, InputGrad x, uint32_t blocks, Product gw, WeightGrad w) {
  __shared__ __attribute__((aligned(16))) Lds<1> lds;
  if (blockIdx.x < blocks) product<1, true, false>(gx, x, Dense<64, Floats>(gx), lds, blockIdx.x, blocks);
  else product<1, true, true>(gw, w, Dense<64, Floats>(gw), lds, blockIdx.x - blocks, gridDim.x - blocks);
}

// the rest of a product's numbers, and its workgroups
template <int W>
uint32_t plan(Product& g) {
  constexpr int T = 64 * W;
  g.p_tiles = cdiv(g.np, T);
  g.items = cdiv(g.nq, T) * g.p_tiles * g.splits;
  return (uint32_t)(g.items < 65536 ? g.items : 65536);
}

template <int W, bool kPT, bool kQT, class Out>
void launch(Product g, const Out& out, hipStream_t stream) {
  const uint32_t blocks = plan<W>(g);
  product_kernel<W, kPT, kQT><<<blocks, kThreads, 0, stream>>>(g, out);
}

// 128 x 128 tiles where there are two rounds of them, else 64 x 64. Activations take the larger ones only where k is long
// and 128 columns fit no worse than 64. Measured (us, 128 / 64): activations of 150,000 x 80 -> 160 75 / 53, 128 -> 128 64 /
// 59, 192 -> 192 167 / 135, 256 -> 256 233 / 235, 60,000 x 1024 -> 1024 1163 / 1215; input's gradients of 150,000 x 256 ->
// 256 210 / 257, 60,000 x 1024 -> 1024 1074 / 1658.
bool wide(int64_t np, int64_t nq) { return np > 64 && nq > 64 && cdiv(np, 128) * cdiv(nq, 128) >= 2 * kCus; }
bool wide_forward(int64_t np, int64_t nq, int64_t nk) { return wide(np, nq) && nk >= 192 && cdiv(np, 64) % 2 == 0; }

// The weights' gradient: the rows split so that there are about two workgroups a CU, none with fewer than 256 rows. 128 x 128
// tiles for many rows where they hold at most 1.2 times what 64 x 64 ones do: 150,000 x 192 -> 192 191 us (150 with 64), 256 ->
// 256 203 (246), 96 -> 96 58 (68).
struct Cut {
  bool wide;
  int64_t k_split, splits;
};
Cut cut_of(int64_t n, int64_t d_in, int64_t d_out) {
  Cut c;
  const int64_t large = 4 * cdiv(d_in, 128) * cdiv(d_out, 128), small = cdiv(d_in, 64) * cdiv(d_out, 64);
  c.wide = d_in > 64 && d_out > 64 && n >= 32768 && 5 * large <= 6 * small;
  const int64_t t = c.wide ? 128 : 64, tiles = cdiv(d_in, t) * cdiv(d_out, t);
  int64_t splits = 2 * kCus / tiles;
  if (splits > cdiv(n, 256)) splits = cdiv(n, 256);
  if (splits < 1) splits = 1;
  c.k_split = cdiv(cdiv(n, splits), kDepth) * kDepth;
  c.splits = cdiv(n, c.k_split);
  return c;
}

}  // namespace

maestro_status launch_layer(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* x, const void* weight,
                            const float* bias, bool relu, void* y, hipStream_t stream) {
  if (dtype == MAESTRO_BF16) return launch_layer_bf16(n, d_in, d_out, x, weight, bias, relu, y, stream);
  const Product g{{static_cast<const float*>(weight), d_in}, {static_cast<const float*>(x), d_in}, d_out, n, d_in, d_in, 1, 0, 0};
  const Forward out{bias, static_cast<float*>(y), relu};
  if (wide_forward(d_out, n, d_in)) launch<2, false, false>(g, out, stream);
  else launch<1, false, false>(g, out, stream);
  return launch_status();
}

size_t layer_grad_workspace_bytes(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype) {
  if (dtype == MAESTRO_BF16) return layer_grad_bf16_workspace_bytes(n, d_in, d_out);
  if (n == 0) return 0;
  const int64_t splits = cut_of(n, d_in, d_out).splits;
  return splits > 1 ? sizeof(float) * (size_t)(splits * ((int64_t)d_in + 1) * d_out) : 0;
}

maestro_status launch_layer_grad(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* x,
                                 const void* weight, const void* g_z, bool relu_input, void* g_x, float* g_weight,
                                 float* g_bias, void* workspace, hipStream_t stream) {
  const int64_t size = (int64_t)d_in * d_out;
  if (n == 0) return launch_join(nullptr, 0, g_weight, size, nullptr, 0, g_bias, d_out, stream);
  if (dtype == MAESTRO_BF16)
    return launch_layer_grad_bf16(n, d_in, d_out, x, weight, g_z, relu_input, g_x, g_weight, g_bias, workspace, stream);
  const float *xf = static_cast<const float*>(x), *gz = static_cast<const float*>(g_z);
  const Cut c = cut_of(n, d_in, d_out);
  float* parts = static_cast<float*>(workspace);
  Product gw{{xf, d_in}, {gz, d_out}, d_in, d_out, n, c.k_split, c.splits, 0, 0};
  const WeightGrad w{c.splits > 1 ? parts : g_weight, c.splits > 1 ? parts + c.splits * size : g_bias};
  Product gx{{static_cast<const float*>(weight), d_in}, {gz, d_out}, d_in, n, d_out, d_out, 1, 0, 0};
  const InputGrad x_out{xf, static_cast<float*>(g_x), relu_input};
  if (g_x && !c.wide && !wide(d_in, n)) {                   // 20,000 x 128 -> 128 25.6 us (33.5 in two launches)
    const uint32_t blocks = plan<1>(gx), more = plan<1>(gw);
    pair_kernel<<<blocks + more, kThreads, 0, stream>>>(gx, x_out, blocks, gw, w);
  } else {
    if (g_x && wide(d_in, n)) launch<2, true, false>(gx, x_out, stream);
    else if (g_x) launch<1, true, false>(gx, x_out, stream);
    if (c.wide) launch<2, true, true>(gw, w, stream);
    else launch<1, true, true>(gw, w, stream);
  }
  if (c.splits == 1) return launch_status();
  return launch_join(parts, (int32_t)c.splits, g_weight, size, parts + c.splits * size, (int32_t)c.splits, g_bias, d_out,
                     stream);
}

}  // namespace maestro
