// The float32 products (products_f32.h) of a layer's gradients from an input kept in 8 bits: codes become values as they are
// loaded for the weights' gradient, and mask the input's. Nothing is unpacked in memory.
#include "layers.h"
#include "products_f32.h"

namespace maestro {
namespace {

using namespace packed_f32;

template <int W, bool kQT, class P, class Out>
__global__ __launch_bounds__(kThreads, 2) void product_kernel(ProductOf<P> g, Out out) {
  __shared__ __attribute__((aligned(16))) Lds<W> lds;
  product<W, true, kQT>(g, out, Dense<64 * W, P>(g), lds, blockIdx.x, gridDim.x);
}

// Both gradients in one launch, in 64 x 64 tiles: the first `blocks` workgroups make the input's, the others the weights'.
template <class P>
__global__ __launch_bounds__(kThreads, 2) void pair_kernel(Product gx, CodesInputGrad x, uint32_t blocks, ProductOf<P> gw, WeightGrad w) {
  __shared__ __attribute__((aligned(16))) Lds<1> lds;
  if (blockIdx.x < blocks) product<1, true, false>(gx, x, Dense<64, Floats>(gx), lds, blockIdx.x, blocks);
  else product<1, true, true>(gw, w, Dense<64, P>(gw), lds, blockIdx.x - blocks, gridDim.x - blocks);
}

// the rest of a product's numbers, and its workgroups
template <int W, class P>
uint32_t plan(ProductOf<P>& g) {
  constexpr int T = 64 * W;
  g.p_tiles = cdiv(g.np, T);
  g.items = cdiv(g.nq, T) * g.p_tiles * g.splits;
  return (uint32_t)(g.items < 65536 ? g.items : 65536);
}

template <int W, bool kQT, class P, class Out>
void launch(ProductOf<P> g, const Out& out, hipStream_t stream) {
  const uint32_t blocks = plan<W>(g);
  product_kernel<W, kQT><<<blocks, kThreads, 0, stream>>>(g, out);
}

template <class Code>
void launch_gradients(int64_t n, int32_t d_in, int32_t d_out, const Codes<Code>& x, const float* weight, const float* gz,
                      bool relu_input, float* g_x, const Cut& c, const WeightGrad& w, hipStream_t stream) {
  ProductOf<Codes<Code>> gw{x, {gz, d_out}, d_in, d_out, n, c.k_split, c.splits, 0, 0};
  Product gx{{weight, d_in}, {gz, d_out}, d_in, n, d_out, d_out, 1, 0, 0};
  const CodesInputGrad x_out{reinterpret_cast<const unsigned char*>(x.m), g_x, relu_input};
  if (g_x && paired(c, n, d_in)) {
    const uint32_t blocks = plan<1>(gx), more = plan<1>(gw);
    pair_kernel<<<blocks + more, kThreads, 0, stream>>>(gx, x_out, blocks, gw, w);
    return;
  }
  if (g_x && wide(d_in, n)) launch<2, false>(gx, x_out, stream);
  else if (g_x) launch<1, false>(gx, x_out, stream);
  if (c.wide) launch<2, true>(gw, w, stream);
  else launch<1, true>(gw, w, stream);
}

}  // namespace

size_t grad_packed_f32_workspace_bytes(int64_t n, int32_t d_in, int32_t d_out) {
  if (n == 0) return 0;
  const int64_t splits = cut_of(n, d_in, d_out).splits;
  return splits > 1 ? sizeof(float) * (size_t)(splits * ((int64_t)d_in + 1) * d_out) : 0;
}

maestro_status launch_grad_packed_f32(int64_t n, int32_t d_in, int32_t d_out, const void* codes, const uint8_t* exponents,
                                      bool rectified, const float* weight, const float* g_z, bool relu_input, float* g_x,
                                      float* g_weight, float* g_bias, void* workspace, hipStream_t stream) {
  const int64_t size = (int64_t)d_in * d_out, blocks = (d_in + 31) / 32;
  const Cut c = cut_of(n, d_in, d_out);
  float* parts = static_cast<float*>(workspace);
  const WeightGrad w{c.splits > 1 ? parts : g_weight, c.splits > 1 ? parts + c.splits * size : g_bias};
  if (rectified)
    launch_gradients(n, d_in, d_out, Codes<uint8_t>{static_cast<const uint8_t*>(codes), exponents, d_in, blocks}, weight, g_z,
                     relu_input, g_x, c, w, stream);
  else
    launch_gradients(n, d_in, d_out, Codes<int8_t>{static_cast<const int8_t*>(codes), exponents, d_in, blocks}, weight, g_z,
                     relu_input, g_x, c, w, stream);
  const maestro_status st = launch_status();
  if (st != MAESTRO_OK || c.splits == 1) return st;
  return launch_join(parts, (int32_t)c.splits, g_weight, size, parts + c.splits * size, (int32_t)c.splits, g_bias, d_out, stream);
}

}  // namespace maestro
