// The bfloat16 products (products_bf16.h) of a layer's gradients from an input kept in 8 bits.
//
// The weights' gradient takes the codes as its operand P and makes values of them on the way into LDS; the input's needs
// them for its mask only. Nothing is unpacked in memory.
#include "layers.h"
#include "products_bf16.h"

namespace maestro {
namespace {

using namespace packed_bf16;

template <int WP, int WQ, bool kQT, int kWaves, class Out>
__global__ __launch_bounds__(64 * kWaves, (Tile<WP, WQ, 64, 2, Out, kWaves>::kSimdWaves)) void product_kernel(Product g, Out out) {
  using L = Tile<WP, WQ, 64, 2, Out, kWaves>;
  __shared__ __attribute__((aligned(16))) unsigned char lds[L::kBytes];
  product<WP, WQ, 64, 2, true, kQT, kWaves>(g, out, Dense<L::TP, L::TQ, 64>(g), lds, blockIdx.x, gridDim.x);
}

// Both gradients in one launch: the first `blocks` workgroups make the input's, in 64 x 64 tiles, the others the weights'.
template <int WP, int WQ, class Code>
__global__ __launch_bounds__(kThreads, (WP * WQ == 1 ? 4 : 2)) void pair_kernel(Product gx, CodesInputGrad x, uint32_t blocks, Product gw, CodesWeightGrad<Code> w) {
  using X = Tile<1, 1, 64, 2, CodesInputGrad>;
  using W = Tile<WP, WQ, 64, 2, CodesWeightGrad<Code>>;
  __shared__ __attribute__((aligned(16))) unsigned char lds[X::kBytes > W::kBytes ? X::kBytes : W::kBytes];
  if (blockIdx.x < blocks) product<1, 1, 64, 2, true, false>(gx, x, Dense<X::TP, X::TQ, 64>(gx), lds, blockIdx.x, blocks);
  else product<WP, WQ, 64, 2, true, true>(gw, w, Dense<W::TP, W::TQ, 64>(gw), lds, blockIdx.x - blocks, gridDim.x - blocks);
}

// the rest of a product's numbers, and its workgroups
template <class Tile>
uint32_t plan(Product& g) {
  g.p_tiles = (int32_t)cdiv(g.np, Tile::TP);
  g.splits = (int32_t)cdiv(g.nk, g.k_split);
  g.items = cdiv(g.nq, Tile::TQ) * g.p_tiles * g.splits;
  const int64_t want = cdiv(g.items, 8) * 8, most = kCus * Tile::kResident;
  return (uint32_t)(want < most ? want : most);
}

template <int WP, int WQ, bool kQT, int kWaves, class Out>
void launch(Product g, const Out& out, hipStream_t stream) {
  const uint32_t blocks = plan<Tile<WP, WQ, 64, 2, Out, kWaves>>(g);
  product_kernel<WP, WQ, kQT, kWaves><<<blocks, 64 * kWaves, 0, stream>>>(g, out);
}

template <int WP, int WQ, class Code>
void launch_pair(Product gx, const CodesInputGrad& x, Product gw, const CodesWeightGrad<Code>& w, hipStream_t stream) {
  const uint32_t blocks = plan<Tile<1, 1, 64, 2, CodesInputGrad>>(gx), more = plan<Tile<WP, WQ, 64, 2, CodesWeightGrad<Code>>>(gw);
  pair_kernel<WP, WQ><<<blocks + more, kThreads, 0, stream>>>(gx, x, blocks, gw, w);
}

template <class Code>
void launch_gradients(int64_t n, const Product& gx, const CodesInputGrad& x, const Product& gw, const CodesWeightGrad<Code>& w,
                      const Cut& c, hipStream_t stream) {
  const int tile = tile_of(gx.np, n);
  if (x.c && tile == 64) {                                  // few enough tiles for it: c.tp is not 256 by any size
    if (c.tp == 64) launch_pair<1, 1>(gx, x, gw, w, stream);
    else launch_pair<2, 2>(gx, x, gw, w, stream);
    return;
  }
  if (x.c && tile == 256) launch<4, 4, false, 4>(gx, x, stream);
  else if (x.c) launch<2, 2, false, 4>(gx, x, stream);
  if (c.tp == 64) launch<1, 1, true, 4>(gw, w, stream);
  else if (c.tq == 256) launch<4, 2, true, 8>(gw, w, stream);
  else if (c.tp == 256) launch<4, 1, true, 4>(gw, w, stream);
  else launch<2, 2, true, 4>(gw, w, stream);
}

}  // namespace

size_t grad_packed_bf16_workspace_bytes(int64_t n, int32_t d_in, int32_t d_out) {
  if (n == 0) return 0;
  const Cut c = cut_of(n, d_in, d_out);
  return c.splits > 1 ? sizeof(float) * (size_t)(c.splits * ((int64_t)d_in + c.parts * 2) * d_out) : 0;
}

maestro_status launch_grad_packed_bf16(int64_t n, int32_t d_in, int32_t d_out, const void* codes, const uint8_t* exponents,
                                       bool rectified, const void* weight, const void* g_z, bool relu_input, void* g_x,
                                       float* g_weight, float* g_bias, void* workspace, hipStream_t stream) {
  const __bf16* gz = static_cast<const __bf16*>(g_z);
  const Cut c = cut_of(n, d_in, d_out);
  float* parts = static_cast<float*>(workspace);
  float* gb_parts = parts + c.splits * d_in * d_out;
  const Product gw{nullptr, gz, d_in, d_out, d_in, d_out, n, c.k_split, 1, 0, 0};
  const Product gx{static_cast<const __bf16*>(weight), gz, d_in, d_out, d_in, n, d_out, d_out, 1, 0, 0};
  const CodesInputGrad x_out{static_cast<const unsigned char*>(codes), static_cast<__bf16*>(g_x), relu_input};
  const WeightGrad w{c.splits > 1 ? parts : g_weight, c.splits > 1 ? gb_parts : g_bias, c.parts};
  const int64_t blocks = (d_in + 31) / 32;
  if (rectified) launch_gradients(n, gx, x_out, gw, CodesWeightGrad<uint8_t>{w, static_cast<const uint8_t*>(codes), exponents, blocks}, c, stream);
  else launch_gradients(n, gx, x_out, gw, CodesWeightGrad<int8_t>{w, static_cast<const int8_t*>(codes), exponents, blocks}, c, stream);
  const maestro_status st = launch_status();
  if (st != MAESTRO_OK || c.splits == 1) return st;
  return launch_join(parts, (int32_t)c.splits, g_weight, (int64_t)d_in * d_out, gb_parts, (int32_t)(c.splits * c.parts * 2),
                     g_bias, d_out, stream);
}

}  // namespace maestro
