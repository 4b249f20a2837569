// The bfloat16 products (products_bf16.h) of a predictor's layer and its gradients: tiles, cuts and launches.
//
// Bound by the matrix cores on wide layers, by HBM on narrow ones. Measured: 262,139 x 1024 -> 1024
// (0.55 TFLOP a product) activations 523 us in the first launches, 550 in a long run and up to 680 in between, while the
// clock settles to the matrix cores' power; input's gradient 535 and 560, weights' 447 and 475, 20 more to join its shares
// (as calls, over changing inputs: 533, and 1,047 for both gradients). A 16,384-cubed library product reaches 1.31 to 1.35
// PFLOP/s on the same card, and the library's products of these shapes 555, 618 and 1,230 us. 512 -> 256: activations 96 us for
// 403 MB, input's gradient 131 to 140 us for 671 MB = 4.8 to 5.1 TB/s, what a copy reaches.
#include "products_bf16.h"

namespace maestro {
namespace {

template <int WP, int WQ, int kDepth, int kBufs, bool kPT, bool kQT, class Out>
__global__ __launch_bounds__(kThreads, (Tile<WP, WQ, kDepth, kBufs, Out>::kResident)) void product_kernel(Product g, Out out) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[Tile<WP, WQ, kDepth, kBufs, Out>::kBytes];
  using L = Tile<WP, WQ, kDepth, kBufs, Out>;
  product<WP, WQ, kDepth, kBufs, kPT, kQT>(g, out, Dense<L::TP, L::TQ, kDepth>(g), lds, blockIdx.x, gridDim.x);
}

// Both gradients in one launch: the first `blocks` workgroups make the input's, in 64 x 64 tiles, the others the weights'.
template <int WP, int WQ>
__global__ __launch_bounds__(kThreads, 2) void pair_kernel(Product gx, InputGrad x, uint32_t blocks, Product gw, WeightGrad w) {
  using X = Tile<1, 1, 64, 2, InputGrad>;
  using W = Tile<WP, WQ, 64, 2, WeightGrad>;
  __shared__ __attribute__((aligned(16))) unsigned char lds[X::kBytes > W::kBytes ? X::kBytes : W::kBytes];
  if (blockIdx.x < blocks) product<1, 1, 64, 2, true, false>(gx, x, Dense<X::TP, X::TQ, 64>(gx), lds, blockIdx.x, blocks);
  else product<WP, WQ, 64, 2, true, true>(gw, w, Dense<W::TP, W::TQ, 64>(gw), lds, blockIdx.x - blocks, gridDim.x - blocks);
}

// g_w and g_b from their shares, summed in a fixed order. A quad of values to each of 256 / G neighbouring threads, its
// shares dealt out over G groups of them, each with the loads of eight shares issued before the first is added. G = 16
// where there are few values for the chip: the gradients of 91,341 x 32 -> 48 float32 (357 shares) take 31 us so and 45 in
// one chain of adds, of 65,536 x 256 -> 512 bfloat16 (64 shares) 42.9 and 44.8.
template <int G>
__global__ __launch_bounds__(kThreads) void join_kernel(const float* gw_parts, int32_t n_gw, float* gw, int64_t size,
                                                        const float* gb_parts, int32_t n_gb, float* gb, int32_t d_out) {
  constexpr int kQuads = kThreads / G;
  const int group = threadIdx.x / kQuads, own = threadIdx.x % kQuads;
  const int64_t quads = n_gw != 1 ? size / 4 : 0, all = quads + d_out / 4;      // one share is g_w itself
  __shared__ float4 s_sum[G][kQuads];
  for (int64_t first = (int64_t)blockIdx.x * kQuads; first < all; first += (int64_t)gridDim.x * kQuads) {
    const int64_t i = first + own;
    const bool w = i < quads;
    const float4* at = w ? reinterpret_cast<const float4*>(gw_parts) + i : reinterpret_cast<const float4*>(gb_parts) + (i - quads);
    const int64_t step = w ? size / 4 : d_out / 4;
    const int32_t n = i < all ? w ? n_gw : n_gb : 0;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    int32_t j = group;
    for (; j + 7 * G < n; j += 8 * G) {
      float4 a[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) a[u] = at[(j + u * G) * step];
#pragma unroll
      for (int u = 0; u < 8; ++u) s.x += a[u].x, s.y += a[u].y, s.z += a[u].z, s.w += a[u].w;
    }
    for (; j < n; j += G) {
      const float4 a = at[j * step];
      s.x += a.x, s.y += a.y, s.z += a.z, s.w += a.w;
    }
    if constexpr (G > 1) {
      __syncthreads();                                      // the last round's sums are read
      s_sum[group][own] = s;
      __syncthreads();
      if (group > 0) continue;
#pragma unroll
      for (int u = 1; u < G; ++u) {
        const float4 a = s_sum[u][own];
        s.x += a.x, s.y += a.y, s.z += a.z, s.w += a.w;
      }
    }
    if (i < all) (w ? reinterpret_cast<float4*>(gw) + i : reinterpret_cast<float4*>(gb) + (i - quads))[0] = s;
  }
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

template <int WP, int WQ, int kDepth, int kBufs, bool kPT, bool kQT, class Out>
maestro_status launch(Product g, const Out& out, hipStream_t stream) {
  const uint32_t blocks = plan<Tile<WP, WQ, kDepth, kBufs, Out>>(g);
  product_kernel<WP, WQ, kDepth, kBufs, kPT, kQT, Out><<<blocks, kThreads, 0, stream>>>(g, out);
  return launch_status();
}

template <int WP, int WQ>
maestro_status launch_pair(Product gx, const InputGrad& x, Product gw, const WeightGrad& w, hipStream_t stream) {
  const uint32_t blocks = plan<Tile<1, 1, 64, 2, InputGrad>>(gx), more = plan<Tile<WP, WQ, 64, 2, WeightGrad>>(gw);
  pair_kernel<WP, WQ><<<blocks + more, kThreads, 0, stream>>>(gx, x, blocks, gw, w);
  return launch_status();
}

// Tile of the activations and the input's gradient. A wavefront of a 256 x 256 tile reads half a KB of LDS for a
// product, of a 128 x 128 tile one, of a 64 x 64 tile two; but each size needs its tiles to be many: two
// rounds of workgroups or more, one for 128. Measured (us, tile 256 / 128 / 64): 262,139 x 1024 -> 1024
// 522 / 659 / 1568, 65,536 x 256 -> 512 (512 and 2,048 tiles) 28 / 30 / 55, 16,384 x 512 -> 512 (128 and 512) 22 / 15 / 23,
// 4,096 x 1024 -> 1024 (64 and 256) 30 / 15 / 20, 16,384 x 1024 -> 64 (128 of 128) 29 / 15 / 12.
int tile_of(int64_t np, int64_t nq) {
  if (np > 128 && cdiv(np, 256) * cdiv(nq, 256) >= 2 * kCus) return 256;
  return cdiv(np, 128) * cdiv(nq, 128) >= kCus ? 128 : 64;
}

// Stages of 64 k: rows whose k is contiguous come as whole 128-byte lines. (With stages of 32 and four buffers
// each line is fetched twice, its halves a stage apart: 552 against 522 us at 262,139 x 1024 -> 1024.)
template <bool kPT, class Out>
maestro_status launch_rows(const Product& g, const Out& out, hipStream_t stream) {
  const int tile = tile_of(g.np, g.nq);
  if (tile == 256) return launch<4, 4, 64, 2, kPT, false>(g, out, stream);
  if constexpr (!kPT)                                       // the input's gradient of this size: pair_kernel
    if (tile == 64) return launch<1, 1, 64, 2, kPT, false>(g, out, stream);
  return launch<2, 2, 64, 2, kPT, false>(g, out, stream);
}

// How the weights' gradient is cut: tile, k of one split, splits of the n rows, and workgroups that share the
// biases' sum (one where the rows are not split, so that no second launch is needed). 256 x 256 tiles for many rows, else 256 (d_in) x 64, or 128 x 128 where d_in is narrow;
// rows split so that there is one round of workgroups, none with fewer than 512 rows. Measured (us,
// 256 x 256 / 256 x 64 / 128 x 128): 262,139 x 1024 -> 1024 505 / 668 / 591, 512 -> 512 163 / 199 / 194,
// 1024 -> 64 153 / 149 / 154, 64 -> 1024 155 / 170 / 118; 65,536 x 512 -> 512 68 / 58 / 65; 16,384 41 / 32 / 38.
struct Cut {
  int32_t tp, tq;
  int64_t k_split, splits;
  int32_t parts;
};

Cut cut_of(int64_t n, int64_t d_in, int64_t d_out) {
  Cut c;
  c.tp = d_in > 128 ? 256 : 128;
  c.tq = c.tp == 128 ? 128 : d_out > 128 && n >= 131072 ? 256 : 64;
  const int64_t tiles = cdiv(d_in, c.tp) * cdiv(d_out, c.tq), resident = c.tq == 256 ? 1 : 2;
  int64_t splits = kCus * resident / tiles;
  if (splits > cdiv(n, 512)) splits = cdiv(n, 512);
  if (splits < 1) splits = 1;
  c.k_split = cdiv(cdiv(n, splits), 64) * 64;
  c.splits = cdiv(n, c.k_split);
  c.parts = c.splits > 1 ? (int32_t)cdiv(d_in, c.tp) : 1;
  return c;
}

}  // namespace

maestro_status launch_layer_bf16(int64_t n, int32_t d_in, int32_t d_out, const void* x, const void* weight,
                                 const float* bias, bool relu, void* y, hipStream_t stream) {
  Product g{static_cast<const __bf16*>(weight), static_cast<const __bf16*>(x), d_in, d_in, d_out, n, d_in, d_in, 1, 0, 0};
  return launch_rows<false>(g, Forward{bias, static_cast<__bf16*>(y), relu}, stream);
}

size_t layer_grad_bf16_workspace_bytes(int64_t n, int32_t d_in, int32_t d_out) {
  if (n == 0) return 0;
  const Cut c = cut_of(n, d_in, d_out);
  return c.splits > 1 ? sizeof(float) * (size_t)(c.splits * ((int64_t)d_in + c.parts * 2) * d_out) : 0;
}

maestro_status launch_layer_grad_bf16(int64_t n, int32_t d_in, int32_t d_out, const void* x, const void* weight,
                                      const void* g_z, bool relu_input, void* g_x, float* g_weight, float* g_bias,
                                      void* workspace, hipStream_t stream) {
  const __bf16 *xb = static_cast<const __bf16*>(x), *gz = static_cast<const __bf16*>(g_z);
  const Cut c = cut_of(n, d_in, d_out);
  float* parts = static_cast<float*>(workspace);
  float* gb_parts = parts + c.splits * d_in * d_out;
  const Product gw{xb, gz, d_in, d_out, d_in, d_out, n, c.k_split, 1, 0, 0};
  const WeightGrad w{c.splits > 1 ? parts : g_weight, c.splits > 1 ? gb_parts : g_bias, c.parts};
  const Product gx{static_cast<const __bf16*>(weight), gz, d_in, d_out, d_in, n, d_out, d_out, 1, 0, 0};
  const InputGrad x_out{xb, static_cast<__bf16*>(g_x), relu_input};
  maestro_status st = MAESTRO_OK;
  // Little work: a launch less, and the two products side by side. 300 x 256 -> 512 11.8 us (14.6 in two launches),
  // 2,000 x 512 -> 512 16.7 (22.6), 30,000 x 64 -> 128 18.7 (20.2)
  if (g_x && tile_of(d_in, n) == 64) {
    st = c.tp == 256 ? launch_pair<4, 1>(gx, x_out, gw, w, stream) : launch_pair<2, 2>(gx, x_out, gw, w, stream);
  } else {
    if (g_x) st = launch_rows<true>(gx, x_out, stream);
    if (st != MAESTRO_OK) return st;
    st = c.tq == 256   ? launch<4, 4, 32, 4, true, true>(gw, w, stream)
         : c.tp == 256 ? launch<4, 1, 64, 2, true, true>(gw, w, stream)
                       : launch<2, 2, 64, 2, true, true>(gw, w, stream);
  }
  if (st != MAESTRO_OK || c.splits == 1) return st;
  return launch_join(parts, (int32_t)c.splits, g_weight, (int64_t)d_in * d_out, gb_parts, (int32_t)(c.splits * c.parts * 2),
                     g_bias, d_out, stream);
}

maestro_status launch_join(const float* gw_parts, int32_t n_gw, float* gw, int64_t size, const float* gb_parts,
                           int32_t n_gb, float* gb, int32_t d_out, hipStream_t stream) {
  const int64_t quads = (n_gw != 1 ? size / 4 : 0) + d_out / 4, blocks = cdiv(quads, kThreads);
  if (blocks < kCus && n_gb > 8)
    join_kernel<16><<<(unsigned)cdiv(quads, kThreads / 16), kThreads, 0, stream>>>(gw_parts, n_gw, gw, size, gb_parts, n_gb, gb, d_out);
  else
    join_kernel<1><<<(unsigned)(blocks < 4096 ? blocks : 4096), kThreads, 0, stream>>>(gw_parts, n_gw, gw, size, gb_parts, n_gb, gb, d_out);
  return launch_status();
}

}  // namespace maestro
