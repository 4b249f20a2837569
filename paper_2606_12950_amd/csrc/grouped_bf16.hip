// The bfloat16 products (products_bf16.h) of a grouped layer and its gradients.
//
// Rows of a group make tiles of their own, each against the group's weights; workgroups are persistent and find a tile's group
// in a table of the groups' rows that each wavefront builds. The weights' gradients cut the rows of all groups together into shares of
// k_split, which a workgroup takes group after group, or, where rows are few, every group's by itself into units of k_split; a group of one
// part writes its gradient, of more its parts, which a second launch adds in order.
#include "groups.h"
#include "layers.h"
#include "products_bf16.h"

namespace maestro {
namespace {

using namespace grouped_bf16;

template <int TP, int TQ, int kDepth>
struct GroupedRows : GroupedRowsWay<8> {
  const Product& g;
  __device__ __forceinline__ Item item(const Way& c) const {
    const Place at = place(c, TQ);
    Item t;
    t.group = at.group;
    t.p = g.p + at.group * (g.np * g.nk);
    t.q = g.q;
    t.q0 = at.q0;
    t.q_end = at.q_end;
    t.p0 = at.p_tile * TP;
    t.k0 = 0;
    t.kn = g.nk;
    t.stages = (g.nk + kDepth - 1) / kDepth;
    t.slot = 0;
    t.whole = t.direct = true;
    return t;
  }
};

template <int TP, int TQ, int kDepth, GroupUnits kUnits, bool kShared>
struct GroupedSums : GroupedSumsWay<8, kUnits, kShared> {
  using Way = typename GroupedSumsWay<8, kUnits, kShared>::Way;
  const Product& g;
  __device__ __forceinline__ Item item(const Way& c) const {
    const auto at = this->place(c);
    const int q_tile = quotient(at.tile, g.p_tiles);
    Item t;
    t.group = at.group;
    t.p = g.p;
    t.q = g.q;
    t.q0 = q_tile * TQ;
    t.q_end = g.nq;
    t.p0 = (at.tile - q_tile * g.p_tiles) * TP;
    t.k0 = at.k0;
    t.kn = at.k_end - at.k0;
    t.stages = (at.k_end - at.k0 + kDepth - 1) / kDepth;
    t.slot = at.slot;
    t.whole = true;
    t.direct = at.direct;
    return t;
  }
};

struct GroupedWeightGrad {
  static constexpr bool kBias = false, kInt8 = false, kCodes = false;
  float *gw, *gb, *gw_parts, *gb_parts;
  int32_t parts;                     // 1
  __device__ __forceinline__ float* weights(const Product& g, const Item& t) const {
    return t.direct ? gw + t.group * (g.nq * g.np) : gw_parts + t.slot * (g.nq * g.np);
  }
  __device__ __forceinline__ float* biases(const Product& g, const Item& t, int64_t, int) const {
    return t.direct ? gb + t.group * g.nq : gb_parts + t.slot * g.nq;
  }
};

template <int WP, int WQ, int kDepth, int kBufs, bool kPT, int kWaves, class Out>
__global__ __launch_bounds__(64 * kWaves, (Tile<WP, WQ, kDepth, kBufs, Out, kWaves>::kSimdWaves)) void rows_kernel(
    Product g, Out out, const int64_t* offsets, int32_t n_groups, int32_t n) {
  using L = Tile<WP, WQ, kDepth, kBufs, Out, kWaves>;
  __shared__ __attribute__((aligned(16))) unsigned char lds[L::kBytes];
  GroupTable table;
  table.build<kTiles>(offsets, n_groups, n, L::TQ);
  product<WP, WQ, kDepth, kBufs, kPT, false, kWaves>(g, out, GroupedRows<L::TP, L::TQ, kDepth>{{table, g.p_tiles}, g}, lds, blockIdx.x, gridDim.x);
}

// alone: no group has more than one unit, and no second launch follows.
template <int WP, int WQ, int kDepth, int kBufs, int kWaves, GroupUnits kUnits, bool kShared>
__global__ __launch_bounds__(64 * kWaves, (Tile<WP, WQ, kDepth, kBufs, GroupedWeightGrad, kWaves>::kSimdWaves)) void sums_kernel(
    Product g, GroupedWeightGrad out, const int64_t* offsets, int32_t n_groups, int32_t n, bool alone) {
  using L = Tile<WP, WQ, kDepth, kBufs, GroupedWeightGrad, kWaves>;
  __shared__ __attribute__((aligned(16))) unsigned char lds[L::kBytes];
  GroupTable table;
  table.build<kUnits>(offsets, n_groups, n, (int)g.k_split);
  const int tiles = (int)((g.nq + L::TQ - 1) / L::TQ) * g.p_tiles;
  product<WP, WQ, kDepth, kBufs, true, true, kWaves>(g, out, GroupedSums<L::TP, L::TQ, kDepth, kUnits, kShared>{{table, tiles, (int)g.k_split}, g}, lds, blockIdx.x,
                                                gridDim.x);
  if (alone) clear_empty_groups(table, out.gw, g.np * g.nq, out.gb, (int)g.nq, blockIdx.x, gridDim.x);
}

// Both gradients in one launch, in 64 x 64 tiles: the first `blocks` workgroups make the input's, the others the weights'.
template <bool kShared>
__global__ __launch_bounds__(kThreads, 4) void pair_kernel(Product gx, InputGrad x, uint32_t blocks, Product gw, GroupedWeightGrad w,
                                                           const int64_t* offsets, int32_t n_groups, int32_t n, bool alone) {
  using X = Tile<1, 1, 64, 2, InputGrad>;
  using W = Tile<1, 1, 64, 2, GroupedWeightGrad>;
  __shared__ __attribute__((aligned(16))) unsigned char lds[X::kBytes > W::kBytes ? X::kBytes : W::kBytes];
  GroupTable table;
  if (blockIdx.x < blocks) {
    table.build<kTiles>(offsets, n_groups, n, X::TQ);
    product<1, 1, 64, 2, true, false>(gx, x, GroupedRows<X::TP, X::TQ, 64>{{table, gx.p_tiles}, gx}, lds, blockIdx.x, blocks);
    return;
  }
  table.build<kTiles>(offsets, n_groups, n, (int)gw.k_split);
  const int tiles = (int)((gw.nq + W::TQ - 1) / W::TQ) * gw.p_tiles;
  product<1, 1, 64, 2, true, true>(gw, w, GroupedSums<W::TP, W::TQ, 64, kTiles, kShared>{{table, tiles, (int)gw.k_split}, gw}, lds,
                                   blockIdx.x - blocks, gridDim.x - blocks);
  if (alone) clear_empty_groups(table, w.gw, gw.np * gw.nq, w.gb, (int)gw.nq, blockIdx.x - blocks, gridDim.x - blocks);
}

uint32_t blocks_of(int64_t items, int64_t resident) {
  const int64_t want = cdiv(items, 8) * 8, most = kCus * resident;
  return (uint32_t)(want < most ? want : most);
}

template <int WP, int WQ, bool kPT, int kWaves, class Out>
void launch_tiles(Product g, const Out& out, const int64_t* offsets, int32_t n_groups, int64_t n, hipStream_t stream) {
  using L = Tile<WP, WQ, 64, 2, Out, kWaves>;
  g.p_tiles = (int32_t)cdiv(g.np, L::TP);
  const uint32_t blocks = blocks_of((n / L::TQ + n_groups) * g.p_tiles, L::kResident);
  rows_kernel<WP, WQ, 64, 2, kPT, kWaves><<<blocks, 64 * kWaves, 0, stream>>>(g, out, offsets, n_groups, (int32_t)n);
}

template <bool kPT, class Out>
void launch_rows(const Product& g, const Out& out, const int64_t* offsets, int32_t n_groups, int64_t n, hipStream_t stream) {
  const int tile = tile_of(kPT, g.np, n);
  if (tile == 256) {
    if constexpr (kPT) launch_tiles<4, 4, kPT, 4>(g, out, offsets, n_groups, n, stream);
    else launch_tiles<4, 2, kPT, 8>(g, out, offsets, n_groups, n, stream);
  } else if (tile == 128) {
    launch_tiles<2, 2, kPT, 4>(g, out, offsets, n_groups, n, stream);
  } else {
    launch_tiles<1, 1, kPT, 4>(g, out, offsets, n_groups, n, stream);
  }
}

template <int WP, int WQ, int kDepth, int kBufs, int kWaves>
void launch_sums(Product g, const GroupedWeightGrad& out, const int64_t* offsets, int32_t n_groups, int32_t n, bool by_group,
                 bool alone, hipStream_t stream) {
  using L = Tile<WP, WQ, kDepth, kBufs, GroupedWeightGrad, kWaves>;
  g.p_tiles = (int32_t)cdiv(g.np, L::TP);
  const int64_t pieces = by_group ? n / g.k_split + n_groups : cdiv(n, g.k_split);
  const uint32_t blocks = blocks_of(pieces * g.p_tiles * cdiv(g.nq, L::TQ), L::kResident);
  auto of = [&](auto shared) {
    constexpr bool kShared = decltype(shared)::value;
    if constexpr (WP * WQ == 1) return sums_kernel<WP, WQ, kDepth, kBufs, kWaves, kTiles, kShared>;          // always by group
    else if constexpr (WP * WQ == 8) return sums_kernel<WP, WQ, kDepth, kBufs, kWaves, kShares, kShared>;    // 131,072 rows and more: never
    else return by_group ? sums_kernel<WP, WQ, kDepth, kBufs, kWaves, kTiles, kShared> : sums_kernel<WP, WQ, kDepth, kBufs, kWaves, kShares, kShared>;
  };
  auto kernel = shared_places(n, n_groups, g.k_split) ? of(std::true_type{}) : of(std::false_type{});
  kernel<<<blocks, 64 * kWaves, 0, stream>>>(g, out, offsets, n_groups, n, alone);
}

void launch_pair(Product gx, const InputGrad& x, Product gw, const GroupedWeightGrad& w, const int64_t* offsets, int32_t n_groups,
                 int32_t n, bool alone, hipStream_t stream) {
  gx.p_tiles = (int32_t)cdiv(gx.np, 64);
  gw.p_tiles = (int32_t)cdiv(gw.np, 64);
  const uint32_t blocks = blocks_of((n / 64 + n_groups) * gx.p_tiles, 4);
  const uint32_t more = blocks_of((n / gw.k_split + n_groups) * gw.p_tiles * cdiv(gw.nq, 64), 4);
  auto kernel = shared_places(n, n_groups, gw.k_split) ? pair_kernel<true> : pair_kernel<false>;
  kernel<<<blocks + more, kThreads, 0, stream>>>(gx, x, blocks, gw, w, offsets, n_groups, n, alone);
}

}  // namespace

maestro_status launch_layer_grouped_bf16(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, const void* x,
                                         const void* weight, const float* bias, const int64_t* offsets, bool relu, void* y,
                                         hipStream_t stream) {
  const Product g{static_cast<const __bf16*>(weight), static_cast<const __bf16*>(x), d_in, d_in, d_out, n, d_in, d_in, 1, 0, 0};
  launch_rows<false>(g, Forward{bias, static_cast<__bf16*>(y), relu}, offsets, n_groups, n, stream);
  return launch_status();
}

size_t grouped_grad_bf16_workspace_bytes(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out) {
  if (n == 0) return 0;
  const Cut c = cut_of(n, n_groups, d_in, d_out);
  return n <= c.k_split ? 0 : sizeof(float) * (size_t)(places_of(n, n_groups, c.k_split) * ((int64_t)d_in + 1) * d_out);
}

maestro_status launch_grouped_grad_bf16(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, const void* x,
                                        const void* weight, const void* g_z, const int64_t* offsets, bool relu_input,
                                        void* g_x, float* g_weight, float* g_bias, void* workspace, hipStream_t stream) {
  const int64_t size = (int64_t)d_in * d_out;
  if (n == 0) return launch_join_groups(0, n_groups, offsets, 1, true, nullptr, g_weight, size, nullptr, g_bias, d_out, stream);
  const __bf16 *xb = static_cast<const __bf16*>(x), *gz = static_cast<const __bf16*>(g_z);
  const Cut c = cut_of(n, n_groups, d_in, d_out);
  float *gw_parts = static_cast<float*>(workspace), *gb_parts = gw_parts + places_of(n, n_groups, c.k_split) * size;
  const Product gx{static_cast<const __bf16*>(weight), gz, d_in, d_out, d_in, n, d_out, d_out, 1, 0, 0};
  const InputGrad x_out{xb, static_cast<__bf16*>(g_x), relu_input};
  const Product gw{xb, gz, d_in, d_out, d_in, d_out, n, c.k_split, 1, 0, 0};
  const GroupedWeightGrad out{g_weight, g_bias, gw_parts, gb_parts, 1};
  const bool alone = n <= c.k_split;
  if (g_x && paired(c, n, d_in)) {
    launch_pair(gx, x_out, gw, out, offsets, n_groups, (int32_t)n, alone, stream);
  } else {
    if (g_x) launch_rows<true>(gx, x_out, offsets, n_groups, n, stream);
    auto sums = c.tp == 64 ? launch_sums<1, 1, 64, 2, 4> : c.tq == 256 ? launch_sums<4, 2, 32, 4, 8>
              : c.tp == 256 ? launch_sums<4, 1, 64, 2, 4> : launch_sums<2, 2, 64, 2, 4>;
    sums(gw, out, offsets, n_groups, (int32_t)n, c.by_group, alone, stream);
  }
  const maestro_status st = launch_status();
  if (st != MAESTRO_OK || alone) return st;
  return launch_join_groups(n, n_groups, offsets, c.k_split, c.by_group, gw_parts, g_weight, size, gb_parts, g_bias, d_out, stream);
}

}  // namespace maestro
