// The float32 products (products_f32.h) of a grouped layer and its gradients, and the join of a group's shares.
//
// Rows of a group make tiles of their own, each against the group's weights. The weights' gradients cut the rows of all groups together
// into shares of k_split, or, where rows are few, every group's by itself into units of k_split; a group of one part writes its gradient, of
// more its parts, which a second launch adds in order.
#include "groups.h"
#include "layers.h"
#include "products_f32.h"

namespace maestro {
namespace {

using namespace grouped_f32;

template <int T>
struct GroupedRows : GroupedRowsWay<1> {
  const Product& g;
  __device__ __forceinline__ Item item(const Way& c) const {
    const Place at = place(c, T);
    Item t;
    t.group = at.group;
    t.p_shift = at.group * (g.np * g.nk);
    t.q0 = at.q0;
    t.q_end = at.q_end;
    t.p0 = at.p_tile * T;
    t.k0 = 0;
    t.k_end = g.nk;
    t.slot = 0;
    t.direct = true;
    return t;
  }
};

template <int T, GroupUnits kUnits, bool kShared>
struct GroupedSums : GroupedSumsWay<1, kUnits, kShared> {
  using Way = typename GroupedSumsWay<1, kUnits, kShared>::Way;
  const Product& g;
  __device__ __forceinline__ Item item(const Way& c) const {
    const auto at = this->place(c);
    const int p_tiles = (int)g.p_tiles, q_tile = quotient(at.tile, p_tiles);
    Item t;
    t.group = at.group;
    t.p_shift = 0;
    t.q0 = q_tile * T;
    t.q_end = g.nq;
    t.p0 = (at.tile - q_tile * p_tiles) * T;
    t.k0 = at.k0;
    t.k_end = at.k_end;
    t.slot = at.slot;
    t.direct = at.direct;
    return t;
  }
};

struct GroupedWeightGrad {
  float *gw, *gb, *gw_parts, *gb_parts;
  __device__ __forceinline__ void finish(const Item& t, int64_t np, int64_t nq, int64_t q, int64_t p, float4 c) const {
    float* at = t.direct ? gw + t.group * nq * np : gw_parts + t.slot * nq * np;
    *reinterpret_cast<float4*>(at + q * np + p) = c;
  }
  __device__ __forceinline__ float* bias(const Item& t, int64_t nq, int64_t q) const {
    return (t.direct ? gb + t.group * nq : gb_parts + t.slot * nq) + q;
  }
};

template <int W, bool kPT, class Out>
__global__ __launch_bounds__(kThreads, 2) void rows_kernel(Product g, Out out, const int64_t* offsets, int32_t n_groups, int32_t n) {
  __shared__ __attribute__((aligned(16))) Lds<W> lds;
  GroupTable table;
  table.build<kTiles>(offsets, n_groups, n, 64 * W);
  product<W, kPT, false>(g, out, GroupedRows<64 * W>{{table, (int)g.p_tiles}, g}, lds, blockIdx.x, gridDim.x);
}

// alone: no group has more than one unit, and no second launch follows.
template <int W, GroupUnits kUnits, bool kShared>
__global__ __launch_bounds__(kThreads, 2) void sums_kernel(Product g, GroupedWeightGrad out, const int64_t* offsets, int32_t n_groups,
                                                           int32_t n, bool alone) {
  __shared__ __attribute__((aligned(16))) Lds<W> lds;
  GroupTable table;
  table.build<kUnits>(offsets, n_groups, n, (int)g.k_split);
  const int tiles = (int)((g.nq + 64 * W - 1) / (64 * W) * g.p_tiles);
  product<W, true, true>(g, out, GroupedSums<64 * W, kUnits, kShared>{{table, tiles, (int)g.k_split}, g}, lds, blockIdx.x, gridDim.x);
  if (alone) clear_empty_groups(table, out.gw, g.np * g.nq, out.gb, (int)g.nq, blockIdx.x, gridDim.x);
}

// Both gradients in one launch, in 64 x 64 tiles: the first `blocks` workgroups make the input's, the others the weights'.
template <bool kShared>
__global__ __launch_bounds__(kThreads, 2) void pair_kernel(Product gx, InputGrad x, uint32_t blocks, Product gw, GroupedWeightGrad w,
                                                           const int64_t* offsets, int32_t n_groups, int32_t n, bool alone) {
  __shared__ __attribute__((aligned(16))) Lds<1> lds;
  GroupTable table;
  if (blockIdx.x < blocks) {
    table.build<kTiles>(offsets, n_groups, n, 64);
    product<1, true, false>(gx, x, GroupedRows<64>{{table, (int)gx.p_tiles}, gx}, lds, blockIdx.x, blocks);
    return;
  }
  table.build<kTiles>(offsets, n_groups, n, (int)gw.k_split);
  const int tiles = (int)((gw.nq + 63) / 64 * gw.p_tiles);
  product<1, true, true>(gw, w, GroupedSums<64, kTiles, kShared>{{table, tiles, (int)gw.k_split}, gw}, lds, blockIdx.x - blocks,
                         gridDim.x - blocks);
  if (alone) clear_empty_groups(table, w.gw, gw.np * gw.nq, w.gb, (int)gw.nq, blockIdx.x - blocks, gridDim.x - blocks);
}

// Group blockIdx.y's units added in a fixed order; zeros where it has none. A quad of values to each of 256 / G neighbouring threads,
// its units dealt out over G groups of them. G = 16 where there are few values, else 1. Measured (us, weights' gradient, G = 1 / 16): float32 100,000 x 64 ->
// 64 in 4 groups 36.9 / 22.8, 22,266 x 64 -> 80 in 2 21.3 / 16.9, bfloat16 60,000 x 64 -> 64 in 3 16.9 / 13.6; 31,065 x 384 -> 48 in 8 15.4 / 16.5.
template <GroupUnits kUnits, bool kShared, int G>
__global__ __launch_bounds__(kThreads) void join_groups_kernel(int32_t n, int32_t n_groups, const int64_t* offsets, int32_t k_split,
                                                               const float* gw_parts, float* gw, int64_t size,
                                                               const float* gb_parts, float* gb, int32_t d_out) {
  GroupTable table;
  table.build<kUnits>(offsets, n_groups, n, k_split);
  const int group = blockIdx.y;
  int first = table.first_unit(group), last = table.first_unit(group + 1);
  if (last - first == 1) return;
  if (kShared && last > first) {
    const int place = first_place(group, table.first_row(group) - table.first_row(0), k_split);
    last += place - first, first = place;
  }
  constexpr int kQuads = kThreads / G;
  const int part = threadIdx.x / kQuads, own = threadIdx.x % kQuads;
  const int64_t quads = size / 4, all = quads + d_out / 4;
  __shared__ float4 s_sum[G][kQuads];
  for (int64_t from = (int64_t)blockIdx.x * kQuads; from < all; from += (int64_t)gridDim.x * kQuads) {
    const int64_t i = from + own;
    const bool w = i < quads;
    const float4* at = w ? reinterpret_cast<const float4*>(gw_parts) + i : reinterpret_cast<const float4*>(gb_parts) + (i - quads);
    const int64_t step = w ? quads : d_out / 4;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const int end = i < all ? last : first;
    int j = first + part;
    for (; j + 7 * G < end; j += 8 * G) {
      float4 a[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) a[u] = at[(j + u * G) * step];
#pragma unroll
      for (int u = 0; u < 8; ++u) s.x += a[u].x, s.y += a[u].y, s.z += a[u].z, s.w += a[u].w;
    }
    for (; j < end; j += G) {
      const float4 a = at[j * step];
      s.x += a.x, s.y += a.y, s.z += a.z, s.w += a.w;
    }
    if constexpr (G > 1) {
      __syncthreads();                                      // the last round's sums are read
      s_sum[part][own] = s;
      __syncthreads();
      if (part > 0) continue;
#pragma unroll
      for (int u = 1; u < G; ++u) {
        const float4 a = s_sum[u][own];
        s.x += a.x, s.y += a.y, s.z += a.z, s.w += a.w;
      }
    }
    if (i >= all) continue;
    float4* to = w ? reinterpret_cast<float4*>(gw) + group * quads + i : reinterpret_cast<float4*>(gb) + group * step + (i - quads);
    *to = s;
  }
}

template <int W, bool kPT, class Out>
void launch_rows(Product g, const Out& out, const int64_t* offsets, int32_t n_groups, int64_t n, hipStream_t stream) {
  g.p_tiles = cdiv(g.np, 64 * W);
  const int64_t most = (n / (64 * W) + n_groups) * g.p_tiles;
  rows_kernel<W, kPT><<<(unsigned)(most < 65536 ? most : 65536), kThreads, 0, stream>>>(g, out, offsets, n_groups, (int32_t)n);
}

template <int W>
void launch_sums(Product g, const GroupedWeightGrad& out, const int64_t* offsets, int32_t n_groups, int32_t n, bool by_group,
                 bool alone, hipStream_t stream) {
  g.p_tiles = cdiv(g.np, 64 * W);
  const int64_t pieces = by_group ? n / g.k_split + n_groups : cdiv(n, g.k_split);
  const int64_t most = pieces * g.p_tiles * cdiv(g.nq, 64 * W);
  const bool shared = shared_places(n, n_groups, g.k_split);
  auto kernel = by_group ? sums_kernel<W, kTiles, false> : shared ? sums_kernel<W, kShares, true> : sums_kernel<W, kShares, false>;
  if constexpr (W == 1)                                     // large tiles by group: units by the hundred, more than half the groups
    if (by_group && shared) kernel = sums_kernel<W, kTiles, true>;
  kernel<<<(unsigned)(most < 65536 ? most : 65536), kThreads, 0, stream>>>(g, out, offsets, n_groups, n, alone);
}

}  // namespace

maestro_status launch_layer_grouped_f32(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, const float* x,
                                        const float* weight, const float* bias, const int64_t* offsets, bool relu, float* y,
                                        hipStream_t stream) {
  const Product g{{weight, d_in}, {x, d_in}, d_out, n, d_in, d_in, 1, 0, 0};
  const Forward out{bias, y, relu};
  if (wide_forward(d_out, n, d_in)) launch_rows<2, false>(g, out, offsets, n_groups, n, stream);
  else launch_rows<1, false>(g, out, offsets, n_groups, n, stream);
  return launch_status();
}

size_t grouped_grad_f32_workspace_bytes(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out) {
  if (n == 0) return 0;
  const Cut c = cut_of(n, d_in, d_out);
  return n <= c.k_split ? 0 : sizeof(float) * (size_t)(places_of(n, n_groups, c.k_split) * ((int64_t)d_in + 1) * d_out);
}

maestro_status launch_grouped_grad_f32(int64_t n, int32_t n_groups, int32_t d_in, int32_t d_out, const float* x,
                                       const float* weight, const float* g_z, const int64_t* offsets, bool relu_input,
                                       float* g_x, float* g_weight, float* g_bias, void* workspace, hipStream_t stream) {
  const int64_t size = (int64_t)d_in * d_out;
  if (n == 0) return launch_join_groups(0, n_groups, offsets, 1, true, nullptr, g_weight, size, nullptr, g_bias, d_out, stream);
  const Cut c = cut_of(n, d_in, d_out);
  float *gw_parts = static_cast<float*>(workspace), *gb_parts = gw_parts + places_of(n, n_groups, c.k_split) * size;
  Product gx{{weight, d_in}, {g_z, d_out}, d_in, n, d_out, d_out, 1, 0, 0};
  const InputGrad x_out{x, g_x, relu_input};
  Product gw{{x, d_in}, {g_z, d_out}, d_in, d_out, n, c.k_split, 1, 0, 0};
  const GroupedWeightGrad out{g_weight, g_bias, gw_parts, gb_parts};
  const bool alone = n <= c.k_split;
  if (g_x && paired(c, n, d_in)) {
    gx.p_tiles = cdiv(d_in, 64);
    gw.p_tiles = cdiv(d_in, 64);
    const int64_t rows = (n / 64 + n_groups) * gx.p_tiles, sums = (n / c.k_split + n_groups) * gw.p_tiles * cdiv(d_out, 64);
    const uint32_t blocks = (uint32_t)(rows < 65536 ? rows : 65536), more = (uint32_t)(sums < 65536 ? sums : 65536);
    auto kernel = shared_places(n, n_groups, c.k_split) ? pair_kernel<true> : pair_kernel<false>;
    kernel<<<blocks + more, kThreads, 0, stream>>>(gx, x_out, blocks, gw, out, offsets, n_groups, (int32_t)n, alone);
  } else {
    if (g_x && wide(d_in, n)) launch_rows<2, true>(gx, x_out, offsets, n_groups, n, stream);
    else if (g_x) launch_rows<1, true>(gx, x_out, offsets, n_groups, n, stream);
    (c.wide ? launch_sums<2> : launch_sums<1>)(gw, out, offsets, n_groups, (int32_t)n, c.by_group, alone, stream);
  }
  const maestro_status st = launch_status();
  if (st != MAESTRO_OK || alone) return st;
  return launch_join_groups(n, n_groups, offsets, c.k_split, c.by_group, gw_parts, g_weight, size, gb_parts, g_bias, d_out, stream);
}

maestro_status launch_join_groups(int64_t n, int32_t n_groups, const int64_t* offsets, int64_t k_split, bool by_group,
                                  const float* gw_parts, float* gw, int64_t size, const float* gb_parts, float* gb, int32_t d_out,
                                  hipStream_t stream) {
  const int64_t quads = size / 4 + d_out / 4;
  const bool dealt = join_dealt(n, n_groups, k_split, size, d_out);
  const int64_t blocks = cdiv(quads, dealt ? kThreads / 16 : kThreads);
  auto of = [&](auto shared) {
    constexpr bool kShared = decltype(shared)::value;
    // few values by shares: units by the hundred, more than half the groups
    return dealt ? by_group ? join_groups_kernel<kTiles, kShared, 16> : join_groups_kernel<kShares, false, 16>
                 : by_group ? join_groups_kernel<kTiles, kShared, 1> : join_groups_kernel<kShares, kShared, 1>;
  };
  auto kernel = shared_places(n, n_groups, k_split) ? of(std::true_type{}) : of(std::false_type{});
  kernel<<<dim3((unsigned)(blocks < 4096 ? blocks : 4096), (unsigned)n_groups), kThreads, 0, stream>>>(
      (int32_t)n, n_groups, offsets, (int32_t)k_split, gw_parts, gw, size, gb_parts, gb, d_out);
  return launch_status();
}

}  // namespace maestro
