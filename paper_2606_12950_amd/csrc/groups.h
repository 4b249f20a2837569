// The rows of a grouped layer's groups and the units of work they make, on the device: offsets are known there only.
//
// Rows, units and tiles are counted in 32 bits (kMaxGroupedRows), which the scalar unit compares by itself. The 64-bit
// comparison of uniform numbers it has not: one that both chooses a value and branches came out of the compiler (22.0, gfx950)
// with the choice made by an older condition (the branch came from a vector comparison, the choice from what a shift had left), and a
// workgroup's way through its groups did not end. Where counts pass 32 bits (rows of one product), 64-bit ones stay; a test of every build
// looks for that form in all of the library's kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "maestro_layers.h"
#include "rules.h"

namespace maestro {

constexpr int64_t kMaxGroupedRows = ((int64_t)1 << 31) - ((int64_t)1 << 16);

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// a / b, neither negative
__device__ __forceinline__ int quotient(int a, int b) { return (int)((uint32_t)a / (uint32_t)b); }

// Group g's rows are row[g] .. row[g + 1], its units unit[g] .. unit[g + 1]: of up to `per` rows each, counted from the group's
// first row (kTiles) or, of all groups together, from row[0] on (kShares: a group's rows are cut where the count of all is a
// multiple of `per`, so that the units of one cut are `per` rows together, whatever the groups' sizes).
enum GroupUnits { kTiles, kShares };

// Every wavefront holds a table of its own, a group a lane in kSets sets of registers: in LDS it would cost the 256 x 64 tiles the
// second workgroup of a CU, and a look-up is a ballot or a lane's read. All of a wavefront's lanes take part in every call.
struct GroupTable {
  static constexpr int kSets = MAESTRO_MAX_LAYER_GROUPS / 64;
  int row_end[kSets], unit_end[kSets];                      // of group 64 s + lane
  int base, n_groups;

  // Whatever the offsets hold, rows are 0 <= first_row(0) <= first_row(1) <= ... <= n.
  template <GroupUnits kUnits>
  __device__ __forceinline__ void build(const int64_t* __restrict__ offsets, int groups, int n, int per) {
    const int lane = threadIdx.x & 63;
    auto clamp = [&](int64_t v) { return v < 0 ? 0 : v > n ? n : (int)v; };
    n_groups = groups;
    base = uniform(clamp(offsets[0]));
    int before = base, units = 0;                           // the last row and unit so far
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
      row_end[s] = unit_end[s] = 0;
      if (64 * s >= n_groups) continue;
      const int g = 64 * s + lane;
      int end = g < n_groups ? clamp(offsets[g + 1]) : 0;
      if (end < before) end = before;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int other = __shfl_up(end, d);
        if (lane >= d && other > end) end = other;
      }
      int start = __shfl_up(end, 1);
      if (lane == 0) start = before;
      int sum = end == start ? 0 : kUnits == kTiles ? quotient(end - start - 1, per) + 1
                                                    : quotient(end - 1 - base, per) - quotient(start - base, per) + 1;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int other = __shfl_up(sum, d);
        if (lane >= d) sum += other;
      }
      row_end[s] = end;
      unit_end[s] = units + sum;
      before = __builtin_amdgcn_readlane(end, 63);
      units = __builtin_amdgcn_readlane(unit_end[s], 63);
    }
  }

  // The group of a unit below first_unit(n_groups), or of a row from first_row(0) on below first_row(n_groups).
  __device__ __forceinline__ int group_of_unit(int u) const { return passed(unit_end, u); }
  __device__ __forceinline__ int group_of_row(int r) const { return passed(row_end, r); }
  __device__ __forceinline__ int passed(const int (&ends)[kSets], int v) const {
    const int lane = threadIdx.x & 63;
    int g = 0;
#pragma unroll
    for (int s = 0; s < kSets; ++s)
      if (64 * s < n_groups) g += __popcll(__ballot(64 * s + lane < n_groups && ends[s] <= v));
    return g;
  }
  // of groups 0 .. n_groups: the last one's is where all end
  __device__ __forceinline__ int first_row(int g) const { return g == 0 ? base : of_group(row_end, g - 1); }
  __device__ __forceinline__ int first_unit(int g) const { return g == 0 ? 0 : of_group(unit_end, g - 1); }
  static __device__ __forceinline__ int of_group(const int (&ends)[kSets], int g) {
    int v = __builtin_amdgcn_readlane(ends[0], g & 63);
#pragma unroll
    for (int s = 1; s < kSets; ++s)
      if (g >= 64 * s) v = __builtin_amdgcn_readlane(ends[s], g & 63);
    return v;
  }
};

// A workgroup's way through `items` units of work, workgroup `block` of `blocks`. kXcds = 8 (blocks a multiple of it): XCD x
// (workgroups go round them) takes a contiguous share; 1: none has one of its own.
template <int kXcds>
struct GroupedCursor {
  int i, last, step;
  __device__ __forceinline__ GroupedCursor(int items, uint32_t block, uint32_t blocks) {
    const int share = (items + kXcds - 1) / kXcds, end = (int)(block % kXcds + 1) * share;
    step = (int)(blocks / kXcds);
    last = end < items ? end : items;
    i = end - share + (int)(block / kXcds);
  }
  __device__ __forceinline__ bool done() const { return i >= last; }
};

// Tiles of TQ rows of a group, all p tiles of one after the other.
template <int kXcds>
struct GroupedRowsWay {
  using Way = GroupedCursor<kXcds>;
  const GroupTable& table;
  int p_tiles;
  struct Place {
    int group, q0, q_end, p_tile;
  };
  __device__ __forceinline__ Way begin(uint32_t block, uint32_t blocks) const {
    return Way(table.first_unit(table.n_groups) * p_tiles, block, blocks);
  }
  __device__ __forceinline__ void next(Way& c) const { c.i += c.step; }
  __device__ __forceinline__ Place place(const Way& c, int tile_rows) const {
    const int unit = quotient(c.i, p_tiles), g = table.group_of_unit(unit);
    return Place{g, table.first_row(g) + (unit - table.first_unit(g)) * tile_rows, table.first_row(g + 1), c.i - unit * p_tiles};
  }
};

// Tiles of a group's weights' gradient over its units of rows. kShares: `per` rows of all groups together are one piece of work
// for every tile, which a workgroup takes group after group. kTiles: a group's unit is one, so that small groups run side by side.
// kShared: only units of groups of two or more have places in the workspace (shared_places).
template <int kXcds, GroupUnits kUnits, bool kShared>
struct GroupedSumsWay {
  struct Way : GroupedCursor<kXcds> {
    int row, end;                    // kShares: the first row of the group's part, and the piece's last
    __device__ __forceinline__ explicit Way(const GroupedCursor<kXcds>& c) : GroupedCursor<kXcds>(c), row(0), end(0) {}
  };
  const GroupTable& table;
  int tiles, per;
  struct Place {
    int group, tile, slot, k0, k_end;
    bool direct;                     // all of the group's rows
  };
  __device__ __forceinline__ void open(Way& c) const {
    if (kUnits == kTiles || c.done()) return;
    const int last = table.first_row(table.n_groups);
    c.row = table.first_row(0) + quotient(c.i, tiles) * per;
    c.end = last - c.row < per ? last : c.row + per;
  }
  __device__ __forceinline__ Way begin(uint32_t block, uint32_t blocks) const {
    const int rows = table.first_row(table.n_groups) - table.first_row(0);
    const int pieces = kUnits == kTiles ? table.first_unit(table.n_groups) : rows > 0 ? quotient(rows - 1, per) + 1 : 0;
    Way c(GroupedCursor<kXcds>(pieces * tiles, block, blocks));
    open(c);
    return c;
  }
  __device__ __forceinline__ void next(Way& c) const {
    if constexpr (kUnits == kShares) {
      const int group_end = table.first_row(table.group_of_row(c.row) + 1);
      c.row = group_end < c.end ? group_end : c.end;
      if (c.row < c.end) return;
    }
    c.i += c.step;
    open(c);
  }
  __device__ __forceinline__ Place place(const Way& c) const {
    const int piece = quotient(c.i, tiles), tile = c.i - piece * tiles;
    const int g = kUnits == kTiles ? table.group_of_unit(piece) : table.group_of_row(c.row);
    const int first = table.first_unit(g), row = table.first_row(g), group_end = table.first_row(g + 1);
    const bool direct = table.first_unit(g + 1) - first == 1;
    if constexpr (kUnits == kTiles) {
      const int k0 = row + (piece - first) * per;
      const int slot = !kShared ? piece : direct ? 0 : first_place(g, row - table.first_row(0), per) + piece - first;
      return Place{g, tile, slot, k0, group_end - k0 < per ? group_end : k0 + per, direct};
    }
    const int from = !kShared ? first : direct ? 0 : first_place(g, row - table.first_row(0), per);
    return Place{g, tile, from + piece - quotient(row - table.first_row(0), per), c.row, group_end < c.end ? group_end : c.end, direct};
  }
};

// Zeros for the groups without rows, by `blocks` workgroups.
__device__ __forceinline__ void clear_empty_groups(const GroupTable& table, float* gw, int64_t size, float* gb, int d_out,
                                                   uint32_t block, uint32_t blocks) {
  const int64_t quads = size / 4, all = quads + d_out / 4;
  for (int g = 0; g < table.n_groups; ++g) {
    if (table.first_unit(g + 1) != table.first_unit(g)) continue;
    for (int64_t i = (int64_t)block * blockDim.x + threadIdx.x; i < all; i += (int64_t)blocks * blockDim.x)
      (i < quads ? reinterpret_cast<float4*>(gw) + g * quads + i : reinterpret_cast<float4*>(gb) + g * (all - quads) + (i - quads))[0] =
          make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  }
}

}  // namespace maestro
