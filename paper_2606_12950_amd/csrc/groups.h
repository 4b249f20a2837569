// The rows of a grouped layer's groups and the units of work they make, on the device: offsets are known there only.
//
// Rows, units and tiles are counted in 32 bits (kMaxGroupedRows), which the scalar unit compares by itself. The 64-bit
// comparison of uniform numbers it has not: one that both chooses a value and branches came out of the compiler (22.0, gfx950)
// with the choice made by an older condition, and a workgroup's way through its groups did not end.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "maestro_layers.h"

namespace maestro {

constexpr int64_t kMaxGroupedRows = ((int64_t)1 << 31) - ((int64_t)1 << 16);

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// a / b, neither negative
__device__ __forceinline__ int quotient(int a, int b) { return (int)((uint32_t)a / (uint32_t)b); }

// Group g's rows are row[g] .. row[g + 1], its units unit[g] .. unit[g + 1]: of up to `per` rows each, counted from the group's
// first row (kTiles) or, of all groups together, from row[0] on (kShares: a group's rows are cut where the count of all is a
// multiple of `per`, so that the units of one cut are `per` rows together, whatever the groups' sizes).
enum GroupUnits { kTiles, kShares };
struct GroupTable {
  int row[MAESTRO_MAX_LAYER_GROUPS + 1], unit[MAESTRO_MAX_LAYER_GROUPS + 1];

  // By every thread of a workgroup; the first wavefront works. Whatever the offsets hold, rows are 0 <= row[0] <= row[1] <= ... <= n.
  template <GroupUnits kUnits>
  __device__ __forceinline__ void build(const int64_t* __restrict__ offsets, int n_groups, int n, int per) {
    if (threadIdx.x < 64) {
      const int lane = threadIdx.x;
      auto clamp = [&](int64_t v) { return v < 0 ? 0 : v > n ? n : (int)v; };
      const int base = clamp(offsets[0]);
      int before = base, units = 0;                         // the last row and unit so far
      if (lane == 0) row[0] = before, unit[0] = 0;
      for (int g0 = 0; g0 < n_groups; g0 += 64) {
        const int g = g0 + lane;
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
        if (g < n_groups) row[g + 1] = end, unit[g + 1] = units + sum;
        before = __shfl(end, 63);
        units += __shfl(sum, 63);
      }
    }
    __syncthreads();
  }

  // The group of a unit below unit[n_groups], or of a row from row[0] on below row[n_groups]; the same for a wavefront's
  // lanes (all of them there).
  __device__ __forceinline__ int group_of_unit(int u, int n_groups) const { return passed(unit, u, n_groups); }
  __device__ __forceinline__ int group_of_row(int r, int n_groups) const { return passed(row, r, n_groups); }
  static __device__ __forceinline__ int passed(const int* first, int v, int n_groups) {
    const int lane = threadIdx.x & 63;
    int g = 0;
    for (int g0 = 0; g0 < n_groups; g0 += 64)
      g += __popcll(__ballot(g0 + lane < n_groups && first[g0 + lane + 1] <= v));
    return g;
  }
  __device__ __forceinline__ int first_row(int g) const { return uniform(row[g]); }
  __device__ __forceinline__ int first_unit(int g) const { return uniform(unit[g]); }
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
  int n_groups, p_tiles;
  struct Place {
    int group, q0, q_end, p_tile;
  };
  __device__ __forceinline__ Way begin(uint32_t block, uint32_t blocks) const {
    return Way(table.first_unit(n_groups) * p_tiles, block, blocks);
  }
  __device__ __forceinline__ void next(Way& c) const { c.i += c.step; }
  __device__ __forceinline__ Place place(const Way& c, int tile_rows) const {
    const int unit = quotient(c.i, p_tiles), g = table.group_of_unit(unit, n_groups);
    return Place{g, table.first_row(g) + (unit - table.first_unit(g)) * tile_rows, table.first_row(g + 1), c.i - unit * p_tiles};
  }
};

// Tiles of a group's weights' gradient over its shares of rows: `share` rows of all groups together are one unit of work for
// every tile, which a workgroup takes group after group.
template <int kXcds>
struct GroupedSumsWay {
  struct Way : GroupedCursor<kXcds> {
    int row, end;                    // the first row of the group's part, and the unit's last
    __device__ __forceinline__ explicit Way(const GroupedCursor<kXcds>& c) : GroupedCursor<kXcds>(c), row(0), end(0) {}
  };
  const GroupTable& table;
  int n_groups, tiles, share;
  struct Place {
    int group, tile, slot, k0, k_end;
    bool direct;                     // all of the group's rows
  };
  __device__ __forceinline__ void open(Way& c) const {
    if (c.done()) return;
    const int last = table.first_row(n_groups);
    c.row = table.first_row(0) + quotient(c.i, tiles) * share;
    c.end = last - c.row < share ? last : c.row + share;
  }
  __device__ __forceinline__ Way begin(uint32_t block, uint32_t blocks) const {
    const int rows = table.first_row(n_groups) - table.first_row(0);
    Way c(GroupedCursor<kXcds>(rows > 0 ? (quotient(rows - 1, share) + 1) * tiles : 0, block, blocks));
    open(c);
    return c;
  }
  __device__ __forceinline__ void next(Way& c) const {
    const int group_end = table.first_row(table.group_of_row(c.row, n_groups) + 1);
    c.row = group_end < c.end ? group_end : c.end;
    if (c.row < c.end) return;
    c.i += c.step;
    open(c);
  }
  __device__ __forceinline__ Place place(const Way& c) const {
    const int unit = quotient(c.i, tiles), g = table.group_of_row(c.row, n_groups), first = table.first_unit(g);
    const int group_end = table.first_row(g + 1);
    return Place{g, c.i - unit * tiles, first + unit - quotient(table.first_row(g) - table.first_row(0), share), c.row,
                 group_end < c.end ? group_end : c.end, table.first_unit(g + 1) - first == 1};
  }
};

}  // namespace maestro
