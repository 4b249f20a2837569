// The rows of a grouped layer's groups and the units of work they make, on the device: offsets are known there only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "maestro_layers.h"

namespace maestro {

__device__ __forceinline__ int64_t uniform64(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// Group g's rows are row[g] .. row[g + 1], its units (of up to `per` rows) unit[g] .. unit[g + 1].
struct GroupTable {
  int64_t row[MAESTRO_MAX_LAYER_GROUPS + 1], unit[MAESTRO_MAX_LAYER_GROUPS + 1];

  // By every thread of a workgroup; the first wavefront works. Whatever the offsets hold, rows are 0 <= row[0] <= row[1] <= ... <= n.
  __device__ __forceinline__ void build(const int64_t* __restrict__ offsets, int n_groups, int64_t n, int64_t per) {
    if (threadIdx.x < 64) {
      const int lane = threadIdx.x;
      auto clamp = [&](int64_t v) { return v < 0 ? 0 : v > n ? n : v; };
      int64_t before = clamp(offsets[0]), units = 0;        // the last row and unit so far
      if (lane == 0) row[0] = before, unit[0] = 0;
      for (int g0 = 0; g0 < n_groups; g0 += 64) {
        const int g = g0 + lane;
        int64_t end = g < n_groups ? clamp(offsets[g + 1]) : 0;
        if (end < before) end = before;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int64_t other = __shfl_up(end, d);
          if (lane >= d && other > end) end = other;
        }
        int64_t start = __shfl_up(end, 1);
        if (lane == 0) start = before;
        int64_t sum = (end - start + per - 1) / per;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int64_t other = __shfl_up(sum, d);
          if (lane >= d) sum += other;
        }
        if (g < n_groups) row[g + 1] = end, unit[g + 1] = units + sum;
        before = __shfl(end, 63);
        units += __shfl(sum, 63);
      }
    }
    __syncthreads();
  }

  // The group of a unit below unit[n_groups], the same for a wavefront's lanes (all of them there).
  __device__ __forceinline__ int group_of(int64_t u, int n_groups) const {
    const int lane = threadIdx.x & 63;
    int g = 0;
    for (int g0 = 0; g0 < n_groups; g0 += 64)
      g += __popcll(__ballot(g0 + lane < n_groups && unit[g0 + lane + 1] <= u));
    return g;
  }
  __device__ __forceinline__ int64_t first_row(int g) const { return uniform64(row[g]); }
  __device__ __forceinline__ int64_t first_unit(int g) const { return uniform64(unit[g]); }
};

}  // namespace maestro
