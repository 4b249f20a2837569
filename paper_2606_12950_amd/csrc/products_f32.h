// Float32 products of a predictor's layer and its gradients on the matrix cores.
//
// As in the bfloat16 kernel all three products are C[q][p] = sum_k P(p, k) Q(q, k) with C's rows contiguous in p;
// here in 32x32x2 float32 MFMAs, four wavefronts of 32 W x 32 W each. Stages of 16 k come through
// registers into two LDS buffers laid out [k][p], so every operand is turned (or not) as it is written, and a product
// reads one word a lane.
#pragma once

#include <type_traits>

#include "mlp.h"
#include "rules.h"
#include "train.h"

namespace maestro {
namespace {

constexpr int kThreads = 256, kDepth = kDepthF32;

// An operand in memory, rows of ld values: four neighbouring ones of a row.
struct Floats {
  const float* m;
  int64_t ld;
  __device__ __forceinline__ float4 at(int64_t row, int64_t col) const {
    return *reinterpret_cast<const float4*>(m + row * ld + col);
  }
  __device__ __forceinline__ Floats from(int64_t values) const { return Floats{m + values, ld}; }
};
// kept activations: a value is its code times 2^(exponent - 127), one exponent to 32 values of a row
template <class Code>
struct Codes {
  const Code* m;
  const unsigned char* exponents;
  int64_t ld, ld_exponents;
  __device__ __forceinline__ float4 at(int64_t row, int64_t col) const {
    const float s = __uint_as_float((uint32_t)exponents[row * ld_exponents + col / 32] << 23);
    Code c[4];
    __builtin_memcpy(c, __builtin_assume_aligned(m + row * ld + col, 4), 4);
    return make_float4((float)c[0] * s, (float)c[1] * s, (float)c[2] * s, (float)c[3] * s);
  }
  __device__ __forceinline__ Codes from(int64_t) const { return *this; }
};

template <class P>
struct ProductOf {
  P p;
  Floats q;
  int64_t np, nq, nk, k_split, splits;
  int64_t p_tiles, items;
};
typedef ProductOf<Floats> Product;

// One tile: its place in C (rows of q from q_end on are not the tile's) and its k.
struct Item {
  int64_t q0, q_end, p0, k0, k_end;
  int64_t slot;                      // which share of C, where k is split
  int64_t p_shift;                   // values from P's first to those of the tile's group
  int32_t group;
  bool direct;                       // the whole of a group's C
};

// A workgroup's way through `items` units of work, workgroup `block` of `blocks`.
// Counts of 64 bits, as in the bfloat16 kernel.
struct Cursor {
  int64_t i, last, step;
  __device__ __forceinline__ Cursor(int64_t items, uint32_t block, uint32_t blocks) : i(block), last(items), step(blocks) {}
  __device__ __forceinline__ bool done() const { return i >= last; }
};

// The tiles of one product, all splits' one after the other.
template <int T, class P>
struct Dense {
  using Way = Cursor;
  const ProductOf<P>& g;
  int64_t per_split;
  __device__ __forceinline__ explicit Dense(const ProductOf<P>& product) : g(product), per_split(product.items / product.splits) {}
  __device__ __forceinline__ Way begin(uint32_t block, uint32_t blocks) const { return Way(g.items, block, blocks); }
  __device__ __forceinline__ void next(Way& c) const { c.i += c.step; }
  __device__ __forceinline__ Item item(const Way& c) const {
    Item t;
    t.slot = c.i / per_split;
    const int64_t tile = c.i % per_split;
    t.q0 = tile / g.p_tiles * T;
    t.q_end = g.nq;
    t.p0 = tile % g.p_tiles * T;
    t.k0 = t.slot * g.k_split;
    t.k_end = t.k0 + g.k_split < g.nk ? t.k0 + g.k_split : g.nk;
    t.p_shift = 0;
    t.group = 0;
    t.direct = false;
    return t;
  }
};

struct Forward {
  const float* bias;                 // [p], of the tile's group
  float* y;
  bool relu;
  // four consecutive p of one q
  __device__ __forceinline__ void finish(const Item& t, int64_t np, int64_t, int64_t q, int64_t p, float4 c) const {
    const float4 b = *reinterpret_cast<const float4*>(bias + t.group * np + p);
    c.x += b.x, c.y += b.y, c.z += b.z, c.w += b.w;
    if (relu) {                                             // a NaN stays one
      c.x = c.x < 0.0f ? 0.0f : c.x, c.y = c.y < 0.0f ? 0.0f : c.y;
      c.z = c.z < 0.0f ? 0.0f : c.z, c.w = c.w < 0.0f ? 0.0f : c.w;
    }
    *reinterpret_cast<float4*>(y + q * np + p) = c;
  }
};
struct InputGrad {
  const float* x;
  float* gx;
  bool relu;
  __device__ __forceinline__ void finish(const Item&, int64_t np, int64_t, int64_t q, int64_t p, float4 c) const {
    if (relu) {
      const float4 m = *reinterpret_cast<const float4*>(x + q * np + p);
      c.x = m.x > 0.0f ? c.x : 0.0f, c.y = m.y > 0.0f ? c.y : 0.0f;
      c.z = m.z > 0.0f ? c.z : 0.0f, c.w = m.w > 0.0f ? c.w : 0.0f;
    }
    *reinterpret_cast<float4*>(gx + q * np + p) = c;
  }
};
// of rectified values kept as codes: 0 where the code is
struct CodesInputGrad {
  const unsigned char* x;
  float* gx;
  bool relu;
  __device__ __forceinline__ void finish(const Item&, int64_t np, int64_t, int64_t q, int64_t p, float4 c) const {
    if (relu) {
      const uint32_t m = *reinterpret_cast<const uint32_t*>(x + q * np + p);
      c.x = m & 0xFFu ? c.x : 0.0f, c.y = m & 0xFF00u ? c.y : 0.0f;
      c.z = m & 0xFF0000u ? c.z : 0.0f, c.w = m & 0xFF000000u ? c.w : 0.0f;
    }
    *reinterpret_cast<float4*>(gx + q * np + p) = c;
  }
};
struct WeightGrad {
  float* gw;                         // [slots][nq][np]
  float* gb;                         // [slots][nq]
  __device__ __forceinline__ void finish(const Item& t, int64_t np, int64_t nq, int64_t q, int64_t p, float4 c) const {
    *reinterpret_cast<float4*>(gw + (t.slot * nq + q) * np + p) = c;
  }
  __device__ __forceinline__ float* bias(const Item& t, int64_t nq, int64_t q) const { return gb + t.slot * nq + q; }
};

// T rows of an operand, kDepth k at a time; kTurned: rows contiguous in memory instead of k. Thread t loads vectors
// t, t + 256, ... of the stage.
template <int T, bool kTurned>
struct Operand {
  static constexpr int kLoads = T * kDepth / 4 / kThreads;
  static constexpr int kRow = T + 4;                        // words of an LDS row: neighbouring k in other banks
  float4 v[kLoads];
  template <class M>
  __device__ __forceinline__ void load(const M& m, int64_t row0, int64_t rows, int64_t k0, int64_t k_end) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i = threadIdx.x + kThreads * j;
      const int64_t k = k0 + (kTurned ? i / (T / 4) : i % (kDepth / 4) * 4);
      const int64_t r = row0 + (kTurned ? i % (T / 4) * 4 : i / (kDepth / 4));
      v[j] = k < k_end && r < rows ? m.at(kTurned ? k : r, kTurned ? r : k) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
  }
  __device__ __forceinline__ void store(float* lds) const {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i = threadIdx.x + kThreads * j;
      if constexpr (kTurned) {
        *reinterpret_cast<float4*>(lds + i / (T / 4) * kRow + i % (T / 4) * 4) = v[j];
      } else {
        float* at = lds + i % (kDepth / 4) * 4 * kRow + i / (kDepth / 4);
        at[0] = v[j].x, at[kRow] = v[j].y, at[2 * kRow] = v[j].z, at[3 * kRow] = v[j].w;
      }
    }
  }
};

template <int W>
struct Lds {
  float at[2][2][kDepth * (64 * W + 4)];
};

// The share of workgroup `block` of `blocks` in the tiles of `work`, products of the sizes of `g`.
template <int W, bool kPT, bool kQT, class P, class Out, class Work>
__device__ __forceinline__ void product(const ProductOf<P>& g, const Out& out, const Work& work, Lds<W>& shared, uint32_t block,
                                        uint32_t blocks) {
  constexpr int T = 64 * W, kRow = T + 4;
  constexpr bool kSums = kQT;                               // the weights' gradient sums Q too (the biases')
  auto& lds = shared.at;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, h = lane >> 5;
  const int wp = wave & 1, wq = wave >> 1;
  for (auto at = work.begin(block, blocks); !at.done(); work.next(at)) {
    const Item t = work.item(at);
    const int64_t q0 = t.q0, p0 = t.p0, k0 = t.k0, k_end = t.k_end;
    const P p_rows = g.p.from(t.p_shift);
    Operand<T, kPT> op;
    Operand<T, kQT> oq;
    f32x16 acc[W][W] = {};
    float sums[W] = {};
    op.load(p_rows, p0, g.np, k0, k_end);
    oq.load(g.q, q0, t.q_end, k0, k_end);
    int buf = 0;
    for (int64_t k = k0; k < k_end; k += kDepth, buf ^= 1) {
      op.store(lds[buf][0]);
      oq.store(lds[buf][1]);
      __syncthreads();
      op.load(p_rows, p0, g.np, k + kDepth, k_end);
      oq.load(g.q, q0, t.q_end, k + kDepth, k_end);
      const float *ps = lds[buf][0] + h * kRow + 32 * W * wp + r, *qs = lds[buf][1] + h * kRow + 32 * W * wq + r;
#pragma unroll
      for (int kk = 0; kk < kDepth; kk += 2) {
        float pf[W], qf[W];
#pragma unroll
        for (int a = 0; a < W; ++a) pf[a] = ps[kk * kRow + 32 * a], qf[a] = qs[kk * kRow + 32 * a];
#pragma unroll
        for (int a = 0; a < W; ++a)
#pragma unroll
          for (int b = 0; b < W; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x2f32(pf[a], qf[b], acc[a][b], 0, 0, 0);
        if constexpr (kSums)
#pragma unroll
          for (int b = 0; b < W; ++b) sums[b] += qf[b];
      }
    }
    __syncthreads();                                        // the buffers are free for the next item
#pragma unroll
    for (int b = 0; b < W; ++b) {
      const int64_t q = q0 + 32 * (W * wq + b) + r;
#pragma unroll
      for (int a = 0; a < W; ++a)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int64_t p = p0 + 32 * (W * wp + a) + acc_row(4 * i, h);
          if (q < t.q_end && p < g.np)
            out.finish(t, g.np, g.nq, q, p,
                   make_float4(acc[a][b][4 * i], acc[a][b][4 * i + 1], acc[a][b][4 * i + 2], acc[a][b][4 * i + 3]));
        }
      if constexpr (kSums) {
        const float s = sums[b] + __shfl_xor(sums[b], 32);
        if (h == 0 && wp == 0 && p0 == 0 && q < t.q_end) *out.bias(t, g.nq, q) = s;
      }
    }
  }
}

}  // namespace
}  // namespace maestro
