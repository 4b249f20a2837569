// A predictor's Linear layer with its activations kept, and the layer's gradients: the float32 products, and the
// choice between them and the bfloat16 ones.
//
// As in the bfloat16 kernel all three products are C[q][p] = sum_k P(p, k) Q(q, k) with C's rows contiguous in p;
// here in 32x32x2 float32 MFMAs, four wavefronts of 32 W x 32 W each. Stages of 16 k come through
// registers into two LDS buffers laid out [k][p], so every operand is turned (or not) as it is written, and a product
// reads one word a lane. Bound by the float32 matrix cores (64 operations a cycle and SIMD, 1/16 of bfloat16) on wide
// layers, by launches on the small ones it is for. Measured: 4,096 x 64 -> 128 5.5 us, 60,000 x 1024 -> 1024
// 1,061 (floor 833), 150,000 x 256 -> 256 195 (130): one 16-k stage ahead does not cover a load; see wide and cut_of for the rest.
#include "mlp.h"
#include "train.h"

namespace maestro {
namespace {

constexpr int kThreads = 256, kDepth = 16;

struct Product {
  const float* p;
  const float* q;
  int64_t ldp, ldq, np, nq, nk, k_split, splits;
  int64_t p_tiles, items;
};

struct Forward {
  const float* bias;
  float* y;
  bool relu;
};
struct InputGrad {
  const float* x;
  float* gx;
  bool relu;
};
struct WeightGrad {
  float* gw;                         // [splits][nq][np]
  float* gb;                         // [splits][nq]
};

// four consecutive p of one q
__device__ __forceinline__ void finish(const Forward& e, const Product& g, int64_t q, int64_t p, int64_t, float4 c) {
  const float4 b = *reinterpret_cast<const float4*>(e.bias + p);
  c.x += b.x, c.y += b.y, c.z += b.z, c.w += b.w;
  if (e.relu) {                                             // a NaN stays one
    c.x = c.x < 0.0f ? 0.0f : c.x, c.y = c.y < 0.0f ? 0.0f : c.y;
    c.z = c.z < 0.0f ? 0.0f : c.z, c.w = c.w < 0.0f ? 0.0f : c.w;
  }
  *reinterpret_cast<float4*>(e.y + q * g.np + p) = c;
}
__device__ __forceinline__ void finish(const InputGrad& e, const Product& g, int64_t q, int64_t p, int64_t, float4 c) {
  if (e.relu) {
    const float4 x = *reinterpret_cast<const float4*>(e.x + q * g.np + p);
    c.x = x.x > 0.0f ? c.x : 0.0f, c.y = x.y > 0.0f ? c.y : 0.0f;
    c.z = x.z > 0.0f ? c.z : 0.0f, c.w = x.w > 0.0f ? c.w : 0.0f;
  }
  *reinterpret_cast<float4*>(e.gx + q * g.np + p) = c;
}
__device__ __forceinline__ void finish(const WeightGrad& e, const Product& g, int64_t q, int64_t p, int64_t split, float4 c) {
  *reinterpret_cast<float4*>(e.gw + (split * g.nq + q) * g.np + p) = c;
}

// T rows of an operand, kDepth k at a time; kTurned: rows contiguous in memory instead of k. Thread t loads vectors
// t, t + 256, ... of the stage.
template <int T, bool kTurned>
struct Operand {
  static constexpr int kLoads = T * kDepth / 4 / kThreads;
  static constexpr int kRow = T + 4;                        // words of an LDS row: neighbouring k in other banks
  float4 v[kLoads];
  __device__ __forceinline__ void load(const float* m, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int64_t k_end) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i = threadIdx.x + kThreads * j;
      const int64_t k = k0 + (kTurned ? i / (T / 4) : i % (kDepth / 4) * 4);
      const int64_t r = row0 + (kTurned ? i % (T / 4) * 4 : i / (kDepth / 4));
      v[j] = k < k_end && r < rows ? *reinterpret_cast<const float4*>(m + (kTurned ? k * ld + r : r * ld + k))
                                   : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
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

// The share of workgroup `block` of `blocks` in a product.
template <int W, bool kPT, bool kQT, class Out>
__device__ __forceinline__ void product(const Product& g, const Out& out, Lds<W>& shared, uint32_t block, uint32_t blocks) {
  constexpr int T = 64 * W, kRow = T + 4;
  constexpr bool kSums = kQT;                               // the weights' gradient sums Q too (the biases')
  auto& lds = shared.at;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, h = lane >> 5;
  const int wp = wave & 1, wq = wave >> 1;
  const int64_t per_split = g.items / g.splits;
  for (int64_t item = block; item < g.items; item += blocks) {
    const int64_t split = item / per_split, tile = item % per_split;
    const int64_t q0 = tile / g.p_tiles * T, p0 = tile % g.p_tiles * T;
    const int64_t k0 = split * g.k_split, k_end = k0 + g.k_split < g.nk ? k0 + g.k_split : g.nk;
    Operand<T, kPT> op;
    Operand<T, kQT> oq;
    f32x16 acc[W][W] = {};
    float sums[W] = {};
    op.load(g.p, g.ldp, p0, g.np, k0, k_end);
    oq.load(g.q, g.ldq, q0, g.nq, k0, k_end);
    int buf = 0;
    for (int64_t k = k0; k < k_end; k += kDepth, buf ^= 1) {
      op.store(lds[buf][0]);
      oq.store(lds[buf][1]);
      __syncthreads();
      op.load(g.p, g.ldp, p0, g.np, k + kDepth, k_end);
      oq.load(g.q, g.ldq, q0, g.nq, k + kDepth, k_end);
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
          if (q < g.nq && p < g.np)
            finish(out, g, q, p, split,
                   make_float4(acc[a][b][4 * i], acc[a][b][4 * i + 1], acc[a][b][4 * i + 2], acc[a][b][4 * i + 3]));
        }
      if constexpr (kSums) {
        const float s = sums[b] + __shfl_xor(sums[b], 32);
        if (h == 0 && wp == 0 && p0 == 0 && q < g.nq) out.gb[split * g.nq + q] = s;
      }
    }
  }
}

template <int W, bool kPT, bool kQT, class Out>
__global__ __launch_bounds__(kThreads, 2) void product_kernel(Product g, Out out) {
  __shared__ __attribute__((aligned(16))) Lds<W> lds;
  product<W, kPT, kQT>(g, out, lds, blockIdx.x, gridDim.x);
}

// Both gradients in one launch, in 64 x 64 tiles: the first `blocks` workgroups make the input's, the others the weights'.
__global__ __launch_bounds__(kThreads, 2) void pair_kernel(Product gx, InputGrad x, uint32_t blocks, Product gw, WeightGrad w) {
  __shared__ __attribute__((aligned(16))) Lds<1> lds;
  if (blockIdx.x < blocks) product<1, true, false>(gx, x, lds, blockIdx.x, blocks);
  else product<1, true, true>(gw, w, lds, blockIdx.x - blocks, gridDim.x - blocks);
}

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t kCus = 256;

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
  const Product g{static_cast<const float*>(weight), static_cast<const float*>(x), d_in, d_in, d_out, n, d_in, d_in, 1, 0, 0};
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
  Product gw{xf, gz, d_in, d_out, d_in, d_out, n, c.k_split, c.splits, 0, 0};
  const WeightGrad w{c.splits > 1 ? parts : g_weight, c.splits > 1 ? parts + c.splits * size : g_bias};
  Product gx{static_cast<const float*>(weight), gz, d_in, d_out, d_in, n, d_out, d_out, 1, 0, 0};
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
