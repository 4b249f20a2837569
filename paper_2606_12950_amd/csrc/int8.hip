// Rows as signed bytes with a scale each, and a layer of rows and weights so quantised.
//
// quantize_kernel: a row's largest magnitude, then code = x / scale to the nearest. A power of two of lanes takes a row, eight
// values each at a time; rows of up to 4,096 values stay in registers, longer ones are read again.
// The products are the tiles of products_bf16.h with pairs of bytes in the place of bfloat16 values: v_mfma_i32_32x32x32_i8
// takes as many bytes of either operand as the bfloat16 product, 32 k of them instead of 16. Both operands' bytes lie in the
// same order, whichever that is, and a whole-number sum does not depend on it.
#include "layers.h"
#include "products_bf16.h"
#include "vectors.h"

namespace maestro {
namespace {

// The whole number nearest to the real quotient x / s, ties to the even one; r = 1 / s rounded. rint(x r) is off by at most one,
// and x - n s is exact: a multiple of 2^-24 s or more, below s.
__device__ __forceinline__ int code_of(float x, float s, float r) {
  const float n = __builtin_rintf(x * r), twice = 2.0f * fmaf(-n, s, x), off = fabsf(twice);
  const int c = (int)n;
  const bool next = off > s || (off == s && (c & 1));
  return c + (next ? twice > 0.0f ? 1 : -1 : 0);
}

// Eight codes: x r rounded once, and what it leaves of x. Where that is less than half a scale for all eight, they are right; at a
// tie, or next to one, code_of decides. (Every value by code_of took 26 vector operations, as long as the memory does.)
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float s, float r, bool none) {
  float t[8], left = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    t[e] = fmaf(v[e], r, kRounder);
    left = fmaxf(left, fabsf(fmaf(kRounder - t[e], s, v[e])));
  }
  uint2 b = low_bytes8(t);
  if (!(left < 0.5f * s)) {
    int q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = code_of(v[e], s, r);
    b = bytes8(q);
  }
  return none ? make_uint2(0, 0) : b;
}

// R units of 8 values a lane; R = 0: any number of them, read twice.
template <class T, int R>
__global__ __launch_bounds__(256) void quantize_kernel(int64_t n, int32_t d, int32_t lanes, const T* __restrict__ x,
                                                       int8_t* __restrict__ codes, float* __restrict__ scale) {
  const int units = d / 8, lane = threadIdx.x & (lanes - 1);
  const int64_t row = (int64_t)blockIdx.x * (256 / lanes) + threadIdx.x / lanes;
  if (row >= n) return;                                     // whole rows: no lane of a row that is there
  const T* from = x + row * d;
  Vector8<T> held[R ? R : 1];
  float v[8];
  uint32_t most = 0;
  if constexpr (R > 0) {
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (lane + lanes * j < units) held[j].load(from + 8 * (lane + lanes * j));
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (lane + lanes * j < units) {
        const uint32_t m = largest8(held[j]);
        most = m > most ? m : most;
      }
  } else {
    for (int u = lane; u < units; u += lanes) {
      held[0].load(from + 8 * u);
      const uint32_t m = largest8(held[0]);
      most = m > most ? m : most;
    }
  }
  for (int step = 1; step < lanes; step <<= 1) {
    const uint32_t m = __shfl_xor(most, step);
    most = m > most ? m : most;
  }
  const bool none = most >= 0x7F800000u;
  const float s = fmaxf(__uint_as_float(most) / 127.0f, 0x1p-126f), r = 1.0f / s;
  uint2* to = reinterpret_cast<uint2*>(codes + row * d);
  if constexpr (R > 0) {
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (lane + lanes * j < units) {
        held[j].get(v);
        to[lane + lanes * j] = codes8(v, s, r, none);
      }
  } else {
    for (int u = lane; u < units; u += lanes) {
      held[0].load(from + 8 * u);
      held[0].get(v);
      to[u] = codes8(v, s, r, none);
    }
  }
  if (lane == 0) scale[row] = none ? __uint_as_float(0x7FC00000u) : s;
}

template <class T>
void launch_quantize(int64_t n, int32_t d, const T* x, int8_t* codes, float* scale, hipStream_t stream) {
  const int8::RowLanes l = int8::row_lanes(d);
  const int64_t rows = 256 / l.lanes;
  const unsigned blocks = (unsigned)((n + rows - 1) / rows);
  auto kernel = l.units == 1 ? quantize_kernel<T, 1> : l.units == 2 ? quantize_kernel<T, 2> : l.units == 4 ? quantize_kernel<T, 4>
              : l.units == 8 ? quantize_kernel<T, 8> : quantize_kernel<T, 0>;
  kernel<<<blocks, 256, 0, stream>>>(n, d, l.lanes, x, codes, scale);
}

template <int WP, int WQ, int kWaves, class T>
__global__ __launch_bounds__(64 * kWaves, (Tile<WP, WQ, 64, 2, Int8Forward<T>, kWaves>::kSimdWaves)) void int8_kernel(Product g, Int8Forward<T> out) {
  using L = Tile<WP, WQ, 64, 2, Int8Forward<T>, kWaves>;
  __shared__ __attribute__((aligned(16))) unsigned char lds[L::kBytes];
  product<WP, WQ, 64, 2, false, false, kWaves>(g, out, Dense<L::TP, L::TQ, 64>(g), lds, blockIdx.x, gridDim.x);
}

template <int WP, int WQ, int kWaves, class T>
void launch_tiles(Product g, const Int8Forward<T>& out, hipStream_t stream) {
  using L = Tile<WP, WQ, 64, 2, Int8Forward<T>, kWaves>;
  g.p_tiles = (int32_t)cdiv(g.np, L::TP);
  g.splits = 1;
  g.items = cdiv(g.nq, L::TQ) * g.p_tiles;
  const int64_t want = cdiv(g.items, 8) * 8, most = kCus * L::kResident;
  int8_kernel<WP, WQ, kWaves, T><<<(unsigned)(want < most ? want : most), 64 * kWaves, 0, stream>>>(g, out);
}

template <class T>
void launch_product(const Product& g, const Int8Forward<T>& out, hipStream_t stream) {
  const int8::ProductTile t = int8::product_tile(g.np, g.nq);
  if (t.tile == 256 && t.wavefronts == 4) launch_tiles<4, 4, 4>(g, out, stream);
  else if (t.tile == 256) launch_tiles<4, 2, 8>(g, out, stream);
  else if (t.tile == 128) launch_tiles<2, 2, 4>(g, out, stream);
  else launch_tiles<1, 1, 4>(g, out, stream);
}

}  // namespace

maestro_status launch_quantize_rows(int64_t n, int32_t d, int32_t dtype, const void* x, int8_t* codes, float* scale,
                                    hipStream_t stream) {
  constexpr int64_t kRows = (int64_t)1 << 25;               // of a launch: 64 threads a row at most, counted in 32 bits
  for (int64_t row = 0; row < n; row += kRows) {
    const int64_t rows = n - row < kRows ? n - row : kRows;
    if (dtype == MAESTRO_BF16)
      launch_quantize(rows, d, static_cast<const __bf16*>(x) + row * d, codes + row * d, scale + row, stream);
    else launch_quantize(rows, d, static_cast<const float*>(x) + row * d, codes + row * d, scale + row, stream);
  }
  return launch_status();
}

maestro_status launch_layer_int8(int64_t n, int32_t d_in, int32_t d_out, const int8_t* x, const float* x_scale,
                                 const int8_t* weight, const float* weight_scale, const float* bias, bool relu, int32_t dtype,
                                 void* y, hipStream_t stream) {
  const Product g{reinterpret_cast<const __bf16*>(weight), reinterpret_cast<const __bf16*>(x), d_in / 2, d_in / 2, d_out, n,
                  d_in / 2, d_in / 2, 1, 0, 0};
  if (dtype == MAESTRO_BF16)
    launch_product(g, Int8Forward<__bf16>{bias, weight_scale, x_scale, static_cast<__bf16*>(y), relu}, stream);
  else launch_product(g, Int8Forward<float>{bias, weight_scale, x_scale, static_cast<float*>(y), relu}, stream);
  return launch_status();
}

}  // namespace maestro
