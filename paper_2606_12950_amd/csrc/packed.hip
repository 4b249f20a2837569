// Activations kept in 8 bits: bytes, and for every 32 of a row a power of two.
//
// pack_kernel, unpack_kernel: eight values a thread; four neighbouring threads hold the 32 values of an exponent (two, at the end
// of a row of an odd number of 16s). The step 2^e is read off the largest magnitude's bits: with most = 127 (255 for
// rectified values, which need no sign) the least e with rint(largest / 2^e) <= most, so largest / 2^e < most + 1/2; the
// quotient by a power of two is exact. A value has at most 8 significant bits then, so bfloat16 holds it exactly. The step that would
// make 2^128 of a finite value is not taken: the one below it is, and codes end at the last one, less than a step from the value.
#include "layers.h"
#include "vectors.h"

namespace maestro {
namespace {

constexpr int kThreads = 256;
constexpr int kRowsBits = 31;        // threads of a launch's part of the rows, counted in 32 bits

// the exponent (127 added) of 32 values whose largest magnitude has these bits; 255: not finite
template <bool kRectified>
__device__ __forceinline__ int exponent_of(uint32_t most) {
  if (most >= 0x7F800000u) return 255;
  constexpr uint32_t kLast = kRectified ? 0x7F8000u : 0x7F0000u;      // mantissa of (most + 1/2) / 2^k
  constexpr int kBelow = kRectified ? 7 : 6;                          // a largest value's exponent over its step's
  const int e = (int)(most >> 23) - kBelow + ((most & 0x7FFFFFu) >= kLast ? 1 : 0);
  return e < 1 ? 1 : e > 254 - kBelow ? 254 - kBelow : e;
}
// 2^(127 - e): the inverse step's bits, for e = 1 .. 248
__device__ __forceinline__ float inverse_step(int e) { return __uint_as_float((uint32_t)(254 - e) << 23); }
__device__ __forceinline__ float step_of(int e) { return __uint_as_float((uint32_t)e << 23); }

// Rows are taken as `padded` units of 8 values, a multiple of four; rows of a launch times padded is below 2^31.
template <class T, bool kRectified>
__global__ __launch_bounds__(kThreads) void pack_kernel(uint32_t rows, uint32_t d, uint32_t padded, const T* __restrict__ x,
                                                        unsigned char* __restrict__ codes, uint8_t* __restrict__ exponents) {
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x, row = i / padded, unit = i % padded;
  const bool there = row < rows && unit * 8 < d;
  float v[8] = {};
  if (there) {
    Vector8<T> w;
    w.load(x + (int64_t)row * d + unit * 8);
    w.get(v);
  }
  if constexpr (kRectified)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] <= 0.0f ? 0.0f : v[e];        // a NaN stays one
  uint32_t most = largest8(v);
#pragma unroll
  for (int step = 1; step < 4; step <<= 1) {
    const uint32_t m = __shfl_xor(most, step);
    most = m > most ? m : most;
  }
  if (!there) return;
  const int e = exponent_of<kRectified>(most);
  const float inverse = inverse_step(e == 255 ? 1 : e);
  float t[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    t[j] = fmaf(v[j], inverse, kRounder);                   // the product is exact
    const float least = !kRectified ? kRounder - 127.0f : v[j] > 0.0f ? kRounder + 1.0f : kRounder;
    t[j] = __builtin_amdgcn_fmed3f(t[j], least, kRounder + (kRectified ? 255.0f : 127.0f));
  }
  *reinterpret_cast<uint2*>(codes + (int64_t)row * d + unit * 8) = e == 255 ? make_uint2(0, 0) : low_bytes8(t);
  if (unit % 4 == 0) exponents[(int64_t)row * (padded / 4) + unit / 4] = (uint8_t)e;
}

template <class T, class Code>
__global__ __launch_bounds__(kThreads) void unpack_kernel(uint32_t rows, uint32_t d, uint32_t units, uint32_t exponents_of_row,
                                                          const Code* __restrict__ codes,
                                                          const uint8_t* __restrict__ exponents, T* __restrict__ x) {
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x, row = i / units, unit = i % units;
  if (row >= rows) return;
  const int64_t at = (int64_t)row * d + unit * 8;
  const float s = step_of(exponents[(int64_t)row * exponents_of_row + unit / 4]);
  const uint2 w = *reinterpret_cast<const uint2*>(codes + at);
  Code c[8];
  __builtin_memcpy(c, &w, 8);
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (float)c[j] * s;
  Vector8<T>::store(x + at, v);
}

// f(first row, rows, blocks) for parts of n rows that `units` threads a row can count
template <class F>
void parts(int64_t n, int64_t units, const F& f) {
  const int64_t most = (((int64_t)1 << kRowsBits) - kThreads) / units;
  for (int64_t row = 0; row < n; row += most) {
    const int64_t rows = n - row < most ? n - row : most;
    f(row, (uint32_t)rows, (unsigned)((rows * units + kThreads - 1) / kThreads));
  }
}

template <class T>
void pack(int64_t n, int32_t d, const T* x, bool rectified, unsigned char* codes, uint8_t* exponents, hipStream_t stream) {
  const int64_t blocks_of_32 = (d + 31) / 32;
  auto kernel = rectified ? pack_kernel<T, true> : pack_kernel<T, false>;
  parts(n, 4 * blocks_of_32, [&](int64_t row, uint32_t rows, unsigned blocks) {
    kernel<<<blocks, kThreads, 0, stream>>>(rows, d, (uint32_t)(4 * blocks_of_32), x + row * d, codes + row * d, exponents + row * blocks_of_32);
  });
}

template <class T, class Code>
void unpack(int64_t n, int32_t d, const Code* codes, const uint8_t* exponents, T* x, hipStream_t stream) {
  const int64_t blocks_of_32 = (d + 31) / 32;
  parts(n, d / 8, [&](int64_t row, uint32_t rows, unsigned blocks) {
    unpack_kernel<T, Code><<<blocks, kThreads, 0, stream>>>(rows, d, d / 8, (uint32_t)blocks_of_32, codes + row * d, exponents + row * blocks_of_32, x + row * d);
  });
}

}  // namespace

maestro_status launch_pack(int64_t n, int32_t d, int32_t dtype, const void* x, bool rectified, void* codes, uint8_t* exponents,
                           hipStream_t stream) {
  auto* c = static_cast<unsigned char*>(codes);
  if (dtype == MAESTRO_BF16) pack(n, d, static_cast<const __bf16*>(x), rectified, c, exponents, stream);
  else pack(n, d, static_cast<const float*>(x), rectified, c, exponents, stream);
  return launch_status();
}

maestro_status launch_unpack(int64_t n, int32_t d, int32_t dtype, const void* codes, const uint8_t* exponents, bool rectified,
                             void* x, hipStream_t stream) {
  auto as = [&](auto* to) {
    if (rectified) unpack(n, d, static_cast<const uint8_t*>(codes), exponents, to, stream);
    else unpack(n, d, static_cast<const int8_t*>(codes), exponents, to, stream);
  };
  if (dtype == MAESTRO_BF16) as(static_cast<__bf16*>(x));
  else as(static_cast<float*>(x));
  return launch_status();
}

size_t grad_packed_workspace_bytes(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype) {
  return dtype == MAESTRO_BF16 ? grad_packed_bf16_workspace_bytes(n, d_in, d_out) : grad_packed_f32_workspace_bytes(n, d_in, d_out);
}

maestro_status launch_grad_packed(int64_t n, int32_t d_in, int32_t d_out, int32_t dtype, const void* codes,
                                  const uint8_t* exponents, bool rectified, const void* weight, const void* g_z, bool relu_input,
                                  void* g_x, float* g_weight, float* g_bias, void* workspace, hipStream_t stream) {
  if (n == 0) return launch_join(nullptr, 0, g_weight, (int64_t)d_in * d_out, nullptr, 0, g_bias, d_out, stream);
  if (dtype == MAESTRO_BF16)
    return launch_grad_packed_bf16(n, d_in, d_out, codes, exponents, rectified, weight, g_z, relu_input, g_x, g_weight, g_bias,
                                   workspace, stream);
  return launch_grad_packed_f32(n, d_in, d_out, codes, exponents, rectified, static_cast<const float*>(weight),
                                static_cast<const float*>(g_z), relu_input, static_cast<float*>(g_x), g_weight, g_bias, workspace,
                                stream);
}

}  // namespace maestro
