// Eight neighbouring values of a float32 or bfloat16 row, in float32.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace maestro {

template <class T>
struct Vector8;
template <>
struct Vector8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
  static __device__ __forceinline__ void store(float* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
};
template <>
struct Vector8<__bf16> {
  uint4 w;
  __device__ __forceinline__ void load(const __bf16* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(u[i] << 16), v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
  // of values that are bfloat16 already
  static __device__ __forceinline__ void store(__bf16* p, const float (&v)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = (__float_as_uint(v[2 * i]) >> 16) | (__float_as_uint(v[2 * i + 1]) & 0xFFFF0000u);
    *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
  }
};

// The largest magnitude of eight values, as bits: NaN above infinity above any number.
__device__ __forceinline__ uint32_t largest8(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t a = __float_as_uint(v[e]) & 0x7FFFFFFFu;
    m = a > m ? a : m;
  }
  return m;
}
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t largest8(const Vector8<float>& w) {
  float v[8];
  w.get(v);
  return largest8(v);
}
__device__ __forceinline__ uint32_t largest8(const Vector8<__bf16>& w) {      // pairs at a time
  auto size = [](uint32_t u) { return __builtin_bit_cast(u16x2, u & 0x7FFF7FFFu); };
  const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(size(w.w.x), size(w.w.y)),
                                            __builtin_elementwise_max(size(w.w.z), size(w.w.w)));
  return (uint32_t)(m.x > m.y ? m.x : m.y) << 16;
}

// x + kRounder is x rounded to a whole number, ties to the even one, in the sum's low bits (|x| < 2^22): its lowest byte is a code.
constexpr float kRounder = 12582912.0f;      // 1.5 * 2^23

// The lowest bytes of eight words.
__device__ __forceinline__ uint2 low_bytes8(const float (&t)[8]) {
  auto u = [&](int e) { return __float_as_uint(t[e]); };
  uint2 b;
  b.x = __builtin_amdgcn_perm(u(1), u(0), 0x0C0C0400u) | __builtin_amdgcn_perm(u(3), u(2), 0x04000C0Cu);
  b.y = __builtin_amdgcn_perm(u(5), u(4), 0x0C0C0400u) | __builtin_amdgcn_perm(u(7), u(6), 0x04000C0Cu);
  return b;
}

// Eight whole numbers as bytes.
__device__ __forceinline__ uint2 bytes8(const int (&q)[8]) {
  uint2 u;
  u.x = (q[0] & 255) | (q[1] & 255) << 8 | (q[2] & 255) << 16 | (uint32_t)q[3] << 24;
  u.y = (q[4] & 255) | (q[5] & 255) << 8 | (q[6] & 255) << 16 | (uint32_t)q[7] << 24;
  return u;
}

}  // namespace maestro
