// The global norm over many gradient tensors, and clipping by it: one pass that leaves sums of squares, one that adds
// them up (every workgroup for itself, in the same order) and scales.
//
// Tensors reach the kernels as tables in the kernel arguments, up to kTensors a launch, so a call keeps
// nothing and a captured graph holds its own copy. Squares are summed in float64: a product of two
// float32 is exact there and cannot overflow, and the sum needs no care for order or length. The scaled value is a float64
// product rounded to float32 (and then to the tensor's type), so no factor is too small for a float32.
//
// Bound by HBM. The second pass goes through the tensors backwards: what the first read last is still in the memory-side
// cache. 320 bfloat16 tensors of 403 million values (805 MB, read twice and written once) 490 us = 4.9 TB/s, their norm
// alone 175 us; two float32 tensors of 145 million 345 us = 5.1; small sets are bound by the two launches.
#include <math.h>

#include "train.h"

namespace maestro {
namespace {

constexpr int kTensors = 160;        // 160 * 22 bytes of table: within the 4 KB of kernel arguments. 400 small tensors 31 us a call (50 with 96 in a table)
constexpr int kFew = 12;             // a smaller table, which is sooner copied to the arguments: six tensors 9.3 us a call (9.8)
constexpr int kThreads = 256;
constexpr int kAhead = 8;            // 16-byte vectors of a thread in flight
constexpr int64_t kChunk = 16 * kThreads * kAhead;        // bytes of one unit of work
constexpr int kBlocks = 2048;        // the most workgroups, and so partial sums, of a launch

template <int N>
struct Table {
  const void* in[N];
  void* out[N];
  uint32_t chunk[N];                 // first chunk of each tensor, over all of the launch's
  uint16_t last[N];                  // values in its last chunk (at most 2^14), and 2^15 for bfloat16
  uint32_t chunks;                   // < 2^32: a tensor has at most 2^24 (kClipMaxBytes)
  int32_t count;
};
static_assert(sizeof(Table<kTensors>) <= 3600, "kernel arguments");

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 __attribute__((aligned(2))) u32x4_at2;        // tensors start anywhere
typedef u32x4 __attribute__((aligned(4))) u32x4_at4;

template <typename T>
constexpr int kVec = 16 / sizeof(T);

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return (float)v; }
__device__ __forceinline__ u32x4 load16(const float* p) { return *reinterpret_cast<const u32x4_at4*>(p); }
__device__ __forceinline__ u32x4 load16(const __bf16* p) { return *reinterpret_cast<const u32x4_at2*>(p); }
__device__ __forceinline__ void store16(float* p, const u32x4& w) { *reinterpret_cast<u32x4_at4*>(p) = w; }
__device__ __forceinline__ void store16(__bf16* p, const u32x4& w) { *reinterpret_cast<u32x4_at2*>(p) = w; }

// the tensor that chunk c lies in: the last one whose first chunk is not past it
template <int N>
__device__ __forceinline__ int tensor_of(const Table<N>& t, uint32_t c) {
  int lo = 0, hi = t.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.chunk[mid] <= c) lo = mid;
    else hi = mid;
  }
  return lo;
}

// chunk c: its tensor, type, and values [lo, hi)
struct Chunk {
  int i;
  bool bf16;
  int64_t lo, hi;
};
template <int N>
__device__ __forceinline__ Chunk chunk_of(const Table<N>& t, uint32_t c) {
  Chunk k;
  k.i = tensor_of(t, c);
  const uint32_t last = t.last[k.i], end = k.i + 1 < t.count ? t.chunk[k.i + 1] : t.chunks;
  k.bf16 = last >> 15;
  const int64_t most = kChunk / (k.bf16 ? 2 : 4);
  k.lo = (c - t.chunk[k.i]) * most;
  k.hi = k.lo + (c + 1 == end ? last & 0x7FFF : most);
  return k;
}

__device__ __forceinline__ double block_sum(double s) {
  __shared__ double part[kThreads / 64];
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  __syncthreads();
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < kThreads / 64; ++w) s += part[w];
  return s;
}

__device__ __forceinline__ void add_squares(const u32x4& w, const float*, double& s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const double v = __uint_as_float(w[i]);
    s = fma(v, v, s);
  }
}
__device__ __forceinline__ void add_squares(const u32x4& w, const __bf16*, double& s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const double lo = __uint_as_float(w[i] << 16), hi = __uint_as_float(w[i] & 0xFFFF0000u);
    s = fma(lo, lo, s);
    s = fma(hi, hi, s);
  }
}
__device__ __forceinline__ float scaled(float v, double f) { return (float)((double)v * f); }
__device__ __forceinline__ u32x4 scale16(const u32x4& w, const float*, double f) {
  return u32x4{__float_as_uint(scaled(__uint_as_float(w[0]), f)), __float_as_uint(scaled(__uint_as_float(w[1]), f)),
               __float_as_uint(scaled(__uint_as_float(w[2]), f)), __float_as_uint(scaled(__uint_as_float(w[3]), f))};
}
__device__ __forceinline__ u32x4 scale16(const u32x4& w, const __bf16*, double f) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 v = {scaled(__uint_as_float(w[i] << 16), f), scaled(__uint_as_float(w[i] & 0xFFFF0000u), f)};
    out[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
  }
  return out;
}

// values [lo, hi), at most a chunk
template <typename T>
__device__ __forceinline__ double square_sum(const T* x, int64_t lo, int64_t hi) {
  constexpr int V = kVec<T>;
  double s = 0.0;
  if (hi - lo == kThreads * kAhead * V) {
    u32x4 w[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) w[u] = load16(x + lo + (u * kThreads + threadIdx.x) * V);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) add_squares(w[u], x, s);
  } else {
    for (int64_t i = lo + threadIdx.x * V; i < hi; i += kThreads * V) {
      if (i + V <= hi) add_squares(load16(x + i), x, s);
      else
        for (int64_t j = i; j < hi; ++j) {
          const double v = to_f32(x[j]);
          s = fma(v, v, s);
        }
    }
  }
  return s;
}

template <typename T>
__device__ __forceinline__ void scale(const T* x, T* y, int64_t lo, int64_t hi, double f) {
  constexpr int V = kVec<T>;
  if (hi - lo == kThreads * kAhead * V) {
    u32x4 w[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) w[u] = load16(x + lo + (u * kThreads + threadIdx.x) * V);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) store16(y + lo + (u * kThreads + threadIdx.x) * V, scale16(w[u], x, f));
  } else {
    for (int64_t i = lo + threadIdx.x * V; i < hi; i += kThreads * V) {
      if (i + V <= hi) store16(y + i, scale16(load16(x + i), x, f));
      else
        for (int64_t j = i; j < hi; ++j) y[j] = (T)scaled(to_f32(x[j]), f);
    }
  }
}

template <int N>
__global__ __launch_bounds__(kThreads) void square_kernel(Table<N> t, double* partial) {
  double s = 0.0;
  for (int64_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const Chunk k = chunk_of(t, (uint32_t)c);
    if (k.bf16) s += square_sum(static_cast<const __bf16*>(t.in[k.i]), k.lo, k.hi);
    else s += square_sum(static_cast<const float*>(t.in[k.i]), k.lo, k.hi);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// the sum of all partial sums, in every thread
__device__ __forceinline__ double total(const double* partial, int64_t n) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += kThreads) s += partial[i];
  return block_sum(s);
}

__global__ __launch_bounds__(kThreads) void norm_kernel(const double* partial, int64_t n, float* norm) {
  const double s = total(partial, n);
  if (threadIdx.x == 0) norm[0] = (float)sqrt(s);
}

// norm: written by the first launch's first workgroup, NULL in the others
template <int N>
__global__ __launch_bounds__(kThreads) void scale_kernel(Table<N> t, const double* partial, int64_t n, double max_norm,
                                                         bool in_place, float* norm) {
  const double all = sqrt(total(partial, n));
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) norm[0] = (float)all;
  const bool over = all > max_norm && all < INFINITY;
  if (!over && in_place) return;
  const double f = over ? max_norm / all : 1.0;
  for (int64_t c = (int64_t)t.chunks - 1 - blockIdx.x; c >= 0; c -= gridDim.x) {
    const Chunk k = chunk_of(t, (uint32_t)c);
    if (k.bf16) scale(static_cast<const __bf16*>(t.in[k.i]), static_cast<__bf16*>(t.out[k.i]), k.lo, k.hi, f);
    else scale(static_cast<const float*>(t.in[k.i]), static_cast<float*>(t.out[k.i]), k.lo, k.hi, f);
  }
}

struct Call {
  int32_t n;
  void* const* tensors;
  void* const* out;
  const int64_t* sizes;
  const int32_t* dtypes;
};

// The table of the tensors [from, to): at most N that are not empty.
template <int N>
void fill(Table<N>& t, const Call& c, int32_t from, int32_t to) {
  t.count = 0;
  t.chunks = 0;
  for (int32_t j = from; j < to; ++j) {
    if (c.sizes[j] == 0) continue;
    const int i = t.count++;
    t.in[i] = c.tensors[j];
    t.out[i] = c.out ? c.out[j] : c.tensors[j];
    t.chunk[i] = t.chunks;
    const bool bf16 = c.dtypes[j] == MAESTRO_BF16;
    const int64_t most = kChunk / (bf16 ? 2 : 4), chunks = (c.sizes[j] + most - 1) / most;
    t.last[i] = (uint16_t)(c.sizes[j] - (chunks - 1) * most + (bf16 ? 0x8000 : 0));
    t.chunks += (uint32_t)chunks;
  }
}

int32_t launches_of(int32_t n) { return (int32_t)(((int64_t)n + kTensors - 1) / kTensors); }

// Workgroups of a launch: fewer where there are many launches, so that the partial sums stay soon added up.
template <int N>
unsigned grid_of(const Table<N>& t, int32_t launches) {
  int64_t most = 2 * kBlocks / launches;
  most = most < 64 ? 64 : most > kBlocks ? kBlocks : most;
  return (unsigned)(t.chunks < most ? t.chunks : most);
}

template <int N>
maestro_status launch(const Call& c, int32_t launches, float max_norm, float* norm, double* partial, hipStream_t stream) {
  int64_t sums = 0;
  Table<N> t;
  for (int32_t l = 0; l < launches; ++l) {
    fill(t, c, l * N, l == launches - 1 ? c.n : (l + 1) * N);
    if (t.count == 0) continue;
    const unsigned grid = grid_of(t, launches);
    square_kernel<<<grid, kThreads, 0, stream>>>(t, partial + sums);
    sums += grid;
  }
  if (max_norm == INFINITY || sums == 0) {
    norm_kernel<<<1, kThreads, 0, stream>>>(partial, sums, norm);
    return launch_status();
  }
  for (int32_t l = launches - 1; l >= 0; --l) {             // backwards: see the top
    if (launches > 1) fill(t, c, l * N, l == launches - 1 ? c.n : (l + 1) * N);
    if (t.count == 0) continue;
    scale_kernel<<<grid_of(t, 1), kThreads, 0, stream>>>(t, partial, sums, max_norm, !c.out, norm);
    norm = nullptr;
  }
  return launch_status();
}

}  // namespace

size_t clip_workspace_bytes(int32_t n_tensors) {
  return 16 + (size_t)launches_of(n_tensors) * kBlocks * sizeof(double);
}

maestro_status launch_clip(int32_t n_tensors, void* const* tensors, void* const* out, const int64_t* sizes,
                           const int32_t* dtypes, float max_norm, float* norm, void* workspace, hipStream_t stream) {
  const Call c{n_tensors, tensors, out, sizes, dtypes};
  double* partial = static_cast<double*>(workspace);
  if (n_tensors <= kFew) return launch<kFew>(c, n_tensors > 0, max_norm, norm, partial, stream);
  return launch<kTensors>(c, launches_of(n_tensors), max_norm, norm, partial, stream);
}

}  // namespace maestro
