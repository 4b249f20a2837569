// The global norm over many gradient tensors, and clipping by it.
//
// Tensors reach the kernels as tables in the kernel arguments, up to kTensors a launch, so a call keeps
// nothing and a captured graph holds its own copy. Squares are summed in float64: a product of two
// float32 is exact there and cannot overflow, and the sum needs no care for order or length.
#include <math.h>

#include "train.h"

namespace maestro {
namespace {

constexpr int kTensors = 96;         // 96 * 32 bytes of table: within the 4 KB of kernel arguments
constexpr int kThreads = 256;
constexpr int kChunk = 16384;        // values of one unit of work
constexpr int kBlocks = 1024;        // workgroups a launch, and partial sums it leaves

struct Table {
  const void* in[kTensors];
  void* out[kTensors];
  int64_t size[kTensors];
  int64_t chunk[kTensors];           // first chunk of each tensor, over all of the launch's
  uint64_t bf16[2];
  int64_t chunks;
  int32_t count;
};

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return (float)v; }

// the tensor that chunk c lies in: the last one whose first chunk is not past it
__device__ __forceinline__ int tensor_of(const Table& t, int64_t c) {
  int lo = 0, hi = t.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.chunk[mid] <= c) lo = mid;
    else hi = mid;
  }
  return lo;
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

template <typename T>
__device__ __forceinline__ double square_sum(const T* x, int64_t lo, int64_t hi) {
  double s = 0.0;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
    const double v = to_f32(x[i]);
    s = fma(v, v, s);
  }
  return s;
}

template <typename T>
__device__ __forceinline__ void scale(const T* x, T* y, int64_t lo, int64_t hi, double f) {
  for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) y[i] = (T)(float)((double)to_f32(x[i]) * f);
}

__global__ __launch_bounds__(kThreads) void square_kernel(Table t, double* partial) {
  double s = 0.0;
  for (int64_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const int i = tensor_of(t, c);
    const int64_t lo = (c - t.chunk[i]) * kChunk, hi = lo + kChunk < t.size[i] ? lo + kChunk : t.size[i];
    if ((t.bf16[i >> 6] >> (i & 63)) & 1) s += square_sum(static_cast<const __bf16*>(t.in[i]), lo, hi);
    else s += square_sum(static_cast<const float*>(t.in[i]), lo, hi);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// total[0] = the sum of squares
__global__ __launch_bounds__(kThreads) void total_kernel(const double* partial, int64_t n, double* total, float* norm) {
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += kThreads) s += partial[i];
  s = block_sum(s);
  if (threadIdx.x == 0) {
    total[0] = s;
    norm[0] = (float)sqrt(s);
  }
}

__global__ __launch_bounds__(kThreads) void scale_kernel(Table t, const double* total, double max_norm, bool in_place) {
  const double norm = sqrt(total[0]);
  const bool over = norm > max_norm && norm < INFINITY;
  if (!over && in_place) return;
  const double f = over ? max_norm / norm : 1.0;
  for (int64_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const int i = tensor_of(t, c);
    const int64_t lo = (c - t.chunk[i]) * kChunk, hi = lo + kChunk < t.size[i] ? lo + kChunk : t.size[i];
    if ((t.bf16[i >> 6] >> (i & 63)) & 1)
      scale(static_cast<const __bf16*>(t.in[i]), static_cast<__bf16*>(t.out[i]), lo, hi, f);
    else
      scale(static_cast<const float*>(t.in[i]), static_cast<float*>(t.out[i]), lo, hi, f);
  }
}

// the next launch's table, from tensor `next` on; empty tensors take no entry
void fill(Table& t, int32_t& next, int32_t n, void* const* tensors, void* const* out, const int64_t* sizes,
          const int32_t* dtypes) {
  t.count = 0;
  t.chunks = 0;
  t.bf16[0] = t.bf16[1] = 0;
  for (; next < n && t.count < kTensors; ++next) {
    if (sizes[next] == 0) continue;
    const int i = t.count++;
    t.in[i] = tensors[next];
    t.out[i] = out ? out[next] : tensors[next];
    t.size[i] = sizes[next];
    t.chunk[i] = t.chunks;
    t.chunks += (sizes[next] + kChunk - 1) / kChunk;
    if (dtypes[next] == MAESTRO_BF16) t.bf16[i >> 6] |= 1ull << (i & 63);
  }
}

unsigned grid_of(const Table& t) { return (unsigned)(t.chunks < kBlocks ? t.chunks : kBlocks); }

}  // namespace

// the total, then every launch's partial sums
size_t clip_workspace_bytes(int32_t n_tensors) {
  return 16 + ((size_t)n_tensors + kTensors - 1) / kTensors * kBlocks * sizeof(double);
}

maestro_status launch_clip(int32_t n_tensors, void* const* tensors, void* const* out, const int64_t* sizes,
                           const int32_t* dtypes, float max_norm, float* norm, void* workspace, hipStream_t stream) {
  double* total = static_cast<double*>(workspace);
  double* partial = total + 2;
  int64_t sums = 0;
  Table t;
  for (int32_t next = 0; next < n_tensors;) {
    fill(t, next, n_tensors, tensors, out, sizes, dtypes);
    if (t.count == 0) break;
    square_kernel<<<grid_of(t), kThreads, 0, stream>>>(t, partial + sums);
    sums += grid_of(t);
  }
  total_kernel<<<1, kThreads, 0, stream>>>(partial, sums, total, norm);
  if (max_norm == INFINITY) return launch_status();
  for (int32_t next = 0; next < n_tensors;) {
    fill(t, next, n_tensors, tensors, out, sizes, dtypes);
    if (t.count == 0) break;
    scale_kernel<<<grid_of(t), kThreads, 0, stream>>>(t, total, max_norm, !out);
  }
  return launch_status();
}

}  // namespace maestro
