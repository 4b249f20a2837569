// Log probabilities of given tokens with entropy and alternatives, and their gradient.
#include "train.h"

namespace maestro {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 256;

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return (float)v; }

// m, S = sum e^(x - m), T = sum e^(x - m) (x - m) of a part of a row; a NaN or +inf makes m NaN or +inf
struct Part {
  float m, s, t;
};

__device__ __forceinline__ Part join(const Part& a, const Part& b) {
  if (!(a.m >= b.m)) {   // b holds the maximum, or one of the two is NaN
    if (b.m > a.m) return join(b, a);
    return Part{NAN, NAN, NAN};
  }
  if (b.m == -INFINITY) return a;
  const float d = b.m - a.m, e = __builtin_amdgcn_exp2f(d * kLog2e);
  return Part{a.m, a.s + e * b.s, a.t + e * b.t + fmaxf(d, -1e30f) * (e * b.s)};
}

template <typename T>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(int64_t n, int32_t v, const T* logits, int64_t stride,
                                                            const int32_t* token, int32_t k, float* logprob,
                                                            float* entropy, int32_t* top_id, float* top_logprob,
                                                            float* stats) {
  __shared__ Part parts[kThreads];
  __shared__ float best[kThreads];
  __shared__ int32_t at[kThreads];
  const int tid = threadIdx.x;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    const T* x = logits + row * stride;
    Part p{-INFINITY, 0.0f, 0.0f};
    for (int64_t j = tid; j < v; j += kThreads) p = join(p, Part{to_f32(x[j]), 1.0f, 0.0f});
    parts[tid] = p;
    __syncthreads();
    for (int w = kThreads / 2; w > 0; w >>= 1) {
      if (tid < w) parts[tid] = join(parts[tid], parts[tid + w]);
      __syncthreads();
    }
    p = parts[0];
    const bool none = p.m == -INFINITY, bad = !(p.m < INFINITY);
    const float log_s = bad ? NAN : none ? -INFINITY : logf(p.s), m = none ? 0.0f : p.m;
    if (tid == 0) {
      if (logprob) {
        const int32_t t = token[row];
        logprob[row] = (uint32_t)t >= (uint32_t)v ? 0.0f : none ? -INFINITY : to_f32(x[t]) - m - log_s;
      }
      if (entropy) entropy[row] = none ? 0.0f : bad ? NAN : log_s - p.t / p.s;
      if (stats) {
        stats[2 * row] = bad ? NAN : p.m;
        stats[2 * row + 1] = log_s;
      }
    }
    float last = INFINITY;
    int32_t last_at = -1;
    for (int i = 0; i < k; ++i) {   // the first value after the last one listed
      float b = -INFINITY;
      int32_t a = -1;
      for (int64_t j = tid; j < v; j += kThreads) {
        const float z = to_f32(x[j]);
        if ((z < last || (z == last && j > last_at)) && z > b) b = z, a = (int32_t)j;
      }
      best[tid] = b;
      at[tid] = a;
      __syncthreads();
      for (int w = kThreads / 2; w > 0; w >>= 1) {
        if (tid < w && (best[tid + w] > best[tid] ||
                        (best[tid + w] == best[tid] && (uint32_t)at[tid + w] < (uint32_t)at[tid])))
          best[tid] = best[tid + w], at[tid] = at[tid + w];
        __syncthreads();
      }
      last = best[0];
      last_at = at[0];
      if (tid == 0) {
        top_id[row * k + i] = bad ? -1 : last_at;
        top_logprob[row * k + i] = bad ? NAN : last_at < 0 ? -INFINITY : last - m - log_s;
      }
      __syncthreads();
    }
    __syncthreads();
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void logprobs_grad_kernel(int64_t n, int32_t v, const T* logits, int64_t stride,
                                                                 const int32_t* token, const float* stats,
                                                                 const float* entropy, const float* g_logprob,
                                                                 const float* g_entropy, T* grad, int64_t grad_stride) {
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    const T* x = logits + row * stride;
    T* out = grad + row * grad_stride;
    const int32_t t = token ? token[row] : -1;
    const float g = (uint32_t)t < (uint32_t)v ? g_logprob[row] : 0.0f;
    const float ge = g_entropy ? g_entropy[row] : 0.0f, h = g_entropy ? entropy[row] : 0.0f;
    const float m = stats[2 * row], log_s = stats[2 * row + 1];
    if (m == -INFINITY || (g == 0.0f && ge == 0.0f)) {
      for (int64_t j = threadIdx.x; j < v; j += kThreads) out[j] = (T)0.0f;
      continue;
    }
    for (int64_t j = threadIdx.x; j < v; j += kThreads) {
      const float lp = (to_f32(x[j]) - m) - log_s;
      const float p = __builtin_amdgcn_exp2f(lp * kLog2e);
      float d = -g * p;
      if (ge != 0.0f) d -= ge * (p * (fmaxf(lp, -1e30f) + h));
      if (j == t) d += g;
      out[j] = (T)d;
    }
  }
}

}  // namespace

size_t logprobs_workspace_bytes(int64_t, int32_t, int32_t, int32_t) { return 0; }

maestro_status launch_logprobs(int64_t n, int32_t v, const void* logits, int64_t row_stride, int32_t dtype,
                               const int32_t* token, int32_t k, float* logprob, float* entropy, int32_t* top_id,
                               float* top_logprob, float* stats, void*, hipStream_t stream) {
  const dim3 grid((unsigned)(n < 65536 ? n : 65536));
  if (dtype == MAESTRO_F32)
    logprobs_kernel<<<grid, kThreads, 0, stream>>>(n, v, static_cast<const float*>(logits), row_stride, token, k,
                                                   logprob, entropy, top_id, top_logprob, stats);
  else
    logprobs_kernel<<<grid, kThreads, 0, stream>>>(n, v, static_cast<const __bf16*>(logits), row_stride, token, k,
                                                   logprob, entropy, top_id, top_logprob, stats);
  return launch_status();
}

maestro_status launch_logprobs_grad(int64_t n, int32_t v, const void* logits, int64_t row_stride, int32_t dtype,
                                    const int32_t* token, const float* stats, const float* entropy,
                                    const float* g_logprob, const float* g_entropy, void* grad, int64_t grad_stride,
                                    hipStream_t stream) {
  const dim3 grid((unsigned)(n < 65536 ? n : 65536));
  if (dtype == MAESTRO_F32)
    logprobs_grad_kernel<<<grid, kThreads, 0, stream>>>(n, v, static_cast<const float*>(logits), row_stride, token,
                                                        stats, entropy, g_logprob, g_entropy, static_cast<float*>(grad),
                                                        grad_stride);
  else
    logprobs_grad_kernel<<<grid, kThreads, 0, stream>>>(n, v, static_cast<const __bf16*>(logits), row_stride, token,
                                                        stats, entropy, g_logprob, g_entropy,
                                                        static_cast<__bf16*>(grad), grad_stride);
  return launch_status();
}

}  // namespace maestro
