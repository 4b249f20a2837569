// Log probabilities of given tokens with entropy and alternatives, and their gradient.
//
// With m the row's maximum and u_j = (x_j - m) log2 e: S = sum 2^u_j, T = sum 2^u_j u_j, ln p_t = (x_t - m) - ln S and
// entropy = ln 2 (log2 S - T / S). The difference comes first, so large logits lose nothing to a rounded
// product; the hardware's 2^x and log2 are good to an ulp. A long row's S and T are chains of v / 64 to v / 512 additions, a chain
// a thread, and then a tree.
//
// A pass reads every logit once and is bound by HBM, but for short rows with alternatives, which are bound by the
// vector ALU. Measured, passes back to back over changing inputs (a copy reaches 5.1 TB/s): 4,096 rows of 50,257 float32 with 5
// alternatives 160 us = 5.1 TB/s, 2,048 of 131,072 bfloat16 with 8 117 us = 4.6; 2^20 rows of 64 bfloat16 37 us without
// alternatives (30 where the logits are still in the memory-side cache), 41 with one and 53 with four (floors 30, 32 and 37).
// Gradient: 2^20 x 64 bfloat16 55 us = 5.2 TB/s, 2,048 x 131,072 187 us = 5.7.
#include "train.h"

namespace maestro {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeast = -1e30f;     // below any log probability in range; times 0 it is 0
constexpr int kMaxAlternatives = MAESTRO_MAX_ALTERNATIVES;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 __attribute__((aligned(2))) u32x4_at2;        // rows start anywhere
typedef u32x4 __attribute__((aligned(4))) u32x4_at4;

template <typename T>
constexpr int kVec = 16 / sizeof(T);

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__bf16 v) { return (float)v; }

__device__ __forceinline__ u32x4 load16(const float* p) { return *reinterpret_cast<const u32x4_at4*>(p); }
__device__ __forceinline__ u32x4 load16(const __bf16* p) { return *reinterpret_cast<const u32x4_at2*>(p); }

__device__ __forceinline__ void unpack(const u32x4& w, float (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ void unpack(const u32x4& w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
}

// the vector at x[j] as it lies in memory, what lies past v filled with -inf
template <class I>
__device__ __forceinline__ u32x4 load_raw(const float* x, I j, I v) {
  if (j + 4 <= v) return load16(x + j);
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = j + i < v ? __float_as_uint(x[j + i]) : 0xFF800000u;
  return w;
}
template <class I>
__device__ __forceinline__ u32x4 load_raw(const __bf16* x, I j, I v) {
  if (j + 8 <= v) return load16(x + j);
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = j + 2 * i < v ? __builtin_bit_cast(uint16_t, x[j + 2 * i]) : 0xFF80;
    const uint32_t hi = j + 2 * i + 1 < v ? __builtin_bit_cast(uint16_t, x[j + 2 * i + 1]) : 0xFF80;
    w[i] = lo | (hi << 16);
  }
  return w;
}

// the same, unpacked
template <typename T>
__device__ __forceinline__ void load_vec(const T* x, int64_t j, int64_t v, float (&out)[kVec<T>]) {
  if (j + kVec<T> <= v) {
    unpack(load16(x + j), out);
  } else {
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) out[i] = j + i < v ? to_f32(x[j + i]) : -INFINITY;
  }
}

// --- reductions over G neighbouring lanes (a power of two) -----------------------------------------

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, kCtrl, 0xF, 0xF, true);
}

// v and the value of a lane that is on the other side of a step, so that after the steps 1, 2, 4, ... < G every
// lane has combined all of them
template <int kStep, class Op>
__device__ __forceinline__ uint32_t step(uint32_t v, const Op& op) {
  if constexpr (kStep == 1) return op(v, dpp<0xB1>(v));     // quad_perm 1,0,3,2
  else if constexpr (kStep == 2) return op(v, dpp<0x4E>(v));     // quad_perm 2,3,0,1
  else if constexpr (kStep == 4) return op(v, dpp<0x141>(v));    // row_half_mirror: the other four of eight
  else if constexpr (kStep == 8) return op(v, dpp<0x140>(v));    // row_mirror: the other eight of sixteen
  else if constexpr (kStep == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);     // even rows, odd rows
    return op(r[0], r[1]);
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);     // lower half, upper half
    return op(r[0], r[1]);
  }
}

template <int G, int kStep = 1, class Op>
__device__ __forceinline__ uint32_t combine(uint32_t v, const Op& op) {
  if constexpr (kStep < G) return combine<G, 2 * kStep>(step<kStep>(v, op), op);
  else return v;
}
// NaN if either is (v_maximum3_f32)
__device__ __forceinline__ float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }

template <int G>
__device__ __forceinline__ float group_max(float v) {
  return __uint_as_float(combine<G>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(maximum(__uint_as_float(a), __uint_as_float(b)));
  }));
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
  return __uint_as_float(combine<G>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}
template <int G>
__device__ __forceinline__ uint32_t group_max_u32(uint32_t v) {
  return combine<G>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
// --- one part of a row ------------------------------------------------------------------------

// maximum m (-inf where nothing is visible, NaN where anything is), and S, T relative to base_of(m)
struct Part {
  float m, s, t;
};

__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }

__device__ __forceinline__ void add(Part& p, float x, float base) {
  const float u = fmaxf((x - base) * kLog2e, kLeast), e = __builtin_amdgcn_exp2f(u);
  p.s += e;
  p.t = fmaf(e, u, p.t);
}

// p relative to a larger maximum m. A part in which nothing is visible has S = T = 0 and stays as it is.
__device__ __forceinline__ void rebase(Part& p, float m) {
  if (p.m != -INFINITY) {
    const float d = fmaxf((p.m - m) * kLog2e, kLeast), f = __builtin_amdgcn_exp2f(d);
    p.t = f * fmaf(p.s, d, p.t);
    p.s *= f;
  }
  p.m = m;
}

// all lanes' parts in every lane of the group
template <int G>
__device__ __forceinline__ Part group_join(Part p) {
  rebase(p, group_max<G>(p.m));
  p.s = group_sum<G>(p.s);
  p.t = group_sum<G>(p.t);
  return p;
}

// What a row's outputs need, from the joined part.
struct RowStats {
  float base, entropy, m, log_s;
  bool none, bad;
};
__device__ __forceinline__ RowStats row_stats(const Part& p) {
  RowStats r;
  r.bad = !(p.m < INFINITY);
  r.none = p.m == -INFINITY;
  r.base = base_of(p.m);
  const float log2_s = __builtin_amdgcn_logf(p.s);
  r.entropy = r.bad ? NAN : r.none ? 0.0f : kLn2 * (log2_s - p.t * __builtin_amdgcn_rcpf(p.s));
  r.m = r.bad ? NAN : p.m;
  r.log_s = r.bad ? NAN : r.none ? -INFINITY : kLn2 * log2_s;
  return r;
}
__device__ __forceinline__ float log_prob(const RowStats& r, float x) {
  return r.bad ? NAN : r.none ? -INFINITY : (x - r.base) - r.log_s;
}

struct Outputs {
  float* logprob;
  float* entropy;
  int32_t* top_id;
  float* top_logprob;
  float* stats;
};

__device__ __forceinline__ void write_row(const Outputs& o, int64_t row, const RowStats& r, bool given, float x) {
  if (o.logprob) o.logprob[row] = given ? log_prob(r, x) : 0.0f;
  if (o.entropy) o.entropy[row] = r.entropy;
  if (o.stats) *reinterpret_cast<float2*>(o.stats + 2 * row) = make_float2(r.m, r.log_s);
}

// --- short rows: a row to G lanes, its logits in registers -------------------------------------------

// A logit with its index as one whole number, larger for what comes first: the value as a two's complement number in the
// upper half (-0 is 0, -inf the least), the index counted down in the lower one.
template <typename T>
struct Key;
template <>
struct Key<__bf16> {
  typedef uint32_t type;
  static constexpr int kBits = 16;
  static constexpr uint32_t kMasked = 0x8080;               // -0x7F80
  // of the pair of logits w with indexes j, j + 1
  static __device__ __forceinline__ void make(uint32_t w, uint32_t j, uint32_t& a, uint32_t& b) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    const s16x2 v = __builtin_bit_cast(s16x2, w), m = v >> 15;
    const uint32_t s = __builtin_bit_cast(uint32_t, ((v & (short)0x7FFF) ^ m) - m);
    a = (s << 16) | (0xFFFF - j);
    b = (s & 0xFFFF0000u) | (0xFFFE - j);
  }
};
template <>
struct Key<float> {
  typedef uint64_t type;
  static constexpr int kBits = 32;
  static constexpr uint32_t kMasked = 0x80800000;           // -0x7F800000
  static __device__ __forceinline__ uint64_t make(uint32_t w, uint32_t j) {
    const int32_t m = (int32_t)w >> 31, s = (((int32_t)w & 0x7FFFFFFF) ^ m) - m;
    return ((uint64_t)(uint32_t)s << 32) | (0xFFFFFFFFu - j);
  }
};

template <int G>
__device__ __forceinline__ uint32_t group_max_key(uint32_t v) { return group_max_u32<G>(v); }
template <int G, int kStep = 1>
__device__ __forceinline__ uint64_t group_max_key(uint64_t v) {
  if constexpr (kStep < G) {
    // both sides of the step, word by word
    uint32_t a[2], b[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t w = (uint32_t)(v >> (32 * i));
      step<kStep>(w, [&](uint32_t x, uint32_t y) { return a[i] = x, b[i] = y, x; });
    }
    const uint64_t x = (uint64_t)a[1] << 32 | a[0], y = (uint64_t)b[1] << 32 | b[0];
    return group_max_key<G, 2 * kStep>(x > y ? x : y);
  } else {
    return v;
  }
}

constexpr int kShortThreads = 256;

// Rows of up to G R vectors of 16 bytes, R to a lane (vector u G + g to lane g); the next row's are loaded before this
// one's are used. Alternatives: the next one after w is the largest of key - w in unsigned arithmetic, which
// puts the keys already taken (and w itself) below all others; there are always more keys than alternatives.
//
// Few lanes to a row: what is done once a row (the reductions, logarithms and outputs) takes a lane's time however
// few logits the lane has. 2^20 x 64 bfloat16 with four alternatives: 85 us with a vector to each of 8 lanes, 52 with four
// to each of two.
template <typename T, int G, int R>
__global__ __launch_bounds__(kShortThreads) void short_kernel(int64_t n, int32_t v, const T* logits, int64_t stride,
                                                              const int32_t* token, int32_t k, Outputs o) {
  constexpr int V = kVec<T>, kRows = kShortThreads / G;
  static_assert(G * R * V >= kMaxAlternatives, "more keys than alternatives");
  typedef typename Key<T>::type K;
  const int g = threadIdx.x % G;
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
  if (row >= n) return;
  // a vector past v, or part of it, is -inf
  auto load = [&](const T* x, u32x4(&w)[R]) {
#pragma unroll
    for (int u = 0; u < R; ++u) w[u] = load_raw(x, (u * G + g) * V, v);
  };
  const T* x = logits + row * stride;
  const int64_t ahead = step * stride;
  u32x4 w[R];
  load(x, w);
  int32_t t = token ? token[row] : -1;
  for (; row < n; row += step) {
    const bool given = (uint32_t)t < (uint32_t)v, more = row + step < n;
    const float xt = given ? to_f32(x[t]) : 0.0f;
    x += ahead;
    u32x4 next[R];
    int32_t t_next = -1;
    if (more) {
      load(x, next);
      if (token) t_next = token[row + step];
    }
    Part p{-INFINITY, 0.0f, 0.0f};
    float z[R * V];
#pragma unroll
    for (int u = 0; u < R; ++u) unpack(w[u], *reinterpret_cast<float(*)[V]>(&z[u * V]));
#pragma unroll
    for (int i = 0; i < R * V; ++i) p.m = maximum(p.m, z[i]);
    p.m = group_max<G>(p.m);
    const float base = base_of(p.m);
#pragma unroll
    for (int i = 0; i < R * V; ++i) add(p, z[i], base);
    p.s = group_sum<G>(p.s);
    p.t = group_sum<G>(p.t);
    const RowStats r = row_stats(p);
    if (g == 0) write_row(o, row, r, given, xt);
    if (k > 0) {
      K key[R * V];
#pragma unroll
      for (int u = 0; u < R; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (V == 4) key[u * V + i] = Key<T>::make(w[u][i], (u * G + g) * V + i);
          else Key<T>::make(w[u][i], (u * G + g) * V + 2 * i, key[u * V + 2 * i], key[u * V + 2 * i + 1]);
        }
      K last = (K)1 << (2 * Key<T>::kBits - 1), mine = 0;   // below every key
      for (int i = 0; i < k; ++i) {
        K best = 0;
#pragma unroll
        for (int e = 0; e < R * V; ++e) {
          const K d = key[e] - last;
          best = d > best ? d : best;
        }
        last += group_max_key<G>(best);
        mine = i % G == g ? last : mine;
        if (i % G == G - 1 || i == k - 1) {                 // the group's lanes write up to G of them together
          const uint32_t s = (uint32_t)(mine >> Key<T>::kBits);
          const int32_t id = (int32_t)(V == 4 ? 0xFFFFFFFFu - (uint32_t)mine : 0xFFFF - (uint32_t)(mine & 0xFFFF));
          const int32_t whole = V == 4 ? (int32_t)s : (int32_t)(s << 16), sign = whole >> 31;
          const float value = __uint_as_float((uint32_t)((whole ^ sign) - sign) | ((uint32_t)sign & 0x80000000u));
          const bool none = r.bad || s == Key<T>::kMasked;
          if (g <= i % G) {
            const int64_t at = row * k + (i - i % G) + g;
            o.top_id[at] = none ? -1 : id;
            o.top_logprob[at] = r.bad ? NAN : none ? -INFINITY : log_prob(r, value);
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < R; ++u) w[u] = next[u];
    t = t_next;
  }
}

// --- longer rows: a row, or a segment of one, to a workgroup -------------------------------------------

constexpr int kCandidates = 512;

__device__ __forceinline__ bool better(float a, int32_t i, float b, int32_t j) { return a > b || (a == b && i < j); }

// A segment's part and its alternatives' logits and ids, for join_kernel.
struct Segments {
  float4* part;                      // [n][count]: m, S, T
  float* value;                      // [n][count][k]
  int32_t* id;
  int32_t count;
  int64_t length;
};

// Thread t takes the vectors t, t + kThreads, ... and keeps their maximum beside its sums. The k-th largest of any of
// those maxima bounds the k-th largest logit from below, so only the vectors of threads that reach it are read again (from
// the cache; hardly more than k of them, by all threads together), and of these only the logits that reach it are ranked. Where more than
// kCandidates do (long runs of equal logits), k scans find them instead.
//
// A wavefront to a row (no barriers, 64 threads) where rows are short (8 KB, any number of them) or many, 512 threads where they
// are few and long, else 256. Measured (us): 16,384 x 4,096 bfloat16 36 with 64 threads and 110 with 256, 4,096 x 20,000 39 and
// 48, 2,500 x 8,000 16.4 and 18.6, but 4,082 x 16,000 float32 60 and 51, 1,000 x 4,000 9.3 and 8.1, 2,048 x 131,072
// bfloat16 171 and 111; 4,082 x 2,000 float32 11.0 and 22.7, 3 of them 6.2 and 6.0; one row of 32,000 with eight
// alternatives 8.6 with 256 and 7.8 with 512 (9.5 with 1,024), one of 5,000 6.6 and 7.5.
template <typename T, int kThreads>
__global__ __launch_bounds__(kThreads) void long_kernel(int64_t n, int32_t v, const T* logits, int64_t stride,
                                                        const int32_t* token, int32_t k, Outputs o, Segments seg) {
  constexpr int V = kVec<T>, kWaves = kThreads / 64, kAhead = 4;
  __shared__ Part s_part[kWaves];
  constexpr int kTop = kThreads / 16 * ((kMaxAlternatives + kThreads / 16 - 1) / (kThreads / 16) + 1);
  __shared__ float s_top[kTop], s_value[kCandidates], s_bound;
  __shared__ int32_t s_id[kCandidates], s_who[kThreads];
  __shared__ uint32_t s_who_count, s_count;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t jobs = n * seg.count;
  for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
    // more than one segment: few rows, and 32 bits do
    const int64_t row = seg.count == 1 ? job : (int64_t)((uint32_t)job / (uint32_t)seg.count);
    const int64_t first = (job - row * seg.count) * seg.length;
    const T* x = logits + row * stride + first;
    const int64_t len = v - first < seg.length ? v - first : seg.length, vecs = (len + V - 1) / V;

    Part p{-INFINITY, 0.0f, 0.0f};
    float b = 0.0f;
    // some values of this thread
    auto take = [&](const auto& z) {
      constexpr int N = sizeof(z) / sizeof(float);
      float m = z[0];
#pragma unroll
      for (int i = 1; i < N; ++i) m = maximum(m, z[i]);
      if (!(m <= p.m)) {
        rebase(p, maximum(p.m, m));
        b = base_of(p.m);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) add(p, z[i], b);
    };
    for (int64_t at = 0; at < vecs; at += kAhead * kThreads) {
      u32x4 w[kAhead];                                      // unpacked when all are on their way
      if ((at + kAhead * kThreads) * V <= len) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) w[u] = load16(x + (at + u * kThreads + tid) * V);
        float z[kAhead * V];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) unpack(w[u], *reinterpret_cast<float(*)[V]>(&z[u * V]));
        take(z);
      } else {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) w[u] = load_raw<int64_t>(x, (at + u * kThreads + tid) * V, len);
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
          if (at + u * kThreads < vecs) {                   // nothing is computed for vectors that no thread has
            float z[V];
            unpack(w[u], z);
            take(z);
          }
      }
    }
    const float own = p.m;
    p = group_join<64>(p);
    if constexpr (kWaves > 1) {
      if (lane == 0) s_part[wave] = p;
      __syncthreads();
      p = s_part[lane % kWaves];
      p = group_join<kWaves>(p);
    }
    const RowStats r = row_stats(p);
    if (tid == 0) {
      if (seg.count > 1) {
        seg.part[job] = make_float4(p.m, p.s, p.t, 0.0f);
      } else {
        const int32_t t = token ? token[row] : -1;
        const bool given = (uint32_t)t < (uint32_t)v;
        write_row(o, row, r, given, given ? to_f32(x[t]) : 0.0f);
      }
      s_who_count = 0;
      s_count = 0;
    }
    if (k > 0) {
      auto put = [&](int i, int32_t id, float z) {          // alternative i of this job
        if (seg.count > 1) {
          seg.value[job * k + i] = z;
          seg.id[job * k + i] = id;
        } else {
          o.top_id[row * k + i] = id < 0 ? -1 : id;
          o.top_logprob[row * k + i] = r.bad ? NAN : id < 0 ? -INFINITY : log_prob(r, z);
        }
      };
      if (r.bad || r.none) {
        if (tid < k) put(tid, -1, -INFINITY);
      } else {
        // every 16 lanes their largest maxima, a few more than k in all, and the k-th of those
        constexpr int kGroups = kThreads / 16;
        const int rounds = (k + kGroups - 1) / kGroups + (2 * k > kGroups), values = kGroups * rounds;
        float left = own;
        for (int i = 0; i < rounds; ++i) {
          const float m = group_max<16>(left);
          if ((lane & 15) == 0) s_top[tid / 16 * rounds + i] = m;
          const uint64_t have = __ballot(left == m) >> (lane & 48) & 0xFFFF;
          if ((lane & 15) == __builtin_ctzll(have)) left = -INFINITY;
        }
        __syncthreads();
        if (tid < values) {
          const float mine = s_top[tid];
          int rank = 0;
#pragma unroll 8
          for (int i = 0; i < values; ++i) rank += s_top[i] > mine || (s_top[i] == mine && i < tid);
          if (rank == k - 1) s_bound = mine;
        }
        __syncthreads();
        const float w = s_bound;
        if (own >= w && own > -INFINITY) s_who[atomicAdd(&s_who_count, 1u)] = tid;
        __syncthreads();
        const uint32_t each = (uint32_t)((vecs + kThreads - 1) / kThreads), all = each * s_who_count;     // < 2^31 / V + 256
        for (uint32_t i = tid; i < all; i += kThreads) {
          const int64_t j = (s_who[i / each] + (int64_t)(i % each) * kThreads) * V;
          if (j < len) {
            float z[V];
            load_vec(x, j, len, z);
#pragma unroll
            for (int e = 0; e < V; ++e)
              if (z[e] >= w && z[e] > -INFINITY) {
                const uint32_t at = atomicAdd(&s_count, 1u);
                if (at < kCandidates) s_value[at] = z[e], s_id[at] = (int32_t)(j + e);
              }
          }
        }
        __syncthreads();
        const int count = (int)s_count;
        if (count <= kCandidates) {
          for (int a = tid; a < count; a += kThreads) {
            const float z = s_value[a];
            const int32_t id = s_id[a];
            int rank = 0;
#pragma unroll 8
            for (int b = 0; b < count; ++b) rank += better(s_value[b], s_id[b], z, id);
            if (rank < k) put(rank, (int32_t)(first + id), z);
          }
          if (tid >= count && tid < k) put(tid, -1, -INFINITY);
        } else {
          float last = INFINITY;
          int32_t last_id = -1;
          for (int i = 0; i < k; ++i) {
            float z = -INFINITY;
            int32_t id = 0x7FFFFFFF;
            for (int64_t j = (int64_t)tid * V; j < len; j += kThreads * V) {
              float y[V];
              load_vec(x, j, len, y);
#pragma unroll
              for (int e = 0; e < V; ++e)
                if (y[e] > z && better(last, last_id, y[e], (int32_t)(j + e))) z = y[e], id = (int32_t)(j + e);
            }
            for (int step = 1; step < 64; step *= 2) {
              const float y = __shfl_xor(z, step);
              const int32_t jd = __shfl_xor(id, step);
              if (better(y, jd, z, id)) z = y, id = jd;
            }
            if constexpr (kWaves > 1) {
              __syncthreads();
              if (lane == 0) s_value[wave] = z, s_id[wave] = id;
              __syncthreads();
              z = s_value[0], id = s_id[0];
              for (int b = 1; b < kWaves; ++b)
                if (better(s_value[b], s_id[b], z, id)) z = s_value[b], id = s_id[b];
            }
            last = z;
            last_id = id;
            if (tid == 0) put(i, z == -INFINITY ? -1 : (int32_t)(first + id), z);
          }
        }
      }
    }
    __syncthreads();
  }
}

// order-preserving bits of a visible logit, never 0; -0 equals 0
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

// The segments of a row joined by one wavefront, a segment to a lane: their parts, then k times the best of the
// segments' next alternatives.
__global__ __launch_bounds__(64) void join_kernel(int64_t n, int32_t v, const void* logits, int64_t stride, bool bf16,
                                                  const int32_t* token, int32_t k, Outputs o, Segments seg) {
  __shared__ float s_value[64 * kMaxAlternatives];
  __shared__ int32_t s_id[64 * kMaxAlternatives];
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x, count = seg.count;
  for (int i = lane; i < count * k; i += 64) {
    s_value[i] = seg.value[row * count * k + i];
    s_id[i] = seg.id[row * count * k + i];
  }
  Part p{-INFINITY, 0.0f, 0.0f};
  if (lane < count) {
    const float4 f = seg.part[row * count + lane];
    p = Part{f.x, f.y, f.z};
  }
  const RowStats r = row_stats(group_join<64>(p));
  if (lane == 0) {
    const int32_t t = token ? token[row] : -1;
    const bool given = (uint32_t)t < (uint32_t)v;
    const int64_t at = row * stride + t;
    write_row(o, row, r, given,
              !given ? 0.0f : bf16 ? to_f32(static_cast<const __bf16*>(logits)[at]) : static_cast<const float*>(logits)[at]);
  }
  __syncthreads();
  int head = 0;
  for (int i = 0; i < k; ++i) {
    float z = -INFINITY;
    int32_t id = -1;
    if (lane < count && head < k) z = s_value[lane * k + head], id = s_id[lane * k + head];
    const uint32_t mine = id < 0 || r.bad ? 0 : order_of(z), w = group_max_u32<64>(mine);
    // segments lie in ascending index, and so do lanes: the first of equal ones
    const uint64_t have = __ballot(mine == w);
    const int who = __builtin_ctzll(have);
    if (lane == who) {
      ++head;
      o.top_id[row * k + i] = w ? id : -1;
      o.top_logprob[row * k + i] = r.bad ? NAN : w ? log_prob(r, z) : -INFINITY;
    }
  }
}

// --- gradient -----------------------------------------------------------------------------------

__device__ __forceinline__ void store16(float* p, const u32x4& w) { *reinterpret_cast<u32x4_at4*>(p) = w; }
__device__ __forceinline__ void store16(__bf16* p, const u32x4& w) { *reinterpret_cast<u32x4_at2*>(p) = w; }

__device__ __forceinline__ u32x4 pack(const float (&d)[4]) {
  return u32x4{__float_as_uint(d[0]), __float_as_uint(d[1]), __float_as_uint(d[2]), __float_as_uint(d[3])};
}
__device__ __forceinline__ u32x4 pack(const float (&d)[8]) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 f = {d[2 * i], d[2 * i + 1]};
    w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
  }
  return w;
}

struct Gradient {
  const int32_t* token;
  const float* stats;
  const float* entropy;
  const float* g_logprob;
  const float* g_entropy;
};

// the row's own numbers, and a vector's gradient: hot_j - p_j g - ge (p_j (ln p_j + entropy)), the product with p_j first: it
// is in range where ge ln p_j is not, and 0 where p_j is
struct GradRow {
  float m, log_s, g, ge, h;
  int32_t t;
  bool zero;
  __device__ __forceinline__ void load(const Gradient& a, int64_t row, int32_t v) {
    t = a.token ? a.token[row] : -1;
    g = (uint32_t)t < (uint32_t)v ? a.g_logprob[row] : 0.0f;
    ge = a.g_entropy ? a.g_entropy[row] : 0.0f;
    h = a.g_entropy ? a.entropy[row] : 0.0f;
    h = ge != 0.0f ? h : 0.0f;
    const float2 s = *reinterpret_cast<const float2*>(a.stats + 2 * row);
    m = s.x;
    log_s = s.y;
    zero = m == -INFINITY || (g == 0.0f && ge == 0.0f);
  }
  // without kEntropy: for rows whose ge is 0
  template <bool kEntropy = true, int V>
  __device__ __forceinline__ void gradient(float (&x)[V], int64_t j) const {
    const int64_t hot = t - j;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float lp = (x[i] - m) - log_s, p = __builtin_amdgcn_exp2f(lp * kLog2e);
      float d = fmaf(-p, g, hot == i ? g : 0.0f);
      if constexpr (kEntropy) d = fmaf(-ge, p * (fmaxf(lp, kLeast) + h), d);
      x[i] = zero ? 0.0f : d;
    }
  }
};

constexpr int kGradAhead = 4;        // vectors of a thread in flight
// the longest row, in vectors, that shares a workgroup with others: 60,000 x 2,000 float32 168 us so and 188 a wavefront to
// a row, but 100,000 x 1,025 bfloat16 103 and 87 (more to compute for a vector)
template <typename T>
constexpr int kGradShort = sizeof(T) == 4 ? 512 : 64;
constexpr int kGradRow = 512;        // and the longest that a wavefront takes

// Rows of `vecs` vectors laid end to end, a vector to a thread, whatever rows a wavefront's lie in, so no lane idles at a
// row's end. magic = ceil(2^21 / vecs): i * magic >> 21 is i / vecs for i < vecs + 1024, vecs <= 1024.
// Measured (us; a row to a power of two of lanes before): 300,000 x 293 bfloat16 105 (164), 450,209 x 34 float32 33
// (44), 10^6 x 3 bfloat16 9.5 (13.9), 2^20 x 64 56 (56). Two or four vectors a thread take 5 to 30% longer (registers).
template <typename T, bool kEntropy>
__global__ __launch_bounds__(256) void grad_short_kernel(int64_t n, int32_t v, const T* logits, int64_t stride, Gradient a,
                                                         T* grad, int64_t grad_stride, uint32_t vecs, uint32_t magic) {
  constexpr int V = kVec<T>;
  const int64_t chunks = (n * vecs + 255) / 256;
  for (int64_t chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
    const int64_t first = chunk * 256;
    const int64_t row0 = first >> 32 ? first / vecs : (uint32_t)first / vecs;      // 32 bits: a sixth of the time
    const uint32_t i = (uint32_t)(first - row0 * vecs) + threadIdx.x, down = i * magic >> 21;
    const int64_t row = row0 + down;
    if (row >= n) continue;
    const int32_t j = (int32_t)(i - down * vecs) * V;
    const u32x4 w = load_raw(logits + row * stride, j, v);
    GradRow r;
    r.load(a, row, v);
    float x[V];
    unpack(w, x);
    r.template gradient<kEntropy>(x, j);
    T* out = grad + row * grad_stride + j;
    if (j + V <= v) {
      store16(out, pack(x));
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (j + e < v) out[e] = (T)x[e];
    }
  }
}

// a wavefront to a row
template <typename T>
__global__ __launch_bounds__(256) void grad_row_kernel(int64_t n, int32_t v, const T* logits, int64_t stride, Gradient a,
                                                       T* grad, int64_t grad_stride) {
  constexpr int V = kVec<T>;
  const int lane = threadIdx.x & 63;
  for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < n; row += (int64_t)gridDim.x * 4) {
    GradRow r;
    r.load(a, row, v);
    for (int j = V * lane; j < v; j += V * 64) {
      float x[V];
      load_vec(logits + row * stride, j, v, x);
      r.gradient(x, j);
      T* out = grad + row * grad_stride + j;
      if (j + V <= v) {
        store16(out, pack(x));
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (j + i < v) out[i] = (T)x[i];
      }
    }
  }
}

// a workgroup takes 256 kGradAhead vectors of a row
template <typename T>
__global__ __launch_bounds__(256) void grad_long_kernel(int64_t n, int32_t v, const T* logits, int64_t stride, Gradient a,
                                                        T* grad, int64_t grad_stride, int32_t parts) {
  constexpr int V = kVec<T>;
  const int64_t jobs = n * parts;
  for (int64_t job = blockIdx.x; job < jobs; job += gridDim.x) {
    const int64_t row = job / parts, first = (job - row * parts) * (256 * kGradAhead * V);
    const T* in = logits + row * stride;
    T* out = grad + row * grad_stride;
    GradRow r;
    r.load(a, row, v);
    if (first + 256 * kGradAhead * V <= v) {
      u32x4 w[kGradAhead];
#pragma unroll
      for (int u = 0; u < kGradAhead; ++u) w[u] = load16(in + first + (u * 256 + threadIdx.x) * V);
#pragma unroll
      for (int u = 0; u < kGradAhead; ++u) {
        const int64_t j = first + (u * 256 + threadIdx.x) * V;
        float x[V];
        unpack(w[u], x);
        r.gradient(x, j);
        store16(out + j, pack(x));
      }
    } else {
      for (int64_t j = first + threadIdx.x * V; j < v; j += 256 * V) {
        float x[V];
        load_vec(in, j, v, x);
        r.gradient(x, j);
        if (j + V <= v) {
          store16(out + j, pack(x));
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i)
            if (j + i < v) out[j + i] = (T)x[i];
        }
      }
    }
  }
}

// --- launches -----------------------------------------------------------------------------------

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

constexpr int64_t kCus = 256;

// Segments of a row: one where there are rows enough for the chip, or the row is soon read. One row of 131,072
// float32 with eight alternatives takes 22 us in one piece and 10 in 16 to 32 (both launches); one of 32,000 bfloat16 8 in one, 11
// in four.
int64_t segments_of(int64_t n, int64_t bytes) {
  if (n >= kCus || bytes < 131072) return 1;
  return least(least(64, cdiv(2 * kCus, n)), bytes / 16384);
}

// Alternatives up to which a row of 129 to 256 vectors stays in a wavefront's registers: each costs a pass over them there,
// of 64-bit keys for float32. Measured (us, short / long with 0, 2, 5 alternatives): 41,004 x 700 float32 25 / 31,
// 43 / 49, 65 / 58; 60,000 x 2,048 bfloat16 43 / 50, 67 / 75, 90 / 90; 20,000 x 1,100 22 / 22, 31 / 32, 38 / 36.
template <typename T>
constexpr int32_t kWideShort = sizeof(T) == 4 ? 2 : 4;

template <typename T, int G, int R>
void launch_short(int64_t n, int32_t v, const T* x, int64_t stride, const int32_t* token, int32_t k, const Outputs& o,
                  hipStream_t stream) {
  const int64_t blocks = cdiv(n, kShortThreads / G);
  short_kernel<T, G, R><<<(unsigned)least(blocks, kCus * 8), kShortThreads, 0, stream>>>(n, v, x, stride, token, k, o);
}

template <typename T>
maestro_status launch(int64_t n, int32_t v, const T* x, int64_t stride, const int32_t* token, int32_t k, const Outputs& o,
                      void* workspace, hipStream_t stream) {
  const int64_t vecs = cdiv(v, kVec<T>);
  if (vecs <= 4) launch_short<T, 2, 2>(n, v, x, stride, token, k, o, stream);
  else if (vecs <= 8) launch_short<T, 2, 4>(n, v, x, stride, token, k, o, stream);
  else if (vecs <= 16) launch_short<T, 4, 4>(n, v, x, stride, token, k, o, stream);
  else if (vecs <= 32) launch_short<T, 8, 4>(n, v, x, stride, token, k, o, stream);
  else if (vecs <= 64) launch_short<T, 16, 4>(n, v, x, stride, token, k, o, stream);
  else if (vecs <= 128) launch_short<T, 32, 4>(n, v, x, stride, token, k, o, stream);
  else if (vecs <= 256 && k <= kWideShort<T>) launch_short<T, 64, 4>(n, v, x, stride, token, k, o, stream);
  else {
    Segments seg{nullptr, nullptr, nullptr, (int32_t)segments_of(n, (int64_t)v * sizeof(T)), v};
    if (seg.count > 1) {
      seg.length = cdiv(cdiv(v, seg.count), kVec<T>) * kVec<T>;
      seg.count = (int32_t)cdiv(v, seg.length);
      seg.part = static_cast<float4*>(workspace);
      seg.value = reinterpret_cast<float*>(seg.part + n * seg.count);
      seg.id = reinterpret_cast<int32_t*>(seg.value + n * seg.count * k);
    }
    const int64_t jobs = n * seg.count;
    const int64_t bytes = seg.length * (int64_t)sizeof(T);
    if (bytes <= 8192 || (bytes <= 40960 && jobs >= 2048))
      long_kernel<T, 64><<<(unsigned)least(jobs, kCus * 32), 64, 0, stream>>>(n, v, x, stride, token, k, o, seg);
    else if (jobs <= 2 * kCus && seg.length >= 16384)
      long_kernel<T, 512><<<(unsigned)jobs, 512, 0, stream>>>(n, v, x, stride, token, k, o, seg);
    else
      long_kernel<T, 256><<<(unsigned)least(jobs, kCus * 8), 256, 0, stream>>>(n, v, x, stride, token, k, o, seg);
    if (seg.count > 1)
      join_kernel<<<(unsigned)n, 64, 0, stream>>>(n, v, x, stride, sizeof(T) == 2, token, k, o, seg);
  }
  return launch_status();
}

template <typename T>
maestro_status launch_grad(int64_t n, int32_t v, const T* x, int64_t stride, const Gradient& a, T* grad,
                           int64_t grad_stride, hipStream_t stream) {
  const int64_t vecs = cdiv(v, kVec<T>);
  if (vecs <= kGradShort<T>) {
    auto kernel = a.g_entropy ? grad_short_kernel<T, true> : grad_short_kernel<T, false>;
    kernel<<<(unsigned)least(cdiv(n * vecs, 256), kCus * 64), 256, 0, stream>>>(
        n, v, x, stride, a, grad, grad_stride, (uint32_t)vecs, (uint32_t)cdiv(1 << 21, vecs));
  } else if (vecs <= kGradRow) {
    if constexpr (kGradShort<T> < kGradRow)
      grad_row_kernel<T><<<(unsigned)least(cdiv(n, 4), kCus * 64), 256, 0, stream>>>(n, v, x, stride, a, grad, grad_stride);
  } else {
    const int32_t parts = (int32_t)cdiv(vecs, 256 * kGradAhead);
    grad_long_kernel<T><<<(unsigned)least(n * parts, kCus * 64), 256, 0, stream>>>(n, v, x, stride, a, grad, grad_stride, parts);
  }
  return launch_status();
}

}  // namespace

size_t logprobs_workspace_bytes(int64_t n, int32_t v, int32_t k, int32_t dtype) {
  const int64_t count = v <= 128 * (dtype == MAESTRO_F32 ? kVec<float> : kVec<__bf16>) ? 1 : segments_of(n, (int64_t)v * (dtype == MAESTRO_F32 ? 4 : 2));
  return count > 1 ? (size_t)(n * count) * (sizeof(float4) + (sizeof(float) + sizeof(int32_t)) * k) : 0;
}

maestro_status launch_logprobs(int64_t n, int32_t v, const void* logits, int64_t row_stride, int32_t dtype,
                               const int32_t* token, int32_t k, float* logprob, float* entropy, int32_t* top_id,
                               float* top_logprob, float* stats, void* workspace, hipStream_t stream) {
  const Outputs o{logprob, entropy, top_id, top_logprob, stats};
  if (dtype == MAESTRO_F32)
    return launch(n, v, static_cast<const float*>(logits), row_stride, token, k, o, workspace, stream);
  return launch(n, v, static_cast<const __bf16*>(logits), row_stride, token, k, o, workspace, stream);
}

maestro_status launch_logprobs_grad(int64_t n, int32_t v, const void* logits, int64_t row_stride, int32_t dtype,
                                    const int32_t* token, const float* stats, const float* entropy,
                                    const float* g_logprob, const float* g_entropy, void* grad, int64_t grad_stride,
                                    hipStream_t stream) {
  const Gradient a{token, stats, entropy, g_logprob, g_entropy};
  if (dtype == MAESTRO_F32)
    return launch_grad(n, v, static_cast<const float*>(logits), row_stride, a, static_cast<float*>(grad), grad_stride, stream);
  return launch_grad(n, v, static_cast<const __bf16*>(logits), row_stride, a, static_cast<__bf16*>(grad), grad_stride, stream);
}

}  // namespace maestro
