// The bfloat16 products of a predictor's layer and its gradients on the matrix cores.
//
// All three are C[q][p] = sum_k P(p, k) Q(q, k) with C's rows contiguous in p:
//   activations      y[n][o]   P = weight (k contiguous)   Q = x   (k contiguous)   k over d_in
//   input's gradient g_x[n][i] P = weight (p contiguous)   Q = g_z (k contiguous)   k over d_out
//   weights'         g_w[o][i] P = x      (p contiguous)   Q = g_z (q contiguous)   k over the n rows
// A workgroup of four wavefronts makes a tile of TP x TQ of C, each wavefront 32 WP x 32 WQ of it in
// 32x32x16 MFMAs. k advances in stages of 32; a stage's TP + TQ rows of 64 bytes come straight into LDS
// (four buffers, three stages ahead of their use). An operand whose k is contiguous lies in LDS as
// [p][32 k]; one whose p (or q) is contiguous as [32 k][p], and is turned by the transposing LDS read
// (ds_read_b64_tr_b16: sixteen lanes read a 4 x 16 block row-wise and get it column-wise).
// P's 32 rows of a block are taken in an order (tile_row_neuron) that leaves every lane runs of 8 consecutive p.
// Workgroups are persistent: the loads of the next tile's first stages run under a tile's last
// products and its stores.
#include "mlp.h"
#include "train.h"

namespace maestro {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kThreads = 256;
constexpr int kDepth = 32;           // k of a stage
constexpr int kBufs = 4;

struct Product {
  const __bf16* p;                   // P and Q and their leading dimensions (elements)
  const __bf16* q;
  int64_t ldp, ldq;
  int64_t np, nq, nk;                // extents
  int64_t k_split;                   // k of one split, a multiple of kDepth (>= nk: one split)
  int32_t splits, p_tiles;
  int64_t items;                     // splits * tiles
};

// What becomes of C, for a run of 8 consecutive p of one q.
struct Forward {
  const float* bias;
  __bf16* y;
  int32_t relu;
};
struct InputGrad {
  const __bf16* x;
  __bf16* gx;
  int32_t relu;
};
struct WeightGrad {
  float* gw;                         // [splits][nq][np]
  float* gb;                         // [splits * parts][nq]
  int32_t parts;                     // workgroups (of one split and q) that share the sum over Q
};

template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (0 << 8));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ bf16x8 read_turned(const unsigned char* at, int step) {
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + step));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// One operand of a tile: T rows (p or q), kTurned: rows contiguous in memory instead of k.
template <int T, bool kTurned>
struct Operand {
  static constexpr int kLoads = T / 64;                     // 1 KB loads of a wavefront and stage
  uint32_t off[kLoads];                                     // per lane, within the resource
  uint32_t unit;                                            // k-contiguous: the 16-byte unit this lane loads
  const unsigned char* base;
  i32x4 rsrc;
  int64_t ld2;                                              // bytes

  // 64-byte blocks of a turned row k are stored at block ^ turn(k), so that the four rows of a
  // transposing read lie in different banks
  static __device__ __forceinline__ int turn(int k) { return T >= 128 ? k & 3 : (k >> 1) & 1; }

  __device__ __forceinline__ void tile(const __bf16* m, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int wave,
                                       int lane) {
    ld2 = ld * 2;
    if constexpr (kTurned) {
      base = reinterpret_cast<const unsigned char*>(m) + k0 * ld2;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int o = 1024 * (wave * kLoads + j) + 16 * lane, k = o / (2 * T), slot = o % (2 * T) / 16;
        off[j] = (uint32_t)(k * ld2 + row0 * 2) + ((slot ^ (4 * turn(k))) << 4);
      }
    } else {
      base = reinterpret_cast<const unsigned char*>(m) + row0 * ld2;
      const int64_t left = rows - row0;
      rsrc = buffer_rsrc(base, (uint32_t)((left < T ? left : T) * ld2));
      unit = ((lane & 3) ^ ((lane >> 4) & 3)) << 4;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) off[j] = (uint32_t)((16 * (wave * kLoads + j) + (lane >> 2)) * ld2) + unit;
    }
  }
  // stage s of k_n values of k in all, into the buffer at LDS address lds (uniform)
  __device__ __forceinline__ void fetch(int64_t s, int64_t k_n, uint32_t lds, int wave) {
    const int64_t left = k_n - s * kDepth;                  // <= 0: past the end, nothing is read
    const uint32_t at = __builtin_amdgcn_readfirstlane(lds + 1024 * kLoads * wave);
    if constexpr (kTurned) {
      const i32x4 r = buffer_rsrc(base + (left > 0 ? s * kDepth * ld2 : 0),
                                  left > 0 ? (uint32_t)((left < kDepth ? left : kDepth) * ld2) : 0);
#pragma unroll
      for (int j = 0; j < kLoads; ++j) dma16(r, off[j], 0, at, 1024 * j);
    } else {
      const bool in = (int64_t)unit < left * 2;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) dma16(rsrc, in ? off[j] + (uint32_t)(s * 64) : 0x80000000u, 0, at, 1024 * j);
    }
  }
};

// LDS offsets of a lane's fragments in an operand's stage: block b (of 32 rows) of the wavefront's, k half kk.
template <int T, bool kTurned, int W, bool kPermuted>
struct Fragments {
  int at[kTurned ? W : 1];
  __device__ __forceinline__ void init(int block0, int lane) {
    const int r = lane & 31, h = lane >> 5;
    if constexpr (kTurned) {
      const int s = lane & 15, g = (lane >> 4) & 1;
      const int quad = 4 * g + (s & 3);
      const int c = kPermuted ? 4 * (quad >> 2) + 2 * (quad & 1) + ((quad >> 1) & 1) : quad;
      const int k = 8 * h + (s >> 2);
#pragma unroll
      for (int b = 0; b < W; ++b)
        at[b] = k * 2 * T + 64 * ((block0 + b) ^ Operand<T, true>::turn(k)) + 8 * c;
    } else {
      const int row = 32 * block0 + (kPermuted ? tile_row_neuron(r) : r);
      at[0] = row * 64 + ((h ^ ((row >> 2) & 3)) << 4);
    }
  }
  __device__ __forceinline__ void read(const unsigned char* stage, int kk, bf16x8 (&f)[W]) const {
#pragma unroll
    for (int b = 0; b < W; ++b) {
      if constexpr (kTurned) f[b] = read_turned(stage + at[b] + kk * 16 * 2 * T, 4 * 2 * T);
      else f[b] = *reinterpret_cast<const bf16x8*>(stage + (at[0] ^ (kk * 32)) + b * 32 * 64);
    }
  }
};

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

__device__ __forceinline__ void store8(__bf16* at, const float (&c)[8]) {
  *reinterpret_cast<uint4*>(at) = make_uint4(pack2(c[0], c[1]), pack2(c[2], c[3]), pack2(c[4], c[5]), pack2(c[6], c[7]));
}

// what a run of 8 consecutive p needs for every q: the biases
__device__ __forceinline__ void begin(const Forward& e, int64_t p, float (&b)[8]) {
  const float4 b0 = *reinterpret_cast<const float4*>(e.bias + p), b1 = *reinterpret_cast<const float4*>(e.bias + p + 4);
  b[0] = b0.x, b[1] = b0.y, b[2] = b0.z, b[3] = b0.w, b[4] = b1.x, b[5] = b1.y, b[6] = b1.z, b[7] = b1.w;
}
template <class Out>
__device__ __forceinline__ void begin(const Out&, int64_t, float (&)[8]) {}

__device__ __forceinline__ void finish(const Forward& e, const Product& g, int64_t q, int64_t p, int64_t,
                                       const float (&b)[8], float (&c)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    c[i] += b[i];
    c[i] = e.relu && c[i] < 0.0f ? 0.0f : c[i];
  }
  store8(e.y + q * g.np + p, c);
}

__device__ __forceinline__ void finish(const InputGrad& e, const Product& g, int64_t q, int64_t p, int64_t,
                                       const float (&)[8], float (&c)[8]) {
  if (e.relu) {
    const bf16x8 x = *reinterpret_cast<const bf16x8*>(e.x + q * g.np + p);
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = (float)x[i] > 0.0f ? c[i] : 0.0f;
  }
  store8(e.gx + q * g.np + p, c);
}

__device__ __forceinline__ void finish(const WeightGrad& e, const Product& g, int64_t q, int64_t p, int64_t split,
                                       const float (&)[8], float (&c)[8]) {
  float* at = e.gw + (split * g.nq + q) * g.np + p;
  *reinterpret_cast<float4*>(at) = make_float4(c[0], c[1], c[2], c[3]);
  *reinterpret_cast<float4*>(at + 4) = make_float4(c[4], c[5], c[6], c[7]);
}

template <int WP, int WQ, int NP, int NQ, bool kPT, bool kQT, class Out>
__global__ __launch_bounds__(kThreads, WP * WQ > 8 ? 1 : WP * WQ > 2 ? 2 : 4) void product_kernel(Product g, Out out) {
  static_assert(NP * NQ == 4, "four wavefronts");
  constexpr int TP = 32 * WP * NP, TQ = 32 * WQ * NQ;
  constexpr int kStage = (TP + TQ) * 64, kLoads = TP / 64 + TQ / 64;
  constexpr bool kSums = kQT;                               // the weights' gradient sums Q too (the biases')
  extern __shared__ unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wp = wave % NP, wq = wave / NP;

  // XCD x (of 8; workgroups go round them) takes a contiguous share of the items, so that the tiles that read
  // the same rows of Q run side by side on one L2
  const int64_t share = (g.items + 7) / 8, xcd = blockIdx.x & 7, step = gridDim.x >> 3;
  const int64_t last = (xcd + 1) * share < g.items ? (xcd + 1) * share : g.items;
  const int64_t first = xcd * share + (blockIdx.x >> 3);
  if (first >= last) return;

  struct Item {
    int64_t q0, p0, k0, kn, split, stages;
  };
  const int64_t per_split = g.items / g.splits;
  auto item = [&](int64_t i) {
    Item t;
    t.split = i / per_split;
    const int64_t tile = i % per_split;
    t.q0 = tile / g.p_tiles * TQ;
    t.p0 = tile % g.p_tiles * TP;
    t.k0 = t.split * g.k_split;
    t.kn = g.nk - t.k0 < g.k_split ? g.nk - t.k0 : g.k_split;
    t.stages = (t.kn + kDepth - 1) / kDepth;
    return t;
  };

  Operand<TP, kPT> op;
  Operand<TQ, kQT> oq;
  int64_t fetch_item = first, fetch_stage = 0, fetch_kn = 0, fetch_stages = 0;
  auto open = [&]() {
    if (fetch_item >= last) {                               // no more tiles: loads that read nothing
      fetch_kn = 0;
      fetch_stages = INT64_MAX;
      return;
    }
    const Item t = item(fetch_item);
    op.tile(g.p, g.ldp, t.p0, g.np, t.k0, wave, lane);
    oq.tile(g.q, g.ldq, t.q0, g.nq, t.k0, wave, lane);
    fetch_kn = t.kn;
    fetch_stages = t.stages;
  };
  const uint32_t lds0 = lds_addr(lds);
  auto fetch = [&](int buf) {
    op.fetch(fetch_stage, fetch_kn, lds0 + buf * kStage, wave);
    oq.fetch(fetch_stage, fetch_kn, lds0 + buf * kStage + TP * 64, wave);
    if (++fetch_stage == fetch_stages) {
      fetch_stage = 0;
      fetch_item += step;
      open();
    }
  };

  Fragments<TP, kPT, WP, true> fp;
  Fragments<TQ, kQT, WQ, false> fq;
  fp.init(wp * WP, lane);
  fq.init(wq * WQ, lane);

  open();
#pragma unroll
  for (int b = 0; b < kBufs; ++b) fetch(b);
  wait_loads<kLoads * (kBufs - 1)>();

  bf16x8 p0[WP], q0[WQ], p1[WP], q1[WQ];
  fp.read(lds, 0, p0);
  fq.read(lds + TP * 64, 0, q0);
  int buf = 0;
  for (int64_t i = first; i < last; i += step) {
    const Item t = item(i);
    f32x16 acc[WP][WQ] = {};
    float sums[kSums ? WQ : 1] = {};
    int64_t mine = 0;                                       // the next stage whose Q this workgroup sums
    int64_t parts = 1;
    if constexpr (kSums) {
      parts = out.parts;
      mine = t.p0 / TP;
    }
    for (int64_t s = 0; s < t.stages; ++s) {
      const unsigned char* stage = lds + buf * kStage;
      fp.read(stage, 1, p1);
      fq.read(stage + TP * 64, 1, q1);
#pragma unroll
      for (int a = 0; a < WP; ++a)
#pragma unroll
        for (int b = 0; b < WQ; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(p0[a], q0[b], acc[a][b], 0, 0, 0);
      if constexpr (kSums) {
        if (s == mine) {                                    // wavefronts of the same Q rows take a half each
          mine += parts;
#pragma unroll
          for (int b = 0; b < WQ; ++b) {
            if (NP == 1 || wp == 0)
#pragma unroll
              for (int e = 0; e < 8; ++e) sums[b] += (float)q0[b][e];
            if (NP == 1 || wp == 1)
#pragma unroll
              for (int e = 0; e < 8; ++e) sums[b] += (float)q1[b][e];
          }
        }
      }
      wait_loads<kLoads * (kBufs - 2)>();                   // the next stage is there, this one read by all
      fetch(buf);
      buf = (buf + 1) & (kBufs - 1);
      fp.read(lds + buf * kStage, 0, p0);
      fq.read(lds + buf * kStage + TP * 64, 0, q0);
#pragma unroll
      for (int a = 0; a < WP; ++a)
#pragma unroll
        for (int b = 0; b < WQ; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(p1[a], q1[b], acc[a][b], 0, 0, 0);
    }
    const int r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int a = 0; a < WP; ++a) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        asm volatile("" ::: "memory");                      // one run's loads at a time: registers
        const int64_t p = t.p0 + 32 * (wp * WP + a) + 16 * half + 8 * h;
        if (p < g.np) {
          float bias[8];
          begin(out, p, bias);
#pragma unroll
          for (int b = 0; b < WQ; ++b) {
            const int64_t q = t.q0 + 32 * (wq * WQ + b) + r;
            if (q < g.nq) {
              float c[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) c[e] = acc[a][b][8 * half + e];
              finish(out, g, q, p, t.split, bias, c);
            }
          }
        }
      }
    }
    if constexpr (kSums) {
      // NP wavefronts and `parts` workgroups hold shares of the sum over Q
      const int64_t part = t.p0 / TP;
#pragma unroll
      for (int b = 0; b < WQ; ++b) {
        const int64_t q = t.q0 + 32 * (wq * WQ + b) + r;
        const float s = sums[b] + __shfl_xor(sums[b], 32);
        if (h == 0 && q < g.nq) out.gb[((t.split * out.parts + part) * NP + wp) * g.nq + q] = s;
      }
    }
  }
  wait_loads<0>();                                          // no load into LDS outlives the workgroup
}

// g_w and g_b from their shares, summed in order
__global__ __launch_bounds__(kThreads) void join_kernel(const float* gw_parts, int32_t n_gw, float* gw, int64_t size,
                                                        const float* gb_parts, int32_t n_gb, float* gb, int32_t d_out) {
  const int64_t quads = n_gw != 1 ? size / 4 : 0, all = quads + d_out;      // one share is g_w itself
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < all; i += (int64_t)gridDim.x * kThreads) {
    if (i < quads) {
      float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      for (int32_t j = 0; j < n_gw; ++j) {
        const float4 a = reinterpret_cast<const float4*>(gw_parts + j * size)[i];
        s.x += a.x, s.y += a.y, s.z += a.z, s.w += a.w;
      }
      reinterpret_cast<float4*>(gw)[i] = s;
    } else {
      const int64_t c = i - quads;
      float s = 0.0f;
      for (int32_t j = 0; j < n_gb; ++j) s += gb_parts[(int64_t)j * d_out + c];
      gb[c] = s;
    }
  }
}

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t kCus = 256;

template <int WP, int WQ, int NP, int NQ, bool kPT, bool kQT, class Out>
maestro_status launch(Product g, const Out& out, hipStream_t stream) {
  constexpr int TP = 32 * WP * NP, TQ = 32 * WQ * NQ;
  constexpr int kLds = kBufs * (TP + TQ) * 64;
  constexpr int64_t kResident = kLds > 81920 ? 1 : kLds > 40960 ? 2 : 4;     // workgroups of a CU
  g.p_tiles = (int32_t)cdiv(g.np, TP);
  g.splits = (int32_t)cdiv(g.nk, g.k_split);
  g.items = cdiv(g.nq, TQ) * g.p_tiles * g.splits;
  const auto kernel = product_kernel<WP, WQ, NP, NQ, kPT, kQT, Out>;
  if (kLds > 65536 &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds) != hipSuccess)
    return MAESTRO_ERR_LAUNCH;
  const int64_t want = cdiv(g.items, 8) * 8, most = kCus * kResident;
  kernel<<<(unsigned)(want < most ? want : most), kThreads, kLds, stream>>>(g, out);
  return launch_status();
}

// Tiles of 256 x 256 keep the matrix cores fed best; smaller ones where 256 x 256 would leave CUs idle or most
// of a tile outside the product.
int tile_of(int64_t np, int64_t nq) {
  for (int t = 256; t > 64; t /= 2)
    if (np > t / 2 && nq > t / 2 && cdiv(np, t) * cdiv(nq, t) >= kCus) return t;
  return 64;
}

template <bool kPT, bool kQT, class Out>
maestro_status dispatch(int tile, const Product& g, const Out& out, hipStream_t stream) {
  if (tile == 256) return launch<4, 4, 2, 2, kPT, kQT>(g, out, stream);
  if (tile == 128) return launch<2, 2, 2, 2, kPT, kQT>(g, out, stream);
  return launch<1, 1, 2, 2, kPT, kQT>(g, out, stream);
}

// How the weights' gradient is cut: tile, splits of the n rows, and workgroups that share the biases' sum.
struct Cut {
  int tile;
  int64_t k_split, splits;
  int32_t parts;
};

Cut cut_of(int64_t n, int64_t d_in, int64_t d_out) {
  Cut c;
  c.tile = d_in > 128 && d_out > 128 && n >= 32768 ? 256 : d_in > 64 && d_out > 64 && n >= 8192 ? 128 : 64;
  const int64_t tiles = cdiv(d_in, c.tile) * cdiv(d_out, c.tile);
  const int64_t resident = c.tile == 256 ? 1 : c.tile == 128 ? 2 : 4;
  // one round of workgroups, none with fewer than 512 rows
  int64_t splits = kCus * resident / tiles;
  if (splits > cdiv(n, 512)) splits = cdiv(n, 512);
  if (splits < 1) splits = 1;
  c.k_split = cdiv(cdiv(n, splits), kDepth) * kDepth;
  c.splits = cdiv(n, c.k_split);
  c.parts = (int32_t)cdiv(d_in, c.tile);
  return c;
}

}  // namespace

maestro_status launch_layer_bf16(int64_t n, int32_t d_in, int32_t d_out, const void* x, const void* weight,
                                 const float* bias, bool relu, void* y, hipStream_t stream) {
  Product g{static_cast<const __bf16*>(weight), static_cast<const __bf16*>(x), d_in, d_in, d_out, n, d_in, d_in, 1, 0, 0};
  return dispatch<false, false>(tile_of(d_out, n), g, Forward{bias, static_cast<__bf16*>(y), relu}, stream);
}

size_t layer_grad_bf16_workspace_bytes(int64_t n, int32_t d_in, int32_t d_out) {
  if (n == 0) return 0;
  const Cut c = cut_of(n, d_in, d_out);
  return sizeof(float) * (size_t)((c.splits > 1 ? c.splits * d_in * d_out : 0) + c.splits * c.parts * 2 * d_out);
}

maestro_status launch_layer_grad_bf16(int64_t n, int32_t d_in, int32_t d_out, const void* x, const void* weight,
                                      const void* g_z, bool relu_input, void* g_x, float* g_weight, float* g_bias,
                                      void* workspace, hipStream_t stream) {
  const __bf16 *xb = static_cast<const __bf16*>(x), *gz = static_cast<const __bf16*>(g_z);
  if (n == 0) {
    join_kernel<<<(unsigned)cdiv((int64_t)d_in * d_out / 4 + d_out, kThreads), kThreads, 0, stream>>>(
        nullptr, 0, g_weight, (int64_t)d_in * d_out, nullptr, 0, g_bias, d_out);
    return launch_status();
  }
  if (g_x) {
    Product g{static_cast<const __bf16*>(weight), gz, d_in, d_out, d_in, n, d_out, d_out, 1, 0, 0};
    const maestro_status st =
        dispatch<true, false>(tile_of(d_in, n), g, InputGrad{xb, static_cast<__bf16*>(g_x), relu_input}, stream);
    if (st != MAESTRO_OK) return st;
  }
  const Cut c = cut_of(n, d_in, d_out);
  float* parts = static_cast<float*>(workspace);
  float* gb_parts = parts + (c.splits > 1 ? c.splits * d_in * d_out : 0);
  Product g{xb, gz, d_in, d_out, d_in, d_out, n, c.k_split, 1, 0, 0};
  const maestro_status st =
      dispatch<true, true>(c.tile, g, WeightGrad{c.splits > 1 ? parts : g_weight, gb_parts, c.parts}, stream);
  if (st != MAESTRO_OK) return st;
  const int64_t work = (c.splits > 1 ? (int64_t)d_in * d_out / 4 : 0) + d_out, blocks = cdiv(work, kThreads);
  join_kernel<<<(unsigned)(blocks < 4096 ? blocks : 4096), kThreads, 0, stream>>>(
      parts, (int32_t)c.splits, g_weight, (int64_t)d_in * d_out, gb_parts, (int32_t)(c.splits * c.parts * 2), g_bias, d_out);
  return launch_status();
}

}  // namespace maestro
