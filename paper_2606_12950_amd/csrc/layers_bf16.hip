// The bfloat16 products of a predictor's layer and its gradients on the matrix cores.
//
// All three are C[q][p] = sum_k P(p, k) Q(q, k) with C's rows contiguous in p:
//   activations      y[n][o]   P = weight (k contiguous)   Q = x   (k contiguous)   k over d_in
//   input's gradient g_x[n][i] P = weight (p contiguous)   Q = g_z (k contiguous)   k over d_out
//   weights'         g_w[o][i] P = x      (p contiguous)   Q = g_z (q contiguous)   k over the n rows
// A workgroup of four wavefronts makes a tile of TP x TQ of C, each wavefront 32 WP x 32 WQ of it in
// 32x32x16 MFMAs. k advances in stages of kDepth (32 or 64) that come straight into LDS, kBufs buffers round. An
// operand whose k is contiguous lies in LDS as [p][k]; one whose p (or q) is contiguous as [k][p], and
// is turned by the transposing LDS read (ds_read_b64_tr_b16: sixteen lanes read a 4 x 16 block row-wise
// and get it column-wise). P's 32 rows of a block are taken in an order (tile_row_neuron) that leaves every lane runs
// of 8 consecutive p. Workgroups are persistent: the loads of the next tile's first stages run under a
// tile's last products and its stores, and its stores under the next tile's products.
//
// Bound by the matrix cores on wide layers, by HBM on narrow ones. Measured: 262,139 x 1024 -> 1024
// (0.55 TFLOP a product) activations 523 us in the first launches, 550 in a long run and up to 680 in between, while the
// clock settles to the matrix cores' power; input's gradient 535 and 560, weights' 447 and 475, 20 more to join its shares
// (as calls, over changing inputs: 533, and 1,047 for both gradients). A 16,384-cubed library product reaches 1.31 to 1.35
// PFLOP/s on the same card, and the library's products of these shapes 555, 618 and 1,230 us. 512 -> 256: activations 96 us for
// 403 MB, input's gradient 131 to 140 us for 671 MB = 4.8 to 5.1 TB/s, what a copy reaches.
#include <type_traits>

#include "mlp.h"
#include "train.h"

namespace maestro {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kThreads = 256;

struct Product {
  const __bf16* p;                   // P and Q and their leading dimensions (elements)
  const __bf16* q;
  int64_t ldp, ldq;
  int64_t np, nq, nk;                // extents
  int64_t k_split;                   // k of one split, a multiple of kDepth (>= nk: one split)
  int32_t splits, p_tiles;
  int64_t items;                     // splits * tiles
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Rows of a bfloat16 matrix seen through a buffer resource: accesses past its end read zeros and write nothing.
struct Rows {
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ __forceinline__ void init(const void* m, int64_t row0, int64_t rows, int64_t most, int64_t row_bytes) {
    const int64_t left = rows - row0 < most ? rows - row0 : most;
    rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(static_cast<const unsigned char*>(m)) +
                                                 (left > 0 ? row0 * row_bytes : 0),
                                             0, (uint32_t)(left > 0 ? left * row_bytes : 0), 0x00020000);
  }
  __device__ __forceinline__ u32x4 load(uint32_t off) const {
    return __builtin_amdgcn_raw_buffer_load_b128(rsrc, off, 0, 0);
  }
  __device__ __forceinline__ void store(const u32x4& v, uint32_t off) const {
    __builtin_amdgcn_raw_buffer_store_b128(v, rsrc, off, 0, 0);
  }
};

// What becomes of C. kMasked: C is 0 wherever `x`, of C's shape, is not positive. kBias: `bias` [p] is added and,
// with relu, negative values become 0.
struct Forward {
  static constexpr bool kMasked = false, kBias = true;
  const float* bias;
  __bf16* c;
  int32_t relu;
};
struct InputGrad {
  static constexpr bool kMasked = true, kBias = false;
  const __bf16* x;
  __bf16* c;
  int32_t relu;
};
struct WeightGrad {
  static constexpr bool kBias = false;
  float* gw;                         // [splits][nq][np]
  float* gb;                         // one split: [nq], whole; else [splits][parts][two wavefronts][nq]
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

// Of this wavefront alone: at most N of its vector memory operations outstanding.
template <int N>
__device__ __forceinline__ void wait_own() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
  asm volatile("" ::: "memory");
}

// One operand of a tile: T rows (p or q), kTurned: rows contiguous in memory instead of k.
template <int T, int kDepth, bool kTurned>
struct Operand {
  static constexpr int kLoads = T * kDepth / 2048;          // 1 KB loads of a wavefront and stage
  static constexpr int kUnits = kDepth / 8;                 // k contiguous: 16-byte units of a row
  static constexpr int kRows = 64 / kUnits;                 // k contiguous: rows of a load
  uint32_t off[kLoads];                                     // per lane, within the resource
  uint32_t unit;                                            // k contiguous: the byte of the row this lane loads next
  uint32_t row_bytes;                                       // k contiguous: bytes of k; turned: bytes of a row of k
  const unsigned char* base;                                // turned: the next stage's first row
  int64_t left;                                             // turned: rows of k from there on
  uint32_t bytes;                                           // k contiguous: of the resource
  i32x4 rsrc;                                               // of the stage being fetched, and its place
  uint32_t to;

  // 64-byte blocks of a turned row k are stored at block ^ turn(k), so that the four rows of a
  // transposing read lie in different banks
  static __device__ __forceinline__ int turn(int k) { return T >= 128 ? k & 3 : (k >> 1) & 1; }
  // unit u of a row whose k is contiguous is stored at u ^ place(row): sixteen rows' reads of one unit meet all banks
  static __device__ __forceinline__ int place(int row) { return (row / (16 / kUnits)) & (kUnits - 1); }

  // place() goes round in 16 rows: where a load has 8, the odd ones take the other half of its values
  static __device__ __forceinline__ uint32_t odd(int j) {
    static_assert(kRows == 16 || (kRows == 8 && kLoads % 2 == 0), "place()'s period");
    return kRows == 8 && j % 2 ? 64 : 0;
  }

  __device__ __forceinline__ void tile(const __bf16* m, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int64_t kn,
                                       int wave, int lane) {
    const int64_t ld2 = ld * 2;
    if constexpr (kTurned) {
      base = reinterpret_cast<const unsigned char*>(m) + k0 * ld2;
      left = kn;
      row_bytes = (uint32_t)ld2;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int o = 1024 * (wave * kLoads + j) + 16 * lane, k = o / (2 * T), slot = o % (2 * T) / 16;
        off[j] = (uint32_t)(k * ld2 + row0 * 2) + ((slot ^ (4 * turn(k))) << 4);
      }
    } else {
      base = reinterpret_cast<const unsigned char*>(m) + row0 * ld2;
      bytes = (uint32_t)((rows - row0 < T ? rows - row0 : T) * ld2);
      row_bytes = (uint32_t)(kn * 2);
      unit = ((lane % kUnits) ^ place(lane / kUnits)) << 4;
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        off[j] = (uint32_t)((kRows * (wave * kLoads + j) + lane / kUnits) * ld2) + (unit ^ odd(j));
    }
  }
  // no tile: the loads read nothing
  __device__ __forceinline__ void none() {
    left = 0;
    bytes = 0;
  }
  // The next stage, into the buffer at LDS address lds (uniform): aim, every load, advance.
  __device__ __forceinline__ void aim(uint32_t lds, int wave) {
    to = __builtin_amdgcn_readfirstlane(lds + 1024 * kLoads * wave);
    rsrc = buffer_rsrc(base, kTurned ? (uint32_t)(left < kDepth ? left < 0 ? 0 : left : kDepth) * row_bytes : bytes);
  }
  __device__ __forceinline__ void fetch(int j) const {
    if constexpr (kTurned) dma16(rsrc, off[j], 0, to, 1024 * j);
    else dma16(rsrc, (unit ^ odd(j)) < row_bytes ? off[j] : 0x80000000u, 0, to, 1024 * j);
  }
  __device__ __forceinline__ void advance() {
    if constexpr (kTurned) {
      base += kDepth * row_bytes;
      left -= kDepth;
    } else {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) off[j] += 2 * kDepth;
      unit += 2 * kDepth;
    }
  }
  __device__ __forceinline__ void fetch_all(uint32_t lds, int wave) {
    aim(lds, wave);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) fetch(j);
    advance();
  }
};

// LDS offsets of a lane's fragments in an operand's stage: block b (of 32 rows) of the wavefront's, k half kk.
template <int T, int kDepth, bool kTurned, int W, bool kPermuted>
struct Fragments {
  using Op = Operand<T, kDepth, kTurned>;
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
        at[b] = k * 2 * T + 64 * ((block0 + b) ^ Op::turn(k)) + 8 * c;
    } else {
      const int row = 32 * block0 + (kPermuted ? tile_row_neuron(r) : r);
      at[0] = row * 2 * kDepth + ((h ^ Op::place(row)) << 4);
    }
  }
  __device__ __forceinline__ bf16x8 read(const unsigned char* stage, int kk, int b) const {
    if constexpr (kTurned) return read_turned(stage + at[b] + kk * 16 * 2 * T, 4 * 2 * T);
    else return *reinterpret_cast<const bf16x8*>(stage + (at[0] ^ (kk * 32)) + b * 32 * 2 * kDepth);
  }
};

__device__ __forceinline__ float add8(const u32x4& v) {
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) s += __uint_as_float(v[e] << 16) + __uint_as_float(v[e] & 0xFFFF0000u);
  return s;
}

template <class Out>
__device__ __forceinline__ int32_t parts_of(const Out& out) {
  if constexpr (std::is_same<Out, WeightGrad>::value) return out.parts;
  else return 1;
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

// eight consecutive values rounded
__device__ __forceinline__ u32x4 pack8(const float (&v)[8]) {
  return u32x4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
}

// the bfloat16 pair c where the pair x is positive
__device__ __forceinline__ uint32_t where_positive(uint32_t c, uint32_t x) {
  const float lo = __uint_as_float(x << 16), hi = __uint_as_float(x & 0xFFFF0000u);
  return c & ((lo > 0.0f ? 0xFFFFu : 0u) | (hi > 0.0f ? 0xFFFF0000u : 0u));
}

// max(., 0) of a bfloat16 pair; a NaN stays one
__device__ __forceinline__ uint32_t rectify(uint32_t c) {
  const float lo = __uint_as_float(c << 16), hi = __uint_as_float(c & 0xFFFF0000u);
  return c & ((lo < 0.0f ? 0u : 0xFFFFu) | (hi < 0.0f ? 0u : 0xFFFF0000u));
}

// A wavefront's 32 WP x 32 WQ part of C in bfloat16, by way of LDS, so that memory sees whole lines: a lane holds
// runs of 8 p (16 bytes) of one q and leaves them at their place in [32 q][32 WS p]; then 4 WS lanes take a
// row together. Units of 16 bytes are stored at unit ^ place(q): neither access meets bank conflicts. Every
// wavefront issues 2 WP WQ stores, whatever lies outside C: the main loop's waits count them.
template <int WP>
struct Staging {
  static constexpr int WS = WP < 4 ? 1 : 2;                 // blocks of 32 p at a time
  static constexpr int kRowBytes = 64 * WS, kUnits = 4 * WS, kRows = 64 / kUnits;
  static constexpr int kBytes = 32 * kRowBytes;             // of a wavefront
  static __device__ __forceinline__ int place(int q) { return (q / (16 / kUnits)) & (kUnits - 1); }
};

template <int WP, int WQ, class Out>
__device__ __forceinline__ void store_rows(const Out& out, const Product& g, unsigned char* staging, int64_t q0, int64_t p0,
                                           int lane, const f32x16 (&acc)[WP][WQ]) {
  using S = Staging<WP>;
  constexpr int kStores = 32 / S::kRows;                    // of one q block and WS p blocks
  const int r = lane & 31, h = lane >> 5;
  const int row0 = lane / S::kUnits, unit0 = lane % S::kUnits;
  const uint32_t ld = (uint32_t)g.np * 2, step = S::kRows * ld;
  Rows c, x;
  c.init(out.c, q0, g.nq, 32 * WQ, ld);
  uint32_t at[WP / S::WS];                                  // of the first row's unit, outside C: past the resource
#pragma unroll
  for (int w = 0; w < WP / S::WS; ++w) {
    const int64_t p = p0 + 32 * S::WS * w + 8 * unit0;
    at[w] = p < g.np ? (uint32_t)(row0 * ld + p * 2) : 0x80000000u;
  }
  u32x4 xv[WP / S::WS][kStores];
  const bool relu = out.relu;
  if constexpr (Out::kMasked) {
    x.init(out.x, q0, g.nq, 32 * WQ, relu ? ld : 0);
#pragma unroll
    for (int w = 0; w < WP / S::WS; ++w)
#pragma unroll
      for (int j = 0; j < kStores; ++j) xv[w][j] = x.load(at[w] + j * step);
  }
#pragma unroll
  for (int b = 0; b < WQ; ++b) {
#pragma unroll
    for (int w = 0; w < WP / S::WS; ++w) {
#pragma unroll
      for (int a = 0; a < S::WS; ++a)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = acc[w * S::WS + a][b][8 * half + e];
          *reinterpret_cast<u32x4*>(staging + r * S::kRowBytes + (((4 * a + 2 * half + h) ^ S::place(r)) << 4)) = pack8(v);
        }
      u32x4 v[kStores];
#pragma unroll
      for (int j = 0; j < kStores; ++j) {
        const int row = j * S::kRows + row0;
        v[j] = *reinterpret_cast<const u32x4*>(staging + row * S::kRowBytes + ((unit0 ^ S::place(row)) << 4));
      }
      if constexpr (!Out::kMasked) {
        if (relu)
#pragma unroll
          for (int j = 0; j < kStores; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[j][e] = rectify(v[j][e]);
      } else {
#pragma unroll
        for (int j = 0; j < kStores; ++j) {
          if (relu)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[j][e] = where_positive(v[j][e], xv[w][j][e]);
          if (b + 1 < WQ) xv[w][j] = x.load(at[w] + ((b + 1) * kStores + j) * step);
        }
      }
#pragma unroll
      for (int j = 0; j < kStores; ++j) c.store(v[j], at[w] + (b * kStores + j) * step);
      asm volatile("" ::: "memory");                        // one block's values at a time: registers
    }
  }
}

// Sizes of a product's tile, and its LDS.
template <int WP, int WQ, int kDepth, int kBufs, class Out>
struct Tile {
  static constexpr int TP = 64 * WP, TQ = 64 * WQ;          // four wavefronts
  static constexpr int kStage = (TP + TQ) * 2 * kDepth;
  static constexpr bool kStores = !std::is_same<Out, WeightGrad>::value;      // by way of LDS
  static constexpr int kBiasLoads = Out::kBias ? (WP + 1) / 2 : 0;
  static constexpr int kBiasBytes = 2 * 4 * 256 * kBiasLoads;                 // two places for each wavefront
  static constexpr int kBytes = kBufs * kStage + (kStores ? 4 * Staging<WP>::kBytes : 0) + kBiasBytes;
  // workgroups of a CU that a launch plans for, and that registers allow. LDS lets three run of the activations' 64 x 64
  // (43,008 bytes of 160 KB) and two of pair_kernel<4, 1> (81,920, the larger tile's, in all of them).
  static constexpr int kResident = WP * WQ > 8 ? 1 : WP * WQ > 2 ? 2 : 4;
};

// The share of workgroup `block` of `blocks` (a multiple of 8) in a product.
template <int WP, int WQ, int kDepth, int kBufs, bool kPT, bool kQT, class Out>
__device__ __forceinline__ void product(const Product& g, const Out& out, unsigned char* lds, uint32_t block, uint32_t blocks) {
  using L = Tile<WP, WQ, kDepth, kBufs, Out>;
  constexpr int NP = 2, TP = L::TP, TQ = L::TQ;
  constexpr int kStage = L::kStage, kLoads = (TP + TQ) * kDepth / 2048, kHalves = kDepth / 16;
  constexpr int kQ = TP * 2 * kDepth;                       // Q's place in a stage
  constexpr bool kSums = kQT;                               // the weights' gradient sums Q too (the biases')
  constexpr int kBiasLoads = L::kBiasLoads;
  constexpr int kStores = kSums ? 0 : 2 * WP * WQ + kBiasLoads;      // between two tiles, exactly
  static_assert(kSums != L::kStores && kLoads * (kBufs - 2) + kStores < 64, "vmcnt range");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wp = wave % NP, wq = wave / NP;

  // XCD x (of 8; workgroups go round them) takes a contiguous share of the items, so that the tiles that read
  // the same rows of Q run side by side on one L2
  const int64_t share = (g.items + 7) / 8, xcd = block & 7, step = blocks >> 3;
  const int64_t last = (xcd + 1) * share < g.items ? (xcd + 1) * share : g.items;
  const int64_t first = xcd * share + (block >> 3);
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

  Operand<TP, kDepth, kPT> op;
  Operand<TQ, kDepth, kQT> oq;
  int64_t fetch_item = first, fetch_left = 0;               // the tile being loaded, and its stages still to load
  auto open = [&]() {
    if (fetch_item >= last) {
      op.none();
      oq.none();
      fetch_left = INT64_MAX;
      return;
    }
    const Item t = item(fetch_item);
    op.tile(g.p, g.ldp, t.p0, g.np, t.k0, t.kn, wave, lane);
    oq.tile(g.q, g.ldq, t.q0, g.nq, t.k0, t.kn, wave, lane);
    fetch_left = t.stages;
  };
  const uint32_t lds0 = lds_addr(lds);
  auto fetched = [&]() {
    if (--fetch_left == 0) {
      fetch_item += step;
      open();
    }
  };

  Fragments<TP, kDepth, kPT, WP, true> fp;
  Fragments<TQ, kDepth, kQT, WQ, false> fq;
  fp.init(wp * WP, lane);
  fq.init(wq * WQ, lane);

  // this wavefront's biases of item j, into LDS a tile ahead of their use; two places in turn
  float* biases = reinterpret_cast<float*>(lds + kBufs * kStage + 4 * Staging<WP>::kBytes) + wave * 128 * kBiasLoads;
  int parity = 0;
  auto fetch_biases = [&](int64_t j) {
    if constexpr (Out::kBias) {
      const int64_t pw = item(j).p0 + 32 * WP * wp;
      const i32x4 r = buffer_rsrc(out.bias, j < last ? (uint32_t)(g.np * 4) : 0);
#pragma unroll
      for (int l = 0; l < kBiasLoads; ++l)
        dma4(r, (uint32_t)(pw + 64 * l + lane) * 4,
             __builtin_amdgcn_readfirstlane(lds_addr(biases + (parity ? 64 * kBiasLoads : 0)) + 256 * l));
    }
  };
  fetch_biases(first);

  open();
#pragma unroll
  for (int b = 0; b < kBufs; ++b) {
    op.fetch_all(lds0 + b * kStage, wave);
    oq.fetch_all(lds0 + b * kStage + kQ, wave);
    fetched();
  }
  wait_loads<kLoads * (kBufs - 1)>();

  bf16x8 pf[2][WP], qf[2][WQ];                              // this step's fragments and the next one's
#pragma unroll
  for (int a = 0; a < WP; ++a) pf[0][a] = fp.read(lds, 0, a);
#pragma unroll
  for (int b = 0; b < WQ; ++b) qf[0][b] = fq.read(lds + kQ, 0, b);
  int buf = 0;
#pragma clang loop unroll(disable)
  for (int64_t i = first; i < last; i += step) {
    const Item t = item(i);
    f32x16 acc[WP][WQ];
    if constexpr (Out::kBias) {                             // the sums begin with the biases
      const float* bias = biases + (parity ? 64 * kBiasLoads : 0) + 8 * (lane >> 5);
      parity ^= 1;
#pragma unroll
      for (int a = 0; a < WP; ++a)
#pragma unroll
        for (int b = 0; b < WQ; ++b)
#pragma unroll
          for (int v = 0; v < 16; v += 4) {
            const float4 f = *reinterpret_cast<const float4*>(bias + 32 * a + 2 * (v & 8) + (v & 4));
            acc[a][b][v] = f.x, acc[a][b][v + 1] = f.y, acc[a][b][v + 2] = f.z, acc[a][b][v + 3] = f.w;
          }
      fetch_biases(i + step);
    } else {
#pragma unroll
      for (int a = 0; a < WP; ++a)
#pragma unroll
        for (int b = 0; b < WQ; ++b)
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.0f;
    }
    float sums[kSums ? WQ : 1] = {};
    // the sum over Q's k (the biases' gradient): a stage's by one of the workgroups with these rows of Q,
    // half of k by each of the wavefronts
    const int64_t turns = parts_of(out);
    int64_t mine = kSums && t.p0 / TP < turns ? t.p0 / TP : INT64_MAX;
#pragma clang loop unroll(disable)                            // nor peel: copies of 256 accumulators
    for (int64_t s = 0; s < t.stages; ++s) {
      const unsigned char* stage = lds + buf * kStage;
      uint32_t into = 0;
#pragma unroll
      for (int kk = 0; kk < kHalves; ++kk) {
        // One step of 16 k. A wavefront has its SIMD's matrix core to itself (256 x 256), and whatever does not fit
        // between one product's issue and the next is a gap: so the next step's fragments are read, and with
        // the stage's last step the loads of a later stage issued, a few after each product.
        const bool end = kk == kHalves - 1;
        bf16x8(&pc)[WP] = pf[kk & 1], (&pn)[WP] = pf[1 - (kk & 1)];
        bf16x8(&qc)[WQ] = qf[kk & 1], (&qn)[WQ] = qf[1 - (kk & 1)];
        if constexpr (kSums) {
          if (kk % 2 && s == mine) {                        // steps kk - 1 and kk: one for each wavefront, or both
#pragma unroll
            for (int b = 0; b < WQ; ++b) {
              // each whole: a choice between references becomes one between registers by number
              const float c = add8(__builtin_bit_cast(u32x4, qc[b])), n = add8(__builtin_bit_cast(u32x4, qn[b]));
              sums[b] += g.splits == 1 ? n + c : wp ? c : n;
            }
            if (end) mine += turns;
          }
        }
        if (end) {
          // The next stage is there, and this one read by all. Vector memory operations complete in order:
          // for the first stages after a tile's stores, those are newer than the loads waited for.
          if (kStores && s < kBufs - 1 && i != first) wait_loads<kLoads * (kBufs - 2) + kStores>();
          else wait_loads<kLoads * (kBufs - 2)>();
          into = lds0 + buf * kStage;
          buf = buf == kBufs - 1 ? 0 : buf + 1;
          stage = lds + buf * kStage;
        }
        const int to = end ? 0 : kk + 1;
        if (end) {
          op.aim(into, wave);
          oq.aim(into + kQ, wave);
        }
        // of the products, the first half is followed by a share of the reads each, all by one of the loads
        constexpr int kProducts = WP * WQ, kHalf = (kProducts + 1) / 2, kFrags = WP + WQ;
#pragma unroll
        for (int m = 0; m < kProducts; ++m) {
          const int a = m / WQ, b = m % WQ;
          acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pc[a], qc[b], acc[a][b], 0, 0, 0);
#pragma unroll
          for (int f = m * kFrags / kHalf; f < (m + 1) * kFrags / kHalf && f < kFrags; ++f) {
            if (f < WQ) qn[f] = fq.read(stage + kQ, to, f);
            else pn[f - WQ] = fp.read(stage, to, f - WQ);
          }
          if (end) {
#pragma unroll
            for (int l = m * kLoads / kProducts; l < (m + 1) * kLoads / kProducts; ++l) {
              if (l < op.kLoads) op.fetch(l);
              else oq.fetch(l - op.kLoads);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (end) {
          op.advance();
          oq.advance();
        }
      }
      fetched();
    }
    if (Out::kBias && t.stages < kBufs) wait_own<0>();      // else a stage's wait has covered the next biases
    const int64_t qw = t.q0 + 32 * WQ * wq, pw = t.p0 + 32 * WP * wp;        // this wavefront's part
    if constexpr (!kSums) {
      store_rows<WP, WQ>(out, g, lds + kBufs * kStage + wave * Staging<WP>::kBytes, qw, pw, lane, acc);
    } else {
      const int r = lane & 31, h = lane >> 5;
#pragma unroll
      for (int b = 0; b < WQ; ++b) {
        const int64_t q = qw + 32 * b + r;
#pragma unroll
        for (int a = 0; a < WP; ++a)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int64_t p = pw + 32 * a + 16 * half + 8 * h;
            float* at = out.gw + (t.split * g.nq + q) * g.np + p;
            if (q < g.nq && p < g.np) {
#pragma unroll
              for (int e = 0; e < 2; ++e)
                reinterpret_cast<float4*>(at)[e] = make_float4(acc[a][b][8 * half + 4 * e], acc[a][b][8 * half + 4 * e + 1],
                                                               acc[a][b][8 * half + 4 * e + 2], acc[a][b][8 * half + 4 * e + 3]);
            }
          }
        // NP wavefronts and `parts` workgroups hold shares of the sum over Q; of a single split, each the whole
        const float s = sums[b] + __shfl_xor(sums[b], 32);
        const int64_t part = t.p0 / TP;
        if (g.splits > 1) {
          if (h == 0 && part < out.parts && q < g.nq) out.gb[((t.split * out.parts + part) * NP + wp) * g.nq + q] = s;
        } else if (h == 0 && part == 0 && wp == 0 && q < g.nq) {
          out.gb[q] = s;
        }
      }
    }
  }
  wait_loads<0>();                                          // no load into LDS outlives the workgroup
}

template <int WP, int WQ, int kDepth, int kBufs, bool kPT, bool kQT, class Out>
__global__ __launch_bounds__(kThreads, (Tile<WP, WQ, kDepth, kBufs, Out>::kResident)) void product_kernel(Product g, Out out) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[Tile<WP, WQ, kDepth, kBufs, Out>::kBytes];
  product<WP, WQ, kDepth, kBufs, kPT, kQT>(g, out, lds, blockIdx.x, gridDim.x);
}

// Both gradients in one launch: the first `blocks` workgroups make the input's, in 64 x 64 tiles, the others the weights'.
template <int WP, int WQ>
__global__ __launch_bounds__(kThreads, 2) void pair_kernel(Product gx, InputGrad x, uint32_t blocks, Product gw, WeightGrad w) {
  using X = Tile<1, 1, 64, 2, InputGrad>;
  using W = Tile<WP, WQ, 64, 2, WeightGrad>;
  __shared__ __attribute__((aligned(16))) unsigned char lds[X::kBytes > W::kBytes ? X::kBytes : W::kBytes];
  if (blockIdx.x < blocks) product<1, 1, 64, 2, true, false>(gx, x, lds, blockIdx.x, blocks);
  else product<WP, WQ, 64, 2, true, true>(gw, w, lds, blockIdx.x - blocks, gridDim.x - blocks);
}

// g_w and g_b from their shares, summed in a fixed order. A quad of values to each of 256 / G neighbouring threads, its
// shares dealt out over G groups of them, each with the loads of eight shares issued before the first is added. G = 16
// where there are few values for the chip: the gradients of 91,341 x 32 -> 48 float32 (357 shares) take 31 us so and 45 in
// one chain of adds, of 65,536 x 256 -> 512 bfloat16 (64 shares) 42.9 and 44.8.
template <int G>
__global__ __launch_bounds__(kThreads) void join_kernel(const float* gw_parts, int32_t n_gw, float* gw, int64_t size,
                                                        const float* gb_parts, int32_t n_gb, float* gb, int32_t d_out) {
  constexpr int kQuads = kThreads / G;
  const int group = threadIdx.x / kQuads, own = threadIdx.x % kQuads;
  const int64_t quads = n_gw != 1 ? size / 4 : 0, all = quads + d_out / 4;      // one share is g_w itself
  __shared__ float4 s_sum[G][kQuads];
  for (int64_t first = (int64_t)blockIdx.x * kQuads; first < all; first += (int64_t)gridDim.x * kQuads) {
    const int64_t i = first + own;
    const bool w = i < quads;
    const float4* at = w ? reinterpret_cast<const float4*>(gw_parts) + i : reinterpret_cast<const float4*>(gb_parts) + (i - quads);
    const int64_t step = w ? size / 4 : d_out / 4;
    const int32_t n = i < all ? w ? n_gw : n_gb : 0;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    int32_t j = group;
    for (; j + 7 * G < n; j += 8 * G) {
      float4 a[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) a[u] = at[(j + u * G) * step];
#pragma unroll
      for (int u = 0; u < 8; ++u) s.x += a[u].x, s.y += a[u].y, s.z += a[u].z, s.w += a[u].w;
    }
    for (; j < n; j += G) {
      const float4 a = at[j * step];
      s.x += a.x, s.y += a.y, s.z += a.z, s.w += a.w;
    }
    if constexpr (G > 1) {
      __syncthreads();                                      // the last round's sums are read
      s_sum[group][own] = s;
      __syncthreads();
      if (group > 0) continue;
#pragma unroll
      for (int u = 1; u < G; ++u) {
        const float4 a = s_sum[u][own];
        s.x += a.x, s.y += a.y, s.z += a.z, s.w += a.w;
      }
    }
    if (i < all) (w ? reinterpret_cast<float4*>(gw) + i : reinterpret_cast<float4*>(gb) + (i - quads))[0] = s;
  }
}

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t kCus = 256;

// the rest of a product's numbers, and its workgroups
template <class Tile>
uint32_t plan(Product& g) {
  g.p_tiles = (int32_t)cdiv(g.np, Tile::TP);
  g.splits = (int32_t)cdiv(g.nk, g.k_split);
  g.items = cdiv(g.nq, Tile::TQ) * g.p_tiles * g.splits;
  const int64_t want = cdiv(g.items, 8) * 8, most = kCus * Tile::kResident;
  return (uint32_t)(want < most ? want : most);
}

template <int WP, int WQ, int kDepth, int kBufs, bool kPT, bool kQT, class Out>
maestro_status launch(Product g, const Out& out, hipStream_t stream) {
  const uint32_t blocks = plan<Tile<WP, WQ, kDepth, kBufs, Out>>(g);
  product_kernel<WP, WQ, kDepth, kBufs, kPT, kQT, Out><<<blocks, kThreads, 0, stream>>>(g, out);
  return launch_status();
}

template <int WP, int WQ>
maestro_status launch_pair(Product gx, const InputGrad& x, Product gw, const WeightGrad& w, hipStream_t stream) {
  const uint32_t blocks = plan<Tile<1, 1, 64, 2, InputGrad>>(gx), more = plan<Tile<WP, WQ, 64, 2, WeightGrad>>(gw);
  pair_kernel<WP, WQ><<<blocks + more, kThreads, 0, stream>>>(gx, x, blocks, gw, w);
  return launch_status();
}

// Tile of the activations and the input's gradient. A wavefront of a 256 x 256 tile reads half a KB of LDS for a
// product, of a 128 x 128 tile one, of a 64 x 64 tile two; but each size needs its tiles to be many: two
// rounds of workgroups or more, one for 128. Measured (us, tile 256 / 128 / 64): 262,139 x 1024 -> 1024
// 522 / 659 / 1568, 65,536 x 256 -> 512 (512 and 2,048 tiles) 28 / 30 / 55, 16,384 x 512 -> 512 (128 and 512) 22 / 15 / 23,
// 4,096 x 1024 -> 1024 (64 and 256) 30 / 15 / 20, 16,384 x 1024 -> 64 (128 of 128) 29 / 15 / 12.
int tile_of(int64_t np, int64_t nq) {
  if (np > 128 && cdiv(np, 256) * cdiv(nq, 256) >= 2 * kCus) return 256;
  return cdiv(np, 128) * cdiv(nq, 128) >= kCus ? 128 : 64;
}

// Stages of 64 k: rows whose k is contiguous come as whole 128-byte lines. (With stages of 32 and four buffers
// each line is fetched twice, its halves a stage apart: 552 against 522 us at 262,139 x 1024 -> 1024.)
template <bool kPT, class Out>
maestro_status launch_rows(const Product& g, const Out& out, hipStream_t stream) {
  const int tile = tile_of(g.np, g.nq);
  if (tile == 256) return launch<4, 4, 64, 2, kPT, false>(g, out, stream);
  if constexpr (!kPT)                                       // the input's gradient of this size: pair_kernel
    if (tile == 64) return launch<1, 1, 64, 2, kPT, false>(g, out, stream);
  return launch<2, 2, 64, 2, kPT, false>(g, out, stream);
}

// How the weights' gradient is cut: tile, k of one split, splits of the n rows, and workgroups that share the
// biases' sum (one where the rows are not split, so that no second launch is needed). 256 x 256 tiles for many rows, else 256 (d_in) x 64, or 128 x 128 where d_in is narrow;
// rows split so that there is one round of workgroups, none with fewer than 512 rows. Measured (us,
// 256 x 256 / 256 x 64 / 128 x 128): 262,139 x 1024 -> 1024 505 / 668 / 591, 512 -> 512 163 / 199 / 194,
// 1024 -> 64 153 / 149 / 154, 64 -> 1024 155 / 170 / 118; 65,536 x 512 -> 512 68 / 58 / 65; 16,384 41 / 32 / 38.
struct Cut {
  int32_t tp, tq;
  int64_t k_split, splits;
  int32_t parts;
};

Cut cut_of(int64_t n, int64_t d_in, int64_t d_out) {
  Cut c;
  c.tp = d_in > 128 ? 256 : 128;
  c.tq = c.tp == 128 ? 128 : d_out > 128 && n >= 131072 ? 256 : 64;
  const int64_t tiles = cdiv(d_in, c.tp) * cdiv(d_out, c.tq), resident = c.tq == 256 ? 1 : 2;
  int64_t splits = kCus * resident / tiles;
  if (splits > cdiv(n, 512)) splits = cdiv(n, 512);
  if (splits < 1) splits = 1;
  c.k_split = cdiv(cdiv(n, splits), 64) * 64;
  c.splits = cdiv(n, c.k_split);
  c.parts = c.splits > 1 ? (int32_t)cdiv(d_in, c.tp) : 1;
  return c;
}

}  // namespace

maestro_status launch_layer_bf16(int64_t n, int32_t d_in, int32_t d_out, const void* x, const void* weight,
                                 const float* bias, bool relu, void* y, hipStream_t stream) {
  Product g{static_cast<const __bf16*>(weight), static_cast<const __bf16*>(x), d_in, d_in, d_out, n, d_in, d_in, 1, 0, 0};
  return launch_rows<false>(g, Forward{bias, static_cast<__bf16*>(y), relu}, stream);
}

size_t layer_grad_bf16_workspace_bytes(int64_t n, int32_t d_in, int32_t d_out) {
  if (n == 0) return 0;
  const Cut c = cut_of(n, d_in, d_out);
  return c.splits > 1 ? sizeof(float) * (size_t)(c.splits * ((int64_t)d_in + c.parts * 2) * d_out) : 0;
}

maestro_status launch_layer_grad_bf16(int64_t n, int32_t d_in, int32_t d_out, const void* x, const void* weight,
                                      const void* g_z, bool relu_input, void* g_x, float* g_weight, float* g_bias,
                                      void* workspace, hipStream_t stream) {
  const __bf16 *xb = static_cast<const __bf16*>(x), *gz = static_cast<const __bf16*>(g_z);
  const Cut c = cut_of(n, d_in, d_out);
  float* parts = static_cast<float*>(workspace);
  float* gb_parts = parts + c.splits * d_in * d_out;
  const Product gw{xb, gz, d_in, d_out, d_in, d_out, n, c.k_split, 1, 0, 0};
  const WeightGrad w{c.splits > 1 ? parts : g_weight, c.splits > 1 ? gb_parts : g_bias, c.parts};
  const Product gx{static_cast<const __bf16*>(weight), gz, d_in, d_out, d_in, n, d_out, d_out, 1, 0, 0};
  const InputGrad x_out{xb, static_cast<__bf16*>(g_x), relu_input};
  maestro_status st = MAESTRO_OK;
  // Little work: a launch less, and the two products side by side. 300 x 256 -> 512 11.8 us (14.6 in two launches),
  // 2,000 x 512 -> 512 16.7 (22.6), 30,000 x 64 -> 128 18.7 (20.2)
  if (g_x && tile_of(d_in, n) == 64) {
    st = c.tp == 256 ? launch_pair<4, 1>(gx, x_out, gw, w, stream) : launch_pair<2, 2>(gx, x_out, gw, w, stream);
  } else {
    if (g_x) st = launch_rows<true>(gx, x_out, stream);
    if (st != MAESTRO_OK) return st;
    st = c.tq == 256   ? launch<4, 4, 32, 4, true, true>(gw, w, stream)
         : c.tp == 256 ? launch<4, 1, 64, 2, true, true>(gw, w, stream)
                       : launch<2, 2, 64, 2, true, true>(gw, w, stream);
  }
  if (st != MAESTRO_OK || c.splits == 1) return st;
  return launch_join(parts, (int32_t)c.splits, g_weight, (int64_t)d_in * d_out, gb_parts, (int32_t)(c.splits * c.parts * 2),
                     g_bias, d_out, stream);
}

maestro_status launch_join(const float* gw_parts, int32_t n_gw, float* gw, int64_t size, const float* gb_parts,
                           int32_t n_gb, float* gb, int32_t d_out, hipStream_t stream) {
  const int64_t quads = (n_gw != 1 ? size / 4 : 0) + d_out / 4, blocks = cdiv(quads, kThreads);
  if (blocks < kCus && n_gb > 8)
    join_kernel<16><<<(unsigned)cdiv(quads, kThreads / 16), kThreads, 0, stream>>>(gw_parts, n_gw, gw, size, gb_parts, n_gb, gb, d_out);
  else
    join_kernel<1><<<(unsigned)(blocks < 4096 ? blocks : 4096), kThreads, 0, stream>>>(gw_parts, n_gw, gw, size, gb_parts, n_gb, gb, d_out);
  return launch_status();
}

}  // namespace maestro
