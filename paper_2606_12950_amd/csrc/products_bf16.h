// The products of a predictor's layer and its gradients on the matrix cores, of bfloat16 values or of signed bytes.
//
// All three are C[q][p] = sum_k P(p, k) Q(q, k) with C's rows contiguous in p:
//   activations      y[n][o]   P = weight (k contiguous)   Q = x   (k contiguous)   k over d_in
//   input's gradient g_x[n][i] P = weight (p contiguous)   Q = g_z (k contiguous)   k over d_out
//   weights'         g_w[o][i] P = x      (p contiguous)   Q = g_z (q contiguous)   k over the n rows
// A workgroup of four wavefronts (or eight) makes a tile of TP x TQ of C, each wavefront 32 WP x 32 WQ of it in
// 32x32x16 MFMAs. k advances in stages of kDepth (32 or 64) that come straight into LDS, kBufs buffers round. An
// operand whose k is contiguous lies in LDS as [p][k]; one whose p (or q) is contiguous as [k][p], and
// is turned by the transposing LDS read (ds_read_b64_tr_b16: sixteen lanes read a 4 x 16 block row-wise
// and get it column-wise). P's 32 rows of a block are taken in an order (tile_row_neuron) that leaves every lane runs
// of 8 consecutive p. Workgroups are persistent: the loads of the next tile's first stages run under a
// tile's last products and its stores, and its stores under the next tile's products.
#pragma once

#include <type_traits>

#include "mlp.h"
#include "rules.h"
#include "train.h"

namespace maestro {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kThreads = 256;         // of a workgroup of four wavefronts

struct Product {
  const __bf16* p;                   // P and Q and their leading dimensions (elements)
  const __bf16* q;
  int64_t ldp, ldq;
  int64_t np, nq, nk;                // extents
  int64_t k_split;                   // k of one split, a multiple of kDepth (>= nk: one split)
  int32_t splits, p_tiles;
  int64_t items;                     // splits * tiles
};

// One tile: its operands, its place in C (rows of q from q_end on are not the tile's) and its k.
struct Item {
  const __bf16 *p, *q;
  int64_t q0, q_end, p0, k0, kn, stages;
  int64_t slot;                      // which share of C, where k is split
  int32_t group;
  bool whole;                        // the sum over Q is not shared between workgroups
  bool direct;                       // the whole of a group's C
};

// A workgroup's way through `items` units of work, workgroup `block` of `blocks` (a multiple of 8). XCD x (of 8; workgroups go
// round them) takes a contiguous share, so that the tiles that read the same rows of Q run side by side on one L2.
// Counts of 64 bits: a product has up to 2^40 rows. The scalar unit does not compare them; a test looks at what becomes of it (groups.h).
struct Cursor {
  int64_t i, last, step;
  __device__ __forceinline__ Cursor(int64_t items, uint32_t block, uint32_t blocks) {
    const int64_t share = (items + 7) / 8, xcd = block & 7;
    step = blocks >> 3;
    last = (xcd + 1) * share < items ? (xcd + 1) * share : items;
    i = xcd * share + (block >> 3);
  }
  __device__ __forceinline__ bool done() const { return i >= last; }
};

// The tiles of one product, all splits' one after the other.
template <int TP, int TQ, int kDepth>
struct Dense {
  using Way = Cursor;
  const Product& g;
  int64_t per_split;
  __device__ __forceinline__ explicit Dense(const Product& product) : g(product), per_split(product.items / product.splits) {}
  __device__ __forceinline__ Way begin(uint32_t block, uint32_t blocks) const { return Way(g.items, block, blocks); }
  __device__ __forceinline__ void next(Way& c) const { c.i += c.step; }
  __device__ __forceinline__ Item item(const Way& c) const {
    Item t;
    t.p = g.p;
    t.q = g.q;
    t.group = 0;
    t.whole = t.direct = g.splits == 1;
    t.slot = c.i / per_split;
    const int64_t tile = c.i % per_split;
    t.q0 = tile / g.p_tiles * TQ;
    t.q_end = g.nq;
    t.p0 = tile % g.p_tiles * TP;
    t.k0 = t.slot * g.k_split;
    t.kn = g.nk - t.k0 < g.k_split ? g.nk - t.k0 : g.k_split;
    t.stages = (t.kn + kDepth - 1) / kDepth;
    return t;
  }
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

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
  __device__ __forceinline__ u32x2 load8(uint32_t off) const {
    return __builtin_amdgcn_raw_buffer_load_b64(rsrc, off, 0, 0);
  }
  __device__ __forceinline__ void store(const u32x4& v, uint32_t off) const {
    __builtin_amdgcn_raw_buffer_store_b128(v, rsrc, off, 0, 0);
  }
};

// What becomes of C. kMask: C is 0 wherever `x`, of C's shape, is not positive (kMaskBf16), or not zero (kMaskCodes,
// unsigned bytes). kBias: `bias` [p], of the tile's group, is added and, with relu, negative values become 0. kInt8: the
// operands are signed bytes, and a sum counts scale_q[q] * scale_p[p]; the products' extents of k are in pairs of them. kCodes: P
// is the values of kept activations (CodesOperand).
enum { kMaskNone, kMaskBf16, kMaskCodes };
struct Forward {
  static constexpr int kMask = kMaskNone;
  static constexpr bool kBias = true, kInt8 = false, kCodes = false;
  typedef __bf16 type;
  const float* bias;
  __bf16* c;
  int32_t relu;
};
struct InputGrad {
  static constexpr int kMask = kMaskBf16;
  static constexpr bool kBias = false, kInt8 = false, kCodes = false;
  typedef __bf16 type;
  const __bf16* x;
  __bf16* c;
  int32_t relu;
};
struct CodesInputGrad {
  static constexpr int kMask = kMaskCodes;
  static constexpr bool kBias = false, kInt8 = false, kCodes = false;
  typedef __bf16 type;
  const unsigned char* x;
  __bf16* c;
  int32_t relu;
};
template <class T>
struct Int8Forward {
  static constexpr int kMask = kMaskNone;
  static constexpr bool kBias = true, kInt8 = true, kCodes = false;
  typedef T type;
  const float *bias, *scale_p, *scale_q;
  T* c;
  int32_t relu;
};
struct WeightGrad {
  static constexpr bool kBias = false, kInt8 = false, kCodes = false;
  float* gw;                         // [splits][nq][np]
  float* gb;                         // one split: [nq], whole; else [splits][parts][two wavefronts][nq]
  int32_t parts;                     // workgroups (of one split and q) that share the sum over Q
  __device__ __forceinline__ float* weights(const Product& g, const Item& t) const { return gw + t.slot * g.nq * g.np; }
  __device__ __forceinline__ float* biases(const Product& g, const Item& t, int64_t part, int wp) const {
    return t.whole ? gb : gb + ((t.slot * parts + part) * 2 + wp) * g.nq;
  }
};

template <class C>
struct CodesWeightGrad : WeightGrad {
  static constexpr bool kCodes = true;
  typedef C Code;                    // int8_t or uint8_t
  const Code* codes;                 // [nk][np]
  const unsigned char* exponents;    // [nk][ld_exponents]
  int64_t ld_exponents;
};
template <class Out, class = void>
struct CodeOf {
  typedef uint8_t type;
};
template <class Out>
struct CodeOf<Out, std::void_t<typename Out::Code>> {
  typedef typename Out::Code type;
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
template <int T, int kDepth, bool kTurned, int kWaves = 4>
struct Operand {
  static constexpr int kLoads = T * kDepth / (512 * kWaves);      // 1 KB loads of a wavefront and stage
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

// A turned operand that memory holds as codes, bytes, and for every 32 of a row a power of two. A stage's codes come through
// registers, 16 to a unit, and are values before they lie in LDS: a value has at most eight significant bits, so bfloat16
// holds it exactly. They are loaded two stages ahead of the products' and turned into values one ahead, a pair after a product.
template <int T, int kDepth, class Code, int kWaves = 4>
struct CodesOperand {
  static constexpr int kUnits = T * kDepth / 16 / (64 * kWaves), kRowUnits = T / 16, kRows = 64 * kWaves / kRowUnits;
  static constexpr int kPairs = 8 * kUnits;
  u32x4 ahead[kUnits], now[kUnits];                         // the stages being loaded and turned into values
  uint8_t ahead_exponent[kUnits];
  float step[kUnits];
  u32x4 packed;
  const unsigned char *codes, *exponents;                   // of the next stage to load
  int64_t left;                                             // its rows and all after it
  uint32_t ld, ld_exponents, off, off_exponents;
  uint32_t to;                                              // in the stage, the 16 bytes it writes first of a unit's 32
  bool second;                                              // those are the unit's second ones

  template <class Out>
  __device__ __forceinline__ void init(const Out& out, int64_t ldp) {
    const int k = threadIdx.x / kRowUnits, unit = threadIdx.x % kRowUnits;
    ld = (uint32_t)ldp;
    ld_exponents = (uint32_t)out.ld_exponents;
    // eight lanes write 128 bytes at a time: neighbouring fours of them begin with other halves, and meet all banks
    second = (unit & 4) != 0;
    to = k * 2 * T + (((2 * unit + second) ^ (4 * Operand<T, kDepth, true>::turn(k))) << 4);
  }
  template <class Out>
  __device__ __forceinline__ void tile(const Out& out, int64_t p0, int64_t k0, int64_t kn) {
    const int k = threadIdx.x / kRowUnits, unit = threadIdx.x % kRowUnits;
    codes = reinterpret_cast<const unsigned char*>(out.codes) + k0 * ld;
    exponents = out.exponents + k0 * ld_exponents;
    left = kn;
    off = (uint32_t)(k * ld + p0 + 16 * unit);
    off_exponents = (uint32_t)(k * ld_exponents + p0 / 32 + unit / 2);
  }
  __device__ __forceinline__ void none() { left = 0; }
  __device__ __forceinline__ void load() {
    const uint32_t rows = (uint32_t)(left < kDepth ? left < 0 ? 0 : left : kDepth);
    const auto c = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(codes), 0, rows * ld, 0x00020000);
    const auto e = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(exponents), 0, rows * ld_exponents, 0x00020000);
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      ahead[j] = __builtin_amdgcn_raw_buffer_load_b128(c, off + j * kRows * ld, 0, 0);
      ahead_exponent[j] = __builtin_amdgcn_raw_buffer_load_b8(e, off_exponents + j * kRows * ld_exponents, 0, 0);
    }
    codes += kDepth * (int64_t)ld;
    exponents += kDepth * (int64_t)ld_exponents;
    left -= kDepth;
  }
  __device__ __forceinline__ void take() {
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      now[j] = second ? __builtin_shufflevector(ahead[j], ahead[j], 2, 3, 0, 1) : ahead[j];
      step[j] = __uint_as_float((uint32_t)ahead_exponent[j] << 23);
      // here and not after the next loads, whose registers would then be others, and waited for to be copied
      asm volatile("" : "+v"(now[j]), "+v"(step[j]));
    }
  }
  // pair i of the stage, into the stage's buffer when it completes 16 bytes
  __device__ __forceinline__ void pair(int i, unsigned char* stage) {
    const int j = i / 8, r = i % 8;
    const uint32_t w = now[j][r / 2] >> (16 * (r & 1));
    const float a = (float)(Code)w * step[j], b = (float)(Code)(w >> 8) * step[j];
    packed[r % 4] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    if (r % 4 == 3) *reinterpret_cast<u32x4*>(stage + (to ^ (16 * (r / 4))) + j * kRows * 2 * T) = packed;
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

template <class Out, class = void>
struct IsWeightGrad : std::false_type {};
template <class Out>
struct IsWeightGrad<Out, std::void_t<decltype(std::declval<Out>().parts)>> : std::true_type {};

template <class Out>
__device__ __forceinline__ int32_t parts_of(const Out& out) {
  if constexpr (IsWeightGrad<Out>::value) return out.parts;
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

// the bfloat16 pair c where bytes 2 e and 2 e + 1 of x are not zero
__device__ __forceinline__ uint32_t where_coded(uint32_t c, uint32_t x, int e) {
  const uint32_t two = x >> (16 * e);
  return c & ((two & 0xFFu ? 0xFFFFu : 0u) | (two & 0xFF00u ? 0xFFFF0000u : 0u));
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
template <int WP, int kWaves = 4>
struct Staging {
  static constexpr int WS = WP < 4 || kWaves > 4 ? 1 : 2;   // blocks of 32 p at a time
  static constexpr int kRowBytes = 64 * WS, kUnits = 4 * WS, kRows = 64 / kUnits;
  static constexpr int kBytes = 32 * kRowBytes;             // of a wavefront
  static __device__ __forceinline__ int place(int q) { return (q / (16 / kUnits)) & (kUnits - 1); }
};

// Keeps the sums of one block where the products left them, up to here: of 256 x 256 tiles they fill the accumulation registers,
// and copies of other blocks made ahead would take the vector registers of the main loop's addresses.
template <int WP, int WQ, class Acc>
__device__ __forceinline__ void in_place(Acc& acc) {
  if constexpr (WP * WQ == 16) asm volatile("" : "+a"(acc));
}

template <int WP, int WQ, int kWaves, class Out, class Acc>
__device__ __forceinline__ void store_rows(const Out& out, const Product& g, const Item& t, unsigned char* staging, int64_t q0,
                                           int64_t p0, int lane, Acc (&acc)[WP][WQ]) {
  using S = Staging<WP, kWaves>;
  constexpr int kStores = 32 / S::kRows;                    // of one q block and WS p blocks
  const int r = lane & 31, h = lane >> 5;
  const int row0 = lane / S::kUnits, unit0 = lane % S::kUnits;
  const uint32_t ld = (uint32_t)g.np * 2, step = S::kRows * ld;
  Rows c, x;
  c.init(out.c, q0, t.q_end, 32 * WQ, ld);
  uint32_t at[WP / S::WS];                                  // of the first row's unit, outside C: past the resource
#pragma unroll
  for (int w = 0; w < WP / S::WS; ++w) {
    const int64_t p = p0 + 32 * S::WS * w + 8 * unit0;
    at[w] = p < g.np ? (uint32_t)(row0 * ld + p * 2) : 0x80000000u;
  }
  using Mask = std::conditional_t<Out::kMask == kMaskCodes, u32x2, u32x4>;
  Mask xv[WP / S::WS][kStores];
  const bool relu = out.relu;
  auto mask = [&](uint32_t off) -> Mask {                   // a code has half a value's bytes
    if constexpr (Out::kMask == kMaskCodes) return x.load8(off >> 1);
    else return x.load(off);
  };
  if constexpr (Out::kMask != kMaskNone) {
    x.init(out.x, q0, t.q_end, 32 * WQ, !relu ? 0 : Out::kMask == kMaskCodes ? ld / 2 : ld);
#pragma unroll
    for (int w = 0; w < WP / S::WS; ++w)
#pragma unroll
      for (int j = 0; j < kStores; ++j) xv[w][j] = mask(at[w] + j * step);
  }
#pragma unroll
  for (int b = 0; b < WQ; ++b) {
#pragma unroll
    for (int w = 0; w < WP / S::WS; ++w) {
#pragma unroll
      for (int a = 0; a < S::WS; ++a) in_place<WP, WQ>(acc[w * S::WS + a][b]);
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
      if constexpr (Out::kMask == kMaskNone) {
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
            for (int e = 0; e < 4; ++e) {
              if constexpr (Out::kMask == kMaskCodes) v[j][e] = where_coded(v[j][e], xv[w][j][e / 2], e & 1);
              else v[j][e] = where_positive(v[j][e], xv[w][j][e]);
            }
          if (b + 1 < WQ) xv[w][j] = mask(at[w] + ((b + 1) * kStores + j) * step);
        }
      }
#pragma unroll
      for (int j = 0; j < kStores; ++j) c.store(v[j], at[w] + (b * kStores + j) * step);
      asm volatile("" ::: "memory");                        // one block's values at a time: registers
    }
  }
}

// A wavefront's part of C from sums of 8-bit products: fma(sum * scale_q, scale_p, bias), not below `least` (a NaN stays one).
// `place`: the biases and, kPlace / 2 further, the scales of the wavefront's 32 WP p. bfloat16 by way of LDS as above; float32
// straight from the lanes, eight values (32 bytes) of a row each, in stores that the main loop's waits do not count.
template <int WP, int WQ, int kWaves, class Out>
__device__ __forceinline__ void store_scaled(const Out& out, const Product& g, const Item& t, unsigned char* staging, int64_t q0,
                                             int64_t p0, int lane, i32x16 (&acc)[WP][WQ], const float* place, int scales) {
  typedef typename Out::type T;
  constexpr bool kStaged = std::is_same<T, __bf16>::value;
  using S = Staging<WP, kWaves>;
  constexpr int kStores = 32 / S::kRows;
  const int r = lane & 31, h = lane >> 5;
  const int row0 = lane / S::kUnits, unit0 = lane % S::kUnits;
  const uint32_t ld = (uint32_t)g.np * 2, step = S::kRows * ld;
  const float least = out.relu ? 0.0f : -INFINITY;
  Rows c;
  c.init(out.c, q0, t.q_end, 32 * WQ, ld);
  float scale_q[WQ];
#pragma unroll
  for (int b = 0; b < WQ; ++b) {
    const int64_t q = q0 + 32 * b + r;
    scale_q[b] = q < t.q_end ? out.scale_q[q] : 0.0f;
  }
#pragma unroll
  for (int w = 0; w < WP / S::WS; ++w) {
    float4 bias[S::WS][4], scale[S::WS][4];                 // of the lane's p
#pragma unroll
    for (int a = 0; a < S::WS; ++a)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* from = place + 32 * (w * S::WS + a) + 16 * (i / 2) + 8 * h + 4 * (i % 2);
        bias[a][i] = *reinterpret_cast<const float4*>(from);
        scale[a][i] = *reinterpret_cast<const float4*>(from + scales);
      }
    const int64_t p_unit = p0 + 32 * S::WS * w + 8 * unit0;
    const uint32_t at = p_unit < g.np ? (uint32_t)(row0 * ld + p_unit * 2) : 0x80000000u;
#pragma unroll
    for (int b = 0; b < WQ; ++b) {
#pragma unroll
      for (int a = 0; a < S::WS; ++a) in_place<WP, WQ>(acc[w * S::WS + a][b]);
#pragma unroll
      for (int a = 0; a < S::WS; ++a)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float4 &s = scale[a][2 * half + e / 4], &z = bias[a][2 * half + e / 4];
            const float sum = (float)acc[w * S::WS + a][b][8 * half + e] * scale_q[b];
            v[e] = __builtin_elementwise_maximum(
                fmaf(sum, e % 4 == 0 ? s.x : e % 4 == 1 ? s.y : e % 4 == 2 ? s.z : s.w,
                     e % 4 == 0 ? z.x : e % 4 == 1 ? z.y : e % 4 == 2 ? z.z : z.w), least);
          }
          if constexpr (kStaged) {
            *reinterpret_cast<u32x4*>(staging + r * S::kRowBytes + (((4 * a + 2 * half + h) ^ S::place(r)) << 4)) = pack8(v);
          } else {
            const int64_t q = q0 + 32 * b + r, p = p0 + 32 * (w * S::WS + a) + 16 * half + 8 * h;
            if (q < t.q_end && p < g.np) {
              float4* to = reinterpret_cast<float4*>(out.c + q * g.np + p);
              to[0] = make_float4(v[0], v[1], v[2], v[3]);
              to[1] = make_float4(v[4], v[5], v[6], v[7]);
            }
          }
        }
      if constexpr (kStaged) {
        u32x4 v[kStores];
#pragma unroll
        for (int j = 0; j < kStores; ++j) {
          const int row = j * S::kRows + row0;
          v[j] = *reinterpret_cast<const u32x4*>(staging + row * S::kRowBytes + ((unit0 ^ S::place(row)) << 4));
        }
#pragma unroll
        for (int j = 0; j < kStores; ++j) c.store(v[j], at + (b * kStores + j) * step);
      }
      asm volatile("" ::: "memory");                        // one block's values at a time: registers
    }
  }
}

// Whether C goes by way of LDS, in a number of stores that the main loop's waits count.
template <class Out>
constexpr bool staged() {
  if constexpr (IsWeightGrad<Out>::value) return false;
  else return std::is_same<typename Out::type, __bf16>::value;
}

// Sizes of a product's tile, and its LDS.
template <int WP, int WQ, int kDepth, int kBufs, class Out, int kWaves = 4>
struct Tile {
  static constexpr int TP = 64 * WP, TQ = 16 * kWaves * WQ;       // two wavefronts by two, or by four
  static constexpr int kStage = (TP + TQ) * 2 * kDepth;
  static constexpr bool kStores = staged<Out>();            // by way of LDS
  static constexpr int kBiasLoads = Out::kBias ? (WP + 1) / 2 : 0;            // and as many of scale_p
  static constexpr int kEpilogueLoads = kBiasLoads * (Out::kInt8 ? 2 : 1);
  static constexpr int kBiasBytes = 2 * kWaves * 256 * kEpilogueLoads;             // two places for each wavefront
  static constexpr int kBytes = kBufs * kStage + (kStores ? kWaves * Staging<WP, kWaves>::kBytes : 0) + kBiasBytes;
  // workgroups of a CU that a launch plans for, and that registers allow. LDS lets three run of the activations' 64 x 64
  // (43,008 bytes of 160 KB, with scales for 8-bit products 45,056: the fourth's start when others end) and two of pair_kernel<4, 1>
  // (81,920, the larger tile's, in all of them).
  static constexpr int kBlocks = WP * WQ * kWaves / 4;      // of 32 x 32, a SIMD's
  static constexpr int kResident = kBlocks > 8 ? 1 : kBlocks > 2 ? 2 : 4;
  static constexpr int kSimdWaves = kResident * kWaves / 4;
};

// The share of workgroup `block` of `blocks` (a multiple of 8) in the tiles of `work`, products of the sizes of `g`.
template <int WP, int WQ, int kDepth, int kBufs, bool kPT, bool kQT, int kWaves = 4, class Out, class Work>
__device__ __forceinline__ void product(const Product& g, const Out& out, const Work& work, unsigned char* lds, uint32_t block,
                                        uint32_t blocks) {
  using L = Tile<WP, WQ, kDepth, kBufs, Out, kWaves>;
  constexpr int NP = 2, TP = L::TP, TQ = L::TQ;
  constexpr bool kCodes = Out::kCodes;
  constexpr int kStage = L::kStage, kPLoads = kCodes ? 0 : TP * kDepth / (512 * kWaves), kHalves = kDepth / 16;
  constexpr int kLoads = kPLoads + TQ * kDepth / (512 * kWaves);
  static_assert(!kCodes || (kBufs == 2 && kPT), "a stage's end waits for all loads");
  constexpr int kQ = TP * 2 * kDepth;                       // Q's place in a stage
  constexpr bool kSums = kQT;                               // the weights' gradient sums Q too (the biases')
  constexpr int kBiasLoads = L::kBiasLoads, kEpilogueLoads = L::kEpilogueLoads;
  constexpr int kStores = L::kStores ? 2 * WP * WQ + kEpilogueLoads : 0;      // between two tiles, exactly
  static_assert(kSums == IsWeightGrad<Out>::value && kLoads * (kBufs - 2) + kStores < 64, "vmcnt range");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wp = wave % NP, wq = wave / NP;

  typename Work::Way at = work.begin(block, blocks);
  if (at.done()) return;

  Operand<TP, kDepth, kPT, kWaves> op;
  Operand<TQ, kDepth, kQT, kWaves> oq;
  auto fetch_at = at;                                       // the tile being loaded, and its stages still to load
  int64_t fetch_left = 0;
  auto open = [&]() {
    if (fetch_at.done()) {
      if constexpr (!kCodes) op.none();
      oq.none();
      fetch_left = INT64_MAX;
      return;
    }
    const Item t = work.item(fetch_at);
    if constexpr (!kCodes) op.tile(t.p, g.ldp, t.p0, g.np, t.k0, t.kn, wave, lane);
    oq.tile(t.q, g.ldq, t.q0, t.q_end, t.k0, t.kn, wave, lane);
    fetch_left = t.stages;
  };
  const uint32_t lds0 = lds_addr(lds);
  auto fetched = [&]() {
    if (--fetch_left == 0) {
      work.next(fetch_at);
      open();
    }
  };

  Fragments<TP, kDepth, kPT, WP, true> fp;
  Fragments<TQ, kDepth, kQT, WQ, false> fq;
  fp.init(wp * WP, lane);
  fq.init(wq * WQ, lane);

  // this wavefront's biases (and scales) of a tile, into LDS a tile ahead of their use; two places in turn
  constexpr int kPlace = 64 * kEpilogueLoads;
  float* biases = reinterpret_cast<float*>(lds + kBufs * kStage + (L::kStores ? kWaves * Staging<WP, kWaves>::kBytes : 0)) + wave * 2 * kPlace;
  int parity = 0;
  auto fetch_biases = [&](const typename Work::Way& j) {
    if constexpr (Out::kBias) {
      const bool there = !j.done();                         // else its place is nowhere, and nothing is read
      const Item t = work.item(j);
      const int64_t pw = t.p0 + 32 * WP * wp;
      const i32x4 r = buffer_rsrc(out.bias + (int64_t)t.group * g.np, there ? (uint32_t)(g.np * 4) : 0);
      const uint32_t to = lds_addr(biases + (parity ? kPlace : 0));
#pragma unroll
      for (int l = 0; l < kBiasLoads; ++l)
        dma4(r, (uint32_t)(pw + 64 * l + lane) * 4, __builtin_amdgcn_readfirstlane(to + 256 * l));
      if constexpr (Out::kInt8) {
        const i32x4 s = buffer_rsrc(out.scale_p, there ? (uint32_t)(g.np * 4) : 0);
#pragma unroll
        for (int l = 0; l < kBiasLoads; ++l)
          dma4(s, (uint32_t)(pw + 64 * l + lane) * 4, __builtin_amdgcn_readfirstlane(to + 256 * (kBiasLoads + l)));
      }
    }
  };
  fetch_biases(at);

  // P's codes: a stage further ahead than Q
  CodesOperand<TP, kDepth, typename CodeOf<Out>::type, kWaves> codes;
  auto codes_at = at;
  int64_t codes_left = 0;
  auto open_codes = [&]() {
    if constexpr (kCodes) {
      if (codes_at.done()) {
        codes.none();
        codes_left = INT64_MAX;
        return;
      }
      const Item t = work.item(codes_at);
      codes.tile(out, t.p0, t.k0, t.kn);
      codes_left = t.stages;
    }
  };
  auto load_codes = [&]() {
    if constexpr (kCodes) {
      codes.load();
      if (--codes_left == 0) {
        work.next(codes_at);
        open_codes();
      }
    }
  };

  open();
  if constexpr (kCodes) {
    codes.init(out, g.ldp);
    open_codes();
    load_codes();
    codes.take();
    load_codes();
  }
#pragma unroll
  for (int b = 0; b < kBufs; ++b) {
    if constexpr (!kCodes) op.fetch_all(lds0 + b * kStage, wave);
    oq.fetch_all(lds0 + b * kStage + kQ, wave);
    fetched();
  }
  if constexpr (kCodes) {
#pragma unroll
    for (int i = 0; i < codes.kPairs; ++i) codes.pair(i, lds);
    codes.take();
    load_codes();
    wait_loads<0>();
  } else {
    wait_loads<kLoads * (kBufs - 1)>();
  }

  bf16x8 pf[2][WP], qf[2][WQ];                              // this step's fragments and the next one's
#pragma unroll
  for (int a = 0; a < WP; ++a) pf[0][a] = fp.read(lds, 0, a);
#pragma unroll
  for (int b = 0; b < WQ; ++b) qf[0][b] = fq.read(lds + kQ, 0, b);
  int buf = 0;
#pragma clang loop unroll(disable)
  for (bool first = true; !at.done(); first = false) {
    const Item t = work.item(at);
    work.next(at);
    using Acc = std::conditional_t<Out::kInt8, i32x16, f32x16>;
    Acc acc[WP][WQ];
    const float* place = biases + (parity ? kPlace : 0);
    if constexpr (Out::kBias) parity ^= 1;
    if constexpr (Out::kBias && !Out::kInt8) {              // the sums begin with the biases
      const float* bias = place + 8 * (lane >> 5);
#pragma unroll
      for (int a = 0; a < WP; ++a)
#pragma unroll
        for (int b = 0; b < WQ; ++b)
#pragma unroll
          for (int v = 0; v < 16; v += 4) {
            const float4 f = *reinterpret_cast<const float4*>(bias + 32 * a + 2 * (v & 8) + (v & 4));
            acc[a][b][v] = f.x, acc[a][b][v + 1] = f.y, acc[a][b][v + 2] = f.z, acc[a][b][v + 3] = f.w;
          }
      fetch_biases(at);
    } else {
#pragma unroll
      for (int a = 0; a < WP; ++a)
#pragma unroll
        for (int b = 0; b < WQ; ++b)
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[a][b][v] = 0;
      fetch_biases(at);
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
              sums[b] += t.whole ? n + c : wp ? c : n;
            }
            if (end) mine += turns;
          }
        }
        if (end) {
          // The next stage is there, and this one read by all. Vector memory operations complete in order:
          // for the first stages after a tile's stores, those are newer than the loads waited for.
          if (kStores && s < kBufs - 1 && !first) wait_loads<kLoads * (kBufs - 2) + kStores>();
          else wait_loads<kLoads * (kBufs - 2)>();
          into = lds0 + buf * kStage;
          buf = buf == kBufs - 1 ? 0 : buf + 1;
          stage = lds + buf * kStage;
        }
        const int to = end ? 0 : kk + 1;
        if (end) {
          if constexpr (kCodes) {
            codes.take();
            load_codes();
          } else {
            op.aim(into, wave);
          }
          oq.aim(into + kQ, wave);
        }
        // of the products, the first half is followed by a share of the reads each, all by one of the loads
        constexpr int kProducts = WP * WQ, kHalf = (kProducts + 1) / 2, kFrags = WP + WQ;
#pragma unroll
        for (int m = 0; m < kProducts; ++m) {
          const int a = m / WQ, b = m % WQ;
          if constexpr (Out::kInt8)                         // 32 k: both operands' bytes lie in the same order
            acc[a][b] = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, pc[a]), __builtin_bit_cast(i32x4, qc[b]),
                                                              acc[a][b], 0, 0, 0);
          else acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(pc[a], qc[b], acc[a][b], 0, 0, 0);
#pragma unroll
          for (int f = m * kFrags / kHalf; f < (m + 1) * kFrags / kHalf && f < kFrags; ++f) {
            if (f < WQ) qn[f] = fq.read(stage + kQ, to, f);
            else pn[f - WQ] = fp.read(stage, to, f - WQ);
          }
          if (end) {
#pragma unroll
            for (int l = m * kLoads / kProducts; l < (m + 1) * kLoads / kProducts; ++l) {
              if (l < kPLoads) op.fetch(l);
              else oq.fetch(l - kPLoads);
            }
          }
          if constexpr (kCodes) {                           // the next stage's values, before its end and beside the reads
            constexpr int kFree = kProducts > kHalf ? kProducts - kHalf : kProducts, kSlots = (kHalves - 1) * kFree;
            const int slot = kk * kFree + m - (kProducts - kFree);
            if (!end && m >= kProducts - kFree)
#pragma unroll
              for (int i = slot * codes.kPairs / kSlots; i < (slot + 1) * codes.kPairs / kSlots; ++i)
                codes.pair(i, lds + (buf ^ 1) * kStage);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (end) {
          if constexpr (!kCodes) op.advance();
          oq.advance();
        }
      }
      fetched();
    }
    if (Out::kBias && t.stages < kBufs) wait_own<0>();      // else a stage's wait has covered the next biases
    const int64_t qw = t.q0 + 32 * WQ * wq, pw = t.p0 + 32 * WP * wp;        // this wavefront's part
    if constexpr (!kSums) {
      unsigned char* staging = lds + kBufs * kStage + wave * Staging<WP, kWaves>::kBytes;
      if constexpr (Out::kInt8) store_scaled<WP, WQ, kWaves>(out, g, t, staging, qw, pw, lane, acc, place, 64 * kBiasLoads);
      else store_rows<WP, WQ, kWaves>(out, g, t, staging, qw, pw, lane, acc);
    } else {
      const int r = lane & 31, h = lane >> 5;
      float* gw = out.weights(g, t);
#pragma unroll
      for (int b = 0; b < WQ; ++b) {
        const int64_t q = qw + 32 * b + r;
#pragma unroll
        for (int a = 0; a < WP; ++a)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int64_t p = pw + 32 * a + 16 * half + 8 * h;
            float* at = gw + q * g.np + p;
            if (q < g.nq && p < g.np) {
#pragma unroll
              for (int e = 0; e < 2; ++e)
                reinterpret_cast<float4*>(at)[e] = make_float4(acc[a][b][8 * half + 4 * e], acc[a][b][8 * half + 4 * e + 1],
                                                               acc[a][b][8 * half + 4 * e + 2], acc[a][b][8 * half + 4 * e + 3]);
            }
          }
        // NP wavefronts and `parts` workgroups hold shares of the sum over Q, or each the whole
        const float s = sums[b] + __shfl_xor(sums[b], 32);
        const int64_t part = t.p0 / TP;
        if (h == 0 && q < g.nq && (t.whole ? part == 0 && wp == 0 : part < out.parts)) out.biases(g, t, part, wp)[q] = s;
      }
    }
  }
  wait_loads<0>();                                          // no load into LDS outlives the workgroup
}

}  // namespace
}  // namespace maestro
