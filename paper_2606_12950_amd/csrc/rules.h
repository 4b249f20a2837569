// Which tile, cut and launch a layer by role, in 8-bit integers or from kept bytes takes, by its sizes. Host code alone: every choice
// of these operators' launchers is here, so that a test without a GPU can ask which of the kernels a call runs.
#pragma once

#include <stdint.h>

namespace maestro {

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t kCus = 256;
constexpr int kDepthF32 = 16;         // k of a stage of the float32 products

// Widths that tiles of 256 fit as well as tiles of 128, nearly: those above 128, but for 257 .. 384. Measured (us, 256 / 128): grouped
// layers 100,000 x 256 -> 384 43 / 37, 1024 -> 304 108 / 97, 200,000 x 512 -> 640 190 / 196; packed gradients 100,000 x 384 -> 512 172 / 156.
inline bool fits256(int64_t width) { return 5 * cdiv(width, 128) > 8 * cdiv(width, 256); }

// Tile of a weights' gradient, of d_in and of d_out: 256 x 256 for many rows where it fits, 256 x 64 for few outputs, else 128 x 128.
// Measured (us, 256 x 256 / 128 x 128, kept bytes and then groups): 262,139 x 1024 -> 1024 545 / 687 and 540 / 637, 146,481 x 288 -> 896
// 175 / 157 and 177 / 144, 140,000 x 768 -> 512 149 / 173 and 167 / 159; 256 x 64 / 128 x 128: 100,000 x 512 -> 512 98 / 88 and 82 / 81,
// 60,000 x 256 -> 128 23.7 / 22.4 and 23.7 / 23.7, 40,000 x 512 -> 64 22.2 / 24.6.
struct WeightTile {
  int32_t tp, tq;
};
inline WeightTile weight_tile(int64_t n, int64_t d_in, int64_t d_out) {
  const int64_t large = 4 * cdiv(d_in, 256) * cdiv(d_out, 256), small = cdiv(d_in, 128) * cdiv(d_out, 128);
  if (d_in > 128 && d_out > 128 && n >= 131072 && 5 * large <= 6 * small) return {256, 256};
  return d_in > 128 && d_out <= 64 ? WeightTile{256, 64} : WeightTile{128, 128};
}

// 128 x 128 float32 tiles of a weights' gradient for many rows where they hold at most 1.2 times what 64 x 64 ones do.
inline bool weight_wide_f32(int64_t n, int64_t d_in, int64_t d_out) {
  const int64_t large = 4 * cdiv(d_in, 128) * cdiv(d_out, 128), small = cdiv(d_in, 64) * cdiv(d_out, 64);
  return d_in > 64 && d_out > 64 && n >= 32768 && 5 * large <= 6 * small;
}

// The places of the groups' weights' gradients in the workspace, one for a unit of up to `per` rows. Where groups are few, units are
// numbered as they come, a place each. Where they are more than twice what `per` goes into the rows, most are one unit, which writes its gradient
// itself, and only groups of u >= 2 units have places, u neighbouring ones from first_place on: `row`, its first row, and `end`, the next group's,
// count from the first group's. From row / per to end / per are u - 1 or more and at least one, whether units begin at the group's first row or
// at multiples of `per`; and min(group, row / per) rises by one then, so that the next group's first place is u or more further. (Numbered so throughout,
// the divisions cost every call 0.2 to 0.5 us of 12 to 15, and the widest 1 % of their time.)
constexpr int first_place(int group, int row, int per) {
  const int passed = (int)((uint32_t)row / (uint32_t)per);
  return passed + (group < passed ? group : passed);
}
inline bool shared_places(int64_t n, int64_t n_groups, int64_t per) { return n > per && n_groups > 2 * (n / per); }      // n <= per: no places
inline int64_t places_of(int64_t n, int64_t n_groups, int64_t per) {
  return shared_places(n, n_groups, per) ? first_place((int)n_groups, (int)n, (int)per) : n / per + n_groups;
}

namespace grouped_bf16 {

// Tile by how many there are, as for a layer of one group. 256 x 256 ones by eight wavefronts, two to a SIMD, or by four: the layer
// with eight 546 us, four 544 (262,139 x 1024 -> 1024, 16 groups); the input's gradient, whose mask wants registers, 612 and 575.
// The input's gradient no wider than 64 takes tiles that are not either (us, both gradients, 128 x 128 / 64 x 64: 100,000 x 64 -> 64 28.0 / 23.8, 100,000 x
// 16 -> 256 36.7 / 30.5, 200,000 x 48 -> 1024 186 / 180); the layer does not gain (63,399 x 112 -> 48 8.4 / 9.9).
inline int tile_of(bool input_grad, int64_t np, int64_t n) {
  if (input_grad && np <= 64) return 64;
  if (fits256(np) && cdiv(np, 256) * (n / 256) >= 2 * kCus) return 256;
  return cdiv(np, 128) * (n / 128) >= kCus ? 128 : 64;
}

// Tile of the weights' gradient and rows of a unit, as for a layer of one group. by_group: too few rows for a unit of them
// in every workgroup. 64 x 64 tiles and units of 512 rows of a group where four to a CU hold them all. Measured (us, 64 x 64 / 256 x 64 or 128 x 128): 300 rows in 5
// groups 256 -> 512 5.8 / 7.9, 4,000 in 4 256 -> 256 12.1 / 15.8, 8,000 in 16 512 -> 64 10.3 / 14.0, 20,000 in 60 128 -> 128 9.8 / 12.8.
struct Cut {
  int32_t tp, tq;
  int64_t k_split;
  bool by_group;
};
inline Cut cut_of(int64_t n, int64_t n_groups, int64_t d_in, int64_t d_out) {
  Cut c;
  const WeightTile tile = weight_tile(n, d_in, d_out);
  c.tp = tile.tp, c.tq = tile.tq;
  const int64_t tiles = cdiv(d_in, c.tp) * cdiv(d_out, c.tq), resident = c.tq == 256 ? 1 : 2;
  int64_t splits = kCus * resident / tiles;
  c.by_group = splits > cdiv(n, 512);
  if (c.by_group) splits = cdiv(n, 512);
  if (splits < 1) splits = 1;
  c.k_split = cdiv(cdiv(n, splits), 64) * 64;
  if ((n / 512 + n_groups) * cdiv(d_in, 64) * cdiv(d_out, 64) <= 4 * kCus) {
    c.tp = c.tq = 64;
    c.by_group = true;
    c.k_split = cdiv(cdiv(n, cdiv(n, 512)), 64) * 64;
  }
  return c;
}

// Both gradients in one launch.
inline bool paired(const Cut& c, int64_t n, int64_t d_in) { return c.tp == 64 && tile_of(true, d_in, n) == 64; }

}  // namespace grouped_bf16

namespace grouped_f32 {

// 128 x 128 tiles where there are two rounds of them, else 64 x 64, as a layer of one group.
inline bool wide(int64_t np, int64_t n) { return np > 64 && cdiv(np, 128) * (n / 128) >= 2 * kCus; }
inline bool wide_forward(int64_t np, int64_t n, int64_t nk) { return wide(np, n) && nk >= 192 && cdiv(np, 64) % 2 == 0; }

// As for a layer of one group, and twice the workgroups where each has 256 rows then (150,000 x 80 -> 160 in 10 groups 92 / 83 us). by_group: too few rows for a unit of 256 in every workgroup; units of 128 then (us, weights' gradient, 256 / 128 / 64 rows:
// 4,096 x 64 -> 128 in 3 groups 14.7 / 11.4 / 10.6, with the input's 14.8 / 11.7 / 12.8, 20,000 x 128 -> 128 in 30 both 29.8 / 26.7 / 26.7).
struct Cut {
  bool wide, by_group;
  int64_t k_split;                   // rows of a unit
};
inline Cut cut_of(int64_t n, int64_t d_in, int64_t d_out) {
  Cut c;
  c.wide = weight_wide_f32(n, d_in, d_out);
  const int64_t t = c.wide ? 128 : 64, tiles = cdiv(d_in, t) * cdiv(d_out, t);
  int64_t splits = (c.wide || 4 * kCus / tiles > n / 256 ? 2 : 4) * kCus / tiles;
  c.by_group = splits > cdiv(n, 256);
  const int64_t least = n <= 256 ? 256 : 128;
  if (splits > cdiv(n, least)) splits = cdiv(n, least);
  if (splits < 1) splits = 1;
  c.k_split = cdiv(cdiv(n, splits), kDepthF32) * kDepthF32;
  return c;
}

// Both gradients in one launch.
inline bool paired(const Cut& c, int64_t n, int64_t d_in) { return c.by_group && !c.wide && !wide(d_in, n); }

// The join of a group's units: a quad's dealt out over 16 threads where there are few values.
inline bool join_dealt(int64_t n, int64_t n_groups, int64_t k_split, int64_t size, int64_t d_out) {
  return cdiv(size / 4 + d_out / 4, 256) * n_groups <= kCus / 2 && n / k_split > 8;
}

}  // namespace grouped_f32

namespace packed_bf16 {

// As for the gradients of an input in bfloat16, but the input's 64 wide where it is no wider (us, 128 x 128 / 64 x 64, both gradients: 100,000 x 64
// -> 64 24.6 / 19.8, 100,000 x 16 -> 256 36.4 / 33.6, 200,000 x 48 -> 1024 190 / 196, 40,000 x 64 -> 512 34.5 / 29.0), and for little work 64 x 64 tiles of the weights' gradient, with splits of 256 rows
// or more, where four to a CU hold them all. Measured (us, both gradients, 64 x 64 with 256 / 512 rows / the larger tiles): 300 x 256 -> 512
// 9.1 / 6.8 (one split) / 11.7 (weights), 1,000 x 1024 -> 64 9.3 / 11.5, 4,000 x 256 -> 256 11.5 / 12.8, 30,000 x 64 -> 128 13.8 / 15.0 / 17.0 (weights).
// A tile of 64 is the input's in the launch of both gradients.
inline int tile_of(int64_t np, int64_t nq) {
  if (np <= 64) return 64;
  if (fits256(np) && cdiv(np, 256) * cdiv(nq, 256) >= 2 * kCus) return 256;
  return cdiv(np, 128) * cdiv(nq, 128) >= kCus ? 128 : 64;
}

struct Cut {
  int32_t tp, tq;
  int64_t k_split, splits;
  int32_t parts;
};
inline Cut cut_of(int64_t n, int64_t d_in, int64_t d_out) {
  Cut c;
  const WeightTile tile = weight_tile(n, d_in, d_out);
  c.tp = tile.tp, c.tq = tile.tq;
  int64_t tiles = cdiv(d_in, c.tp) * cdiv(d_out, c.tq), most = kCus * (c.tq == 256 ? 1 : 2), least = 512;
  const int64_t small = cdiv(d_in, 64) * cdiv(d_out, 64), few = n <= 512 ? 512 : 256;
  if (small * cdiv(n, few) <= 4 * kCus) c.tp = c.tq = 64, tiles = small, most = 4 * kCus, least = few;
  int64_t splits = most / tiles;
  if (splits > cdiv(n, least)) splits = cdiv(n, least);
  if (splits < 1) splits = 1;
  c.k_split = cdiv(cdiv(n, splits), 64) * 64;
  c.splits = cdiv(n, c.k_split);
  c.parts = c.splits > 1 ? (int32_t)cdiv(d_in, c.tp) : 1;
  return c;
}

}  // namespace packed_bf16

namespace packed_f32 {

inline bool wide(int64_t np, int64_t nq) { return np > 64 && nq > 64 && cdiv(np, 128) * cdiv(nq, 128) >= 2 * kCus; }

// The weights' gradient's tiles as for an input in float32; the rows split so that there are about two workgroups a CU, four where each has 256 rows
// then. Measured (us, two / four): 150,000 x 80 -> 160 98 / 88, 66,255 x 256 -> 16 37.8 / 34.1, 131,365 x 48 -> 240 62 / 57, 200,000 x 64 -> 64 32.5 / 32.7.
constexpr int64_t kLeastRows = 64;
struct Cut {
  bool wide;
  int64_t k_split, splits;
};
inline Cut cut_of(int64_t n, int64_t d_in, int64_t d_out) {
  Cut c;
  c.wide = weight_wide_f32(n, d_in, d_out);
  const int64_t t = c.wide ? 128 : 64, tiles = cdiv(d_in, t) * cdiv(d_out, t);
  int64_t splits = (c.wide || 4 * kCus / tiles > n / 256 ? 2 : 4) * kCus / tiles;
  if (splits > cdiv(n, kLeastRows)) splits = cdiv(n, kLeastRows);
  if (splits < 1) splits = 1;
  c.k_split = cdiv(cdiv(n, splits), kDepthF32) * kDepthF32;
  c.splits = cdiv(n, c.k_split);
  return c;
}

// Both gradients in one launch.
inline bool paired(const Cut& c, int64_t n, int64_t d_in) { return !c.wide && !wide(d_in, n); }

}  // namespace packed_f32

namespace int8 {

// Lanes of a row, a power of two, and units of 8 values of each, kept in registers up to 8.
struct RowLanes {
  int32_t lanes, units;              // units 1, 2, 4 or 8; 0: more, read twice
};
inline RowLanes row_lanes(int32_t d) {
  int32_t lanes = 2;
  while (lanes < 64 && lanes < d / 8) lanes *= 2;
  const int32_t each = (d / 8 + lanes - 1) / lanes;
  return {lanes, each <= 1 ? 1 : each <= 2 ? 2 : each <= 4 ? 4 : each <= 8 ? 8 : 0};
}

// 256 x 256 tiles by eight wavefronts, two to a SIMD, so that one's scaling and stores run under the other's products; by four, which
// read a quarter less of LDS, where a dozen rounds of them or more let the matrix cores' power set the clock. Measured (us with the rows'
// quantisation, eight / four): 262,139 x 1024 -> 1024 (16 rounds) 500 / 484, 120,001 x 768 -> 1008 (7) 218 / 224, 65,536 x 512 -> 512 (2)
// 57 / 58; without it 65,536 x 256 -> 512 23.5 / 27.4, 200,000 x 256 -> 256 39.1 / 43.5.
struct ProductTile {
  int32_t tile, wavefronts;
};
inline ProductTile product_tile(int64_t np, int64_t nq) {
  const int64_t large = cdiv(np, 256) * cdiv(nq, 256);
  if (np > 128 && large >= 12 * kCus) return {256, 4};
  if (np > 128 && large >= 2 * kCus) return {256, 8};
  return cdiv(np, 128) * cdiv(nq, 128) >= kCus ? ProductTile{128, 4} : ProductTile{64, 4};
}

}  // namespace int8

}  // namespace maestro
