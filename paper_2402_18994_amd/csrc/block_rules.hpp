// How calls of the gated block's operators are cut and which kernels they take (host arithmetic only): group norm, gated linear
// recurrence, gated units.
#pragma once
#include <algorithm>

#include "ops_host.hpp"

namespace snn {

inline size_t type_bytes(int32_t type) { return type == SNN_TYPE_FP32 ? 4 : 2; }

// ---------------------------------------------------------------- group norm
constexpr int AHEAD = 4, AHEAD_BWD = 2;      // rows in flight a thread (reverse: of x and dy each)

// How a call is cut, for `vec` channels a vector.
struct NormCut {
  int nt, tpr_log2, K, R, loops, blocks;       // threads; threads a row (log2); column blocks; rows a thread; lots; workgroups a unit and group
  bool chunks;
  int long_row;                                // vectors a lane where a wavefront has a row (or AGAIN_ROW), 0: otherwise
};
constexpr int AGAIN_ROW = -1;
inline NormCut norm_cut(const snn_norm_args &a, int vec, bool backward) {
  const size_t z = a.type == SNN_TYPE_FP32 ? 4 : 2;
  const int C = a.D / a.groups, slots = vec * z == 16 ? 8 : 16;
  const int64_t rows = a.per_step ? (int64_t)a.T * a.B : a.T, units = a.per_step ? 1 : a.B;
  NormCut c;
  auto blocks_of = [&](int64_t each) { return std::max<int64_t>(1, (rows + each - 1) / each); };
  c.nt = 256;
  c.tpr_log2 = 0;
  while ((vec << c.tpr_log2) < C && (1 << c.tpr_log2) < c.nt) ++c.tpr_log2;
  c.K = (C + (vec << c.tpr_log2) - 1) / (vec << c.tpr_log2);
  c.loops = 1;
  c.chunks = false;
  c.long_row = 0;
  if (a.per_step && C > 64 * vec) {
    const int need = (C + 64 * vec - 1) / (64 * vec);
    const int most = vec <= 2 ? 64 / vec : 16;
    // Reverse no more than 4 vectors, as x and dy and what is formed of them fill the registers.  (us, held and loaded again: 8192 rows of
    // 4096, fp32, forward 45 and 79, reverse 175 and 163; 4800 of 4095, 43 and 62, 216 and 122; 4096 of 4096, bf16, 18.7 and 18.9, 62 and 49.)
    c.long_row = need <= 4 ? 4 : backward ? AGAIN_ROW : need <= 16 ? 16 : need <= most ? most : AGAIN_ROW;
    const int64_t across = (a.D + 64 * vec - 1) / (64 * vec);
    c.R = 256;                                 // rows of a chunk of dw and db, in workgroups of 64 vectors of columns
    while (c.R > 16 && blocks_of(c.R) * across < 1024) c.R /= 2;
    while (blocks_of(c.R) > 32768) c.R *= 2;
    c.blocks = (int)blocks_of(c.R);
    return c;
  }
  if (a.per_step) {
    const int64_t rp = c.nt >> c.tpr_log2;
    c.R = blocks_of(rp * 2) * a.groups >= 512 ? 2 : 1;
    const int64_t n = blocks_of(rp * c.R);
    while (c.loops < 64 && blocks_of(rp * c.R * c.loops * 2) * a.groups >= 2048) c.loops *= 2;
    c.blocks = (int)((n + c.loops - 1) / c.loops);
    return c;
  }
  c.R = slots;
  c.blocks = 1;
  // A sequence's group at once, where the registers of 256 threads hold it, or those of 512 and there are 64 groups at least; reverse with
  // 16-byte vectors never, since x and dy with what is formed of them do not
  // fit.  (us of a forward and a reverse call: 51 of 257 steps, 130 channels in 5 groups, fp32, 7.8 and 16.1, in chunks 12.6 and 18.6; 16 of
  // 500 steps, 512 channels in 8, bf16, reverse at once 41.8, in chunks 22.2.)
  if (c.K == 1 && !(backward && vec * z == 16)) {
    if (blocks_of((256 >> c.tpr_log2) * slots) == 1) return c;
    if (units * a.groups >= 64 && blocks_of((512 >> c.tpr_log2) * slots) == 1) {
      c.nt = 512;
      return c;
    }
  }
  const int64_t rp = 256 >> c.tpr_log2;
  c.chunks = true;
  c.R = 64;                                    // rows a thread: as many as leave 512 workgroups (1024: 2 to 25 % slower)
  while (c.R > AHEAD && blocks_of(rp * c.R) * units * a.groups < 512) c.R /= 2;
  c.blocks = (int)blocks_of(rp * c.R);
  return c;
}
inline int norm_vector(const snn_norm_args &a, const snn_norm_grads *g) {
  const size_t z = a.type == SNN_TYPE_FP32 ? 4 : 2;
  for (int vec : {(int)(16 / z), 2}) {
    auto take = [&](const snn_rows &r) { return rows_take(r, a.T, a.B, vec, z); };
    if (a.D / a.groups % vec == 0 && take(a.x) && (g ? take(g->dy) && take(g->dx) : take(a.y))) return vec;
  }
  return 1;
}

// ---------------------------------------------------------------- gated linear recurrence
constexpr int STEPS = 8;                     // a run; the state before every run is what `saved` holds
constexpr int CH = 64;                       // channels of a workgroup

// How time is cut: `waves` wavefronts a workgroup and segments of `tiles` tiles.  Segments cost a second reading, and are taken where
// there are fewer (sequence, 64 channels) than workgroups that keep the chip busy: us of a forward (reverse) call in one piece and cut, by
// their number and steps, bf16: 64 of 1024 27 and 18 (52 and 28), of 4096 101 and 55 (185 and 71); 128 of 1024 29 and 32 (54 and 43), of 4096 103 and 95
// (201 and 141); 140 of 8192 217 and 248 (396 and 356); 153 of 333 15.5 and 18.4 (27 and 29); 180 of 200 11.7 and 16.9 (22 and 29).  fp32: 128 of
// 4096 150 and 212 (299 and 259), 153 of 333 15.2 and 20.1 (30 and 29), 180 of 200 13.3 and 18.7 (26 and 28).  The number of steps is not looked at:
// few and short ones (64 of 128: 11.5 and 16.7, reverse 19 and 23) would be faster in one piece.  As many segments as make 1024 workgroups, reverse 512
// (16 of 8192 steps, bf16, with 1024 and with 512: 36 and 37, reverse 51 and 42).
struct RecCut {
  int waves, tiles, nseg;
};
inline RecCut recurrence_cut(const snn_recurrence_args &a, int vec, bool backward) {
  RecCut c;
  const int64_t groups = (int64_t)(a.D + CH - 1) / CH * a.B;
  const bool enough = groups >= (backward ? 144 : 128);
  c.waves = !enough || a.T <= 64 ? 4 : backward ? 8 : 16;
  const int tile = c.waves * vec * STEPS;                  // (Shape::TILE)
  const int all = std::max(1, (int)(((int64_t)a.T + tile - 1) / tile));
  const int64_t want = enough ? 1 : std::min<int64_t>(64, ((backward ? 512 : 1024) + groups - 1) / groups);
  c.tiles = (int)((all + want - 1) / want);
  c.nseg = (all + c.tiles - 1) / c.tiles;
  return c;
}
// Four bytes a lane: of bfloat16 two channels where rows allow it, of fp32 one (1024 steps of 8 x 2048 channels, two and one: 47.8 and 44.2 us,
// reverse 102 and 96).
inline bool two_channels(const snn_recurrence_args &a, const snn_recurrence_grads *g) {
  const size_t z = type_bytes(a.type);
  auto take = [&](const snn_rows &r) { return rows_take(r, a.T, a.B, 2, z); };
  return a.type == SNN_TYPE_BF16 && a.D % 2 == 0 && take(a.x) && take(a.i) && take(a.r) && (g ? take(g->dy) && take(g->dx) && take(g->di) && take(g->dr) : take(a.y));
}

// ---------------------------------------------------------------- gated units
constexpr int KS = 64;                       // k of a stage: a row of it is 128 bytes
constexpr int FEW = 64;                      // rows that a workgroup of the kernels for few rows takes
constexpr int KEPT = 32 * 32 * 2;            // values of G and U of 32 rows by 32 units

inline int panels_of(int64_t n) { return (int)((n + KS - 1) / KS); }
inline int64_t panel_bytes(int64_t rows, int64_t k, int planes) { return rows * panels_of(k) * 128 * planes; }
inline int pitch_of(int n) { return (n + 3) & ~3; }

// x as it lies: one stride between rows, 16-byte pieces, whole stages, and tiles whose offsets fit 31 bits.
inline bool x_direct(const snn_units_args &a, int64_t &row) {
  const bool one = a.T <= 1 || a.B <= 1 || a.x.stride_t == a.x.stride_b * a.B;
  row = (a.B > 1 ? a.x.stride_b : a.T > 1 ? a.x.stride_t : a.D) * 2;
  return a.type == SNN_TYPE_BF16 && a.D % KS == 0 && one && aligned(a.x.p, 16) && row % 16 == 0 && row >= 0 && row < (1 << 22);
}
inline bool weights_direct(const snn_units_args &a) { return a.type == SNN_TYPE_BF16 && a.D % KS == 0 && aligned(a.gate, 16) && aligned(a.up, 16); }

struct Tile {
  int bm, bn;                                // of the product; wide: 256 x 256
  bool wide;
};
inline Tile tile_of(int64_t m, int64_t n) {
  const int64_t wide = ((m + 255) / 256) * ((n + 255) / 256);
  return wide >= 192 ? Tile{256, 256, true} : Tile{128, 128, false};
}
struct Product {
  Tile tile;
  int mt, nt, splits;
};
inline size_t part_bytes(const Product &p, int64_t m, int n) { return p.splits > 1 ? rup256((size_t)p.splits * m * pitch_of(n) * 4) : 0; }

inline int64_t kept_size(const snn_units_args &a) { return ((int64_t)a.T * a.B + 31) / 32 * ((a.F + 31) / 32) * KEPT; }
// The forward product.  Its parts' sums cost 16 bytes a unit and part, and a launch: where tiles fill a third of
// the chip at most, and have 32 stages (us without and with: 300 rows, 2048 -> 1024, bf16 20.4 and 15.9, fp32 95 and 44; 1000 rows,
// 1000 -> 300, bf16, 16 stages 18.1 and 19.7; 2000 rows, 2048 -> 512, 128 tiles 21.6 and 22.5).
inline Product units_product(const snn_units_args &a) {
  const int64_t M = (int64_t)a.T * a.B, stages = (int64_t)panels_of(a.D) * (a.type == SNN_TYPE_FP32 ? 6 : 1);
  Product p;
  p.tile = tile_of(M, 2 * (int64_t)a.F);
  p.mt = (int)((M + p.tile.bm - 1) / p.tile.bm);
  p.nt = (a.F + p.tile.bn / 2 - 1) / (p.tile.bn / 2);
  const int64_t tiles = std::max<int64_t>(1, (int64_t)p.mt * p.nt);
  p.splits = stages >= 32 && tiles <= 85 ? (int)std::min<int64_t>({stages / 8, 16, 256 / tiles}) : 1;
  return p;
}

// Stages in LDS.  Small tiles, up to one a compute unit: four, three of them on their way; more: two, and two workgroups a compute unit.
inline int gemm_stages(int64_t workgroups, bool wide) { return !wide && workgroups <= 256 ? 4 : 2; }

struct UnitsPlan {                           // of the reverse pass
  int64_t M;
  int planes, segs;
  Product dx, dw;
  size_t rows, cols, xt, wt, part_dx, part_dw;   // bytes of each piece of the workspace
};
// Both products are one launch.  Small tiles, and parts of the contraction, where there are too few tiles for the chip: so many parts
// that the workgroups (one a compute unit of wide tiles, two of small ones) have about the same number of stages, eight at least.
inline UnitsPlan units_plan(const snn_units_args &a) {
  UnitsPlan u;
  u.M = (int64_t)a.T * a.B;
  u.planes = a.type == SNN_TYPE_FP32 ? 3 : 1;
  u.segs = u.planes == 3 ? 6 : 1;
  const int64_t F2 = 2 * (int64_t)panels_of(a.F) * KS;
  auto tiles = [](int64_t m, int64_t n, int b) { return (m + b - 1) / b * ((n + b - 1) / b); };
  const bool wide = tiles(u.M, a.D, 256) + tiles(2 * (int64_t)a.F, a.D, 256) >= 192;
  const int64_t stages_dx = (int64_t)2 * panels_of(a.F) * u.segs, stages_dw = (int64_t)panels_of(u.M) * u.segs;
  const int b = wide ? 256 : 128;
  const int64_t all = tiles(u.M, a.D, b) * stages_dx + tiles(2 * (int64_t)a.F, a.D, b) * stages_dw, each = std::max<int64_t>(8, all / (wide ? 256 : 512));
  auto product = [&](int64_t m, int64_t stages) {
    Product p;
    p.tile = Tile{b, b, wide};
    p.mt = (int)((m + b - 1) / b);
    p.nt = (a.D + b - 1) / b;
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(16, stages / each));
    return p;
  };
  u.dx = product(u.M, stages_dx);
  u.dw = product(2 * (int64_t)a.F, stages_dw);
  u.rows = rup256(panel_bytes(u.M, F2, u.planes));
  u.cols = rup256(panel_bytes(2 * (int64_t)a.F, u.M, u.planes));
  u.xt = rup256(panel_bytes(a.D, u.M, u.planes));
  u.wt = rup256(panel_bytes(a.D, F2, u.planes));
  u.part_dx = part_bytes(u.dx, u.M, a.D);
  u.part_dw = part_bytes(u.dw, 2 * (int64_t)a.F, a.D);
  return u;
}

// Up to 128 rows, of fp32 256, which the tiles would lay out first (us here and as tiles, 2048 -> 4096: bf16, 128 rows 16.8 and 19.4; fp32, 256
// rows 90 and 114; 2048 -> 1024: 8.7 and 15.5, 23 and 44).
inline bool few_rows(const snn_units_args &a) { return (int64_t)a.T * a.B <= (a.type == SNN_TYPE_FP32 ? 4 * FEW : 2 * FEW); }
// Blocks of 16 rows that a workgroup takes.
inline int few_blocks(int rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : FEW / 16; }
// Rows in 16-byte pieces, those of x within 2^30 bytes of the first.
inline bool few_in_pieces(const snn_units_args &a) {
  const int z = (int)type_bytes(a.type), e = 16 / z;
  auto apart = [](int n, int64_t stride) { return n <= 1 ? 0 : stride < 0 || stride > (1 << 30) ? (int64_t)1 << 40 : (n - 1) * stride; };
  return a.D % e == 0 && aligned(a.gate, 16) && aligned(a.up, 16) && rows_take(a.x, a.T, a.B, e, z) && (apart(a.T, a.x.stride_t) + apart(a.B, a.x.stride_b)) * z < (1 << 30);
}

}  // namespace snn
