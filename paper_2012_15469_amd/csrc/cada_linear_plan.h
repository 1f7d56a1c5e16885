// How a layer's products are cut into tiles and parts, which way their operands are read and what that takes of the workspace: plain C++ without
// device code, so that a test can go over it on the host.
#pragma once

#include <algorithm>
#include <cmath>

#include "cada_ops_sizes.h"

namespace cada {

constexpr int kStepBytes = 128;      // of a row per step of the contraction: 64 bf16 or 32 float32
constexpr int kFewRows = 2;          // rows that are a read of the weights
constexpr int64_t eights(int64_t n) { return (n + 7) / 8 * 8; }

constexpr int kCUs = 256;

// How a product is cut: the tile's edge, and into how many parts its contraction.
struct Cut { int tile, splits; int64_t k_per_split; };

// What a tile costs, in microseconds, measured (one product of random values, whole tiles, operands in the caches): a step alone on its CU, what all CUs at work add to
// it, a step's share of a full CU, and the tile's way in and out.  At 8192 x 4096 x 4096 bf16: 256 x 256 tiles 1220 TFLOP/s, 128 x 128 1080, 64 x 64 640; a single
// tile per CU: 870 (128), 460 (64).  Float32 is bound by the matrix instructions at any of them (146 TFLOP/s, 64 x 64 as 128 x 128), so it takes the smallest.
// These are of bare products: what an epilogue reads and writes is in none of them (8192 x 784 x 512 bf16 with z kept: 9.9 us by the estimate, 15.6 measured; the gradients of
// 120 x 784 x 500 float32: 4.8 and 8.8), so times are compared with times, not with clocks.
struct TileCost { int tile, slots; double alone, crowd, share, ends; };
constexpr TileCost kCostBf16[] = {{32, 5, 0.135, 0.05, 0.13, 1.0}, {64, 5, 0.20, 0.05, 0.215, 1.7}, {128, 2, 0.40, 0.13, 0.46, 3.0}, {256, 1, 1.1, 0.57, 1.68, 7.5}};
constexpr TileCost kCostF32[] = {{32, 5, 0.21, 0.02, 0.155, 1.1}, {64, 5, 0.51, 0.05, 0.50, 1.3}};
// Through registers (up to 64 x 64): 8192 x 4001 x 2003 bf16 340 us where 4000 x 2000 takes 108 directly, float32 1100 and 960.
constexpr TileCost kCostBf16Registers[] = {{32, 5, 0.30, 0.03, 0.16, 1.7}, {64, 5, 0.35, 0.1, 0.30, 2.1}}, kCostF32Registers[] = {{32, 5, 0.44, 0.03, 0.24, 1.3}, {64, 5, 0.69, 0.05, 0.57, 2.2}};
constexpr double kJoinLaunch = 4.0, kJoinBytesPerUs = 3.5e6;

struct Shape { int64_t M, N, K; };
constexpr int64_t kMostTiles = ((int64_t)1 << 23) - 8;        // of a product: 512 threads each, two products, less than 2^32 threads in a launch
// The cheapest cut of one or two products in one launch (one tile for both) by that estimate, which it returns; tiles up to `widest`.  `more_ends`: what each tile's way out costs besides.
inline double cut(const Shape *s, int n, int type, bool direct, int widest, Cut *out, int most_splits = 32, const double *more_ends = nullptr) {
  const int64_t step = kStepBytes / (int64_t)type_bytes(type);
  const TileCost *costs = type == CADA_BF16 ? (direct ? kCostBf16 : kCostBf16Registers) : direct ? kCostF32 : kCostF32Registers;
  const int n_costs = type == CADA_BF16 && direct ? 4 : 2;
  int64_t steps[2] = {0, 0};
  for (int i = 0; i < n; ++i) steps[i] = ceil_div(s[i].K, step);
  double best = 1e300;
  for (int c = 0; c < n_costs; ++c) {
    const TileCost &t = costs[c];
    if (t.tile > widest) break;
    // each product's splits that may help (none that leave less than two steps, or make more tiles than two, for a product alone six, for every CU), with tiles, steps and the join's time
    struct Option { int splits; double tiles, steps, join; } opt[2][16];
    int n_opt[2] = {0, 0};
    for (int i = 0; i < n; ++i) {
      const int64_t tiles = ceil_div(s[i].M, t.tile) * ceil_div(s[i].N, t.tile);
      for (int k : {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 16, 24, 32}) {
        if (k > most_splits || (k > 1 && (steps[i] < 2 * k || tiles * k > (n == 1 ? 6 : 2) * kCUs))) break;
        if (tiles > kMostTiles) break;
        opt[i][n_opt[i]++] = Option{k, (double)(tiles * k), (double)ceil_div(steps[i], k), k > 1 ? (k * 4.0 + 2.0) * (double)s[i].M * (double)s[i].N / kJoinBytesPerUs : 0.0};
      }
    }
    if (n_opt[0] == 0 || (n > 1 && n_opt[1] == 0)) continue;      // (too many of the smallest tiles for one launch)
    for (int i = 0; i < n_opt[0]; ++i) {
      for (int j = 0; j < (n > 1 ? n_opt[1] : 1); ++j) {
        const Option &a = opt[0][i], *b = n > 1 ? &opt[1][j] : nullptr;
        const double tiles = a.tiles + (b ? b->tiles : 0.0), most = b ? std::max(a.steps, b->steps) : a.steps, join = a.join + (b ? b->join : 0.0);
        const double mean = (a.tiles * a.steps + (b ? b->tiles * b->steps : 0.0)) / tiles, per_cu = std::ceil(tiles / kCUs);
        const double e = std::max(most * (t.alone + t.crowd * std::min(1.0, tiles / kCUs)), per_cu * mean * t.share) + t.ends * std::ceil(per_cu / t.slots) + (more_ends ? more_ends[c] * per_cu : 0.0) + (join > 0.0 ? join + kJoinLaunch : 0.0);
        if (e >= best) continue;
        best = e;
        for (int q = 0; q < n; ++q) {
          const int64_t per = ceil_div(steps[q], (q == 0 ? a : *b).splits);
          out[q] = Cut{t.tile, (int)ceil_div(steps[q], per), per * step};
        }
      }
    }
  }
  return best;
}
// What a copy of a table to aligned rows costs, in the same microseconds (a launch for one or two of them).
constexpr double kPackLaunch = 4.0, kPackBytesPerUs = 3.5e6;
inline double pack_cost(int64_t rows, int64_t cols, size_t elem) { return 2.0 * elem * (double)rows * (double)cols / kPackBytesPerUs; }
inline int64_t packed_ld(int64_t cols) { return ceil_div(cols, 8) * 8; }
// Tiles whose rows of a copy (or of dz) lie within offsets of 32 bits; those of up to 128 do at any width that a call may have (2^24).
inline int widest_tile(int64_t cols, size_t elem) { return 256 * packed_ld(cols) * (int64_t)elem < (int64_t)1 << 32 ? 256 : 128; }
inline size_t packed_bytes(int64_t rows, int64_t cols, size_t elem) { return ops_align((size_t)rows * packed_ld(cols) * elem); }

inline size_t partial_bytes(const Cut &c, int64_t M, int64_t N) { return c.splits > 1 ? ops_align((size_t)c.splits * M * eights(N) * 4) : 0; }

// Whether a table can be read by LDS-direct loads: rows on 16-byte boundaries, offsets of a tile in 32 bits, and, read across the contraction, whole pieces.
inline bool direct_kc(const void *p, int64_t ld, size_t elem) { return aligned16(p, ld, elem) && 128 * ld * (int64_t)elem < (int64_t)1 << 31; }
inline bool direct_oc(const void *p, int64_t ld, int64_t cols, size_t elem) { return direct_kc(p, ld, elem) && cols % (int64_t)(16 / elem) == 0; }

// Whether a table is too small for a read of 16 bytes, or a tile of it too large for offsets in 32 bits.
inline bool no_tiles(int64_t rows, int64_t ld, int64_t cols, size_t elem) { return ((rows - 1) * ld + cols) * (int64_t)elem < 16 || 64 * ld * (int64_t)elem >= (int64_t)1 << 32; }

// Rows and outputs that are a read of the weights; more rows cost little or no more as 32 x 32 tiles (4 x 1024 x 4096 bf16 7.4 us as rows, 6.0 as tiles, from
// memory 9.8 and 7.9; float32 8.5 and 10.8, 13.4 and 13.3), and more outputs would make a second workgroup for some CUs (1 x 4096 x 50000 bf16 118 us as rows,
// 91 as tiles; float32 186 and 157).
inline bool few_rows(int64_t rows, int64_t out) { return rows <= kFewRows && out <= 64 * kCUs; }
// Columns of a workgroup there: a line of memory of bf16 weights (half a line each from two: 4096 x 4096 17 us, not 11); of float32 ones a line, for twice the workgroups, or
// two lines where that fills the CUs (single row from memory, contraction not split: 4096 x 1024 28 us with 32 columns and 36 with 64, 8192 x 16384 127 and 104).
inline int few_columns(size_t elem, int64_t out) { return elem == 2 || out > 32 * kCUs ? 64 : 32; }
// Their contraction is split where CUs would stand idle and a workgroup have more than two reads of memory one after the other: a join costs 3 us, 1024 rows of weights 4 where they
// come from memory (single row, bf16, from memory: 4096 x 1024 19.5 -> 11.2 us, 3000 x 1000 17.0 -> 11.5, 16384 x 4096 71 -> 32; 2048 x 2048 11.8 -> 11.1, and within L2 7.0 -> 8.7).
inline Cut cut_few(size_t elem, int64_t in, int64_t out) {
  const int64_t groups = ceil_div(out, few_columns(elem, out)), most = in <= 2 * 1024 ? 1 : std::min(kCUs / groups, ceil_div(in, 1024));
  const int64_t per = ceil_div(ceil_div(in, std::clamp<int64_t>(most, 1, 16)), 1024) * 1024;
  return Cut{64, (int)ceil_div(in, per), per};
}

struct ForwardPlan { bool few, by_element, direct, pack_x, pack_w; Cut cut; size_t off_x, off_w, bytes; };
inline ForwardPlan plan_forward(const cada_linear *a) {
  ForwardPlan f{};
  if (a->rows == 0) return f;
  f.few = few_rows(a->rows, a->out);
  const size_t elem = type_bytes(a->type);
  f.cut = f.few ? cut_few(elem, a->in, a->out) : Cut{64, 1, a->in};
  f.by_element = no_tiles(a->rows, a->ldx, a->in, elem) || no_tiles(a->in, a->ldw, a->out, elem);
  if (f.few) f.bytes = partial_bytes(f.cut, a->rows, a->out);
  if (f.few || f.by_element) return f;
  const bool x_direct = direct_kc(a->x, a->ldx, elem), w_direct = direct_oc(a->w, a->ldw, a->out, elem);
  const Shape s = {a->rows, a->out, a->in};
  f.direct = x_direct && w_direct;
  const int widest = widest_tile(a->in, elem);
  const double time = cut(&s, 1, a->type, f.direct, widest, &f.cut);
  if (!f.direct) {
    Cut c;
    const double packed = cut(&s, 1, a->type, true, widest, &c) + kPackLaunch + (x_direct ? 0 : pack_cost(a->rows, a->in, elem)) + (w_direct ? 0 : pack_cost(a->in, a->out, elem));
    if (packed < time) {
      f.direct = true; f.pack_x = !x_direct; f.pack_w = !w_direct;
      f.cut = c;
    }
  }
  f.off_x = partial_bytes(f.cut, a->rows, a->out);
  f.off_w = f.off_x + (f.pack_x ? packed_bytes(a->rows, a->in, elem) : 0);
  f.bytes = f.off_w + (f.pack_w ? packed_bytes(a->in, a->out, elem) : 0);
  return f;
}

// Below this many operations (both gradients), dz is formed on its way into the products' tiles: one launch for three, with tiles that read their operands
// through registers and each form the part of dz that they need.  bf16, us (the three launches): 128 x 362 x 286 12.0 (14.2), 16 x 128 x 128 7.6 (8.6); above it the
// other way round: 120 x 784 x 500 18.3 (15.9), 128 x 784 x 512 15.6 (10.0).
constexpr double kSmallGradients = 1e8;

struct BackwardPlan {
  bool small, by_element, own_dz, direct, pack_x, pack_w;
  Cut dx, dw;
  int signal_lanes;
  int64_t signal_columns, lddz, rows_per_block, row_blocks;
  size_t off_db, off_dx, off_dw, off_x, off_w, bytes;
};
inline BackwardPlan plan_backward(const cada_linear_grad *a) {
  BackwardPlan b{};
  if (a->rows == 0) return b;
  const int64_t rows = a->rows, in = a->in, out = a->out;
  const size_t elem = type_bytes(a->type);
  const bool products = a->dx || a->dw;
  b.dx = Cut{64, 1, out};
  b.dw = Cut{64, 1, rows};
  b.lddz = ceil_div(out, 8) * 8;
  // What dx and dw read by tiles: w and x, and dy and pre, but for dx and db without dw, where the pass that sums db writes dz as well (or dy itself will do: then its rows are whole pieces).
  const bool signal_too_small = no_tiles(rows, a->lddy, out, elem) || (a->act != CADA_ACT_NONE && no_tiles(rows, a->ldpre, out, elem)), w_too_small = a->dx && no_tiles(in, a->ldw, out, elem);
  const bool dz_too_small = ((rows - 1) * b.lddz + out) * (int64_t)elem < 16;
  b.by_element = a->dw ? signal_too_small || w_too_small || no_tiles(rows, a->ldx, in, elem) : w_too_small || (a->dx && (a->db ? dz_too_small : signal_too_small));
  if (b.by_element) {
    if (a->dw || !a->db) return b;
  } else {
    b.small = products && (a->dw || !a->db) && 4.0 * rows * in * out < kSmallGradients;
    // dz in the workspace, unless dy itself will do
    b.own_dz = products && !b.small && (a->act != CADA_ACT_NONE || !direct_oc(a->dy, a->lddy, out, elem));
    const bool w_direct = !a->dx || direct_kc(a->w, a->ldw, elem), x_direct = !a->dw || direct_oc(a->x, a->ldx, in, elem);
    b.direct = !b.small && w_direct && x_direct;
    const Shape s[2] = {{rows, in, out}, {in, out, rows}};
    const int n = (a->dx ? 1 : 0) + (a->dw ? 1 : 0);
    Cut c[2], d[2];
    if (n > 0) {
      const Shape *first = a->dx ? s : s + 1;
      const int widest = a->dx ? widest_tile(out, elem) : 256;
      const double time = cut(first, n, a->type, b.direct, widest, c);
      if (!b.small && !b.direct) {
        const double packed = cut(first, n, a->type, true, widest, d) + kPackLaunch + (x_direct ? 0 : pack_cost(rows, in, elem)) + (w_direct ? 0 : pack_cost(in, out, elem));
        if (packed < time) {
          b.direct = true; b.pack_x = !x_direct; b.pack_w = !w_direct;
          c[0] = d[0]; c[1] = d[1];
        }
      }
      if (a->dx) b.dx = c[0];
      if (a->dw) b.dw = c[n - 1];
    }
  }
  // (workgroups for every CU several times over, but no more parts of the column sums than a workgroup's rows at a time, or two, make)
  while (b.signal_lanes < 5 && (8 << b.signal_lanes) < out) ++b.signal_lanes;
  const int64_t high = 256 >> b.signal_lanes;
  b.signal_columns = ceil_div(out, 8 << b.signal_lanes);
  b.rows_per_block = std::max<int64_t>(b.signal_lanes == 5 ? high : 2 * high, ceil_div(ceil_div(rows * b.signal_columns, 2048), high) * high);
  b.row_blocks = b.small ? b.dw.splits : ceil_div(rows, b.rows_per_block);
  size_t off = b.own_dz ? ops_align((size_t)rows * b.lddz * elem) : 0;
  b.off_db = off;
  if (a->db && (!b.small || b.dw.splits > 1)) off += ops_align((size_t)b.row_blocks * out * 4);
  b.off_dx = off;
  if (a->dx) off += partial_bytes(b.dx, rows, in);
  b.off_dw = off;
  if (a->dw) off += partial_bytes(b.dw, in, out);
  b.off_x = off;
  if (b.pack_x) off += packed_bytes(rows, in, elem);
  b.off_w = off;
  if (b.pack_w) off += packed_bytes(in, out, elem);
  b.bytes = off;
  return b;
}

// A last layer's loss: the product [rows, classes] is formed whole once, for each row's statistics, and again in pieces of the classes, whose signal (softmax - target, [rows, piece]) lies in the
// workspace while both gradients' products read it.
constexpr int64_t kSignalBytes = (int64_t)192 << 20, kPieceStep = 256, kLeastPiece = 1024;
// Where all classes are one piece anyway and a float32 copy of the logits is no larger than a piece may be, the logits are kept between the two, which saves
// the second product: they go to a pass over the rows as the product's float32 sums (in parts, where its contraction is split).
constexpr int64_t kKeptClasses = 16384;        // a workgroup's registers hold a row; the logits of longer ones are left behind by the statistics' tiles, and a pass over them makes the signal
constexpr int64_t kLeftColumns = 2048;         // of a workgroup of that pass
// (bf16 8192 x 4096 x 4000 975 -> 820 us, 1000 x 4096 x 16000 570 -> 490, 8192 x 512 x 1000 88 -> 84; float32 4096 x 256 x 4000 336 -> 272, 120 x 500 x 1001
// 41 -> 32.5; bf16 2048 x 128 x 10000 110 -> 113)
constexpr double kKeptBytesPerUs = 3.2e6, kKeptLaunch = 3.0;
struct KeptShape { int lanes, pieces; int64_t groups; };        // of a row, pieces of four classes per lane, and workgroups at most
inline KeptShape kept_shape(int64_t rows, int64_t classes) {
  const int64_t n = ceil_div(classes, 4);
  if (n <= 64) return {64, 1, 512};
  if (n <= 256 && rows <= 2048) return {256, 1, 1024};        // (120 x 1001 with four rows to a workgroup 12.9 us)
  if (n <= 256) return {64, 4, 512};
  if (n <= 1024) return {256, 4, 1024};
  return {512, 8, 256};
}
constexpr int kLossGroups = 256, kMostGroups = 1024;        // workgroups of the rows' statistics, at most: each leaves a part of the losses' sum
constexpr int kCounters = 64, kLineWords = 32;              // workgroups that are done are counted in so many places of a line each, and the places that are full in one more
struct LossHead {
  float factor;
  uint32_t pad[kLineWords - 1], full[kLineWords], done[kCounters * kLineWords];
  double loss[kMostGroups];
  int64_t used[kMostGroups];
};
// Up to so many rows, dw is an outer product each lane forms of its columns, and not tiles whose way in and out is all that they are (6 x 3104 x 35488 float32: both gradients by tiles 306 us, where
// reading and writing the two tables takes 184).
constexpr int64_t kOuterRows = 16;
constexpr int kWideColumns = 128;
// What a tile's exponentials cost on its way out, in the microseconds of the table above: 4096 x 1024 x 50001 bf16, all four products, with logits in tiles of
// 64 2616 us, of 128 2086, of 256 1905; 8192 x 512 x 32000 1923, 1560 and 1372; 1000 x 768 x 30000 344, 288 and 270.
constexpr double kLossEnds[] = {0.2, 0.7, 3.5, 3.0};
constexpr int strip_columns(int tile) { return tile == 256 ? 64 : 32; }        // of a wavefront's strip of a tile, which has one entry in a row's statistics
struct LossPlan {
  bool grads, signal, kept, left, wide, outer, direct, copy_x, copy_w;
  Cut logits, piece_logits, dx, dw;
  int64_t piece, pieces, chunks, ldz, strips, left_rows;      // strips: of the signal's rows, each with a part of db; left_rows: of a workgroup of the pass over logits that were left behind
  int stat_floats;
  size_t off_bias, off_stats, off_left, off_info, off_label, off_loss, off_signal, off_dx, off_dw, off_db, off_x, off_w, bytes;
};
inline LossPlan plan_loss(const cada_linear_xent *a) {
  LossPlan f{};
  if (a->rows == 0) return f;
  const int64_t rows = a->rows, in = a->in, classes = a->classes;
  const size_t elem = type_bytes(a->type);
  f.signal = a->dx || a->dw || a->db;
  f.grads = a->dx || a->dw;
  // x is read along the contraction for the logits and across it for dw; for gradients it is copied without the rows that do not count (what they hold is not looked at).
  const bool x_direct = f.signal || direct_kc(a->x, a->ldx, elem), w_direct = direct_oc(a->w, a->ldw, classes, elem);
  const bool tiny = no_tiles(rows, a->ldx, in, elem) || no_tiles(in, a->ldw, classes, elem);
  const Shape whole = {rows, classes, in};
  f.outer = a->dw && rows <= kOuterRows;
  const int n = (a->dx ? 1 : 0) + (a->dw && !f.outer ? 1 : 0);
  // As few pieces as kSignalBytes allow, or up to three more where their tiles come out more evenly (8192 x 4096 x 65536 bf16 in 6 pieces 15.7 ms, in 8 14.3).
  const int64_t logits_bytes = rows * eights(classes) * 4;
  const bool may_keep = f.signal && logits_bytes <= kSignalBytes;
  Cut c[2][4] = {};
  bool kept[2] = {}, left[2] = {};
  double time[2], best[2] = {1e300, 1e300};
  int64_t piece[2] = {classes, classes};
  for (int direct = 0; direct < 2; ++direct) {
    time[direct] = cut(&whole, 1, a->type, direct, widest_tile(in, elem), &c[direct][0], 1, kLossEnds);
    if (!f.signal) continue;
    const int64_t least = ceil_div(classes, std::max<int64_t>(kSignalBytes / (rows * (int64_t)elem) / kPieceStep * kPieceStep, kLeastPiece));
    for (int64_t pieces = least; pieces <= (least == 1 ? 1 : least + 3); ++pieces) {
      const int64_t p = pieces == 1 ? classes : std::max(kLeastPiece, ceil_div(ceil_div(classes, pieces), kPieceStep) * kPieceStep);
      const Shape part = {rows, p, in}, grads[2] = {{rows, in, p}, {in, p, rows}};
      Cut mine[3] = {};
      double t = cut(&part, 1, a->type, direct, widest_tile(in, elem), &mine[0], 1, kLossEnds);
      if (n > 0) t += cut(a->dx ? grads : grads + 1, n, a->type, direct, widest_tile(classes, elem), mine + 1);
      t *= ceil_div(classes, p);
      if (pieces == 1 && may_keep) {
        // (the part of the estimate that is the gradients' products is the same)
        Cut k;
        const double again = cut(&part, 1, a->type, direct, widest_tile(in, elem), &mine[0], 1, kLossEnds), pass = kKeptLaunch + (double)logits_bytes * (1.5 + 0.25 * elem / 2) / kKeptBytesPerUs;
        if (classes > kKeptClasses) {
          left[direct] = pass < again;
          if (left[direct]) t += pass - again;
        } else {
          const double formed_twice = time[direct] + again;
          const double once = cut(&whole, 1, a->type, direct, widest_tile(in, elem), &k, (int)std::min<int64_t>(32, kSignalBytes / logits_bytes)) + pass;
          kept[direct] = once < formed_twice;
          if (kept[direct]) {
            c[direct][0] = k;
            t += once - formed_twice;
          }
        }
      }
      if (t >= best[direct]) continue;
      best[direct] = t;
      piece[direct] = p;
      std::copy(mine, mine + 3, c[direct] + 1);
    }
    time[direct] += best[direct];
  }
  if (!x_direct || !w_direct) time[1] += kPackLaunch + (x_direct ? 0 : pack_cost(rows, in, elem)) + (w_direct ? 0 : pack_cost(in, classes, elem));
  f.direct = (x_direct && w_direct) || tiny || time[1] < time[0];
  f.copy_x = f.signal || (f.direct && !x_direct) || tiny;
  f.copy_w = (f.direct && !w_direct) || tiny;
  const Cut *mine = c[f.direct];
  f.piece = piece[f.direct];
  f.pieces = ceil_div(classes, f.piece);
  f.kept = kept[f.direct];
  f.left = left[f.direct];
  f.logits = mine[0];
  f.piece_logits = mine[1];
  if (a->dx) f.dx = mine[2];
  if (a->dw && !f.outer) f.dw = mine[2 + n - 1];
  // Up to 64 rows of bf16 read the weights in tiles of 128 columns where these fill the CUs and leave no round of them mostly empty (64 x 1024 x 50001
  // 48 -> 39 us, 1 x 4096 x 65536 113 -> 98; 64 x 1024 x 10000 15.4 and 21, 40 x 4096 x 65537 148 and 164; float32 50 x 1000 x 30000 47 and 48).
  const int64_t wide_tiles = ceil_div(classes, kWideColumns), slots = (f.direct ? 3 : 2) * kCUs;
  f.wide = a->type == CADA_BF16 && rows <= 64 && f.logits.tile == 64 && !f.kept && !f.left && wide_tiles >= kCUs && (wide_tiles <= slots || 4 * wide_tiles >= 3 * ceil_div(wide_tiles, slots) * slots);
  f.chunks = f.wide ? wide_tiles * (kWideColumns / 32) : ceil_div(classes, f.logits.tile) * (f.logits.tile / strip_columns(f.logits.tile));
  f.stat_floats = a->smoothing != 0.0 ? 4 : 2;
  f.ldz = eights(f.piece);
  const KeptShape shape = kept_shape(rows, classes);
  // (workgroups of the pass for every CU several times over, and no more parts of db than that takes)
  f.left_rows = std::max<int64_t>(1, ceil_div(rows * ceil_div(classes, kLeftColumns), 8 * kCUs));
  if (f.signal) f.strips = f.kept ? std::min(ceil_div(rows, std::max(1, 256 / shape.lanes)), shape.groups) : f.left ? ceil_div(rows, f.left_rows) : 2 * ceil_div(rows, f.piece_logits.tile);
  size_t off = ops_align(sizeof(LossHead));
  f.off_bias = off; off += f.kept ? ops_align((size_t)eights(classes) * 4) : 0;
  f.off_stats = off; off += f.kept ? ops_align((size_t)f.logits.splits * logits_bytes) : ops_align((size_t)f.chunks * rows * f.stat_floats * 4);
  f.off_left = off; off += f.left ? ops_align((size_t)logits_bytes) : 0;
  f.off_info = off; off += ops_align((size_t)rows * 16);
  f.off_label = off; off += ops_align((size_t)rows * 4);
  f.off_loss = off; off += a->loss ? 0 : ops_align((size_t)rows * 4);
  f.off_signal = off; off += f.grads ? ops_align((size_t)rows * f.ldz * elem) : 0;
  f.off_dx = off; off += a->dx && (f.pieces > 1 || f.dx.splits > 1) ? ops_align((size_t)f.dx.splits * rows * eights(in) * 4) : 0;
  f.off_dw = off; off += a->dw ? partial_bytes(f.dw, in, f.piece) : 0;
  f.off_db = off; off += a->db ? ops_align((size_t)f.strips * f.piece * 4) : 0;
  f.off_x = off; off += f.copy_x ? packed_bytes(rows, in, elem) : 0;
  f.off_w = off; off += f.copy_w ? packed_bytes(in, classes, elem) : 0;
  f.bytes = off;
  return f;
}

}  // namespace cada
