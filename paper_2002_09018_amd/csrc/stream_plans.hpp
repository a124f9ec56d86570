// How the loss from the last activations and the gated feed-forward block cut their
// work: plain host arithmetic on sizes and types.
#pragma once

#include <cmath>

#include "layer_plans.hpp"

namespace shp {

enum { kShapeSolo = 0, kShapeFew = 1, kShapeMid = 2, kShapeBig = 3, kShapeDirect = 4 };

// Shapes of a product: tiles of 32 rows whose waves share the contraction (Solo), of 32
// rows (Few; small tiles of a weight gradient), of 128 x 128, and larger ones; and those of
// few rows whose other matrix is not copied (Direct, few_rows.hpp).

// How a product is cut: tiles of C, and parts of the contraction.
struct MmaPlan {
  int shape = kShapeMid, splits = 1, per_split = 0;  // (per_split: stages of a part)
  int64_t tiles_m = 0, tiles_n = 0, seg_stages = 0;
  int64_t ld_part = 0;
  size_t part = 0;  // bytes of the parts
  double us = 0;    // estimated time
};

// A tile and what it takes: us of a stage with 1, 2, .. workgroups on a compute unit
// (`alone`: one, and half the chip idle), us of a launch beside its stages.
struct MmaCost {
  int m, n, slots;
  double alone, stage[4], start;
  int bk;  // contraction indices of a stage
};
// By shape, for operands of one plane (bf16) and of three (fp32).  Measured: at full
// load a compute unit reaches 5.1 TFLOP/s with the largest tiles of one plane and
// 4.7 with those of three (six products), 4.0 and 4.7 with 128 x 128; a library product
// of 8192^3 in bf16 5.1.
constexpr MmaCost kCost1[] = {{32, 64, 1, 0.09, {0.145}, 4, 32},
                              {32, 128, 4, 0.28, {0.30, 0.38, 0.49, 0.62}, 4, 32},
                              {128, 128, 2, 0.58, {0.64, 1.05}, 5, 64},
                              {256, 256, 1, 1.15, {1.65}, 10, 64}};
constexpr MmaCost kCost3[] = {{32, 64, 1, 0.24, {0.46}, 5, 32},
                              {32, 128, 2, 0.70, {0.80, 1.17}, 5, 32},
                              {128, 128, 1, 0.86, {1.33}, 6, 32},
                              {256, 128, 1, 1.55, {2.34}, 10, 32}};
// Weight gradients, whose contraction runs over rows: small tiles take the place of those
// for few rows (few rows are short sums there, and many tiles at once keep the stores
// flowing); for one plane, one and three (three products), three.
constexpr MmaCost kWeight1[] = {{},
                                {64, 64, 4, 0.30, {0.30, 0.32, 0.36, 0.45}, 4, 32},
                                {128, 128, 2, 0.58, {0.64, 1.05}, 5, 64},
                                {256, 256, 1, 0.57, {0.83}, 9, 32}};
constexpr MmaCost kWeight31[] = {{},
                                 {64, 64, 4, 0.35, {0.40, 0.45, 0.60, 0.80}, 4, 32},
                                 {128, 128, 1, 0.55, {0.72}, 6, 32},
                                 {256, 128, 1, 1.03, {1.45}, 9, 32}};
constexpr MmaCost kWeight3[] = {{},
                                {64, 64, 3, 0.50, {0.60, 0.80, 1.10}, 4, 32},
                                {128, 128, 1, 0.86, {1.33}, 6, 32},
                                {256, 128, 1, 1.55, {2.34}, 10, 32}};
inline const MmaCost* mma_cost(int planes) { return planes == 1 ? kCost1 : kCost3; }
inline const MmaCost* weight_cost(int x_planes, int d_planes) {
  return x_planes == 3 ? kWeight3 : d_planes == 3 ? kWeight31 : kWeight1;
}

// Time of `groups` workgroups of `per` stages: full rounds of the chip, then the rest.
inline double mma_us(const MmaCost& t, int64_t groups, double per) {
  const int64_t full = 256 * t.slots, rest = groups % full;
  double us = (double)(groups / full) * (per * t.stage[t.slots - 1] + t.start);
  if (rest) us += per * (rest <= 128 ? t.alone : t.stage[(rest - 1) / 256]) + t.start;
  return us;
}

// A product in tiles of shape i (cost t) and up to `want` parts; `us` is left out.
inline MmaPlan mma_cut(int64_t M, int64_t N, int64_t K, const MmaCost& t, int i, int segs, bool pair, int64_t want,
                       bool always_part) {
  MmaPlan p;
  p.shape = i;
  p.seg_stages = cdiv64(K, t.bk);
  const int64_t stages = p.seg_stages * segs;
  p.per_split = (int)cdiv64(stages, want);
  p.splits = (int)cdiv64(stages, p.per_split);
  p.tiles_m = cdiv64(M, t.m);
  p.tiles_n = cdiv64(N, pair ? t.n / 2 : t.n);
  p.ld_part = cdiv64(N, 8) * 8 * (pair ? 2 : 1);
  p.part = p.splits > 1 || always_part ? (size_t)(p.splits * M * p.ld_part) * sizeof(float) : 0;
  return p;
}
// What parts cost: their way to memory and back (more where the last-level cache does
// not hold them) and the launch that adds them.
inline double parts_us(const MmaPlan& p) {
  const double mb = 1e-6 * (double)p.part;
  return p.splits > 1 ? 5 + 0.3 * mb + 0.25 * std::max(0., mb - 256) : 0;
}

// The cheapest tile and number of parts (at most most_splits) by estimated time.  `segs`
// products of one contraction length are summed.  rounds: terms of A beside a B of one plane;
// tiles of 128 rows and more take every stage once for each, 32 x 128 ones take half again as
// long for a second (1, 1.5 and 2 times as long measured: 700 x 768 x 5000 113, 88 and 91 us,
// 64 x 1024 over 32768 92, 90 and 103), and 32 x 64 ones are bound by B.
inline MmaPlan mma_plan(int64_t M, int64_t N, int64_t K, const MmaCost* cost, int segs, bool pair, int least_shape,
                        int most_splits, bool always_part, int rounds = 1) {
  MmaPlan best;
  for (int i = least_shape; i <= kShapeBig; ++i) {
    const MmaCost& t = cost[i];
    const int64_t tiles = cdiv64(M, t.m) * cdiv64(N, pair ? t.n / 2 : t.n);
    for (int want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      if (want > cdiv64(K, t.bk) * segs || want > most_splits || (want > 1 && want * tiles > 1024)) break;
      MmaPlan p = mma_cut(M, N, K, t, i, segs, pair, want, always_part);
      const double each = i >= kShapeMid ? rounds : i == kShapeFew ? 0.5 + 0.5 * rounds : 1;
      p.us = mma_us(t, tiles * p.splits, each * p.per_split) + parts_us(p);
      if (best.us == 0 || p.us < best.us) best = p;
    }
  }
  return best;
}

// Whether a call reads its table or weights (so many elements) where they lie whatever
// their type and address, once for each 32 rows, instead of copies in planes.  Both
// measured, copies first: a block of 16 and 64 rows over 1024 x 4096 in fp32 33 and 33 us,
// 17 and 20, with odd rows in bf16 15 and 20, 10 and 15; its gradients of 14 rows in fp32
// 75, 57, of 40 rows 57, 58; a loss of 5 and 40 rows over 40960 x 2589 in fp32 330 and 424,
// 167 and 249, in bf16 122, 105 (71 where rows begin at 16 bytes), but over 4096 x 2589
// in bf16 25, 30; a loss' gradients of 64 rows over 32768 x 1024 in fp32 233, 242, of 56
// rows in bf16 48, 81.  (Along rows a lane's 16 bytes are in a line of their own, and
// bf16 ones mostly across two words.)
inline bool few_direct(int64_t rows, int64_t weights, int dtype, bool along_rows, bool grad) {
  const bool odd = dtype == SHAMPOO_BF16 && along_rows;
  return rows <= (grad || odd ? 32 : 64) && (!odd || weights >= (1 << 24));
}
// Its tile; a stage is 64 bytes of a lane's row where the contraction lies along rows.
inline MmaCost few_tile(int planes, bool along_rows) { return {32, 64, 1, 0, {0}, 4, !along_rows ? 16 : planes == 1 ? 64 : 32}; }

// Such a product: the most of its memory time (of the chip, and of the compute units that
// have a part) and of its waves' stages, and parts.
inline MmaPlan few_plan(int64_t M, int64_t N, int64_t K, int planes, bool along_rows, int segs, bool pair,
                        int most_splits, bool always_part) {
  const MmaCost t = few_tile(planes, along_rows);
  const int64_t tiles = cdiv64(M, t.m) * cdiv64(N, pair ? t.n / 2 : t.n);
  // MB a us of a compute unit: lanes whose 16 bytes lie in lines of their own, at any
  // address, are served one by one
  const double each = !along_rows ? 0.04 : planes == 1 ? 0.009 : 0.012;
  const double mb = 1e-6 * (double)(N * K) * segs * (pair ? 2 : 1) * (planes == 1 ? 2 : 4) * (double)cdiv64(M, t.m);
  MmaPlan best;
  for (int want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
    if (want > cdiv64(K, t.bk) * segs || want > most_splits || (want > 1 && want * tiles > 1024)) break;
    MmaPlan p = mma_cut(M, N, K, t, kShapeDirect, segs, pair, want, always_part);
    const double groups = (double)(tiles * p.splits), rounds = std::ceil(groups / 256);
    p.us = std::max(mb / std::min(4.5, each * groups), rounds * 0.6 * (double)cdiv64(p.per_split, 8)) + 4 + rounds +
           parts_us(p);
    if (best.us == 0 || p.us < best.us) best = p;
  }
  return best;
}

// The two products of a gradient, dX (x) and the weights' (w), in one launch of 128 x 128
// tiles where that is estimated to take less time than theirs one after the other
// (`on`): each alone often leaves compute units idle, and a launch and a join are saved.
// Both products have operands of the same number of planes (and so the same waves); a
// second term of a gradient of few rows is not counted (8 and 30 rows x 2048 over 2000 22
// and 25 us, 24 and 28 if it is).
// Measured, whole calls, two launches and one: 1003 x 333 x 1339 in fp32 70.3 and 58.9
// us, in bf16 36.0 and 28.0; 2048 x 512 x 1344 in bf16 47.5 and 34.2; a vocabulary of
// 1000 for 4096 x 1024 in bf16 54.5 and 45.1, where 512 x 1024 x 4096 fills the chip
// either way and keeps two.
struct TwoPlan {
  bool on = false;
  MmaPlan x, w;
};
inline TwoPlan two_plan(const MmaPlan& x, int64_t Mx, int64_t Nx, int64_t Kx, int segs, const MmaPlan& w, int64_t Mw,
                        int64_t Nw, int64_t Kw, int planes) {
  TwoPlan best;
  const MmaCost &tx = mma_cost(planes)[kShapeMid], &tw = weight_cost(planes, planes)[kShapeMid];
  const double slots = 256. * tx.slots;
  const int64_t tiles_x = cdiv64(Mx, tx.m) * cdiv64(Nx, tx.n), tiles_w = cdiv64(Mw, tw.m) * cdiv64(Nw, tw.n);
  if (tiles_x > 1024 || tiles_w > 1024) return best;  // enough for the chip by itself
  double best_us = x.us + w.us;
  for (int wx : {1, 2, 3, 4, 6, 8, 12, 16}) {
    if (wx > cdiv64(Kx, tx.bk) * segs || wx * tiles_x > 1024) break;
    const MmaPlan px = mma_cut(Mx, Nx, Kx, tx, kShapeMid, segs, false, wx, false);
    for (int ww : {1, 2, 3, 4, 6, 8, 12, 16}) {
      if (ww > cdiv64(Kw, tw.bk) || (ww > 1 && ww * tiles_w > 1024)) break;
      const MmaPlan pw = mma_cut(Mw, Nw, Kw, tw, kShapeMid, 1, false, ww, false);
      // workgroups run one after another in the slots, dX's first
      const double gx = (double)(tiles_x * px.splits), gw = (double)(tiles_w * pw.splits);
      const int busy = gx + gw <= 256 ? 0 : tx.slots - 1;
      const double ux = px.per_split * tx.stage[busy] + tx.start, uw = pw.per_split * tw.stage[busy] + tw.start;
      const double us = std::max({ux, uw, (gx * ux + gw * uw) / slots + (gx + gw > slots ? std::min(ux, uw) / 2 : 0)}) +
                        std::max(parts_us(px), parts_us(pw)) + 0.5 * std::min(parts_us(px), parts_us(pw));
      if (us < best_us) {
        best_us = us;
        best = {true, px, pw};
      }
    }
  }
  return best;
}

// Most tiles of a launch (it holds fewer than 2^32 threads, and their numbers 31 bits).
constexpr int64_t kMostTiles = INT32_MAX / 512;
inline bool fits(const MmaPlan& p) { return p.tiles_m * p.tiles_n * p.splits <= kMostTiles; }

// A matrix copied into bf16 planes: one, or three of an fp32 one.
struct PackPlan {
  int planes = 1;
  int64_t ld = 0, plane = 0;  // elements
  size_t bytes = 0;
};
inline PackPlan pack_plan(int64_t rows, int64_t cols, int dtype) {
  PackPlan p;
  p.planes = dtype == SHAMPOO_BF16 ? 1 : 3;
  p.ld = cdiv64(cols, 64) * 64;
  p.plane = rows * p.ld;
  p.bytes = (size_t)(p.plane * p.planes) * 2;
  return p;
}

// Offsets of buffers in a workspace, each aligned to 256 bytes; spared: bytes of copies
// that this call does without, for which a workspace has room all the same (whether a
// matrix is copied hangs on its address and stride).
struct Room {
  size_t at = 0, spared = 0;
  size_t take(size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  }
  size_t copy(bool made, size_t bytes) {
    if (made) return take(bytes);
    spared += (bytes + 255) / 256 * 256;
    return 0;
  }
};

// Most bytes of one piece of the vocabulary: of the logits' gradient (it is read twice
// soon after it was written, and the last-level cache holds 256 MB), and of packed
// rows of the table.
constexpr int64_t kPieceB = 256 << 20;

inline int64_t vocab_piece(int64_t vocab, int64_t bytes_each) {
  const int64_t most = std::max<int64_t>(256, kPieceB / bytes_each / 256 * 256);
  return std::min(vocab, cdiv64(cdiv64(vocab, cdiv64(vocab, most)), 256) * 256);
}

// Columns of a row of logits whose statistics are one entry, where the logits were
// formed in parts.
constexpr int kStatCols = 512;  // 8 of a lane
// Workgroups of the launch that forms them, four waves to one.  Any piece fits: parts are
// taken for at most 1024 tiles, 2^16 such groups.
inline int64_t stat_groups(int64_t rows, int64_t n) { return cdiv64(rows * cdiv64(n, kStatCols), 4); }

// The loss: pieces of the vocabulary (one, where the table is read as it lies).
struct VocabPlan {
  int64_t piece = 0, pieces = 0, entries = 0;  // entries: statistics of a row
  bool direct = false;                         // the table is read where it lies by few_rows.hpp
  MmaPlan mma[2];  // of a whole piece and of the last
  PackPlan x, w;
  size_t at_x = 0, at_w = 0, at_stat = 0, at_target = 0, at_part = 0, bytes = 0, need = 0;
};
inline int64_t vocab_entries(const MmaPlan& p, int64_t n) { return p.part ? cdiv64(n, kStatCols) : p.tiles_n; }

// Whether the table is cut the same way copied or not.
inline bool vocab_alike(int64_t rows, int64_t dim, int64_t vocab, int dtype) {
  return dtype == SHAMPOO_F32 || (!few_direct(rows, vocab * dim, dtype, true, false) && vocab_piece(vocab, pack_plan(1, dim, dtype).bytes) == vocab);
}
inline VocabPlan vocab_plan(int64_t rows, int64_t dim, int64_t vocab, int dtype, bool pack_x, bool pack_w) {
  VocabPlan p;
  Room r;
  p.x = pack_plan(rows, dim, dtype);
  p.at_x = r.copy(pack_x, p.x.bytes);
  const bool few = few_direct(rows, vocab * dim, dtype, true, false), copy_w = pack_w && !few;
  p.direct = pack_w && few;
  p.piece = copy_w ? vocab_piece(vocab, pack_plan(1, dim, dtype).bytes) : vocab;
  p.pieces = cdiv64(vocab, p.piece);
  p.w = pack_plan(p.piece, dim, dtype);
  if (!few) p.at_w = r.copy(copy_w, p.w.bytes);
  const int64_t last = vocab - (p.pieces - 1) * p.piece;
  size_t part = 0;
  for (int i = 0; i < 2; ++i) {
    if (i && last == p.piece) {
      p.mma[1] = p.mma[0];
      break;
    }
    const int64_t n = i ? last : p.piece;
    p.mma[i] = p.direct ? few_plan(rows, n, dim, p.x.planes, true, 1, false, 64, false)
                        : mma_plan(rows, n, dim, mma_cost(p.x.planes), 1, false, kShapeFew, 64, false);
    part = std::max(part, p.mma[i].part);
  }
  p.entries = (p.pieces - 1) * vocab_entries(p.mma[0], p.piece) + vocab_entries(p.mma[1], last);
  p.at_stat = r.take((size_t)(rows * p.entries) * 8);
  p.at_target = r.take((size_t)rows * 4);
  p.at_part = r.take(part);
  p.bytes = r.at;
  p.need = r.at + r.spared;
  return p;
}

// Its gradient: the logits of a piece, its share of dX, its rows of dW.
struct VocabGradPlan {
  int64_t piece = 0, pieces = 0, ld_dz = 0;
  int planes = 1;       // bf16 terms of the logits' gradient
  bool second = false;  // another one, where `planes` is one
  bool direct = false;  // as above
  MmaPlan z[2], dx[2], dw[2];
  bool two = false;  // dX and dW in one launch, where both are wanted, cut as follows
  MmaPlan two_dx, two_dw;
  PackPlan x, w;
  size_t at_x = 0, at_w = 0, at_dz = 0, at_second = 0, at_dx = 0, at_part = 0, bytes = 0, need = 0;
  int terms() const { return second ? 2 : planes; }
};

// An fp32 gradient, of inputs of either type, has three terms of dz: with one it
// would keep 9 bits, with two 17.  A bf16 one takes dz as the framework stores a
// bf16 gradient of logits, rounded once.
inline int grad_planes(int dtype, int g_dtype) { return dtype == SHAMPOO_F32 || g_dtype == SHAMPOO_F32 ? 3 : 1; }
// Terms that dX of bf16 inputs takes of a gradient that is kept in three for an fp32 dW: two
// are off by 2^-16, 2^-8 of what dX itself is rounded by.  One, measured, was off by as much
// as that rounding (0.0024 of the norm for 0.0017) and by more than the result where its
// terms cancel; the third is a third product for nothing that bf16 shows (whole calls
// with one, two and three: 2048 x 1024 over 32768 712, 830 and 925 us, 16384 rows through
// 1024 x 4096 1167, 1420 and 1637).
constexpr int kDxTerms = 2;
// Rounds of its product: one for each of them (in small tiles both go beside one read of the
// other matrix).
inline int dx_rounds(int planes, int terms) { return planes == 1 && terms > 1 ? kDxTerms : 1; }

// Up to so many rows dz has two terms also where inputs and gradients are bf16, for dX and
// dW: the entries of few tokens hold most of its norm, and the roundings of one term do not
// average out there (results off by up to 2.8 times their own rounding).  Such calls are
// bound by the table or by launches: 1, 16 and 32 rows x 1024 over 32768 55, 57 and 60 us with one
// term, 58, 56 and 63 with two, 8 rows x 512 over 5000 16 and 19; 64, 128 and 512 rows x 1024
// over 32768 65, 73 and 127, with two 78, 93 and 202.
constexpr int kSecondRows = 32;

inline bool vocab_grad_alike(int64_t rows, int64_t dim, int64_t vocab, int dtype, int planes) {
  return dtype == SHAMPOO_F32 ||
         (!few_direct(rows, vocab * dim, dtype, true, true) && vocab_piece(vocab, pack_plan(1, dim, dtype).bytes) >= vocab_piece(vocab, rows * planes * 2));
}
inline VocabGradPlan vocab_grad_plan(int64_t rows, int64_t dim, int64_t vocab, int dtype, int g_dtype, bool pack_x,
                                     bool pack_w) {
  VocabGradPlan p;
  Room r;
  p.planes = grad_planes(dtype, g_dtype);
  p.x = pack_plan(rows, dim, dtype);
  p.at_x = r.copy(pack_x, p.x.bytes);
  p.piece = vocab_piece(vocab, rows * p.planes * 2);
  const bool few = few_direct(rows, vocab * dim, dtype, true, true), copy_w = pack_w && !few;
  p.direct = pack_w && few;
  if (copy_w) p.piece = std::min(p.piece, vocab_piece(vocab, pack_plan(1, dim, dtype).bytes));
  p.pieces = cdiv64(vocab, p.piece);
  p.w = pack_plan(p.piece, dim, dtype);
  if (!few) p.at_w = r.copy(copy_w, p.w.bytes);
  p.ld_dz = cdiv64(p.piece, 64) * 64;
  p.at_dz = r.take((size_t)(rows * p.ld_dz * p.planes) * 2);
  p.second = p.planes == 1 && rows <= kSecondRows;  // (in a buffer of its own)
  if (p.second) p.at_second = r.take((size_t)(rows * p.ld_dz) * 2);
  size_t part = 0;
  const int64_t last = vocab - (p.pieces - 1) * p.piece;
  for (int i = 0; i < 2; ++i) {
    const int64_t n = i ? last : p.piece;
    if (i && last == p.piece) {
      p.z[1] = p.z[0];
      p.dx[1] = p.dx[0];
      p.dw[1] = p.dw[0];
      break;
    }
    const MmaCost* cost = mma_cost(p.x.planes);
    const int most = i ? p.dx[0].splits : 64;
    if (p.direct) {
      p.z[i] = few_plan(rows, n, dim, p.x.planes, true, 1, false, 64, false);
      p.dx[i] = few_plan(rows, dim, n, p.x.planes, false, 1, false, most, p.pieces > 1);
    } else {
      p.z[i] = mma_plan(rows, n, dim, cost, 1, false, kShapeSolo, 64, false);
      p.dx[i] = mma_plan(rows, dim, n, cost, 1, false, kShapeSolo, most, p.pieces > 1, dx_rounds(p.x.planes, p.terms()));
    }
    p.dw[i] = mma_plan(n, dim, rows, weight_cost(p.x.planes, p.planes), 1, false, kShapeFew, 64, false, p.second ? 2 : 1);
    part = std::max({part, p.z[i].part, p.dw[i].part});
  }
  if (!p.direct && p.pieces == 1 && p.planes == p.x.planes) {
    const TwoPlan t = two_plan(p.dx[0], rows, dim, vocab, 1, p.dw[0], vocab, dim, rows, p.planes);
    p.two = t.on;
    p.two_dx = t.x;
    p.two_dw = t.w;
  }
  p.at_dx = r.take(std::max(p.dx[0].part, p.two_dx.part));
  p.at_part = r.take(std::max(part, p.two_dw.part));
  p.bytes = r.at;
  p.need = r.at + r.spared;
  return p;
}

// The feed-forward block.
struct FfnPlan {
  MmaPlan mma;
  bool direct = false;  // the weights are read where they lie by few_rows.hpp
  PackPlan x, wg, wu;
  size_t at_x = 0, at_wg = 0, at_wu = 0, at_part = 0, bytes = 0, need = 0;
};
// Whether the products are cut the same way for weights copied or not.
inline bool ffn_alike(int64_t rows, int64_t dim, int64_t width, int dtype, bool grad) {
  return dtype == SHAMPOO_F32 || !few_direct(rows, 2 * dim * width, dtype, grad, grad);
}
inline FfnPlan ffn_plan(int64_t rows, int64_t dim, int64_t width, int dtype, bool pack_x, bool pack_wg, bool pack_wu) {
  FfnPlan p;
  Room r;
  p.x = pack_plan(rows, dim, dtype);
  p.wg = p.wu = pack_plan(dim, width, dtype);
  const bool few = few_direct(rows, 2 * dim * width, dtype, false, false);
  p.direct = few && (dtype == SHAMPOO_F32 || pack_wg || pack_wu);
  p.at_x = r.copy(pack_x, p.x.bytes);
  if (!few) {
    p.at_wg = r.copy(pack_wg, p.wg.bytes);
    p.at_wu = r.copy(pack_wu, p.wu.bytes);
  }
  p.mma = p.direct ? few_plan(rows, width, dim, p.x.planes, false, 1, true, 64, false)
                   : mma_plan(rows, width, dim, mma_cost(p.x.planes), 1, true, kShapeSolo, 64, false);
  p.at_part = r.take(p.mma.part);
  p.bytes = r.at;
  p.need = r.at + r.spared;
  return p;
}

// Its gradient.  dG and dU lie side by side in rows of 2 ld_d, so that dWg and dWu are
// one product.
struct FfnGradPlan {
  MmaPlan gu, dx, dw;
  bool direct = false, two = false;  // as above
  MmaPlan two_dx, two_dw;
  PackPlan x, wg, wu;
  int64_t ld_d = 0;
  int planes = 1;
  size_t at_x = 0, at_wg = 0, at_wu = 0, at_d = 0, at_dx = 0, at_part = 0, bytes = 0, need = 0;
};
inline FfnGradPlan ffn_grad_plan(int64_t rows, int64_t dim, int64_t width, int dtype, int g_dtype, bool pack_x,
                                 bool pack_wg, bool pack_wu) {
  FfnGradPlan p;
  Room r;
  p.planes = grad_planes(dtype, g_dtype);
  p.x = pack_plan(rows, dim, dtype);
  p.wg = p.wu = pack_plan(dim, width, dtype);
  const bool few = few_direct(rows, 2 * dim * width, dtype, true, true);
  p.direct = few && (dtype == SHAMPOO_F32 || pack_wg || pack_wu);
  p.at_x = r.copy(pack_x, p.x.bytes);
  if (!few) {
    p.at_wg = r.copy(pack_wg, p.wg.bytes);
    p.at_wu = r.copy(pack_wu, p.wu.bytes);
  }
  p.ld_d = cdiv64(width, 64) * 64;
  p.at_d = r.take((size_t)(rows * 2 * p.ld_d * p.planes) * 2);
  if (p.direct) {
    p.gu = few_plan(rows, width, dim, p.x.planes, false, 1, true, 64, false);
    p.dx = few_plan(rows, dim, width, p.x.planes, true, 2, false, 64, false);
  } else {
    p.gu = mma_plan(rows, width, dim, mma_cost(p.x.planes), 1, true, kShapeSolo, 64, false);
    p.dx = mma_plan(rows, dim, width, mma_cost(p.x.planes), 2, false, kShapeSolo, 64, false,
                    dx_rounds(p.x.planes, p.planes));
  }
  p.dw = mma_plan(dim, 2 * p.ld_d, rows, weight_cost(p.x.planes, p.planes), 1, false, kShapeFew, 64, false);
  if (!p.direct && p.planes == p.x.planes) {
    const TwoPlan t = two_plan(p.dx, rows, dim, width, 2, p.dw, dim, 2 * p.ld_d, rows, p.planes);
    p.two = t.on;
    p.two_dx = t.x;
    p.two_dw = t.w;
  }
  p.at_part = r.take(std::max({p.gu.part, p.dx.part, p.dw.part, p.two_dw.part}));
  p.at_dx = p.two ? r.take(p.two_dx.part) : p.at_part;
  p.bytes = r.at;
  p.need = r.at + r.spared;
  return p;
}

}  // namespace shp
