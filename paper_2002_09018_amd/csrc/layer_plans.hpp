// How the calls from the loss to the gradient cut their work, and whether their
// buffers overlap: plain host arithmetic on sizes, types and addresses.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "shampoo.h"

namespace shp {

inline int64_t cdiv64(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The bytes of a buffer: rows of `row` bytes, `pitch` apart.
struct Span {
  uintptr_t p;
  int64_t rows, row, pitch;
};
inline Span span(const void* p, int64_t rows, int64_t cols, int64_t ld, int dtype) {
  const int64_t b = dtype == SHAMPOO_BF16 ? 2 : 4;
  return {reinterpret_cast<uintptr_t>(p), p ? rows : 0, cols * b, ld * b};
}
inline Span span(const void* p, int64_t bytes) { return {reinterpret_cast<uintptr_t>(p), p ? 1 : 0, bytes, bytes}; }

// Whether two buffers share no byte: one lies past the other, or the rows of each
// lie between those of the other.  (Rows of different pitches in one range are
// taken as shared.)
inline bool apart(const Span& a, const Span& b) {
  if (a.rows == 0 || b.rows == 0 || a.row == 0 || b.row == 0) return true;
  auto end = [](const Span& x) { return x.p + (uintptr_t)(x.rows - 1) * (uintptr_t)x.pitch + (uintptr_t)x.row; };
  if (end(a) <= b.p || end(b) <= a.p) return true;
  if (a.rows == 1 && b.rows == 1) return false;
  if (a.rows > 1 && b.rows > 1 && a.pitch != b.pitch) return false;
  const int64_t pitch = a.rows > 1 ? a.pitch : b.pitch;
  int64_t at = (int64_t)(b.p - a.p) % pitch;
  if (at < 0) at += pitch;
  return at >= a.row && at + b.row <= pitch;
}

constexpr int kLogitBlockB = 4096;  // bytes of a row that a wave takes at a time (LogitBlock)
// Floats of a part of a row: m, s, t, -, k values, k indices.
constexpr int64_t logprob_record(int k) { return 4 + 2 * (int64_t)k; }

// How a row of logits is cut: waves of a workgroup to a row, and workgroups
// (parts) of a row where there are few rows.  About two waves per SIMD are
// wanted: fewer do not keep enough bytes in flight, and each wave of a row pays
// for finding its own first alternatives.  Rows x 131072 in bf16, 8
// alternatives, us with 1 / 2 / 4 / 8 waves: 8192 rows 390 / 384 / 380 / 436, 1024
// rows 75 / 58 / 52 / 58, 256 rows 71 / 44 / 28 / 23; without alternatives 8192
// rows 385 / 377 / 355 / 358, of 65536 205 / 195 / 184 / 187, of 20000 63 / 63 / 67 / 86.
// Below 256 rows long rows are cut into parts of 4 waves and a second launch joins
// them: one row 10.6 us, by one workgroup of 8 waves 18; 64 rows 13 and 19.  Rows of
// few blocks to a wave do without: 1 x 32768 8.8 us, in parts 10.7, 128 x 32768 9.6 and
// 11.4; 1 x 65536 12.2 and 10.4, without alternatives 7.6 and 9.9.
struct LogprobPlan {
  int waves = 1, parts = 1, per_part = 0;
  size_t ws = 0;
};

inline LogprobPlan logprob_plan(int64_t rows, int64_t vocab, int k, int dtype) {
  LogprobPlan p;
  const int64_t block = kLogitBlockB / (dtype == SHAMPOO_BF16 ? 2 : 4);
  const int64_t blocks = cdiv64(vocab, block);
  const int64_t want = std::min(std::max<int64_t>(cdiv64(2048, rows), k == 0 && blocks >= 32 ? 4 : 1), blocks);
  const bool whole = rows >= 256 || blocks <= (k == 0 ? 48 : 16);
  const int most = whole ? 8 : 4;
  while (p.waves < want && p.waves < most) p.waves *= 2;
  const int64_t steps = cdiv64(blocks, p.waves);
  const int64_t parts = whole ? 1 : std::min<int64_t>(cdiv64(want, p.waves), 64);
  const int64_t per = cdiv64(steps, parts);
  p.parts = (int)cdiv64(steps, per);
  p.per_part = (int)std::min<int64_t>(per * p.waves * block, vocab);
  if (p.parts > 1) p.ws = (size_t)(rows * p.parts * logprob_record(k)) * sizeof(float);
  return p;
}

// How the loss gradient is cut: blocks of a wave, and waves of a row.  One block to
// a wave (8192 x 131072 in bf16: 729 us; two 766, four 792), two in short rows, where
// a row's own values cost more (8192 x 5000 with 32 alternatives: 44.6 -> 41.7).
struct LossGradPlan {
  int per = 1, segs = 1;
};

inline LossGradPlan loss_grad_plan(int64_t rows, int64_t vocab, int dtype) {
  LossGradPlan p;
  const int64_t block = kLogitBlockB / (dtype == SHAMPOO_BF16 ? 2 : 4);
  const int64_t blocks = cdiv64(vocab + 7, block);  // a row may begin up to 7 entries into its first
  p.per = blocks > 16 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(2, rows * blocks / 4096));
  p.segs = (int)cdiv64(blocks, p.per);
  return p;
}

// How a weight gradient is cut: the tile, and the splits of the token axis.
struct WgradPlan {
  int tile_m = 256, tile_n = 256, splits = 1;
  int64_t per_split = 0, tiles_m = 0, tiles_n = 0;
  size_t ws = 0;
};

// Estimated time (us) of a stage of every one of `blocks` workgroups: full rounds
// of the chip, then the rest.  `alone` is a stage's time on a lightly filled
// chip, `full` with every slot taken (clock and bandwidth then are shared, and
// compute units where a workgroup leaves room for a second).
inline double wgrad_rounds(int64_t blocks, int64_t slots, double alone, double full) {
  const int64_t rest = blocks % slots;
  const double part = rest == 0      ? 0
                      : slots == 512 ? (rest <= 256 ? alone * (1 + rest / 1280.0) : full)
                      : rest <= 128  ? alone
                                     : alone + (full - alone) * (rest - 128) / 128;
  return (double)(blocks / slots) * full + part;
}

// The cheapest tile, with the token axis in up to 128 parts, by an estimate from
// the measured time of a stage; parts cost their partial tiles' way to memory
// and back (0.2 us per MB) and a second launch.  One workgroup takes a compute
// unit; two of 128 x 128 share one with bf16 gradients, for which alone there is
// 128 x 256.  Measured (bf16, us, best number of parts of 256 x 256 / 128 x 256 /
// 128 x 128): 65536 x 1024 x 4096 492 / 579 / 666; 16384 x 1024 x 1024 53 / 48 / 55;
// 30000 x 300 x 1000 48 / 39 / 43; 2048 x 1024 x 1024 28 / 22 / 19; one part instead of
// the best: 65536 x 1024 x 4096 1321, 32768 x 512 x 512 (128 x 128) 288 instead of 31.
inline WgradPlan wgrad_plan(int64_t rows, int64_t cols, int64_t out, int dtype) {
  const bool bf16 = dtype == SHAMPOO_BF16;
  WgradPlan best;
  double best_us = 0;
  struct Tile {
    int m, n, bk, slots;        // bk: tokens of a stage
    double alone, full, start;  // us: a stage, and a launch beside its stages
  };
  static const Tile bf16_tiles[] = {
      {128, 128, 64, 512, 0.56, 1.31, 3}, {128, 256, 64, 256, 0.81, 1.10, 3}, {256, 256, 64, 256, 1.28, 1.79, 6}};
  static const Tile f32_tiles[] = {{128, 128, 64, 256, 1.37, 1.60, 3}, {256, 256, 32, 256, 2.10, 2.70, 6}};
  const Tile* tiles_of = bf16 ? bf16_tiles : f32_tiles;
  for (int i = 0; i < (bf16 ? 3 : 2); ++i) {
    const Tile& t = tiles_of[i];
    const int64_t tm = cdiv64(cols, t.m), tn = cdiv64(out, t.n), tiles = tm * tn;
    const int64_t stages = std::max<int64_t>(1, cdiv64(rows, t.bk));
    for (int want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128}) {
      if (want > stages || (want > 1 && want * tiles > 2 * t.slots)) break;
      const int64_t per = cdiv64(stages, want), splits = cdiv64(stages, per);
      const size_t ws = splits > 1 ? (size_t)(splits * tiles) * t.m * t.n * sizeof(float) : 0;
      const double us = t.start + wgrad_rounds(tiles * splits, t.slots, t.alone, t.full) * (double)per +
                        (splits > 1 ? 5 + 0.2e-6 * (double)ws : 0);
      if (best_us == 0 || us < best_us) {
        best_us = us;
        best.tile_m = t.m;
        best.tile_n = t.n;
        best.splits = (int)splits;
        best.per_split = per * t.bk;
        best.tiles_m = tm;
        best.tiles_n = tn;
        best.ws = ws;
      }
    }
  }
  return best;
}

}  // namespace shp
