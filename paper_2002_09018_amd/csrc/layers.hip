// Host side of the calls from the loss to the gradient: argument checking and
// launches of logprobs.hpp, act_checkpoint.hpp and weight_grad.hpp.
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>
#include <atomic>
#include <new>
#include <type_traits>

#include "act_checkpoint.hpp"
#include "handle.hpp"
#include "logprobs.hpp"
#include "shampoo.h"
#include "weight_grad.hpp"

using namespace shp;

namespace {

constexpr int64_t kMaxTokens = INT32_MAX;   // rows of logits and activations
constexpr int64_t kMaxVocab = 1 << 30;
constexpr int64_t kMaxCols = 1 << 20;       // columns of activations and output gradients

inline int64_t cdiv64(int64_t a, int64_t b) { return (a + b - 1) / b; }

// An entry point's body: no exception passes the C boundary.
template <typename F>
shampoo_status entry(void* handle, F&& f) {
  Handle* h = static_cast<Handle*>(handle);
  if (!h) return SHAMPOO_EINVAL;
  h->err.clear();
  try {
    return f(h);
  } catch (const std::bad_alloc&) {
    return SHAMPOO_ENOMEM;
  } catch (...) {
    return SHAMPOO_EHIP;
  }
}

shampoo_status check_dtype(Handle* h, int dtype, const char* what) {
  if (dtype != SHAMPOO_F32 && dtype != SHAMPOO_BF16) return fail(h, SHAMPOO_EINVAL, "%s: bad dtype %d", what, dtype);
  return SHAMPOO_OK;
}

shampoo_status check_logits(Handle* h, int dtype, int64_t rows, int64_t vocab, int64_t ld, int k) {
  STATUS_TRY(check_dtype(h, dtype, "logits"));
  if (rows < 0 || rows >= kMaxTokens) return fail(h, SHAMPOO_EINVAL, "rows = %lld outside [0, 2^31 - 1)", (long long)rows);
  if (vocab < 1 || vocab > kMaxVocab) return fail(h, SHAMPOO_EINVAL, "vocab = %lld outside [1, 2^30]", (long long)vocab);
  if (ld < vocab) return fail(h, SHAMPOO_EINVAL, "ld %lld < vocab %lld", (long long)ld, (long long)vocab);
  if (k < 0 || k > SHAMPOO_MAX_TOP) return fail(h, SHAMPOO_EINVAL, "k = %d outside [0, %d]", k, SHAMPOO_MAX_TOP);
  return SHAMPOO_OK;
}

shampoo_status check_act(Handle* h, int dtype, int64_t rows, int64_t cols, int act) {
  STATUS_TRY(check_dtype(h, dtype, "activations"));
  if (rows < 0 || rows >= kMaxTokens) return fail(h, SHAMPOO_EINVAL, "rows = %lld outside [0, 2^31 - 1)", (long long)rows);
  if (cols < 1 || cols > kMaxCols) return fail(h, SHAMPOO_EINVAL, "cols = %lld outside [1, 2^20]", (long long)cols);
  if (act < SHAMPOO_ACT_NONE || act > SHAMPOO_ACT_SILU) return fail(h, SHAMPOO_EINVAL, "bad activation %d", act);
  return SHAMPOO_OK;
}

// Workgroups of an elementwise launch over n items, one per thread and turn: a
// launch holds fewer than 2^32 threads, so larger ones take turns.
unsigned act_grid(int64_t n) { return (unsigned)std::min<int64_t>(cdiv64(n, kThreads), 1 << 20); }

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// The launches of a pass over a rows x cols tensor and its checkpoint: f(shape,
// grid) for each.
template <typename F>
shampoo_status act_launches(Handle* h, int64_t rows, int64_t cols, hipStream_t s, F&& f) {
  ActShape sh{};
  sh.cols = (int)cols;
  sh.upr = (int)(act_ckpt(rows, cols).ldq / 8);  // at least 4
  int bits = 0;
  while ((int64_t(1) << bits) < sh.upr) ++bits;
  sh.magic = (uint32_t)((((uint64_t(1) << bits) - (uint64_t)sh.upr) << 32) / (uint64_t)sh.upr + 1);
  sh.shift = (uint32_t)bits - 1;
  const int64_t most = INT32_MAX / sh.upr;
  for (sh.row0 = 0; sh.row0 < rows; sh.row0 += most) {
    sh.units = std::min(most, rows - sh.row0) * sh.upr;
    STATUS_TRY(launch(h, SHAMPOO_KCLASS_ACT, s, [&] { f(sh, dim3((unsigned)cdiv64(sh.units, kThreads))); }));
  }
  return SHAMPOO_OK;
}
ActCkptPtr act_parts(const void* ckpt, int64_t rows, int64_t cols) {
  char* p = static_cast<char*>(const_cast<void*>(ckpt));
  return {p, p ? reinterpret_cast<uint8_t*>(p) + act_ckpt(rows, cols).scales : nullptr};
}

// Calls f with the activation as a compile-time constant.
template <typename F>
void with_act(int act, F&& f) {
  switch (act) {
    case SHAMPOO_ACT_RELU: f(std::integral_constant<int, SHAMPOO_ACT_RELU>()); break;
    case SHAMPOO_ACT_GELU: f(std::integral_constant<int, SHAMPOO_ACT_GELU>()); break;
    case SHAMPOO_ACT_GELU_TANH: f(std::integral_constant<int, SHAMPOO_ACT_GELU_TANH>()); break;
    case SHAMPOO_ACT_SILU: f(std::integral_constant<int, SHAMPOO_ACT_SILU>()); break;
    default: f(std::integral_constant<int, SHAMPOO_ACT_NONE>()); break;
  }
}

// Calls f with a null pointer of the element type.
template <typename F>
void with_type(int dtype, F&& f) {
  if (dtype == SHAMPOO_F32) f((float*)nullptr);
  else f((uint16_t*)nullptr);
}

constexpr int64_t kMostItems = 1 << 22;  // parts of rows of one launch

// How a row of logits is cut: waves of a workgroup to a row, and workgroups
// (parts) of a row where there are few rows.  About two waves per SIMD are
// wanted: fewer do not keep enough bytes in flight, and each wave of a row pays
// for finding its own first alternatives.  Rows x 131072 in bf16, 8
// alternatives, us with 1 / 2 / 4 / 8 waves: 8192 rows 388 / 384 / 382 / 445, 1024
// rows 74 / 56 / 52 / 60, 256 rows 69 / 43 / 28 / 23; without alternatives 8192
// rows 381 / 377 / 356 / 361, of 65536 205 / 195 / 188 / 203, of 20000 66 / 67 / 75 /
// 106.  Below 256 rows long rows are cut into parts of 4
// waves and a second launch joins them: one row 12 us, by one workgroup of 8
// waves 19; 64 rows 15 and 20.  Rows of few blocks to a wave do without: 1 x 32768
// 10.0 us, in parts 11.9, 128 x 32768 10.7 and 13.1; 1 x 65536 13.3 and 11.3, without
// alternatives 8.8 and 10.8.
struct LogprobPlan {
  int waves = 1, parts = 1, per_part = 0;
  size_t ws = 0;
};

LogprobPlan logprob_plan(int64_t rows, int64_t vocab, int k, int dtype) {
  LogprobPlan p;
  const int64_t block = dtype == SHAMPOO_BF16 ? LogitBlock<uint16_t>::kN : LogitBlock<float>::kN;
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
double wgrad_rounds(int64_t blocks, int64_t slots, double alone, double full) {
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
WgradPlan wgrad_plan(int64_t rows, int64_t cols, int64_t out, int dtype) {
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

template <typename S, typename SG, int TM, int TN, int WM, int WN>
shampoo_status wgrad_launch(Handle* h, const WgradArgs& q, hipStream_t s) {
  using L = WgradTile<S, TM, TN, WM, WN>;
  auto k = weight_grad_kernel<S, SG, TM, TN, WM, WN>;
  // more LDS than a launch may take by default: asked for once per device
  static std::atomic<uint64_t> asked{0};
  const uint64_t bit = h->device < 64 ? uint64_t(1) << h->device : 0;
  if (!(asked.load(std::memory_order_relaxed) & bit) || !bit) {
    HIP_TRY(h, hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, L::kLdsB));
    asked.fetch_or(bit, std::memory_order_relaxed);
  }
  const int64_t tiles = (int64_t)q.tiles_m * q.tiles_n;
  STATUS_TRY(launch(h, SHAMPOO_KCLASS_WGRAD, s, [&] {
    hipLaunchKernelGGL(k, dim3((unsigned)(tiles * q.splits)), dim3(L::kThr), L::kLdsB, s, q);
  }));
  if (q.splits == 1) return SHAMPOO_OK;
  const int64_t pieces = tiles * (TM / 32) * (TN / 32) * 4;
  return launch(h, SHAMPOO_KCLASS_WGRAD, s, [&] {
    hipLaunchKernelGGL((weight_grad_sum_kernel<SG, TM, TN, WM, WN>), dim3((unsigned)cdiv64(pieces, kThreads / 64)),
                       dim3(kThreads), 0, s, q);
  });
}

}  // namespace

extern "C" {

// ---------------------------------------------------------------- loss
size_t shampoo_token_logprobs_workspace_bytes(int64_t rows, int64_t vocab, int k) {
  if (rows < 1 || rows >= kMaxTokens || vocab < 1 || vocab > kMaxVocab || k < 0 || k > SHAMPOO_MAX_TOP) return 0;
  size_t need = 0;
  for (int dtype : {SHAMPOO_F32, SHAMPOO_BF16}) need = std::max(need, logprob_plan(rows, vocab, k, dtype).ws);
  return need;
}

shampoo_status shampoo_token_logprobs(void* handle, const void* logits, int dtype, int64_t rows, int64_t vocab,
                                      int64_t ld, const int32_t* targets, float* logp, float* lse, float* entropy,
                                      int k, int32_t* top_ids, float* top_logp, void* workspace, size_t ws_bytes,
                                      void* stream) {
  return entry(handle, [&](Handle* h) {
    STATUS_TRY(check_logits(h, dtype, rows, vocab, ld, k));
    if (rows == 0) return SHAMPOO_OK;
    if (!logits || !lse || !logp != !targets || (k > 0 && (!top_ids || !top_logp)))
      return fail(h, SHAMPOO_EINVAL, "logits or lse, one of targets and logp, or top_ids or top_logp is NULL");
    const size_t need = shampoo_token_logprobs_workspace_bytes(rows, vocab, k);
    if (need && (!workspace || ws_bytes < need))
      return fail(h, SHAMPOO_ENOMEM, "workspace %zu bytes < %zu needed", ws_bytes, need);
    if (!aligned16(workspace)) return fail(h, SHAMPOO_EINVAL, "workspace not aligned to 16 bytes");
    DeviceGuard g(h->device);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const LogprobPlan p = logprob_plan(rows, vocab, k, dtype);
    LogprobArgs q{logits, ld, rows, (int)vocab, targets, logp, lse, entropy, k, top_ids, top_logp,
                  p.parts, p.per_part, 0, static_cast<float*>(workspace)};
    // a launch holds fewer than 2^32 threads: more rows than that take several
    for (q.first = 0; q.first < rows * p.parts; q.first += kMostItems) {
      STATUS_TRY(launch(h, SHAMPOO_KCLASS_LOGPROBS, s, [&] {
        with_type(dtype, [&](auto* type) {
          using S = std::remove_pointer_t<decltype(type)>;
          const int64_t n = std::min(rows * p.parts - q.first, kMostItems);
          const dim3 grid((unsigned)(p.waves == 1 ? cdiv64(n, 4) : n));
          auto pick = [&](auto ent) {
            constexpr bool kEnt = decltype(ent)::value;
            return p.waves == 1   ? logprobs_kernel<S, 1, kEnt>
                   : p.waves == 2 ? logprobs_kernel<S, 2, kEnt>
                   : p.waves == 4 ? logprobs_kernel<S, 4, kEnt>
                                  : logprobs_kernel<S, 8, kEnt>;
          };
          auto k1 = entropy ? pick(std::true_type()) : pick(std::false_type());
          hipLaunchKernelGGL(k1, grid, dim3(p.waves == 1 ? kThreads : 64 * p.waves), 0, s, q);
        });
      }));
    }
    if (p.parts == 1) return SHAMPOO_OK;
    return launch(h, SHAMPOO_KCLASS_LOGPROBS, s, [&] {
      with_type(dtype, [&](auto* type) {
        using S = std::remove_pointer_t<decltype(type)>;
        hipLaunchKernelGGL(logprobs_join_kernel<S>, dim3((unsigned)rows), dim3(64), 0, s, q);
      });
    });
  });
}

shampoo_status shampoo_token_logprobs_grad(void* handle, const void* logits, int dtype, int64_t rows, int64_t vocab,
                                           int64_t ld, const int32_t* targets, const float* lse,
                                           const float* entropy, int k, const int32_t* top_ids,
                                           const float* g_logp, const float* g_lse, const float* g_entropy,
                                           const float* g_top, void* dlogits, int64_t ld_d, void* stream) {
  return entry(handle, [&](Handle* h) {
    STATUS_TRY(check_logits(h, dtype, rows, vocab, ld, k));
    if (ld_d < vocab) return fail(h, SHAMPOO_EINVAL, "ld_d %lld < vocab %lld", (long long)ld_d, (long long)vocab);
    if (rows == 0) return SHAMPOO_OK;
    if (!logits || !lse || !dlogits) return fail(h, SHAMPOO_EINVAL, "logits, lse or dlogits is NULL");
    if ((g_logp && !targets) || (g_entropy && !entropy) || (g_top && k > 0 && !top_ids))
      return fail(h, SHAMPOO_EINVAL, "g_logp without targets, g_entropy without entropy, or g_top without top_ids");
    if (dlogits == logits && ld_d != ld) return fail(h, SHAMPOO_EINVAL, "in place, ld_d %lld must be ld %lld", (long long)ld_d, (long long)ld);
    DeviceGuard g(h->device);
    hipStream_t s = static_cast<hipStream_t>(stream);
    LossGradArgs q{logits, ld, rows, (int)vocab, targets, lse, entropy, g_top ? k : 0, top_ids, g_logp, g_lse,
                   g_entropy, g_top, dlogits, ld_d, 1, 1};
    const int64_t block = dtype == SHAMPOO_BF16 ? LogitBlock<uint16_t>::kN : LogitBlock<float>::kN;
    const int64_t blocks = cdiv64(vocab + 7, block);  // a row may begin up to 7 entries into its first
    // one block to a wave (8192 x 131072 in bf16: 729 us; two 766, four 792), two
    // in short rows, where a row's own values cost more (8192 x 5000 with 32
    // alternatives: 44.6 -> 41.7)
    q.per = blocks > 16 ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(2, rows * blocks / 4096));
    q.segs = (int)cdiv64(blocks, q.per);
    return launch(h, SHAMPOO_KCLASS_LOGPROBS, s, [&] {
      with_type(dtype, [&](auto* type) {
        using S = std::remove_pointer_t<decltype(type)>;
        auto k1 = g_entropy ? logprobs_grad_kernel<S, true> : logprobs_grad_kernel<S, false>;
        hipLaunchKernelGGL(k1, dim3((unsigned)std::min<int64_t>(cdiv64(rows * q.segs, 4), 1 << 20)), dim3(kThreads), 0,
                           s, q);
      });
    });
  });
}

// ---------------------------------------------------------------- activations
size_t shampoo_act_checkpoint_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || rows >= kMaxTokens || cols < 1 || cols > kMaxCols) return 0;
  return (size_t)act_ckpt(rows, cols).bytes;
}

shampoo_status shampoo_act_encode(void* handle, const void* X, int dtype, int64_t rows, int64_t cols, int64_t ld_x,
                                  int act, void* Y, int64_t ld_y, void* ckpt_x, void* ckpt_y, void* stream) {
  return entry(handle, [&](Handle* h) {
    STATUS_TRY(check_act(h, dtype, rows, cols, act));
    if (ld_x < cols) return fail(h, SHAMPOO_EINVAL, "ld_x %lld < cols %lld", (long long)ld_x, (long long)cols);
    if (Y && ld_y < cols) return fail(h, SHAMPOO_EINVAL, "ld_y %lld < cols %lld", (long long)ld_y, (long long)cols);
    if (rows == 0) return SHAMPOO_OK;
    if (!X || (!Y && !ckpt_x && !ckpt_y)) return fail(h, SHAMPOO_EINVAL, "X is NULL, or no output is asked for");
    if (Y == X && ld_y != ld_x) return fail(h, SHAMPOO_EINVAL, "in place, ld_y %lld must be ld_x %lld", (long long)ld_y, (long long)ld_x);
    if (!aligned16(ckpt_x) || !aligned16(ckpt_y)) return fail(h, SHAMPOO_EINVAL, "checkpoint not aligned to 16 bytes");
    DeviceGuard g(h->device);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return act_launches(h, rows, cols, s, [&](const ActShape& sh, dim3 grid) {
      with_type(dtype, [&](auto* type) {
        using S = std::remove_pointer_t<decltype(type)>;
        with_act(act, [&](auto a) {
          hipLaunchKernelGGL((act_encode_kernel<S, decltype(a)::value>), grid, dim3(kThreads), 0, s, sh,
                             (const S*)X, ld_x, (S*)Y, ld_y, act_parts(ckpt_x, rows, cols),
                             act_parts(ckpt_y, rows, cols));
        });
      });
    });
  });
}

shampoo_status shampoo_act_decode(void* handle, const void* ckpt, int64_t rows, int64_t cols, void* X, int dtype,
                                  int64_t ld_x, void* stream) {
  return entry(handle, [&](Handle* h) {
    STATUS_TRY(check_act(h, dtype, rows, cols, SHAMPOO_ACT_NONE));
    if (ld_x < cols) return fail(h, SHAMPOO_EINVAL, "ld_x %lld < cols %lld", (long long)ld_x, (long long)cols);
    if (rows == 0) return SHAMPOO_OK;
    if (!ckpt || !X) return fail(h, SHAMPOO_EINVAL, "ckpt or X is NULL");
    if (!aligned16(ckpt)) return fail(h, SHAMPOO_EINVAL, "checkpoint not aligned to 16 bytes");
    DeviceGuard g(h->device);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return act_launches(h, rows, cols, s, [&](const ActShape& sh, dim3 grid) {
      with_type(dtype, [&](auto* type) {
        using S = std::remove_pointer_t<decltype(type)>;
        hipLaunchKernelGGL(act_decode_kernel<S>, grid, dim3(kThreads), 0, s, sh, act_parts(ckpt, rows, cols),
                           (S*)X, ld_x);
      });
    });
  });
}

shampoo_status shampoo_act_grad(void* handle, const void* ckpt, int64_t rows, int64_t cols, int act, const void* dY,
                                int dtype, int64_t ld_dy, void* dX, int64_t ld_dx, void* stream) {
  return entry(handle, [&](Handle* h) {
    STATUS_TRY(check_act(h, dtype, rows, cols, act));
    if (ld_dy < cols || ld_dx < cols)
      return fail(h, SHAMPOO_EINVAL, "ld_dy %lld or ld_dx %lld < cols %lld", (long long)ld_dy, (long long)ld_dx, (long long)cols);
    if (rows == 0) return SHAMPOO_OK;
    if (!ckpt || !dY || !dX) return fail(h, SHAMPOO_EINVAL, "ckpt, dY or dX is NULL");
    if (dX == dY && ld_dx != ld_dy) return fail(h, SHAMPOO_EINVAL, "in place, ld_dx %lld must be ld_dy %lld", (long long)ld_dx, (long long)ld_dy);
    if (!aligned16(ckpt)) return fail(h, SHAMPOO_EINVAL, "checkpoint not aligned to 16 bytes");
    DeviceGuard g(h->device);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return act_launches(h, rows, cols, s, [&](const ActShape& sh, dim3 grid) {
      with_type(dtype, [&](auto* type) {
        using S = std::remove_pointer_t<decltype(type)>;
        with_act(act, [&](auto a) {
          hipLaunchKernelGGL((act_grad_kernel<S, decltype(a)::value>), grid, dim3(kThreads), 0, s, sh,
                             act_parts(ckpt, rows, cols), (const S*)dY, ld_dy, (S*)dX, ld_dx);
        });
      });
    });
  });
}

// ---------------------------------------------------------------- weight gradient
size_t shampoo_act_weight_grad_workspace_bytes(int64_t rows, int64_t cols, int64_t out) {
  if (rows < 0 || rows >= kMaxTokens || cols < 1 || cols > kMaxCols || out < 1 || out > kMaxCols) return 0;
  size_t need = 0;
  for (int dtype : {SHAMPOO_F32, SHAMPOO_BF16}) need = std::max(need, wgrad_plan(rows, cols, out, dtype).ws);
  return need;
}

shampoo_status shampoo_act_weight_grad(void* handle, const void* ckpt, int64_t rows, int64_t cols, const void* dY,
                                       int dtype, int64_t out, int64_t ld_dy, void* G, int g_dtype, int64_t ld_g,
                                       float beta, void* workspace, size_t ws_bytes, void* stream) {
  return entry(handle, [&](Handle* h) {
    STATUS_TRY(check_act(h, dtype, rows, cols, SHAMPOO_ACT_NONE));
    STATUS_TRY(check_dtype(h, g_dtype, "G"));
    if (out < 1 || out > kMaxCols) return fail(h, SHAMPOO_EINVAL, "out = %lld outside [1, 2^20]", (long long)out);
    if (ld_dy < out || ld_g < out)
      return fail(h, SHAMPOO_EINVAL, "ld_dy %lld or ld_g %lld < out %lld", (long long)ld_dy, (long long)ld_g, (long long)out);
    if (!isfinite(beta)) return fail(h, SHAMPOO_EINVAL, "beta is not finite");
    if (!G || (rows > 0 && (!ckpt || !dY))) return fail(h, SHAMPOO_EINVAL, "ckpt, dY or G is NULL");
    if (G == dY || G == ckpt) return fail(h, SHAMPOO_EINVAL, "G must not be dY or the checkpoint");
    if (!aligned16(ckpt) || !aligned16(workspace))
      return fail(h, SHAMPOO_EINVAL, "checkpoint or workspace not aligned to 16 bytes");
    const size_t need = shampoo_act_weight_grad_workspace_bytes(rows, cols, out);
    if (need && (!workspace || ws_bytes < need))
      return fail(h, SHAMPOO_ENOMEM, "workspace %zu bytes < %zu needed", ws_bytes, need);
    const WgradPlan p = wgrad_plan(rows, cols, out, dtype);
    if (p.tiles_m * p.tiles_n * p.splits > INT32_MAX / 512)
      return fail(h, SHAMPOO_EUNSUPPORTED, "G of %lld x %lld", (long long)cols, (long long)out);
    DeviceGuard g(h->device);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const ActCkpt c = act_ckpt(rows, cols);
    WgradArgs q{};
    q.codes = static_cast<const char*>(ckpt);
    q.scales = static_cast<const uint8_t*>(ckpt) + c.scales;
    q.ldq = c.ldq;
    q.dY = dY;
    q.ld_dy = ld_dy;
    q.rows = rows;
    q.cols = (int)cols;
    q.out = (int)out;
    q.G = G;
    q.ld_g = ld_g;
    q.beta = beta;
    q.part = p.splits > 1 ? static_cast<float*>(workspace) : nullptr;
    q.splits = p.splits;
    q.per_split = p.per_split;
    q.tiles_m = (int)p.tiles_m;
    q.tiles_n = (int)p.tiles_n;
    shampoo_status st = SHAMPOO_OK;
    with_type(dtype, [&](auto* type) {
      using S = std::remove_pointer_t<decltype(type)>;
      with_type(g_dtype, [&](auto* gtype) {
        using SG = std::remove_pointer_t<decltype(gtype)>;
        if (rows == 0)
          st = launch(h, SHAMPOO_KCLASS_WGRAD, s, [&] {
            hipLaunchKernelGGL(weight_grad_scale_kernel<SG>, dim3(act_grid(cols * out)), dim3(kThreads), 0, s, q);
          });
        else if (p.tile_m == 256)
          st = wgrad_launch<S, SG, 256, 256, 128, 64>(h, q, s);
        else if (p.tile_n == 128)
          st = wgrad_launch<S, SG, 128, 128, 64, 32>(h, q, s);
        else if constexpr (sizeof(S) == 2)
          st = wgrad_launch<S, SG, 128, 256, 64, 64>(h, q, s);
      });
    });
    return st;
  });
}

}  // extern "C"
