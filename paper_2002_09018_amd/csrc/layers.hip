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
#include "layer_host.hpp"
#include "layer_plans.hpp"
#include "logprobs.hpp"
#include "shampoo.h"
#include "weight_grad.hpp"

using namespace shp;

namespace {

shampoo_status check_logits(Handle* h, int dtype, int64_t rows, int64_t vocab, int64_t ld, int k) {
  STATUS_TRY(check_dtype(h, dtype, "logits"));
  if (rows < 0 || rows > kMaxTokens) return fail(h, SHAMPOO_EINVAL, "rows = %lld outside [0, 2^31)", (long long)rows);
  if (vocab < 1 || vocab > kMaxVocab) return fail(h, SHAMPOO_EINVAL, "vocab = %lld outside [1, 2^30]", (long long)vocab);
  if (ld < vocab) return fail(h, SHAMPOO_EINVAL, "ld %lld < vocab %lld", (long long)ld, (long long)vocab);
  if (k < 0 || k > SHAMPOO_MAX_TOP) return fail(h, SHAMPOO_EINVAL, "k = %d outside [0, %d]", k, SHAMPOO_MAX_TOP);
  return SHAMPOO_OK;
}

shampoo_status check_act(Handle* h, int dtype, int64_t rows, int64_t cols, int act) {
  STATUS_TRY(check_dtype(h, dtype, "activations"));
  if (rows < 0 || rows > kMaxTokens) return fail(h, SHAMPOO_EINVAL, "rows = %lld outside [0, 2^31)", (long long)rows);
  if (cols < 1 || cols > kMaxCols) return fail(h, SHAMPOO_EINVAL, "cols = %lld outside [1, 2^20]", (long long)cols);
  if (act < SHAMPOO_ACT_NONE || act > SHAMPOO_ACT_SILU) return fail(h, SHAMPOO_EINVAL, "bad activation %d", act);
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

static_assert(LogitBlock<uint16_t>::kN == kLogitBlockB / 2 && LogitBlock<float>::kN == kLogitBlockB / 4, "");

constexpr int64_t kMostItems = 1 << 22;  // parts of rows of one launch

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
  if (rows < 1 || rows > kMaxTokens || vocab < 1 || vocab > kMaxVocab || k < 0 || k > SHAMPOO_MAX_TOP) return 0;
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
    STATUS_TRY(check_apart(h, span(workspace, (int64_t)need), "workspace", span(logits, rows, vocab, ld, dtype), "logits"));
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
    if (dlogits != logits)
      STATUS_TRY(check_apart(h, span(dlogits, rows, vocab, ld_d, dtype), "dlogits", span(logits, rows, vocab, ld, dtype), "logits"));
    DeviceGuard g(h->device);
    hipStream_t s = static_cast<hipStream_t>(stream);
    LossGradArgs q{logits, ld, rows, (int)vocab, targets, lse, entropy, g_top ? k : 0, top_ids, g_logp, g_lse,
                   g_entropy, g_top, dlogits, ld_d, 1, 1};
    const LossGradPlan p = loss_grad_plan(rows, vocab, dtype);
    q.per = p.per;
    q.segs = p.segs;
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
  if (rows < 0 || rows > kMaxTokens || cols < 1 || cols > kMaxCols) return 0;
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
    const Span x = span(X, rows, cols, ld_x, dtype), y = span(Y, rows, cols, ld_y, dtype);
    const int64_t bytes = act_ckpt(rows, cols).bytes;
    const Span cx = span(ckpt_x, bytes), cy = span(ckpt_y, bytes);
    if (Y != X) STATUS_TRY(check_apart(h, y, "Y", x, "X"));
    STATUS_TRY(check_apart(h, cx, "ckpt_x", x, "X"));
    STATUS_TRY(check_apart(h, cx, "ckpt_x", y, "Y"));
    STATUS_TRY(check_apart(h, cy, "ckpt_y", x, "X"));
    STATUS_TRY(check_apart(h, cy, "ckpt_y", y, "Y"));
    STATUS_TRY(check_apart(h, cx, "ckpt_x", cy, "ckpt_y"));
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
    STATUS_TRY(check_apart(h, span(ckpt, act_ckpt(rows, cols).bytes), "ckpt", span(X, rows, cols, ld_x, dtype), "X"));
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
    const Span c = span(ckpt, act_ckpt(rows, cols).bytes), y = span(dY, rows, cols, ld_dy, dtype);
    const Span x = span(dX, rows, cols, ld_dx, dtype);
    if (dX != dY) STATUS_TRY(check_apart(h, x, "dX", y, "dY"));
    STATUS_TRY(check_apart(h, c, "ckpt", x, "dX"));
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
  if (rows < 0 || rows > kMaxTokens || cols < 1 || cols > kMaxCols || out < 1 || out > kMaxCols) return 0;
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
    if (!aligned16(ckpt) || !aligned16(workspace))
      return fail(h, SHAMPOO_EINVAL, "checkpoint or workspace not aligned to 16 bytes");
    const size_t need = shampoo_act_weight_grad_workspace_bytes(rows, cols, out);
    if (need && (!workspace || ws_bytes < need))
      return fail(h, SHAMPOO_ENOMEM, "workspace %zu bytes < %zu needed", ws_bytes, need);
    const Span sg = span(G, cols, out, ld_g, g_dtype), sy = span(dY, rows, out, ld_dy, dtype);
    const Span sc = span(ckpt, act_ckpt(rows, cols).bytes), sw = span(workspace, (int64_t)need);
    STATUS_TRY(check_apart(h, sg, "G", sy, "dY"));
    STATUS_TRY(check_apart(h, sg, "G", sc, "ckpt"));
    STATUS_TRY(check_apart(h, sw, "workspace", sg, "G"));
    STATUS_TRY(check_apart(h, sw, "workspace", sy, "dY"));
    STATUS_TRY(check_apart(h, sw, "workspace", sc, "ckpt"));
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
