// Host side that the calls around the step share: argument checks, dispatch on
// types, and launches over the units of a tensor.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <new>
#include <type_traits>

#include "act_checkpoint.hpp"
#include "handle.hpp"
#include "layer_plans.hpp"

namespace shp {

constexpr int64_t kMaxTokens = INT32_MAX;   // rows of logits and activations
constexpr int64_t kMaxVocab = 1 << 30;
constexpr int64_t kMaxCols = 1 << 20;       // columns of activations and output gradients

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

inline shampoo_status check_dtype(Handle* h, int dtype, const char* what) {
  if (dtype != SHAMPOO_F32 && dtype != SHAMPOO_BF16) return fail(h, SHAMPOO_EINVAL, "%s: bad dtype %d", what, dtype);
  return SHAMPOO_OK;
}

// Workgroups of an elementwise launch over n items, one per thread and turn: a
// launch holds fewer than 2^32 threads, so larger ones take turns.
inline unsigned act_grid(int64_t n) { return (unsigned)std::min<int64_t>(cdiv64(n, kThreads), 1 << 20); }

// Buffers of a call that must share no memory.
inline shampoo_status check_apart(Handle* h, const Span& a, const char* what_a, const Span& b, const char* what_b) {
  return apart(a, b) ? SHAMPOO_OK : fail(h, SHAMPOO_EINVAL, "%s and %s overlap", what_a, what_b);
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// A tensor of `cols` columns in `upr` units of 8 columns a row (at least 2).
inline ActShape unit_shape(int64_t cols, int64_t upr) {
  ActShape sh{};
  sh.cols = (int)cols;
  sh.upr = (int)upr;
  int bits = 0;
  while ((int64_t(1) << bits) < sh.upr) ++bits;
  sh.magic = (uint32_t)((((uint64_t(1) << bits) - (uint64_t)sh.upr) << 32) / (uint64_t)sh.upr + 1);
  sh.shift = (uint32_t)bits - 1;
  return sh;
}

// The launches of a pass over a rows x cols tensor: f(shape, grid) for each.
template <typename F>
shampoo_status unit_launches(Handle* h, int cls, int64_t rows, int64_t cols, int64_t upr, hipStream_t s, F&& f) {
  ActShape sh = unit_shape(cols, upr);
  const int64_t most = INT32_MAX / sh.upr;
  for (sh.row0 = 0; sh.row0 < rows; sh.row0 += most) {
    sh.units = std::min(most, rows - sh.row0) * sh.upr;
    STATUS_TRY(launch(h, cls, s, [&] { f(sh, dim3((unsigned)cdiv64(sh.units, kThreads))); }));
  }
  return SHAMPOO_OK;
}
// ... and its checkpoint.
template <typename F>
shampoo_status act_launches(Handle* h, int64_t rows, int64_t cols, hipStream_t s, F&& f) {
  return unit_launches(h, SHAMPOO_KCLASS_ACT, rows, cols, act_ckpt(rows, cols).ldq / 8, s, f);
}

// Calls f with a null pointer of the element type.
template <typename F>
void with_type(int dtype, F&& f) {
  if (dtype == SHAMPOO_F32) f((float*)nullptr);
  else f((uint16_t*)nullptr);
}

}  // namespace shp
