// Host side of the calls of a model's own layers: the loss from the last activations,
// the gated feed-forward block, dropout (vocab_loss.hpp, gated_ffn.hpp, dropout.hpp).
#include <hip/hip_runtime.h>

#include <math.h>

#include <algorithm>
#include <atomic>
#include <initializer_list>

#include "dropout.hpp"
#include "few_rows.hpp"
#include "gated_ffn.hpp"
#include "layer_host.hpp"
#include "shampoo.h"
#include "stream_plans.hpp"
#include "vocab_loss.hpp"

using namespace shp;

namespace {

// Shapes of a product whose operands have PA and PB planes.
template <int PA, int PB>
struct Shapes {
  using Solo = MmaShape<32, 64, 32, 64, 2, PA, PB, 4>;
  using Few = MmaShape<32, 128, 32, 64, 2, PA, PB>;
  using Thin = MmaShape<64, 64, 32, 32, 2, PA, PB>;
  using Mid = MmaShape<128, 128, 32, 64, 3, PA, PB>;
  using Big = MmaShape<256, 128, 64, 64, 2, PA, PB>;
  using BigWeight = Big;
};
template <>
struct Shapes<1, 1> {
  using Solo = MmaShape<32, 64, 32, 64, 3, 1, 1, 8>;
  using Few = MmaShape<32, 128, 32, 64, 4>;
  using Thin = MmaShape<64, 64, 32, 32, 2>;
  using Mid = MmaShape<128, 128, 64, 64, 2, 1, 1, 0, 64>;
  using Big = MmaShape<256, 256, 128, 64, 2, 1, 1, 0, 64>;
  using BigWeight = MmaShape<256, 256, 128, 64, 3>;
};

// ... of two and one, whose large tiles take rounds of one.
template <>
struct Shapes<kDxTerms, 1> {
  using Solo = MmaShape<32, 64, 32, 64, 2, kDxTerms, 1, 8>;
  using Few = MmaShape<32, 128, 32, 64, 3, kDxTerms, 1>;
  using Thin = MmaShape<64, 64, 32, 32, 2, kDxTerms, 1>;
  using Mid = Shapes<1, 1>::Mid;
  using Big = Shapes<1, 1>::Big;
  using BigWeight = Shapes<1, 1>::BigWeight;
};

// A buffer of a call and what to call it.
struct Named {
  Span s;
  const char* name;
};

// Every buffer that is written shares no memory with any other.
shampoo_status check_all_apart(Handle* h, std::initializer_list<Named> written, std::initializer_list<Named> read) {
  for (const Named* a = written.begin(); a != written.end(); ++a) {
    for (const Named* b = a + 1; b != written.end(); ++b) STATUS_TRY(check_apart(h, a->s, a->name, b->s, b->name));
    for (const Named& b : read) STATUS_TRY(check_apart(h, a->s, a->name, b.s, b.name));
  }
  return SHAMPOO_OK;
}

shampoo_status check_room(Handle* h, const void* workspace, size_t ws_bytes, size_t need) {
  if (need && (!workspace || ws_bytes < need))
    return fail(h, SHAMPOO_ENOMEM, "workspace %zu bytes < %zu needed", ws_bytes, need);
  if (!aligned16(workspace)) return fail(h, SHAMPOO_EINVAL, "workspace not aligned to 16 bytes");
  return SHAMPOO_OK;
}

shampoo_status check_size(Handle* h, int64_t v, int64_t lo, int64_t hi, const char* what) {
  if (v < lo || v > hi)
    return fail(h, SHAMPOO_EINVAL, "%s = %lld outside [%lld, %lld]", what, (long long)v, (long long)lo, (long long)hi);
  return SHAMPOO_OK;
}
shampoo_status check_ld(Handle* h, int64_t ld, int64_t cols, const char* what) {
  if (ld < cols || ld > (int64_t(1) << 40))
    return fail(h, SHAMPOO_EINVAL, "%s %lld outside [%lld, 2^40]", what, (long long)ld, (long long)cols);
  return SHAMPOO_OK;
}

// Whether the products can read a matrix as it lies: 16-byte chunks that lie whole in
// its rows, and tiles whose offsets fit 31 bits.
bool as_it_lies(const void* p, int64_t ld, int64_t cols, int dtype) {
  return dtype == SHAMPOO_BF16 && aligned16(p) && cols % 8 == 0 && ld % 8 == 0 && ld <= (1 << 21);
}

// An operand's planes: the first, and the elements from one to the next.
struct Planes16 {
  const uint16_t* p;
  int64_t ld, plane;
};

// Collects the matrices of a call that have to be copied, and launches the copies
// together (at most 2^31 units of 8 columns a launch).
struct Packer {
  Handle* h;
  int cls, dtype;
  hipStream_t s;
  PackArgs q{};
  uint32_t blocks = 0;

  shampoo_status flush() {
    if (q.jobs == 0) return SHAMPOO_OK;
    const dim3 grid(blocks);
    STATUS_TRY(launch(h, cls, s, [&] {
      with_type(dtype, [&](auto* type) {
        using S = std::remove_pointer_t<decltype(type)>;
        hipLaunchKernelGGL(pack_kernel<S>, grid, dim3(kThreads), 0, s, q);
      });
    }));
    q.jobs = 0;
    blocks = 0;
    return SHAMPOO_OK;
  }
  // X (rows x cols) as the products read it: itself, or its planes in `room`.
  shampoo_status take(const void* X, int64_t rows, int64_t cols, int64_t ld, bool pack, const PackPlan& p, void* room,
                      Planes16* out) {
    if (!pack) {
      *out = {static_cast<const uint16_t*>(X), ld, 0};
      return SHAMPOO_OK;
    }
    *out = {static_cast<const uint16_t*>(room), p.ld, p.plane};
    ActShape sh = unit_shape(cols, p.ld / 8);
    const int64_t most = (INT32_MAX / 2) / sh.upr;
    for (sh.row0 = 0; sh.row0 < rows; sh.row0 += most) {
      sh.units = std::min(most, rows - sh.row0) * sh.upr;
      const int64_t n = cdiv64(sh.units, kThreads);
      if (q.jobs == kMostPacks || blocks + n > (1 << 23)) STATUS_TRY(flush());
      q.job[q.jobs++] = {sh, X, ld, static_cast<uint16_t*>(room), p.plane, blocks};
      blocks += (uint32_t)n;
    }
    return SHAMPOO_OK;
  }
};

// One more product of the sum.
void add_seg(MmaArgs& q, const Planes16& a, const Planes16& b, const Planes16* b2 = nullptr) {
  q.seg[q.segs++] = {a.p, b.p, b2 ? b2->p : nullptr, a.plane, b.plane, b2 ? b2->plane : 0,
                     (int)a.ld, (int)b.ld, b2 ? (int)b2->ld : 0};
}

// Fills what the plan says; ka and kb are rounded up to 8 where the contraction
// lies along rows (their padding is zeros).
void use_plan(MmaArgs& q, const MmaPlan& p, int64_t M, int64_t N, int64_t K, int la, int lb, void* part) {
  q.M = (int)M;
  q.N = (int)N;
  q.ka = (int)(la == kLayoutRow ? cdiv64(K, 8) * 8 : K);
  q.kb = (int)(lb == kLayoutRow ? cdiv64(K, 8) * 8 : K);
  q.seg_stages = (int)p.seg_stages;
  q.tiles_m = (int)p.tiles_m;
  q.tiles_n = (int)p.tiles_n;
  q.splits = p.splits;
  q.per_split = p.per_split;
  q.part = p.part ? static_cast<float*>(part) : nullptr;
  q.ld_part = p.ld_part;
}

// More LDS than a launch may take by default: asked for once per kernel and device.
template <typename K>
shampoo_status ask_lds(Handle* h, K k, int bytes, std::atomic<uint64_t>& asked) {
  const uint64_t bit = h->device < 64 ? uint64_t(1) << h->device : 0;
  if (!(asked.load(std::memory_order_relaxed) & bit) || !bit) {
    HIP_TRY(h, hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    asked.fetch_or(bit, std::memory_order_relaxed);
  }
  return SHAMPOO_OK;
}

int64_t groups_of(const MmaArgs& q) { return (int64_t)q.tiles_m * q.tiles_n * q.splits; }

template <typename T, int LA, int LB, typename E>
shampoo_status mma_launch(Handle* h, int cls, const MmaArgs& q, const E& e, hipStream_t s) {
  auto k = mma_kernel<T, LA, LB, E>;
  constexpr int kLds = T::kLdsB + (E::kState ? T::kStateB : 0);
  static std::atomic<uint64_t> asked{0};
  STATUS_TRY(ask_lds(h, k, kLds, asked));
  return launch(h, cls, s, [&] {
    hipLaunchKernelGGL(k, dim3((unsigned)groups_of(q)), dim3(T::kThr), kLds, s, q, e);
  });
}

// The product of operands of PA and PB planes; what was cut is left in q.part.
template <int LA, int LB, int PA, int PB, typename E>
shampoo_status product(Handle* h, int cls, int shape, const MmaArgs& q, const E& e, hipStream_t s) {
  using K = Shapes<PA, PB>;
  if constexpr (LA == kLayoutRow && !E::kWhole)
    if (shape == kShapeSolo) return mma_launch<typename K::Solo, LA, LB>(h, cls, q, e, s);
  if (shape == kShapeFew) {
    if constexpr (LA == kLayoutRow) return mma_launch<typename K::Few, LA, LB>(h, cls, q, e, s);
    else return mma_launch<typename K::Thin, LA, LB>(h, cls, q, e, s);
  }
  if (shape == kShapeMid) return mma_launch<typename K::Mid, LA, LB>(h, cls, q, e, s);
  using B = std::conditional_t<LA == kLayoutK, typename K::BigWeight, typename K::Big>;
  return mma_launch<B, LA, LB>(h, cls, q, e, s);
}
// ... of operands that both have one or both three.
template <int LA, int LB, typename E>
shampoo_status product(Handle* h, int cls, int planes, int shape, const MmaArgs& q, const E& e, hipStream_t s) {
  return planes == 1 ? product<LA, LB, 1, 1>(h, cls, shape, q, e, s) : product<LA, LB, 3, 3>(h, cls, shape, q, e, s);
}

// A product that reads B (of the type dtype, at any address) where it lies.
template <typename S, int LB, typename E>
shampoo_status few_product(Handle* h, int cls, const FewArgs& w, const E& e, hipStream_t s) {
  auto k = few_kernel<S, LB, E>;
  constexpr int kLds = FewShape::kLdsB + (E::kState ? FewShape::kStateB : 0);
  static std::atomic<uint64_t> asked{0};
  STATUS_TRY(ask_lds(h, k, kLds, asked));
  return launch(h, cls, s, [&] {
    hipLaunchKernelGGL(k, dim3((unsigned)groups_of(w.q)), dim3(FewShape::kThr), kLds, s, w, e);
  });
}
template <int LB, typename E>
shampoo_status few_product(Handle* h, int cls, int dtype, const FewArgs& w, const E& e, hipStream_t s) {
  return dtype == SHAMPOO_BF16 ? few_product<uint16_t, LB>(h, cls, w, e, s) : few_product<float, LB>(h, cls, w, e, s);
}
FewSeg few_seg(const Planes16& a, const void* b, int64_t ldb, const void* b2 = nullptr, int64_t ldb2 = 0) {
  return {a.p, a.plane, (int)a.ld, b, b2, ldb, ldb2};
}

// The epilogue over the parts.
template <typename E>
shampoo_status join(Handle* h, int cls, const MmaArgs& q, const E& e, hipStream_t s) {
  const int64_t units = (int64_t)q.M * cdiv64(q.N, 8);
  return launch(h, cls, s, [&] {
    hipLaunchKernelGGL(mma_join_kernel<E>, dim3(act_grid(units)), dim3(kThreads), 0, s, q, e);
  });
}

// dX = D B of a gradient D that is kept in d_planes terms: as many as B has planes, or more
// beside a B of one, of which kDxTerms count.  What was cut is left in q.part.
template <int LB>
shampoo_status dx_product(Handle* h, int cls, int planes, int d_planes, int shape, const MmaArgs& q,
                          const OutEpilogue& e, hipStream_t s) {
  if (d_planes == planes) return product<kLayoutRow, LB>(h, cls, planes, shape, q, e, s);
  return product<kLayoutRow, LB, kDxTerms, 1>(h, cls, shape, q, OutTermsEpilogue(e), s);
}
template <int LB>
shampoo_status few_dx_product(Handle* h, int cls, int dtype, int d_planes, const FewArgs& w, const OutEpilogue& e,
                              hipStream_t s) {
  if (dtype == SHAMPOO_F32) return few_product<float, LB>(h, cls, w, e, s);
  return d_planes == 1 ? few_product<uint16_t, LB>(h, cls, w, e, s)
                       : few_product<uint16_t, LB>(h, cls, w, OutTermsEpilogue(e), s);
}

// dX and the weights' gradient in one launch, and what was cut of them in another.
template <int LB, int P, typename E>
shampoo_status two_products(Handle* h, int cls, const MmaArgs& x, const E& ex, const MmaArgs& w, const E& ew,
                            hipStream_t s) {
  using T = typename Shapes<P, P>::Mid;
  auto k = mma_two_kernel<T, LB, E>;
  static std::atomic<uint64_t> asked{0};
  STATUS_TRY(ask_lds(h, k, T::kLdsB, asked));
  const int first = (int)groups_of(x);
  STATUS_TRY(launch(h, cls, s, [&] {
    hipLaunchKernelGGL(k, dim3((unsigned)(first + groups_of(w))), dim3(T::kThr), T::kLdsB, s, x, ex, w, ew, first);
  }));
  if (!x.part || !w.part) {
    if (x.part) return join<OutEpilogue>(h, cls, x, ex, s);
    return w.part ? join<OutEpilogue>(h, cls, w, ew, s) : SHAMPOO_OK;
  }
  const unsigned nx = act_grid((int64_t)x.M * cdiv64(x.N, 8)), nw = act_grid((int64_t)w.M * cdiv64(w.N, 8));
  return launch(h, cls, s, [&] {
    hipLaunchKernelGGL(mma_join_two_kernel<OutEpilogue>, dim3(nx + nw), dim3(kThreads), 0, s, x,
                       static_cast<const OutEpilogue&>(ex), w, static_cast<const OutEpilogue&>(ew), (int)nx);
  });
}
template <int LB>
shampoo_status two_products(Handle* h, int cls, int planes, const MmaArgs& x, const OutEpilogue& ex, const MmaArgs& w,
                            const OutEpilogue& ew, hipStream_t s) {
  return planes == 1 ? two_products<LB, 1>(h, cls, x, ex, w, ew, s) : two_products<LB, 3>(h, cls, x, ex, w, ew, s);
}

// A weight gradient X^T D or D^T X of D's terms: three where X has one plane and D's
// gradient is kept in fp32.
template <bool D_FIRST>
shampoo_status weight_product(Handle* h, int cls, int x_planes, int d_planes, int shape, const MmaArgs& q,
                              const OutEpilogue& e, hipStream_t s) {
  constexpr int K = kLayoutK;
  shampoo_status st;
  if (x_planes == d_planes) st = product<K, K>(h, cls, x_planes, shape, q, e, s);
  else if (D_FIRST && d_planes == kDxTerms) st = product<K, K, kDxTerms, 1>(h, cls, shape, q, OutTermsEpilogue(e), s);
  else st = product<K, K, D_FIRST ? 3 : 1, D_FIRST ? 1 : 3>(h, cls, shape, q, e, s);
  STATUS_TRY(st);
  return q.part ? join(h, cls, q, e, s) : SHAMPOO_OK;
}

// Calls f with a null pointer of the type of the inputs and the number of bf16 terms of a
// gradient between products (grad_planes): fp32 inputs always have three.
template <typename F>
void with_terms(int dtype, int terms, F&& f) {
  if (dtype == SHAMPOO_F32) f((float*)nullptr, std::integral_constant<int, 3>());
  else if (terms == 3) f((uint16_t*)nullptr, std::integral_constant<int, 3>());
  else f((uint16_t*)nullptr, std::integral_constant<int, 1>());
}

shampoo_status scaled(Handle* h, int cls, void* C, int dtype, int64_t rows, int64_t cols, int64_t ld, float beta,
                      hipStream_t s) {
  return launch(h, cls, s, [&] {
    with_type(dtype, [&](auto* type) {
      using S = std::remove_pointer_t<decltype(type)>;
      hipLaunchKernelGGL(scale_kernel<S>, dim3(act_grid(rows * cols)), dim3(kThreads), 0, s, static_cast<S*>(C), rows,
                         cols, ld, beta);
    });
  });
}

// Products that a call would need in more tiles than a launch holds are refused before
// anything is enqueued.
shampoo_status check_tiles(Handle* h, std::initializer_list<MmaPlan> plans) {
  for (const MmaPlan& p : plans)
    if (!fits(p))
      return fail(h, SHAMPOO_EUNSUPPORTED, "a product of %lld x %lld tiles", (long long)p.tiles_m, (long long)p.tiles_n);
  return SHAMPOO_OK;
}

const char* typed(const void* p, int64_t elements, int dtype) {
  return static_cast<const char*>(p) + elements * (dtype == SHAMPOO_BF16 ? 2 : 4);
}

shampoo_status check_vocab(Handle* h, int dtype, int64_t rows, int64_t dim, int64_t vocab, int64_t ld_x, int64_t ld_w) {
  STATUS_TRY(check_dtype(h, dtype, "X and W"));
  STATUS_TRY(check_size(h, rows, 0, kMaxTokens, "rows"));
  STATUS_TRY(check_size(h, dim, 1, kMaxCols, "dim"));
  STATUS_TRY(check_size(h, vocab, 1, kMaxVocab, "vocab"));
  STATUS_TRY(check_ld(h, ld_x, dim, "ld_x"));
  return check_ld(h, ld_w, dim, "ld_w");
}

shampoo_status check_ffn(Handle* h, int dtype, int64_t rows, int64_t dim, int64_t width, int64_t ld_x, int64_t ld_wg,
                         int64_t ld_wu, int act) {
  STATUS_TRY(check_dtype(h, dtype, "X, Wg and Wu"));
  STATUS_TRY(check_size(h, rows, 0, kMaxTokens, "rows"));
  STATUS_TRY(check_size(h, dim, 1, kMaxCols, "dim"));
  STATUS_TRY(check_size(h, width, 1, kMaxCols / 2, "width"));
  if (act < SHAMPOO_ACT_NONE || act > SHAMPOO_ACT_SILU) return fail(h, SHAMPOO_EINVAL, "bad activation %d", act);
  STATUS_TRY(check_ld(h, ld_x, dim, "ld_x"));
  STATUS_TRY(check_ld(h, ld_wg, width, "ld_wg"));
  return check_ld(h, ld_wu, width, "ld_wu");
}

bool sizes_ok(int64_t rows, int64_t dim, int64_t n, int64_t most, int dtype) {
  return rows >= 0 && rows <= kMaxTokens && dim >= 1 && dim <= kMaxCols && n >= 1 && n <= most &&
         (dtype == SHAMPOO_F32 || dtype == SHAMPOO_BF16);
}

}  // namespace

extern "C" {

// ---------------------------------------------------------------- loss
size_t shampoo_vocab_logprobs_workspace_bytes(int64_t rows, int64_t dim, int64_t vocab, int dtype) {
  if (!sizes_ok(rows, dim, vocab, kMaxVocab, dtype) || rows == 0) return 0;
  const size_t need = vocab_plan(rows, dim, vocab, dtype, true, true).need;
  if (vocab_alike(rows, dim, vocab, dtype)) return need;
  return std::max(need, vocab_plan(rows, dim, vocab, dtype, true, false).bytes);
}

shampoo_status shampoo_vocab_logprobs(void* handle, const void* X, const void* W, int dtype, int64_t rows, int64_t dim,
                                      int64_t vocab, int64_t ld_x, int64_t ld_w, const int32_t* targets, float* logp,
                                      float* lse, void* workspace, size_t ws_bytes, void* stream) {
  return entry(handle, [&](Handle* h) {
    STATUS_TRY(check_vocab(h, dtype, rows, dim, vocab, ld_x, ld_w));
    if (rows == 0) return SHAMPOO_OK;
    if (!X || !W || !lse || !logp != !targets)
      return fail(h, SHAMPOO_EINVAL, "X, W or lse, or one of targets and logp is NULL");
    const bool pack_x = !as_it_lies(X, ld_x, dim, dtype), pack_w = !as_it_lies(W, ld_w, dim, dtype);
    const VocabPlan p = vocab_plan(rows, dim, vocab, dtype, pack_x, pack_w);
    const size_t need = vocab_alike(rows, dim, vocab, dtype) ? p.need
                                                       : shampoo_vocab_logprobs_workspace_bytes(rows, dim, vocab, dtype);
    STATUS_TRY(check_room(h, workspace, ws_bytes, need));
    STATUS_TRY(check_all_apart(
        h, {{span(workspace, (int64_t)need), "workspace"}, {span(logp, rows * 4), "logp"}, {span(lse, rows * 4), "lse"}},
        {{span(X, rows, dim, ld_x, dtype), "X"}, {span(W, vocab, dim, ld_w, dtype), "W"}, {span(targets, rows * 4), "targets"}}));
    DeviceGuard g(h->device);
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    constexpr int kCls = SHAMPOO_KCLASS_VOCAB;
    STATUS_TRY(check_tiles(h, {p.mma[0], p.mma[1]}));
    Planes16 x, w;
    Packer packer{h, kCls, dtype, s};
    STATUS_TRY(packer.take(X, rows, dim, ld_x, pack_x, p.x, ws + p.at_x, &x));
    auto* stat = reinterpret_cast<f32x2p*>(ws + p.at_stat);
    auto* z_target = reinterpret_cast<float*>(ws + p.at_target);
    int64_t entry0 = 0;
    for (int64_t i = 0; i < p.pieces; ++i) {
      const int64_t v0 = i * p.piece, n = std::min(p.piece, vocab - v0);
      const MmaPlan& m = p.mma[i == p.pieces - 1];
      const char* here = typed(W, v0 * ld_w, dtype);
      STATUS_TRY(packer.take(here, n, dim, ld_w, pack_w && !p.direct, p.w, ws + p.at_w, &w));
      STATUS_TRY(packer.flush());
      MmaArgs q{};
      add_seg(q, x, w);
      use_plan(q, m, rows, n, dim, kLayoutRow, kLayoutRow, ws + p.at_part);
      const LseEpilogue e({targets, (int)vocab, (int)v0}, stat + entry0, p.entries, z_target, (int)n);
      if (p.direct) STATUS_TRY(few_product<kLayoutRow>(h, kCls, dtype, {q, {few_seg(x, here, ld_w)}, (int)dim}, e, s));
      else STATUS_TRY((product<kLayoutRow, kLayoutRow>(h, kCls, p.x.planes, m.shape, q, e, s)));
      if (q.part) {
        STATUS_TRY(launch(h, kCls, s, [&] {
          hipLaunchKernelGGL(logit_stat_kernel, dim3((unsigned)stat_groups(rows, n)), dim3(kThreads), 0, s, q, e);
        }));
      }
      entry0 += vocab_entries(m, n);
    }
    return launch(h, kCls, s, [&] {
      const int64_t groups = std::min<int64_t>(cdiv64(rows, kThreads / 64), 1 << 20);
      hipLaunchKernelGGL(lse_join_kernel, dim3((unsigned)groups), dim3(kThreads), 0, s, rows, (int)p.entries, stat,
                         VocabTargets{targets, (int)vocab, 0}, z_target, logp, lse);
    });
  });
}

size_t shampoo_vocab_logprobs_grad_workspace_bytes(int64_t rows, int64_t dim, int64_t vocab, int dtype, int g_dtype) {
  if (!sizes_ok(rows, dim, vocab, kMaxVocab, dtype) || rows == 0) return 0;
  if (g_dtype != SHAMPOO_F32 && g_dtype != SHAMPOO_BF16) return 0;
  const size_t need = vocab_grad_plan(rows, dim, vocab, dtype, g_dtype, true, true).need;
  if (vocab_grad_alike(rows, dim, vocab, dtype, grad_planes(dtype, g_dtype))) return need;
  return std::max(need, vocab_grad_plan(rows, dim, vocab, dtype, g_dtype, true, false).bytes);
}

shampoo_status shampoo_vocab_logprobs_grad(void* handle, const void* X, const void* W, int dtype, int64_t rows,
                                           int64_t dim, int64_t vocab, int64_t ld_x, int64_t ld_w,
                                           const int32_t* targets, const float* lse, const float* g_logp,
                                           const float* g_lse, void* dX, int64_t ld_dx, void* dW, int g_dtype,
                                           int64_t ld_dw, float beta, void* workspace, size_t ws_bytes, void* stream) {
  return entry(handle, [&](Handle* h) {
    STATUS_TRY(check_vocab(h, dtype, rows, dim, vocab, ld_x, ld_w));
    STATUS_TRY(check_dtype(h, g_dtype, "dW"));
    if (dX) STATUS_TRY(check_ld(h, ld_dx, dim, "ld_dx"));
    if (dW) STATUS_TRY(check_ld(h, ld_dw, dim, "ld_dw"));
    if (!isfinite(beta)) return fail(h, SHAMPOO_EINVAL, "beta is not finite");
    if (!dX && !dW) return fail(h, SHAMPOO_EINVAL, "dX and dW are NULL");
    DeviceGuard g(h->device);
    hipStream_t s = static_cast<hipStream_t>(stream);
    constexpr int kCls = SHAMPOO_KCLASS_VOCAB;
    if (rows == 0) return dW ? scaled(h, kCls, dW, g_dtype, vocab, dim, ld_dw, beta, s) : SHAMPOO_OK;
    if (!X || !W || !lse) return fail(h, SHAMPOO_EINVAL, "X, W or lse is NULL");
    if (g_logp && !targets) return fail(h, SHAMPOO_EINVAL, "g_logp without targets");
    const bool pack_x = !as_it_lies(X, ld_x, dim, dtype), pack_w = !as_it_lies(W, ld_w, dim, dtype);
    const VocabGradPlan p = vocab_grad_plan(rows, dim, vocab, dtype, g_dtype, pack_x, pack_w);
    const size_t need = vocab_grad_alike(rows, dim, vocab, dtype, p.planes)
                            ? p.need
                            : shampoo_vocab_logprobs_grad_workspace_bytes(rows, dim, vocab, dtype, g_dtype);
    STATUS_TRY(check_room(h, workspace, ws_bytes, need));
    STATUS_TRY(check_all_apart(h,
                               {{span(workspace, (int64_t)need), "workspace"},
                                {span(dX, rows, dim, ld_dx, dtype), "dX"},
                                {span(dW, vocab, dim, ld_dw, g_dtype), "dW"}},
                               {{span(X, rows, dim, ld_x, dtype), "X"},
                                {span(W, vocab, dim, ld_w, dtype), "W"},
                                {span(targets, rows * 4), "targets"},
                                {span(lse, rows * 4), "lse"},
                                {span(g_logp, rows * 4), "g_logp"},
                                {span(g_lse, rows * 4), "g_lse"}}));
    char* ws = static_cast<char*>(workspace);
    STATUS_TRY(check_tiles(h, {p.z[0], p.z[1], p.dx[0], p.dx[1], p.dw[0], p.dw[1]}));
    Planes16 x, w;
    Packer packer{h, kCls, dtype, s};
    STATUS_TRY(packer.take(X, rows, dim, ld_x, pack_x, p.x, ws + p.at_x, &x));
    uint16_t* dz = reinterpret_cast<uint16_t*>(ws + p.at_dz);
    const Planes16 pz{dz, p.ld_dz, p.second ? (int64_t)(p.at_second - p.at_dz) / 2 : rows * p.ld_dz};
    const int nx = p.x.planes;
    MmaArgs qx{};
    const OutEpilogue out_x(dX, ld_dx, nullptr, 0, 0, (int)dim, (int)dim, dtype == SHAMPOO_BF16, 0.f);
    for (int64_t i = 0; i < p.pieces; ++i) {
      const int64_t v0 = i * p.piece, n = std::min(p.piece, vocab - v0);
      const bool last = i == p.pieces - 1;
      const char* here = typed(W, v0 * ld_w, dtype);
      STATUS_TRY(packer.take(here, n, dim, ld_w, pack_w && !p.direct, p.w, ws + p.at_w, &w));
      STATUS_TRY(packer.flush());
      MmaArgs q{};
      add_seg(q, x, w);
      use_plan(q, p.z[last], rows, n, dim, kLayoutRow, kLayoutRow, ws + p.at_part);
      const DlogitEpilogue e({targets, (int)vocab, (int)v0}, lse, g_logp, g_lse, dz, p.ld_dz, pz.plane, (int)n, p.terms());
      if (p.direct) STATUS_TRY(few_product<kLayoutRow>(h, kCls, dtype, {q, {few_seg(x, here, ld_w)}, (int)dim}, e, s));
      else STATUS_TRY((product<kLayoutRow, kLayoutRow>(h, kCls, nx, p.z[last].shape, q, e, s)));
      if (q.part) STATUS_TRY(join(h, kCls, q, e, s));
      const OutEpilogue out(dW ? const_cast<char*>(typed(dW, v0 * ld_dw, g_dtype)) : nullptr, ld_dw, nullptr, 0, 0,
                            (int)dim, (int)dim, g_dtype == SHAMPOO_BF16, beta);
      const bool two = p.two && dX && dW;
      MmaArgs qw{};
      if (dX) {
        const MmaPlan& m = two ? p.two_dx : p.dx[last];
        MmaArgs r{};
        add_seg(r, pz, w);
        use_plan(r, m, rows, dim, n, kLayoutRow, kLayoutK, ws + p.at_dx);
        r.part_add = i > 0;
        if (p.direct)
          STATUS_TRY(few_dx_product<kLayoutK>(h, kCls, dtype, p.terms(), {r, {few_seg(pz, here, ld_w)}, (int)n}, out_x, s));
        else if (!two) STATUS_TRY(dx_product<kLayoutK>(h, kCls, nx, p.terms(), m.shape, r, out_x, s));
        if (i == 0) qx = r;
      }
      if (dW) {
        const MmaPlan& m = two ? p.two_dw : p.dw[last];
        add_seg(qw, pz, x);
        use_plan(qw, m, n, dim, rows, kLayoutK, kLayoutK, ws + p.at_part);
        if (!two) STATUS_TRY(weight_product<true>(h, kCls, nx, p.terms(), m.shape, qw, out, s));
      }
      if (two && p.second)
        return two_products<kLayoutK, 1>(h, kCls, qx, OutTermsEpilogue(out_x), qw, OutTermsEpilogue(out), s);
      if (two) return two_products<kLayoutK>(h, kCls, nx, qx, out_x, qw, out, s);
    }
    return dX && qx.part ? join(h, kCls, qx, out_x, s) : SHAMPOO_OK;
  });
}

// ---------------------------------------------------------------- feed-forward block
size_t shampoo_gated_ffn_workspace_bytes(int64_t rows, int64_t dim, int64_t width, int dtype) {
  if (!sizes_ok(rows, dim, width, kMaxCols / 2, dtype) || rows == 0) return 0;
  const size_t need = ffn_plan(rows, dim, width, dtype, true, true, true).need;
  return ffn_alike(rows, dim, width, dtype, false) ? need : std::max(need, ffn_plan(rows, dim, width, dtype, true, false, false).bytes);
}

shampoo_status shampoo_gated_ffn(void* handle, const void* X, const void* Wg, const void* Wu, int dtype, int64_t rows,
                                 int64_t dim, int64_t width, int64_t ld_x, int64_t ld_wg, int64_t ld_wu, int act,
                                 void* H, int64_t ld_h, void* G, int64_t ld_g, void* U, int64_t ld_u, void* workspace,
                                 size_t ws_bytes, void* stream) {
  return entry(handle, [&](Handle* h) {
    STATUS_TRY(check_ffn(h, dtype, rows, dim, width, ld_x, ld_wg, ld_wu, act));
    STATUS_TRY(check_ld(h, ld_h, width, "ld_h"));
    if (!G != !U) return fail(h, SHAMPOO_EINVAL, "one of G and U is NULL");
    if (G) STATUS_TRY(check_ld(h, ld_g, width, "ld_g"));
    if (U) STATUS_TRY(check_ld(h, ld_u, width, "ld_u"));
    if (rows == 0) return SHAMPOO_OK;
    if (!X || !Wg || !Wu || !H) return fail(h, SHAMPOO_EINVAL, "X, Wg, Wu or H is NULL");
    const bool px = !as_it_lies(X, ld_x, dim, dtype), pg = !as_it_lies(Wg, ld_wg, width, dtype);
    const bool pu = !as_it_lies(Wu, ld_wu, width, dtype);
    const FfnPlan p = ffn_plan(rows, dim, width, dtype, px, pg, pu);
    const size_t need = ffn_alike(rows, dim, width, dtype, false) ? p.need : shampoo_gated_ffn_workspace_bytes(rows, dim, width, dtype);
    STATUS_TRY(check_room(h, workspace, ws_bytes, need));
    STATUS_TRY(check_all_apart(h,
                               {{span(workspace, (int64_t)need), "workspace"},
                                {span(H, rows, width, ld_h, dtype), "H"},
                                {span(G, rows, width, ld_g, dtype), "G"},
                                {span(U, rows, width, ld_u, dtype), "U"}},
                               {{span(X, rows, dim, ld_x, dtype), "X"},
                                {span(Wg, dim, width, ld_wg, dtype), "Wg"},
                                {span(Wu, dim, width, ld_wu, dtype), "Wu"}}));
    DeviceGuard g(h->device);
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    constexpr int kCls = SHAMPOO_KCLASS_FFN;
    STATUS_TRY(check_tiles(h, {p.mma}));
    Planes16 x, wg, wu;
    Packer packer{h, kCls, dtype, s};
    STATUS_TRY(packer.take(X, rows, dim, ld_x, px, p.x, ws + p.at_x, &x));
    STATUS_TRY(packer.take(Wg, dim, width, ld_wg, pg && !p.direct, p.wg, ws + p.at_wg, &wg));
    STATUS_TRY(packer.take(Wu, dim, width, ld_wu, pu && !p.direct, p.wu, ws + p.at_wu, &wu));
    STATUS_TRY(packer.flush());
    MmaArgs q{};
    add_seg(q, x, wg, &wu);
    use_plan(q, p.mma, rows, width, dim, kLayoutRow, kLayoutK, ws + p.at_part);
    shampoo_status st = SHAMPOO_OK;
    with_type(dtype, [&](auto* type) {
      using S = std::remove_pointer_t<decltype(type)>;
      const GatedEpilogue<S> e(act, (int)width, static_cast<S*>(H), static_cast<S*>(G), static_cast<S*>(U), ld_h, ld_g, ld_u);
      constexpr int kP = sizeof(S) == 2 ? 1 : 3;
      if (p.direct)
        st = few_product<S, kLayoutK>(h, kCls, {q, {few_seg(x, Wg, ld_wg, Wu, ld_wu)}, (int)dim}, e, s);
      else st = product<kLayoutRow, kLayoutK, kP, kP>(h, kCls, p.mma.shape, q, e, s);
      if (st == SHAMPOO_OK && q.part) st = join(h, kCls, q, e, s);
    });
    return st;
  });
}

size_t shampoo_gated_ffn_grad_workspace_bytes(int64_t rows, int64_t dim, int64_t width, int dtype, int g_dtype) {
  if (!sizes_ok(rows, dim, width, kMaxCols / 2, dtype) || rows == 0) return 0;
  if (g_dtype != SHAMPOO_F32 && g_dtype != SHAMPOO_BF16) return 0;
  const size_t need = ffn_grad_plan(rows, dim, width, dtype, g_dtype, true, true, true).need;
  if (ffn_alike(rows, dim, width, dtype, true)) return need;
  return std::max(need, ffn_grad_plan(rows, dim, width, dtype, g_dtype, true, false, false).bytes);
}

shampoo_status shampoo_gated_ffn_grad(void* handle, const void* X, const void* Wg, const void* Wu, int dtype,
                                      int64_t rows, int64_t dim, int64_t width, int64_t ld_x, int64_t ld_wg,
                                      int64_t ld_wu, int act, const void* dH, int64_t ld_dh, const void* G,
                                      int64_t ld_g, const void* U, int64_t ld_u, void* dX, int64_t ld_dx, void* dWg,
                                      int64_t ld_dwg, void* dWu, int64_t ld_dwu, int g_dtype, float beta,
                                      void* workspace, size_t ws_bytes, void* stream) {
  return entry(handle, [&](Handle* h) {
    STATUS_TRY(check_ffn(h, dtype, rows, dim, width, ld_x, ld_wg, ld_wu, act));
    STATUS_TRY(check_dtype(h, g_dtype, "dWg and dWu"));
    STATUS_TRY(check_ld(h, ld_dh, width, "ld_dh"));
    if (!G != !U) return fail(h, SHAMPOO_EINVAL, "one of G and U is NULL");
    if (!dWg != !dWu) return fail(h, SHAMPOO_EINVAL, "one of dWg and dWu is NULL");
    if (!dX && !dWg) return fail(h, SHAMPOO_EINVAL, "dX, dWg and dWu are NULL");
    if (G) STATUS_TRY(check_ld(h, ld_g, width, "ld_g"));
    if (U) STATUS_TRY(check_ld(h, ld_u, width, "ld_u"));
    if (dX) STATUS_TRY(check_ld(h, ld_dx, dim, "ld_dx"));
    if (dWg) STATUS_TRY(check_ld(h, ld_dwg, width, "ld_dwg"));
    if (dWu) STATUS_TRY(check_ld(h, ld_dwu, width, "ld_dwu"));
    if (!isfinite(beta)) return fail(h, SHAMPOO_EINVAL, "beta is not finite");
    STATUS_TRY(check_apart(h, span(dWg, dim, width, ld_dwg, g_dtype), "dWg", span(dWu, dim, width, ld_dwu, g_dtype), "dWu"));
    DeviceGuard g(h->device);
    hipStream_t s = static_cast<hipStream_t>(stream);
    constexpr int kCls = SHAMPOO_KCLASS_FFN;
    if (rows == 0) {
      if (!dWg) return SHAMPOO_OK;
      STATUS_TRY(scaled(h, kCls, dWg, g_dtype, dim, width, ld_dwg, beta, s));
      return scaled(h, kCls, dWu, g_dtype, dim, width, ld_dwu, beta, s);
    }
    if (!X || !Wg || !Wu || !dH) return fail(h, SHAMPOO_EINVAL, "X, Wg, Wu or dH is NULL");
    const bool px = (!G || dWg) && !as_it_lies(X, ld_x, dim, dtype);
    const bool pg = (!G || dX) && !as_it_lies(Wg, ld_wg, width, dtype);
    const bool pu = (!G || dX) && !as_it_lies(Wu, ld_wu, width, dtype);
    const FfnGradPlan p = ffn_grad_plan(rows, dim, width, dtype, g_dtype, px, pg, pu);
    const size_t need = ffn_alike(rows, dim, width, dtype, true)
                            ? p.need
                            : shampoo_gated_ffn_grad_workspace_bytes(rows, dim, width, dtype, g_dtype);
    STATUS_TRY(check_room(h, workspace, ws_bytes, need));
    STATUS_TRY(check_all_apart(h,
                               {{span(workspace, (int64_t)need), "workspace"},
                                {span(dX, rows, dim, ld_dx, dtype), "dX"},
                                {span(dWg, dim, width, ld_dwg, g_dtype), "dWg"},
                                {span(dWu, dim, width, ld_dwu, g_dtype), "dWu"}},
                               {{span(X, rows, dim, ld_x, dtype), "X"},
                                {span(Wg, dim, width, ld_wg, dtype), "Wg"},
                                {span(Wu, dim, width, ld_wu, dtype), "Wu"},
                                {span(dH, rows, width, ld_dh, dtype), "dH"},
                                {span(G, rows, width, ld_g, dtype), "G"},
                                {span(U, rows, width, ld_u, dtype), "U"}}));
    char* ws = static_cast<char*>(workspace);
    STATUS_TRY(check_tiles(h, {p.gu, p.dx, p.dw}));
    Planes16 x, wg, wu;
    Packer packer{h, kCls, dtype, s};
    STATUS_TRY(packer.take(X, rows, dim, ld_x, px, p.x, ws + p.at_x, &x));
    STATUS_TRY(packer.take(Wg, dim, width, ld_wg, pg && !p.direct, p.wg, ws + p.at_wg, &wg));
    STATUS_TRY(packer.take(Wu, dim, width, ld_wu, pu && !p.direct, p.wu, ws + p.at_wu, &wu));
    STATUS_TRY(packer.flush());
    const int nx = p.x.planes;
    uint16_t* d = reinterpret_cast<uint16_t*>(ws + p.at_d);
    const Planes16 dg{d, 2 * p.ld_d, rows * 2 * p.ld_d}, du{d + p.ld_d, dg.ld, dg.plane};
    shampoo_status st = SHAMPOO_OK;
    with_terms(dtype, p.planes, [&](auto* type, auto terms) {
      using S = std::remove_pointer_t<decltype(type)>;
      constexpr int kTerms = decltype(terms)::value;
      const GatedGradEpilogue<S, kTerms> e(act, (int)width, static_cast<const S*>(dH), ld_dh, d, d + p.ld_d, dg.ld,
                                           dg.plane);
      if (G) {
        st = unit_launches(h, kCls, rows, width, p.ld_d / 8, s, [&](const ActShape& sh, dim3 grid) {
          hipLaunchKernelGGL((gated_grad_kernel<S, kTerms>), grid, dim3(kThreads), 0, s, sh, static_cast<const S*>(G),
                             ld_g, static_cast<const S*>(U), ld_u, e);
        });
      } else {
        MmaArgs q{};
        add_seg(q, x, wg, &wu);
        use_plan(q, p.gu, rows, width, dim, kLayoutRow, kLayoutK, ws + p.at_part);
        constexpr int kP = sizeof(S) == 2 ? 1 : 3;
        if (p.direct)
          st = few_product<S, kLayoutK>(h, kCls, {q, {few_seg(x, Wg, ld_wg, Wu, ld_wu)}, (int)dim}, e, s);
        else st = product<kLayoutRow, kLayoutK, kP, kP>(h, kCls, p.gu.shape, q, e, s);
        if (st == SHAMPOO_OK && q.part) st = join(h, kCls, q, e, s);
      }
    });
    STATUS_TRY(st);
    const bool two = p.two && dX && dWg;
    const OutEpilogue out_x(dX, ld_dx, nullptr, 0, 0, (int)dim, (int)dim, dtype == SHAMPOO_BF16, 0.f);
    const OutEpilogue out_w(dWg, ld_dwg, dWu, ld_dwu, (int)p.ld_d, (int)width, (int)(2 * p.ld_d), g_dtype == SHAMPOO_BF16,
                            beta);
    MmaArgs qx{}, qw{};
    if (dX) {
      const MmaPlan& m = two ? p.two_dx : p.dx;
      add_seg(qx, dg, wg);
      add_seg(qx, du, wu);
      use_plan(qx, m, rows, dim, width, kLayoutRow, kLayoutRow, ws + (two ? p.at_dx : p.at_part));
      if (!two) {
        if (p.direct)
          STATUS_TRY(few_dx_product<kLayoutRow>(
              h, kCls, dtype, p.planes, {qx, {few_seg(dg, Wg, ld_wg), few_seg(du, Wu, ld_wu)}, (int)width}, out_x, s));
        else STATUS_TRY(dx_product<kLayoutRow>(h, kCls, nx, p.planes, m.shape, qx, out_x, s));
        if (qx.part) STATUS_TRY(join(h, kCls, qx, out_x, s));
      }
    }
    if (!dWg) return SHAMPOO_OK;
    const MmaPlan& m = two ? p.two_dw : p.dw;
    add_seg(qw, x, dg);
    use_plan(qw, m, dim, 2 * p.ld_d, rows, kLayoutK, kLayoutK, ws + p.at_part);
    if (two) return two_products<kLayoutRow>(h, kCls, nx, qx, out_x, qw, out_w, s);
    return weight_product<false>(h, kCls, nx, p.planes, m.shape, qw, out_w, s);
  });
}

// ---------------------------------------------------------------- dropout
shampoo_status shampoo_dropout(void* handle, const void* X, const void* R, void* Y, int dtype, int64_t rows,
                               int64_t cols, int64_t ld_x, int64_t ld_r, int64_t ld_y, double rate, uint64_t seed,
                               uint64_t offset, void* stream) {
  return entry(handle, [&](Handle* h) {
    STATUS_TRY(check_dtype(h, dtype, "X"));
    STATUS_TRY(check_size(h, rows, 0, kMaxTokens, "rows"));
    STATUS_TRY(check_size(h, cols, 1, kMaxCols, "cols"));
    STATUS_TRY(check_ld(h, ld_x, cols, "ld_x"));
    STATUS_TRY(check_ld(h, ld_y, cols, "ld_y"));
    if (R) STATUS_TRY(check_ld(h, ld_r, cols, "ld_r"));
    if (!(rate >= 0 && rate <= 1)) return fail(h, SHAMPOO_EINVAL, "rate %g outside [0, 1]", rate);
    if (rows == 0) return SHAMPOO_OK;
    if (!X || !Y) return fail(h, SHAMPOO_EINVAL, "X or Y is NULL");
    if (Y == X && ld_y != ld_x) return fail(h, SHAMPOO_EINVAL, "in place, ld_y %lld must be ld_x %lld", (long long)ld_y, (long long)ld_x);
    if (Y == R && ld_y != ld_r) return fail(h, SHAMPOO_EINVAL, "in place, ld_y %lld must be ld_r %lld", (long long)ld_y, (long long)ld_r);
    const Span y = span(Y, rows, cols, ld_y, dtype);
    if (Y != X) STATUS_TRY(check_apart(h, y, "Y", span(X, rows, cols, ld_x, dtype), "X"));
    if (Y != R) STATUS_TRY(check_apart(h, y, "Y", span(R, rows, cols, ld_r, dtype), "R"));
    DeviceGuard g(h->device);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const uint32_t least = (uint32_t)nearbyint(rate * 65536);
    const DropoutArgs q{{(uint32_t)seed, (uint32_t)(seed >> 32)}, {(uint32_t)offset, (uint32_t)(offset >> 32)}, least,
                        least < 65536 ? 65536.f / (float)(65536 - least) : 0.f};
    return unit_launches(h, SHAMPOO_KCLASS_DROPOUT, rows, cols, cdiv64(cols, 32) * 4, s, [&](const ActShape& sh, dim3 grid) {
      with_type(dtype, [&](auto* type) {
        using S = std::remove_pointer_t<decltype(type)>;
        hipLaunchKernelGGL(dropout_kernel<S>, grid, dim3(kThreads), 0, s, sh, q, static_cast<const S*>(X), ld_x,
                           static_cast<const S*>(R), ld_r, static_cast<S*>(Y), ld_y);
      });
    });
  });
}

}  // extern "C"
