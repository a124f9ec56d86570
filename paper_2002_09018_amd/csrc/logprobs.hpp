// Device kernels of the output layer's loss: log probabilities of given
// tokens with log-sum-exp, entropy and the largest alternatives, and their
// gradient with respect to the logits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fp32_block.hpp"
#include "shampoo.h"
#include "tile_mfma.hpp"

namespace shp {

template <typename S>
__device__ __forceinline__ S from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ uint16_t from_f32<uint16_t>(float x) {
  return __builtin_bit_cast(uint16_t, (__bf16)x);  // to nearest even
}

// (value, index) order of the alternatives: larger value first, then lower index.
__device__ __forceinline__ bool better(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

// ---------------------------------------------------------------- statistics
// One pass over a row.  Each lane keeps the largest entry m so far and
//   s = sum 2^(L z - c),  t = sum (L z - c) 2^(L z - c),  c = L m,
// L the fp32 value of log2 e, so that lse = (c + log2 s) / L and the entropy is
// (log2 s - t / s) / L.  Everything is relative to the fp32 number c: one fma
// gives an exponent, and c's own rounding cancels (the largest entry's exponent
// is that rounding, at most 2^-24 |c|, not 0).  A largest entry beyond 1e6 in
// size (a type's lowest value used as a mask, alone in its row) would lose too
// much so: it takes (z - m) L instead.
constexpr float kLog2e = 1.44269502f;
constexpr float kHugeLogit = 1e6f;

struct LseStat {
  float m, s, t;  // m = -kHugeLogit and s = 0 before any entry
};

// c as a rounded number: fused into a later sum it would be another one.
__device__ __forceinline__ float lse_ref(float m) {
#pragma clang fp contract(off)
  return m * kLog2e;
}
// Exponent of the factor that carries sums from reference m to reference n >= m.
__device__ __forceinline__ float lse_shift(float m, float n) {
  float d = fabsf(m) > kHugeLogit || fabsf(n) > kHugeLogit ? (m - n) * kLog2e : lse_ref(m) - lse_ref(n);
  if (m == n) d = 0.f;
  return fminf(fmaxf(d, -1e30f), 0.f);  // finite: it multiplies s, which may be 0
}
__device__ __forceinline__ LseStat lse_join(LseStat a, LseStat b) {
  const float n = a.s == 0.f ? b.m : b.s == 0.f ? a.m : fmaxf(a.m, b.m);
  const float da = lse_shift(a.m, n), db = lse_shift(b.m, n);
  const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
  return {n, a.s * fa + b.s * fb, (a.t + da * a.s) * fa + (b.t + db * b.s) * fb};
}
__device__ __forceinline__ LseStat lse_wave(LseStat a) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
    a = lse_join(a, {__shfl_xor(a.m, o, 64), __shfl_xor(a.s, o, 64), __shfl_xor(a.t, o, 64)});
  return a;
}

// The k largest entries of a wave, sorted over its lanes (lane i: the i-th).
struct TopList {
  float v;
  int i;
  // No entry below cut is wanted, and of those equal to it only the ones before
  // entry `last`: the k-th entry of the list, or a bound where it is not full.
  float cut;
  int last;

  __device__ __forceinline__ void clear() { v = cut = -INFINITY, i = last = INT32_MAX; }
  __device__ __forceinline__ bool wants(float x, int j) const { return better(x, j, cut, last) && x > -INFINITY; }
  // One entry, the same in every lane.
  __device__ __forceinline__ void insert(float x, int j, int k, int lane) {
    const int pos = __popcll(__ballot(better(v, i, x, j)));
    const float pv = __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x138, 0xf, 0xf, false));
    const int pi = __builtin_amdgcn_update_dpp(0, i, 0x138, 0xf, 0xf, false);  // lane - 1's
    if (lane == pos) v = x, i = j;
    else if (lane > pos) v = pv, i = pi;
    cut = fmaxf(cut, __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), k - 1)));
    last = __builtin_amdgcn_readlane(i, k - 1);
  }
  // One entry of each lane, in any order.
  __device__ __forceinline__ void insert_lanes(float x, int j, int k, int lane) {
    uint64_t todo = __ballot(wants(x, j));
    while (todo) {
      const int l = __builtin_ctzll(todo);
      insert(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), l)), __builtin_amdgcn_readlane(j, l), k, lane);
      todo &= ~(uint64_t(1) << l) & __ballot(wants(x, j));
    }
  }
};

// The largest float below x (x not NaN); -inf stays.
__device__ __forceinline__ float float_below(float x) {
  const uint32_t b = __float_as_uint(x);
  if (x == 0.f) return -1.401298464e-45f;
  if (x == -INFINITY) return x;
  return __uint_as_float(x > 0.f ? b - 1 : b + 1);
}

// A cut below the k-th largest of the lanes' values x, by bisection over the
// upper 16 bits of their order.
__device__ __forceinline__ float first_cut(float x, int k) {
  const uint32_t b = __float_as_uint(x + 0.f);  // -0 orders with 0
  const uint32_t key = ((b & 0x80000000u) ? ~b : b | 0x80000000u) >> 16;
  uint32_t at = 0;
#pragma unroll
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t t = at | 1u << bit;
    if (__popcll(__ballot(key >= t)) >= k) at = t;
  }
  const uint32_t o = at << 16;
  const uint32_t f = (o & 0x80000000u) ? o & 0x7fffffffu : ~o;
  // at or below the order of -inf: every allowed entry passes
  return at <= 0x007fu ? -INFINITY : float_below(__uint_as_float(f));
}

// A block of a wave: kU 16-byte loads of each lane, 64 lanes apart.
template <typename S>
struct LogitBlock {
  static constexpr int kV = 16 / sizeof(S), kU = 4, kN = 64 * kV * kU;
  u32x4u raw[kU];

  __device__ __forceinline__ void load(const S* z, int lane) {
#pragma unroll
    for (int u = 0; u < kU; ++u) raw[u] = gload<u32x4u>(z + (u * 64 + lane) * kV);
  }
  // Only n entries; the others are not allowed.
  __device__ __forceinline__ void load_part(const S* z, int n, int lane) {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int at = (u * 64 + lane) * kV;
      if (at + kV <= n) {
        raw[u] = gload<u32x4u>(z + at);
      } else {
#pragma unroll
        for (int i = 0; i < kV; ++i) {
          if constexpr (sizeof(S) == 4) {
            raw[u][i] = at + i < n ? gload<uint32_t>(z + at + i) : 0xff800000u;
          } else {
            const uint32_t w = at + i < n ? (uint32_t)gload<uint16_t>(z + at + i) : 0xff80u;
            raw[u][i / 2] = i & 1 ? raw[u][i / 2] | w << 16 : w;
          }
        }
      }
    }
  }
  __device__ __forceinline__ float at(int u, int i) const {
    if constexpr (sizeof(S) == 4) return __uint_as_float(raw[u][i]);
    return __uint_as_float(i & 1 ? raw[u][i / 2] & 0xffff0000u : raw[u][i / 2] << 16);
  }

  template <bool ENT, bool HUGE_>
  __device__ __forceinline__ void sums(float n, float c, bool clamp, float& s, float& t) const {
    s = t = 0.f;
#pragma unroll
    for (int u = 0; u < kU; ++u)
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        const float z = at(u, i);
        float x = HUGE_ ? (z - n) * kLog2e : fmaf(z, kLog2e, -c);
        const float e = __builtin_amdgcn_exp2f(x);
        s += e;
        if (HUGE_ || clamp) x = fmaxf(x, -1e30f);  // 0, not NaN, for an entry that is not allowed
        if (ENT) t = fmaf(x, e, t);
      }
  }

  // Adds the block to st and the wave's alternatives; its first entry is entry
  // `base` of the row.
  template <bool ENT>
  __device__ __forceinline__ void add(LseStat& st, TopList& top, bool& fresh, int base, int k, int lane) const {
    float um[kU], bm;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      um[u] = at(u, 0);
#pragma unroll
      for (int i = 1; i < kV; ++i) um[u] = fmaxf(um[u], at(u, i));
    }
    bm = fmaxf(fmaxf(um[0], um[1]), fmaxf(um[2], um[3]));
    float s, t;
    const float n0 = st.s == 0.f && bm > -INFINITY ? bm : fmaxf(st.m, bm);
    const bool far = fabsf(n0) > kHugeLogit;
    if (__builtin_expect(__any(far), 0)) {
      if (far) sums<ENT, true>(n0, 0.f, true, s, t);
      else sums<ENT, false>(n0, lse_ref(n0), true, s, t);
      st = lse_join(st, {n0, s, t});
    } else {
      const float n = fmaxf(st.m, bm), c = lse_ref(n);
      const float d = fmaxf(lse_ref(st.m) - c, -1e30f), f = __builtin_amdgcn_exp2f(d);
      sums<ENT, false>(n, c, false, s, t);
      if (ENT && __any(t != t)) sums<ENT, false>(n, c, true, s, t);
      st.t = (st.t + d * st.s) * f + t;
      st.s = st.s * f + s;
      st.m = n;
    }
    if (k == 0) return;
    if (fresh) top.cut = first_cut(bm, k);
    fresh = false;
    // entries equal to the cut count only in the block that holds `last`
    if (!__any(base <= top.last ? bm >= top.cut : bm > top.cut)) return;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      if (!__any(um[u] >= top.cut)) continue;
      const int first = base + (u * 64 + lane) * kV;
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        uint64_t todo = __ballot(top.wants(at(u, i), first + i));
        while (todo) {
          const int l = __builtin_ctzll(todo);
          top.insert(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(at(u, i)), l)),
                     base + (u * 64 + l) * kV + i, k, lane);
          todo &= ~(uint64_t(1) << l) & __ballot(top.wants(at(u, i), first + i));
        }
      }
    }
  }
};

struct LogprobArgs {
  const void* logits;
  int64_t ld, rows;
  int vocab;
  const int32_t* targets;
  float *logp, *lse, *entropy;
  int k;
  int32_t* top_ids;
  float* top_logp;
  int parts;     // workgroups of a row
  int per_part;  // entries of one
  float* ws;     // a record for each part of each row: m, s, t, -, k values, k indices
};
__host__ __device__ __forceinline__ int64_t logprob_record(int k) { return 4 + 2 * (int64_t)k; }

// The outputs of a row, from a wave that holds its sums and alternatives; zt is
// the target's logit in lane 0 (where there is one).
__device__ __forceinline__ void logprobs_finish(const LogprobArgs& q, int64_t r, LseStat st, const TopList& top, int tg,
                                                float zt, int lane) {
  const bool huge = fabsf(st.m) > kHugeLogit, empty = st.s == 0.f;
  const float c = lse_ref(st.m), ls = log2f(st.s);
  auto logprob = [&](float z) {
    // log2 p = L z - c - log2 s
    return huge || fabsf(z) > kHugeLogit ? (z - st.m) - ls * (1.f / kLog2e) : (fmaf(z, kLog2e, -c) - ls) / kLog2e;
  };
  if (lane == 0) {
    const double l = huge ? (double)st.m + (double)ls / kLog2e : ((double)c + (double)ls) / kLog2e;
    q.lse[r] = empty ? -INFINITY : st.s != st.s ? NAN : (float)l;
    if (q.entropy) q.entropy[r] = empty ? 0.f : (ls - st.t / st.s) / kLog2e;
    if (q.logp) q.logp[r] = tg < 0 ? 0.f : empty ? -INFINITY : st.s != st.s ? NAN : logprob(zt);
  }
  if (lane < q.k) {
    const bool bad = st.s != st.s, none = bad || top.v == -INFINITY;
    q.top_ids[r * q.k + lane] = none ? -1 : top.i;
    q.top_logp[r * q.k + lane] = bad ? NAN : none ? -INFINITY : logprob(top.v);
  }
}

// The target of row r (-1: none) and its logit, in every lane.
template <typename S>
__device__ __forceinline__ int logprobs_target(const LogprobArgs& q, int64_t r, float& zt) {
  int tg = q.targets ? q.targets[r] : -1;
  if (tg >= q.vocab) tg = -1;
  zt = tg < 0 ? 0.f : cvt<float, S>(static_cast<const S*>(q.logits)[r * q.ld + tg]);
  return tg < 0 ? -1 : tg;
}

// W waves to a row (or to a part of it), 4 / W rows to a workgroup; the waves
// take its blocks in turn.
template <typename S, int W, bool ENT>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(LogprobArgs q) {
  using Block = LogitBlock<S>;
  __shared__ float sm[W > 1 ? W : 1][3];
  __shared__ float sv[W > 1 ? W : 1][SHAMPOO_MAX_TOP];
  __shared__ int si[W > 1 ? W : 1][SHAMPOO_MAX_TOP];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t item = (int64_t)blockIdx.x * (4 / W) + (W == 1 ? wave : 0);
  if (item >= q.rows * q.parts) return;
  const int64_t r = item / q.parts;
  const int part = (int)(item % q.parts), w = W == 1 ? 0 : wave;
  const S* z = static_cast<const S*>(q.logits) + r * q.ld;
  const int begin = part * q.per_part, end = min(q.vocab, begin + q.per_part);
  float zt = 0.f;
  const int tg = q.parts == 1 && w == 0 ? logprobs_target<S>(q, r, zt) : -1;

  LseStat st = {-kHugeLogit, 0.f, 0.f};
  TopList top;
  top.clear();
  bool fresh = true;
  int at = begin + w * Block::kN;
  Block blk, nxt;
  if (at + Block::kN <= end) nxt.load(z + at, lane);
  for (; at + Block::kN <= end; at += W * Block::kN) {
    blk = nxt;
    if (at + (W + 1) * Block::kN <= end) nxt.load(z + at + W * Block::kN, lane);
    blk.template add<ENT>(st, top, fresh, at, q.k, lane);
  }
  if (at < end) {
    blk.load_part(z + at, end - at, lane);
    blk.template add<ENT>(st, top, fresh, at, q.k, lane);
  }
  st = lse_wave(st);
  if constexpr (W > 1) {
    if (lane == 0) sm[w][0] = st.m, sm[w][1] = st.s, sm[w][2] = st.t;
    if (lane < q.k) sv[w][lane] = top.v, si[w][lane] = top.i;
    __syncthreads();
    if (w != 0) return;
#pragma unroll
    for (int o = 1; o < W; ++o) st = lse_join(st, {sm[o][0], sm[o][1], sm[o][2]});
    for (int e = lane; e - lane < (W - 1) * q.k; e += 64) {  // the best of each wave first
      const bool in = e < (W - 1) * q.k;
      const int o = 1 + e % (W - 1), i = e / (W - 1);
      top.insert_lanes(in ? sv[o][i] : -INFINITY, in ? si[o][i] : INT32_MAX, q.k, lane);
    }
  }
  if (q.parts == 1) {
    logprobs_finish(q, r, st, top, tg, zt, lane);
    return;
  }
  float* rec = q.ws + item * logprob_record(q.k);
  if (lane == 0) rec[0] = st.m, rec[1] = st.s, rec[2] = st.t;
  if (lane < q.k) rec[4 + lane] = top.v, rec[4 + q.k + lane] = __int_as_float(top.i);
}

// Joins the parts of a row (at most 64), one wave to a row.
template <typename S>
__global__ __launch_bounds__(64) void logprobs_join_kernel(LogprobArgs q) {
  const int lane = threadIdx.x;
  const int64_t r = blockIdx.x;
  float zt;
  const int tg = logprobs_target<S>(q, r, zt);
  const float* rec = q.ws + r * q.parts * logprob_record(q.k);
  LseStat st = {-kHugeLogit, 0.f, 0.f};
  if (lane < q.parts) {
    const float* p = rec + lane * logprob_record(q.k);
    st = {p[0], p[1], p[2]};
  }
  st = lse_wave(st);
  TopList top;
  top.clear();
  for (int e = lane; e - lane < q.parts * q.k; e += 64) {
    const bool in = e < q.parts * q.k;
    const float* p = rec + (in ? e % q.parts * logprob_record(q.k) + 4 + e / q.parts : 0);
    top.insert_lanes(in ? p[0] : -INFINITY, in ? __float_as_int(p[q.k]) : INT32_MAX, q.k, lane);
  }
  logprobs_finish(q, r, st, top, tg, zt, lane);
}

// One workgroup per row of the gradient.  The entries that also take a
// target's or an alternative's gradient are read before any entry is
// written (the gradient may overwrite the logits) and written again last.
template <typename S>
__global__ __launch_bounds__(kThreads) void logprobs_grad_kernel(
    const S* logits, int64_t ld, int vocab, const int32_t* __restrict__ targets, const float* __restrict__ lse_in,
    const float* __restrict__ entropy, int k, const int32_t* __restrict__ top_ids, const float* __restrict__ g_logp,
    const float* __restrict__ g_lse, const float* __restrict__ g_entropy, const float* __restrict__ g_top, S* dlogits,
    int64_t ld_d) {
  __shared__ float part[SHAMPOO_MAX_TOP + 1];
  __shared__ int ids[SHAMPOO_MAX_TOP + 1];
  const int64_t r = blockIdx.x;
  const S* z = logits + r * ld;
  S* dz = dlogits + r * ld_d;
  const int tid = threadIdx.x;
  const float lse = lse_in[r];
  const float H = g_entropy ? entropy[r] : 0.f, ge = g_entropy ? g_entropy[r] : 0.f;
  // slot 0: the target; slot 1 + i: alternative i
  if (tid <= k) {
    int64_t id = -1;
    float g = 0.f;
    if (tid == 0) {
      if (g_logp) id = targets[r], g = g_logp[r];
    } else if (g_top) {
      id = top_ids[r * k + tid - 1], g = g_top[r * k + tid - 1];
    }
    const bool on = id >= 0 && id < vocab;
    ids[tid] = on ? (int)id : -1;
    part[tid] = on ? g : 0.f;
  }
  __syncthreads();
  float total = g_lse ? g_lse[r] : 0.f;
  for (int i = 0; i <= k; ++i) total -= part[i];
  const bool empty = lse == -INFINITY;
  auto value = [&](float x) {
    const float lp = x - lse;
    const float p = expf(lp);
    return empty ? 0.f : p * (total - ge * (fmaxf(lp, -1e30f) + H));
  };
  float own = 0.f;
  if (tid <= k && ids[tid] >= 0) {
    own = value(cvt<float, S>(z[ids[tid]]));
    for (int i = 0; i <= k; ++i)
      if (ids[i] == ids[tid]) own += part[i];
  }
  __syncthreads();
  for (int j = tid; j < vocab; j += kThreads) dz[j] = from_f32<S>(value(cvt<float, S>(z[j])));
  __syncthreads();
  if (tid <= k && ids[tid] >= 0 && !empty) dz[ids[tid]] = from_f32<S>(own);
}

}  // namespace shp
