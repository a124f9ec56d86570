// Device kernels of the output layer's loss: log probabilities of given
// tokens with log-sum-exp, entropy and the largest alternatives, and their
// gradient with respect to the logits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "layer_plans.hpp"
#include "split_mfma.hpp"
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
//   s = sum e^(z - m),  t = sum (z - m) e^(z - m),
// so that lse = m + log s and the entropy is log s - t / s.  The differences are
// taken before they are scaled for the base-2 exponential: one instruction more
// than a fused L z - L m, whose rounded L m would be another reference than m.
// So the largest term is exactly 1, s >= 1 and t <= 0 hold through every join,
// log probabilities never exceed 0 and entropies never fall below it, and
// logits of any size (a type's lowest value used as a mask, alone in its row) are
// as exact as small ones.
//
// A wave walks its blocks of 4 KB with the next one in flight.  The alternatives
// cost a comparison with a bound per 16-byte piece: only pieces above it are kept
// (in LDS), and they are ranked once, at the end.  8192 x 131072 in bf16 with 8
// alternatives: 390 us, 5.5 TB/s, bound by memory; 4096 x 131072 in fp32 369 us (5.8
// TB/s); 1 x 32768: 9 us, the latency of a launch, a load and the ranking.  A short
// row is a chain of its own - load, sums, six joins across the wave, then bound
// and ranking: 8192 x 5000 takes 20 us without alternatives (4.0 TB/s), 27 with 8,
// 74 with 64; 8192 x 1000 9 and 13.
constexpr float kLog2e = 1.44269502f;
constexpr float kLowest = -3.40282347e38f;

struct LseStat {
  float m, s, t;  // m = kLowest and s = 0 before any entry
};

// What carries sums from reference m to reference n >= m: m - n, finite, for it
// multiplies s, which may be 0.
__device__ __forceinline__ float lse_shift(float m, float n) { return fmaxf(m - n, -1e20f); }
__device__ __forceinline__ float lse_exp(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
__device__ __forceinline__ LseStat lse_join(LseStat a, LseStat b) {
  const float n = fmaxf(a.m, b.m), da = lse_shift(a.m, n), db = lse_shift(b.m, n);
  const float fa = lse_exp(da), fb = lse_exp(db);
  return {n, a.s * fa + b.s * fb, (a.t + da * a.s) * fa + (b.t + db * b.s) * fb};
}
__device__ __forceinline__ LseStat lse_wave(LseStat a) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
    a = lse_join(a, {__shfl_xor(a.m, o, 64), __shfl_xor(a.s, o, 64), __shfl_xor(a.t, o, 64)});
  return a;
}

// The largest float below x (x not NaN); -inf stays.
__device__ __forceinline__ float float_below(float x) {
  const uint32_t b = __float_as_uint(x);
  if (x == 0.f) return -1.401298464e-45f;
  if (x == -INFINITY) return x;
  return __uint_as_float(x > 0.f ? b - 1 : b + 1);
}

// LDS written by some lanes of a wave and read by others: a wave's LDS accesses
// keep their order, the compiler has to keep it too.
__device__ __forceinline__ void wave_lds_order() { asm volatile("" ::: "memory"); }

// Lanes of the wave below this one that are in the mask.
__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// A cut below the k-th largest of the lanes' values x and y, by bisection over
// the upper 16 bits of their order.  Up to k = 32 the larger of a lane's two
// stands for both: half the ballots, and nearly as good a cut.
__device__ __forceinline__ float first_cut(float x, float y, int k) {
  auto order = [](float v) {
    const uint32_t b = __float_as_uint(v + 0.f);  // -0 orders with 0
    return ((b & 0x80000000u) ? ~b : b | 0x80000000u) >> 16;
  };
  uint32_t at = 0;
  if (k <= 32) {
    const uint32_t key = order(fmaxf(x, y));
#pragma unroll
    for (int bit = 15; bit >= 0; --bit) {
      const uint32_t t = at | 1u << bit;
      if (__popcll(__ballot(key >= t)) >= k) at = t;
    }
  } else {
    const uint32_t kx = order(x), ky = order(y);
    for (int bit = 15; bit >= 0; --bit) {
      const uint32_t t = at | 1u << bit;
      if (__popcll(__ballot(kx >= t)) + __popcll(__ballot(ky >= t)) >= k) at = t;
    }
  }
  const uint32_t o = at << 16;
  const uint32_t f = (o & 0x80000000u) ? o & 0x7fffffffu : ~o;
  // at or below the order of -inf: every allowed entry passes
  return at <= 0x007fu ? -INFINITY : float_below(__uint_as_float(f));
}

// The k largest entries of a wave, sorted over its lanes (lane i: the i-th).
struct TopList {
  float v;
  int i;

  __device__ __forceinline__ void clear() { v = -INFINITY, i = INT32_MAX; }
  // One entry, the same in every lane.
  __device__ __forceinline__ void insert(float x, int j, int lane) {
    const int pos = __popcll(__ballot(better(v, i, x, j)));
    const float pv = __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x138, 0xf, 0xf, false));
    const int pi = __builtin_amdgcn_update_dpp(0, i, 0x138, 0xf, 0xf, false);  // lane - 1's
    if (lane == pos) v = x, i = j;
    else if (lane > pos) v = pv, i = pi;
  }
  // One entry of each lane, in any order.
  __device__ __forceinline__ void insert_lanes(float x, int j, int k, int lane) {
    for (;;) {
      const float kv = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), k - 1));
      const int ki = __builtin_amdgcn_readlane(i, k - 1);
      const uint64_t todo = __ballot(x > -INFINITY && better(x, j, kv, ki));
      if (!todo) return;
      const int l = __builtin_ctzll(todo);
      insert(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), l)), __builtin_amdgcn_readlane(j, l), lane);
      if (lane == l) x = -INFINITY;
    }
  }
  // The n <= 64 entries (x, j) of lanes 0..n-1, sorted: each lane counts the
  // entries before its own and passes it to that lane.
  __device__ __forceinline__ void sort(float x, int j, int n, int lane) {
    if (lane >= n) x = -INFINITY, j = INT32_MAX;
    int rank = lane < n ? 0 : lane - n;  // all n come before an absent one, none after
    for (int o = 0; o < n; o += 4)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float y = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), o + u));
        const int i2 = __builtin_amdgcn_readlane(j, o + u);
        rank += better(y, i2, x, j);
      }
    v = __uint_as_float(__builtin_amdgcn_ds_permute(rank * 4, __float_as_uint(x)));
    i = __builtin_amdgcn_ds_permute(rank * 4, j);
  }
  // The 64 best of the 64 < n <= 128 entries in pv and pi (LDS), sorted.
  __device__ __forceinline__ void sort_two(float* pv, int* pi, int n, int lane) {
    const float x = pv[lane], y = lane + 64 < n ? pv[lane + 64] : -INFINITY;
    const int j = pi[lane], l = lane + 64 < n ? pi[lane + 64] : INT32_MAX;
    wave_lds_order();
    int rx = 0, ry = 0;
    auto count = [&](float a, int b, int o) {
      const float z = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(a), o));
      const int i2 = __builtin_amdgcn_readlane(b, o);
      rx += better(z, i2, x, j), ry += better(z, i2, y, l);
    };
#pragma unroll 4
    for (int o = 0; o < 64; ++o) count(x, j, o);
    for (int o = 0; o < n - 64; ++o) count(y, l, o);
    if (rx < 64) pv[rx] = x, pi[rx] = j;
    if (ry < 64) pv[ry] = y, pi[ry] = l;  // an absent one comes after all n
    wave_lds_order();
    v = pv[lane], i = pi[lane];
  }
};

// The k-th largest of the lanes' four largest values (-inf where there are fewer),
// of which the upper kBits bits are not 0.
template <int kBits>
__device__ __forceinline__ float kth_of_four(const float (&m)[4], int k) {
  uint32_t key[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t b = __float_as_uint(m[i] + 0.f);  // -0 orders with 0
    key[i] = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  }
  uint32_t at = 0;
#pragma unroll 1
  for (int bit = 31; bit >= 32 - kBits; --bit) {
    const uint32_t t = at | 1u << bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) n += __popcll(__ballot(key[i] >= t));
    if (n >= k) at = t;
  }
  // a value below 0 has its lower bits inverted in the key
  if (kBits < 32 && !(at & 0x80000000u)) at |= (1u << (32 - kBits)) - 1;
  return at <= 0x007fffffu ? -INFINITY : __uint_as_float((at & 0x80000000u) ? at & 0x7fffffffu : ~at);
}

// The k best of `top` and of `sets` sets of 64 N entries: get(c, x, j) gives a
// lane's N of set c, of consecutive indices from j (x = -inf: none).  No entry up
// to `low` is wanted.  What is above it is gathered in LDS and sorted.
//
// Where that is more than 128 entries (in rows that rise every block lies above the
// bound) and the entries come by index, those of `top` first (ORDERED), a value v
// that the k-th is not below is found from the lanes' four largest; what is above
// it and, as far as k goes, the first that equal it are gathered instead: 8192 x
// 131072 in bf16 with 8 alternatives takes 1.7 ms where rows rise throughout (one by
// one 8.4), 0.4 where they are in random order, fall or are all equal.  Otherwise,
// and where a few lanes hold most of the largest, they go one by one.
template <int N, bool ORDERED, typename G>
__device__ __forceinline__ void top_select(TopList& top, int sets, float low, int k, int lane, float* pv, int* pi,
                                           G&& get) {
  int n = 0;
  auto gather = [&](bool wanted, float x, int j) {
    const uint64_t in = __ballot(wanted);
    const int at = n + lanes_below(in);
    if (wanted && at < 128) pv[at] = x, pi[at] = j;
    n += __popcll(in);
  };
  gather(top.v > low, top.v, top.i);
  for (int c = 0; c < sets; ++c) {
    float x[N];
    int j;
    get(c, x, j);
#pragma unroll
    for (int i = 0; i < N; ++i) gather(x[i] > low, x[i], j + i);
  }
  if (ORDERED && n > 128) {
    float m[4] = {top.v, -INFINITY, -INFINITY, -INFINITY};
    for (int c = 0; c < sets; ++c) {
      float x[N];
      int j;
      get(c, x, j);
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int o = 0; o < 4; ++o) {
          const float y = fmaxf(m[o], x[i]);
          x[i] = fminf(m[o], x[i]);
          m[o] = y;
        }
    }
    const float v = kth_of_four<N == 8 ? 16 : 32>(m, k);
    int more = __popcll(__ballot(top.v > v));
    for (int c = 0; c < sets; ++c) {
      float x[N];
      int j;
      get(c, x, j);
#pragma unroll
      for (int i = 0; i < N; ++i) more += __popcll(__ballot(x[i] > v));
    }
    if (v > -INFINITY && more <= 128) {
      const int equal = k - more;  // entries of value v that are wanted
      int seen = 0;
      n = 0;
      wave_lds_order();
      const uint64_t ties = __ballot(top.v == v);
      gather(top.v > v || (top.v == v && lanes_below(ties) < equal), top.v, top.i);
      seen += __popcll(ties);
      for (int c = 0; c < sets; ++c) {
        float x[N];
        int j, rank = seen;  // of the lane's first entry of value v
        get(c, x, j);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint64_t in = __ballot(x[i] == v);
          rank += lanes_below(in);
          seen += __popcll(in);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
          gather(x[i] > v || (x[i] == v && rank < equal), x[i], j + i);
          rank += x[i] == v;
        }
      }
    } else if (more >= k) {
      low = fmaxf(low, v);
    }
  }
  wave_lds_order();
  if (n <= 64) {
    top.sort(pv[lane], pi[lane], n, lane);
    wave_lds_order();
    return;
  }
  if (n <= 128) {
    top.sort_two(pv, pi, n, lane);
    wave_lds_order();
    return;
  }
  for (int c = 0; c < sets; ++c) {
    float x[N];
    int j;
    get(c, x, j);
#pragma unroll 1
    for (int i = 0; i < N; ++i) {
      float y = x[0];  // x[i]
#pragma unroll
      for (int o = 1; o < N; ++o) y = i == o ? x[o] : y;
      top.insert_lanes(y > low ? y : -INFINITY, j + i, k, lane);
    }
  }
}

// The k best of n entries, get(e, x, j) the e-th.
template <typename G>
__device__ __forceinline__ void top_join(TopList& top, int n, int k, int lane, float* pv, int* pi, G&& get) {
  auto set = [&](int c, float (&x)[1], int& j) {
    const int e = c * 64 + lane;
    x[0] = -INFINITY, j = INT32_MAX;
    if (e < n) get(e, x[0], j);
  };
  const int sets = (n + 63) / 64;
  float most[2] = {-INFINITY, -INFINITY};  // of even and odd sets
#pragma unroll 2
  for (int c = 0; c < sets; c += 2)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float x[1];
      int j;
      set(c + h, x, j);
      most[h] = fmaxf(most[h], x[0]);
    }
  top.clear();
  top_select<1, false>(top, sets, first_cut(most[0], most[1], k), k, lane, pv, pi, set);
}

// The entries of a wave that may be among the k largest, while it walks its
// blocks: 16-byte pieces that hold one, with their first index, in LDS.
struct TopPieces {
  static constexpr int kCap = 320;  // 64, and the 256 of a block
  u32x4 raw[kCap];
  int at[kCap];
  float pv[128];  // for top_select
  int pi[128];
};
struct TopState {
  TopList list;  // the best so far of the pieces already gone through
  float most[2]; // the lane's largest entries so far, of the first and the second halves of blocks
  float low;     // no entry of the row up to it is wanted
  float bar;     // no later entry of this wave up to it is wanted
  int n, blocks;

  __device__ __forceinline__ void clear() { list.clear(), most[0] = most[1] = low = bar = -INFINITY, n = blocks = 0; }
  __device__ __forceinline__ void raise(float x) { low = fmaxf(low, x), bar = fmaxf(bar, x); }
};

// A block of a wave: kU 16-byte loads of each lane, 64 lanes apart.
template <typename S>
struct LogitBlock {
  static constexpr int kV = 16 / sizeof(S), kU = 4, kN = 64 * kV * kU;
  u32x4u raw[kU];

  __device__ __forceinline__ void load(const S* z, int lane) {
#pragma unroll
    for (int u = 0; u < kU; ++u) raw[u] = gload<u32x4u>(z + (u * 64 + lane) * kV);
  }
  // Only entries lo..hi of it; the others are not allowed.
  __device__ __forceinline__ void load_part(const S* z, int lo, int hi, int lane) {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int at = (u * 64 + lane) * kV;
      if (at >= lo && at + kV <= hi) {
        raw[u] = gload<u32x4u>(z + at);
      } else if (at + kV <= lo || at >= hi) {
        raw[u] = sizeof(S) == 4 ? 0xff800000u : 0xff80ff80u;
      } else {
#pragma unroll
        for (int i = 0; i < kV; ++i) {
          const bool in = at + i >= lo && at + i < hi;
          if constexpr (sizeof(S) == 4) {
            raw[u][i] = in ? gload<uint32_t>(z + at + i) : 0xff800000u;
          } else {
            const uint32_t w = in ? (uint32_t)gload<uint16_t>(z + at + i) : 0xff80u;
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

  // The block's s and t against reference n; only its first `count` entries may
  // be allowed (quarters past them are left out: 8192 x 1000 in bf16 15.6 -> 13.9
  // us).  The lower bound on d makes an entry that is not allowed add 0 to t (it
  // would be 0 times -inf).
  template <bool ENT>
  __device__ __forceinline__ void sums(float n, int count, float& s, float& t) const {
    s = t = 0.f;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      if (u * 64 * kV >= count) break;
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        const float d = at(u, i) - n, e = lse_exp(d);
        s += e;
        if (ENT) t = fmaf(fmaxf(d, -1e30f), e, t);
      }
    }
  }

  // Adds the block to st and keeps its pieces that hold a wanted entry; its
  // first entry is entry `base` of the row, `count` are left of the row, no
  // entry up to `floor_` is wanted.
  template <bool ENT>
  __device__ __forceinline__ void add(LseStat& st, TopState& top, TopPieces* pieces, float floor_, int base, int count,
                                      int k, int lane) const {
    float um[kU], bm;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      um[u] = at(u, 0);
#pragma unroll
      for (int i = 1; i < kV; ++i) um[u] = fmaxf(um[u], at(u, i));
    }
    bm = fmaxf(fmaxf(um[0], um[1]), fmaxf(um[2], um[3]));
    float s, t;
    const float n = fmaxf(st.m, bm), d = lse_shift(st.m, n), f = lse_exp(d);
    sums<ENT>(n, count, s, t);
    st.t = (st.t + d * st.s) * f + t;
    st.s = st.s * f + s;
    st.m = n;
    if (k == 0) return;
    top.most[0] = fmaxf(top.most[0], fmaxf(um[0], um[1]));
    top.most[1] = fmaxf(top.most[1], fmaxf(um[2], um[3]));
    top.raise(floor_);
    // k entries are at or above the k-th of the lanes' largest: a bound
    // worth its 16 ballots whenever the number of blocks has doubled
    ++top.blocks;
    if ((top.blocks & (top.blocks - 1)) == 0) top.raise(first_cut(top.most[0], top.most[1], k));
    if (!__any(bm > top.bar)) return;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const bool hit = um[u] > top.bar;
      const uint64_t hits = __ballot(hit);
      if (!hits) continue;
      const int to = top.n + lanes_below(hits);
      if (hit) {
        pieces->raw[to] = raw[u];
        pieces->at[to] = base + (u * 64 + lane) * kV;
      }
      top.n += __popcll(hits);
    }
    if (top.n > TopPieces::kCap - 64 * kU) settle(top, pieces, k, lane);
  }

  // The wave's k best of its list and its pieces.
  static __device__ __forceinline__ void settle(TopState& top, TopPieces* pieces, int k, int lane) {
    wave_lds_order();
    top_select<kV, true>(top.list, (top.n + 63) / 64, top.low, k, lane, pieces->pv, pieces->pi,
                   [&](int c, float (&x)[kV], int& j) {
                     const int e = c * 64 + lane;
                     LogitBlock one;
                     one.raw[0] = pieces->raw[e < top.n ? e : 0];
                     j = pieces->at[e < top.n ? e : 0];
#pragma unroll
                     for (int i = 0; i < kV; ++i) x[i] = e < top.n ? one.at(0, i) : -INFINITY;
                   });
    top.n = 0;
    wave_lds_order();
    // later entries come after these: they must exceed the k-th
    const float kth = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(top.list.v), k - 1));
    top.low = fmaxf(top.low, float_below(kth));
    top.bar = fmaxf(top.bar, kth);
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
  int64_t first; // the launch's first part of all rows' parts
  float* ws;     // a record (logprob_record) for each part of each row
};

// The outputs of a row, from a wave that holds its sums and alternatives; zt is
// the target's logit in lane 0 (where there is one).
__device__ __forceinline__ void logprobs_finish(const LogprobArgs& q, int64_t r, LseStat st, const TopList& top, int tg,
                                                float zt, int lane) {
  const bool empty = st.s == 0.f;
  const float ls = logf(st.s);  // NaN in a row that holds one or +inf
  if (lane == 0) {
    q.lse[r] = empty ? -INFINITY : st.m + ls;
    if (q.entropy) q.entropy[r] = empty ? 0.f : ls - st.t / st.s;
    if (q.logp) q.logp[r] = tg < 0 ? 0.f : empty ? -INFINITY : (zt - st.m) - ls;
  }
  if (lane < q.k) {
    const bool bad = st.s != st.s, none = bad || top.v == -INFINITY;
    q.top_ids[r * q.k + lane] = none ? -1 : top.i;
    q.top_logp[r * q.k + lane] = bad ? NAN : none ? -INFINITY : (top.v - st.m) - ls;
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

// A workgroup of W waves to a row (or to a part of it), which take its blocks in
// turn; W = 1: four rows to a workgroup.
template <typename S, int W, bool ENT>
__global__ __launch_bounds__(W == 1 ? kThreads : 64 * W) void logprobs_kernel(LogprobArgs q) {
  using Block = LogitBlock<S>;
  constexpr int kWaves = W == 1 ? 4 : W;
  __shared__ TopPieces pieces_[kWaves];
  __shared__ float floors[W];
  __shared__ float sm[W][3];
  __shared__ float sv[W][SHAMPOO_MAX_TOP];
  __shared__ int si[W][SHAMPOO_MAX_TOP];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int w = W == 1 ? 0 : wave;
  TopPieces* pieces = &pieces_[wave];
  const int64_t item = q.first + (W == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x);
  if (item >= q.rows * q.parts) return;
  const int64_t r = item / q.parts;
  const int part = (int)(item % q.parts);
  const S* z = static_cast<const S*>(q.logits) + r * q.ld;
  const int begin = part * q.per_part, end = min(q.vocab, begin + q.per_part);

  LseStat st = {kLowest, 0.f, 0.f};
  TopState top;
  top.clear();
  // What a wave does not want its neighbours do not want either, up to equal
  // values: they read each other's bounds, unsynchronised (an old one only lets
  // more entries through).
  volatile float* shared = floors;
  if (W > 1) {
    if (lane == 0) shared[w] = -INFINITY;
    __syncthreads();
  }
  Block blk, nxt;
  auto fetch = [&](int at) {
    if (at + Block::kN <= end) nxt.load(z + at, lane);
    else if (at < end) nxt.load_part(z + at, 0, end - at, lane);
  };
  int at = begin + w * Block::kN;
  fetch(at);
  float zt = 0.f;
  const int tg = q.parts == 1 && w == 0 ? logprobs_target<S>(q, r, zt) : -1;
  for (; at < end; at += W * Block::kN) {
    blk = nxt;
    fetch(at + W * Block::kN);
    float floor_ = -INFINITY;
    if (W > 1 && q.k) {
#pragma unroll
      for (int o = 0; o < W; ++o) floor_ = fmaxf(floor_, shared[o]);
      floor_ = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(floor_)));
    }
    const float old = top.low;
    blk.template add<ENT>(st, top, pieces, floor_, at, end - at, q.k, lane);
    if (W > 1 && q.k && top.low > fmaxf(old, floor_) && lane == 0) shared[w] = top.low;
  }
  if (q.k) Block::settle(top, pieces, q.k, lane);
  st = lse_wave(st);
  if constexpr (W > 1) {
    if (lane == 0) sm[w][0] = st.m, sm[w][1] = st.s, sm[w][2] = st.t;
    if (lane < q.k) sv[w][lane] = top.list.v, si[w][lane] = top.list.i;
    __syncthreads();
    if (w != 0) return;
#pragma unroll
    for (int o = 1; o < W; ++o) st = lse_join(st, {sm[o][0], sm[o][1], sm[o][2]});
    if (q.k)
      top_join(top.list, W * q.k, q.k, lane, pieces->pv, pieces->pi, [&](int e, float& x, int& j) {
        x = sv[e % W][e / W];
        j = si[e % W][e / W];
      });
  }
  if (q.parts == 1) {
    logprobs_finish(q, r, st, top.list, tg, zt, lane);
    return;
  }
  float* rec = q.ws + item * logprob_record(q.k);
  if (lane == 0) rec[0] = st.m, rec[1] = st.s, rec[2] = st.t;
  if (lane < q.k) rec[4 + lane] = top.list.v, rec[4 + q.k + lane] = __int_as_float(top.list.i);
}

// Joins the parts of a row (at most 64), one wave to a row.
template <typename S>
__global__ __launch_bounds__(64) void logprobs_join_kernel(LogprobArgs q) {
  const int lane = threadIdx.x;
  const int64_t r = blockIdx.x;  // fewer than 256 rows are cut into parts
  float zt;
  const int tg = logprobs_target<S>(q, r, zt);
  const float* rec = q.ws + r * q.parts * logprob_record(q.k);
  LseStat st = {kLowest, 0.f, 0.f};
  if (lane < q.parts) {
    const float* p = rec + lane * logprob_record(q.k);
    st = {p[0], p[1], p[2]};
  }
  st = lse_wave(st);
  __shared__ float pv[128];
  __shared__ int pi[128];
  TopList top;
  top.clear();
  if (q.k)
    top_join(top, q.parts * q.k, q.k, lane, pv, pi, [&](int e, float& x, int& j) {
      const float* p = rec + e % q.parts * logprob_record(q.k) + 4 + e / q.parts;
      x = p[0];
      j = __float_as_int(p[q.k]);
    });
  logprobs_finish(q, r, st, top, tg, zt, lane);
}

// ---------------------------------------------------------------- gradient
struct LossGradArgs {
  const void* logits;
  int64_t ld, rows;
  int vocab;
  const int32_t* targets;
  const float *lse, *entropy;
  int k;
  const int32_t* top_ids;
  const float *g_logp, *g_lse, *g_entropy, *g_top;
  void* dlogits;
  int64_t ld_d;
  int per, segs;  // blocks of a wave, and waves of a row
};

// A wave to `per` blocks of a row, which start where stores to the row are aligned
// (a row of odd length or stride begins with a part of a block).  Lane 0 holds
// the target, lane i an alternative.  The entries of these take the outputs'
// own gradients too: their lanes read them before anything of the row is
// written (the gradient may overwrite the logits; no other wave touches these
// blocks) and write them again when the wave's stores have arrived.
//   dz_j = p_j (S - g_H (ln p_j + H)) + the outputs' gradients at their entries,
//   S = g_lse - g_logp - the sum of the alternatives' gradients.
// Bound by memory: 8192 x 131072 in bf16, with entropy and 8 alternatives, in 731
// us (5.9 TB/s); 1021 x 50001 in 39 us (5.2 TB/s).  More waves on the chip than the
// memory needs cost time: fp32 rows take 3 to a SIMD (4096 x 131072: 733 us, 804
// with 4, 828 with 2; 4096 x 5000: 35.0, 33.5 and 39.6), bf16 rows the 4 that their
// registers leave (large 737, with 3 788; 8192 x 5000: 36.9 and 42.0).
template <typename S, bool ENT>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(1, sizeof(S) == 4 ? 3 : 4)))
void logprobs_grad_kernel(LossGradArgs q) {
  using Block = LogitBlock<S>;
  constexpr int kV = Block::kV, kU = Block::kU, kN = Block::kN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t item = (int64_t)blockIdx.x * 4 + wave; item < q.rows * q.segs; item += (int64_t)gridDim.x * 4) {
    const int64_t r = item / q.segs;
    const S* z = static_cast<const S*>(q.logits) + r * q.ld;
    S* dz = static_cast<S*>(q.dlogits) + r * q.ld_d;
    const int shift = (int)(reinterpret_cast<uintptr_t>(dz) / sizeof(S) % kV);
    const int begin = (int)(item % q.segs) * q.per * kN - shift, end = min(q.vocab, begin + q.per * kN);
    Block blk, nxt;
    auto fetch = [&](int at) {
      if (at >= 0 && at + kN <= end) nxt.load(z + at, lane);
      else if (at < end) nxt.load_part(z + at, -at, end - at, lane);
    };
    fetch(begin);
    const float lse = q.lse[r];
    const float H = ENT ? q.entropy[r] : 0.f, ge = ENT ? q.g_entropy[r] : 0.f;
    float base = q.g_lse ? q.g_lse[r] : 0.f;
    // up to 65 of them: alternative 64 is lane 0's second
    int id[2] = {-1, -1};
    float g[2] = {0.f, 0.f};
    if (lane == 0 && q.g_logp) id[0] = q.targets[r], g[0] = q.g_logp[r];
    if (lane > 0 && lane <= q.k) id[0] = q.top_ids[r * q.k + lane - 1], g[0] = q.g_top[r * q.k + lane - 1];
    if (lane == 0 && q.k > 63) id[1] = q.top_ids[r * q.k + 63], g[1] = q.g_top[r * q.k + 63];
#pragma unroll
    for (int o = 0; o < 2; ++o)
      if (id[o] < 0 || id[o] >= q.vocab) id[o] = -1, g[o] = 0.f;
    base -= wave_sum(g[0] + g[1]);
    const bool empty = lse == -INFINITY;  // no entry is allowed: no gradient
    if (ENT) base -= ge * H;
    auto value = [&](float x) {
      const float lp = x - lse;
      const float p = __builtin_amdgcn_exp2f(lp * kLog2e);
      // exp(-200) is 0: the bound keeps 0 times -inf out
      return empty ? 0.f : p * (ENT ? fmaf(-ge, fmaxf(lp, -200.f), base) : base);
    };
    float own[2];
    bool mine[2];
    uint64_t owners[2];
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      mine[o] = id[o] >= begin && id[o] >= 0 && id[o] < end && !empty;
      owners[o] = __ballot(mine[o]);
      own[o] = mine[o] ? value(cvt<float, S>(z[id[o]])) : 0.f;
    }
#pragma unroll
    for (int o = 0; o < 2; ++o)
      for (uint64_t todo = owners[o]; todo; todo &= todo - 1) {
        const int l = __builtin_ctzll(todo);
        const int at = __builtin_amdgcn_readlane(id[o], l);
        const float add = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(g[o]), l));
        own[0] += id[0] == at ? add : 0.f;
        own[1] += id[1] == at ? add : 0.f;
      }

    for (int at = begin; at < end; at += kN) {
      blk = nxt;
      fetch(at + kN);
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int first = at + (u * 64 + lane) * kV;
        u32x4u w;
        if constexpr (sizeof(S) == 4) {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(value(blk.at(u, i)));
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = pack_bf16(value(blk.at(u, 2 * i)), value(blk.at(u, 2 * i + 1)));
        }
        if (first >= 0 && first + kV <= end) {
          gstore<u32x4u>(dz + first, w);
        } else {
#pragma unroll
          for (int i = 0; i < kV; ++i) {
            if (first + i < 0 || first + i >= end) continue;
            if constexpr (sizeof(S) == 4) gstore<uint32_t>(dz + first + i, w[i]);
            else gstore<uint16_t>(dz + first + i, (uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2]));
          }
        }
      }
    }
    if (owners[0] | owners[1]) {
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
      asm volatile("" ::: "memory");
#pragma unroll
      for (int o = 0; o < 2; ++o)
        if (mine[o]) gstore<S>(dz + id[o], from_f32<S>(own[o]));
    }
  }
}

}  // namespace shp
