// Device kernels of the loss from the last activations: log probabilities of given
// tokens from X and the vocabulary's table W, the logits z = X W^T never in memory.
//
// Forward: the tile's epilogue takes the largest entry m and sum s = sum e^(z - m) of
// every row over the tile's columns, and the target's logit where it lies there; a
// second kernel joins the tiles of a row.  Backward: the logits are formed again in
// pieces of the vocabulary, dz_j = c p_j + [j = t] g (c = g_lse - g) is stored in
// bf16 terms, and two products take it to dX and dW.
//
// What bounds them.  Few rows: the table's bytes (4 x 1024 over 32768 rows, 67 MB, 13.6
// us = 5.0 TB/s, 15.9 with the join).  Many: the products (8192 x 1024 over 131072:
// 1.95-2.0 ms = 1.1 PFLOP/s), of whose 256 x 256 tile of 31 us the statistics take 3.5
// (65536 exponentials, not beside matrix instructions).  Gradient of the same: 6.15-6.25
// ms, three products at 1.07 PFLOP/s; pieces of 256 MB keep dz near the last-level cache
// (pieces of 64, 128, 256, 384, 512 and 1024 MB 7340, 6657, 6451, 6953, 6526 and 6279 us
// on one card: the largest gains 3% for three quarters of a GB of workspace).
#pragma once

#include "stream_mma.hpp"
#include "stream_plans.hpp"

namespace shp {

struct VocabTargets {
  const int32_t* targets;  // or NULL
  int vocab;
  int first;               // of the piece
  // Column of the row's target, counted from the piece's first (a target elsewhere
  // is negative or past it), or kNone.
  static constexpr int kNone = -(1 << 30);
  __device__ __forceinline__ int at(int64_t row) const {
    const int t = targets ? targets[row] : -1;
    return t >= 0 && t < vocab ? t - first : kNone;
  }
};

// (m, s) of a part of a row: s = sum e^(z - m); m = kLowest and s = 0 before any
// entry.  Differences are taken before they are scaled, as in logprobs.hpp.
typedef float f32x2p __attribute__((ext_vector_type(2)));
__device__ __forceinline__ f32x2p ms_join(f32x2p a, f32x2p b) {
  const float n = fmaxf(a[0], b[0]);
  return {n, a[1] * lse_exp(lse_shift(a[0], n)) + b[1] * lse_exp(lse_shift(b[0], n))};
}

struct LseEpilogue : UnitEpilogue<LseEpilogue> {
  static constexpr bool kWhole = true;
  VocabTargets t;
  f32x2p* stat;      // rows x ld_stat
  int64_t ld_stat;
  float* z_target;   // rows
  int N;

  LseEpilogue(VocabTargets tt, f32x2p* s, int64_t ld, float* z, int n)
      : t(tt), stat(s), ld_stat(ld), z_target(z), N(n) {}
  __device__ __forceinline__ void operator()(int, const f32x4&, int, float (&)[8], float (&)[8]) const {}

  template <typename T, typename Core>
  __device__ __forceinline__ void whole(const MmaArgs& q, const Core& core, lds_char* lds, int m0, int n0,
                                        int tn) const {
    typedef __attribute__((address_space(3))) f32x2p lds_f32x2;
    lds_f32x2* rows = (lds_f32x2*)lds;  // [wave column][row]
    const int lane = threadIdx.x & 63;
    const int c0 = n0 + core.wn * T::WN + (lane >> 5) * 4;  // column of (j, v): c0 + j 32 + (v / 4) 8 + v % 4
    const bool full = n0 + T::TN <= q.N;
#pragma unroll
    for (int i = 0; i < T::kBm; ++i) {
      const int r = core.wm + i * 32 + (lane & 31);
      float z[T::kBn][16];
#pragma unroll
      for (int j = 0; j < T::kBn; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          z[j][v] = core.acc[i][j][v];
          if (!full && c0 + j * 32 + v / 4 * 8 + v % 4 >= q.N) z[j][v] = -INFINITY;
        }
      float m = kLowest;
#pragma unroll
      for (int j = 0; j < T::kBn; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) m = fmaxf(m, z[j][v]);
      m = fmaxf(m, __shfl_xor(m, 32, 64));
      const int at = m0 + r < q.M ? t.at(m0 + r) - c0 : -1;
      if (__any(at >= 0 && at < T::WN)) {
#pragma unroll
        for (int j = 0; j < T::kBn; ++j)
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (at == j * 32 + v / 4 * 8 + v % 4) z_target[m0 + r] = z[j][v];
      }
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < T::kBn; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) s += lse_exp(z[j][v] - m);
      s += __shfl_xor(s, 32, 64);
      if (lane < 32) rows[core.wn * T::TM + r] = f32x2p{m, s};
    }
    __syncthreads();
    for (int r = threadIdx.x; r < T::TM; r += T::kThr) {
      f32x2p a = rows[r];
#pragma unroll
      for (int w = 1; w < T::kWavesN; ++w) a = ms_join(a, rows[w * T::TM + r]);
      if (m0 + r < q.M) stat[(int64_t)(m0 + r) * ld_stat + tn] = a;
    }
  }

  // The same of a tile of few rows, whose waves hold shares of the contraction: 8 lanes to
  // a row of 64 columns.
  template <typename T, typename Core>
  __device__ __forceinline__ void few(const MmaArgs& q, const Core& core, lds_char* lds, int m0, int n0, int tn) const {
    mma_rows_out<T>(core.acc[0], lds + (threadIdx.x >> 6) * T::kRingB, threadIdx.x & 63);
    __syncthreads();
    const int r = threadIdx.x / 8, c = threadIdx.x % 8 * 8;
    if (r >= T::TM) return;
    float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < T::kSolo; ++w) lds_add8(z, lds + w * T::kRingB + r * T::kPitch + c * 4);
    const int at = m0 + r < q.M ? t.at(m0 + r) - n0 - c : -1;
    f32x2p a = {kLowest, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (n0 + c + i >= q.N) z[i] = -INFINITY;
      else if (i == at) z_target[m0 + r] = z[i];
      a[0] = fmaxf(a[0], z[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) a[1] += lse_exp(z[i] - a[0]);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) a = ms_join(a, f32x2p{__shfl_xor(a[0], o, 64), __shfl_xor(a[1], o, 64)});
    if (c == 0 && m0 + r < q.M) stat[(int64_t)(m0 + r) * ld_stat + tn] = a;
  }
};

// (m, s) of kStatCols columns of a row of logits that were formed in parts: a wave
// each, its columns in registers.
__global__ __launch_bounds__(kThreads) inline void logit_stat_kernel(MmaArgs q, LseEpilogue e) {
  const int lane = threadIdx.x & 63, parts = (q.N + kStatCols - 1) / kStatCols;
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (w >= (int64_t)q.M * parts) return;
  const int row = (int)(w / parts), p = (int)(w % parts);
  constexpr int kEach = kStatCols / 64;
  const int c0 = p * kStatCols + lane * kEach, t = e.t.at(row) - c0;
  const float* at = q.part + (int64_t)row * q.ld_part + c0;
  float z[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) z[i] = 0.f;
  if (c0 < q.N) {  // whole units of 8 lie in the part
#pragma unroll 4
    for (int s = 0; s < q.splits; ++s)
#pragma unroll
      for (int i = 0; i < kEach / 4; ++i) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(at + (int64_t)s * q.M * q.ld_part + 4 * i);
#pragma unroll
        for (int k = 0; k < 4; ++k) z[4 * i + k] += x[k];
      }
  }
  f32x2p a = {kLowest, 0.f};
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if (c0 + i >= q.N) z[i] = -INFINITY;
    else if (i == t) e.z_target[row] = z[i];
    a[0] = fmaxf(a[0], z[i]);
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i) a[1] += lse_exp(z[i] - a[0]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) a = ms_join(a, f32x2p{__shfl_xor(a[0], o, 64), __shfl_xor(a[1], o, 64)});
  if (lane == 0) e.stat[(int64_t)row * e.ld_stat + p] = a;
}

// lse and log probability from the parts of a row: a wave to a row.
__global__ __launch_bounds__(kThreads) inline void lse_join_kernel(int64_t rows, int parts, const f32x2p* stat,
                                                                   VocabTargets t, const float* z_target, float* logp,
                                                                   float* lse) {
  const int lane = threadIdx.x & 63;
  const int64_t step = (int64_t)gridDim.x * (kThreads / 64);
  for (int64_t row = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); row < rows; row += step) {
    f32x2p a = {kLowest, 0.f};
#pragma unroll 4
    for (int p = lane; p < parts; p += 64) a = ms_join(a, stat[row * parts + p]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) a = ms_join(a, f32x2p{__shfl_xor(a[0], o, 64), __shfl_xor(a[1], o, 64)});
    if (lane) continue;
    const float ls = logf(a[1]);
    lse[row] = a[0] + ls;
    if (logp) logp[row] = t.at(row) != t.kNone ? (z_target[row] - a[0]) - ls : 0.f;
  }
}

// The gradient of the logits, in one, two or three bf16 terms.  A row's state: c, g (0
// without a target), lse and the target's column.  One term (of bf16 inputs with bf16
// gradients) rounds each dz once, half a step of 2^-8 of it: what a bf16 tensor of
// logits' gradients holds, beside the result's own rounding of the same size.  Of many rows
// errors are about sqrt(2) times those of the result's rounding alone (0.0024 and 0.0017 of
// the norm).  Where a few entries hold most of the norm their roundings do not average out
// (of 40 random calls each, 1 row up to 2.8 times, 16 rows 2.0, 64 rows 1.7, 512 rows 1.6):
// calls of up to kSecondRows rows have two terms, off by 2^-16.  Of more rows a second term
// would double both products that read dz (8192 x 1024 over 131072 6.2 -> about 10 ms): a
// caller who wants it takes dW in fp32.
struct DlogitEpilogue : UnitEpilogue<DlogitEpilogue> {
  static constexpr bool kState = true;
  VocabTargets t;
  const float *lse, *g_logp, *g_lse;
  uint16_t* dz;  // M x ld
  int64_t ld, plane;
  int N, planes;

  DlogitEpilogue(VocabTargets tt, const float* l, const float* gp, const float* gs, uint16_t* d, int64_t ld_d,
                 int64_t pl, int n, int np)
      : t(tt), lse(l), g_logp(gp), g_lse(gs), dz(d), ld(ld_d), plane(pl), N(n), planes(np) {}
  __device__ __forceinline__ f32x4 state(int row) const {
    const int target = t.at(row);
    const float l = lse[row], given = g_logp ? g_logp[row] : 0.f, penalty = g_lse ? g_lse[row] : 0.f;
    const float g = target != t.kNone ? given : 0.f;
    return {penalty - g, g, l, __int_as_float(target)};
  }
  __device__ __forceinline__ void operator()(int row, const f32x4& st, int col, float (&z)[8], float (&)[8]) const {
    const float c = st[0], g = st[1], l = st[2];
    const int at = __float_as_int(st[3]) - col;
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = c * lse_exp(z[i] - l);
    if (at >= 0 && at < 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i == at) z[i] += g;
    }
    // columns past the last, and rows of nothing: without entries, or without gradients (those
    // of a padded batch, whose lse may hold anything: exp may be infinite there, and 0 times
    // it a NaN that the products would carry to other rows)
    const bool nothing = l == -INFINITY || (c == 0.f && g == 0.f);
    if (col + 8 > N || nothing) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i >= N || nothing) z[i] = 0.f;
    }
    uint16_t* d = dz + row * ld + col;
    if (planes == 1) {
      ActVec<uint16_t> v;
      v.set(z);
      gstore<u32x4u>(d, v.raw[0]);
    } else {
      u32x4u p[3];
      planes_of(z, p);
#pragma unroll
      for (int s = 0; s < 3; ++s)
        if (s < planes) gstore<u32x4u>(d + s * plane, p[s]);
    }
  }
};

}  // namespace shp
