// Device kernels of the output layer's loss: log probabilities of given
// tokens with log-sum-exp, entropy and the largest alternatives, and their
// gradient with respect to the logits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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

// One workgroup per row.  The row is read twice for the statistics (largest
// entry, then sums) and once per alternative.
template <typename S>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(const S* __restrict__ logits, int64_t ld, int vocab,
                                                           const int32_t* __restrict__ targets,
                                                           float* __restrict__ logp, float* __restrict__ lse_out,
                                                           float* __restrict__ entropy, int k,
                                                           int32_t* __restrict__ top_ids,
                                                           float* __restrict__ top_logp) {
  __shared__ float redv[kThreads / 64];
  __shared__ int redi[kThreads / 64];
  const int64_t r = blockIdx.x;
  const S* z = logits + r * ld;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto sum = [&](float v) {
    v = wave_sum(v);
    __syncthreads();
    if (lane == 0) redv[wave] = v;
    __syncthreads();
    return redv[0] + redv[1] + redv[2] + redv[3];
  };
  float m = -INFINITY;
  for (int j = tid; j < vocab; j += kThreads) m = fmaxf(m, cvt<float, S>(z[j]));
  m = wave_max(m);
  if (lane == 0) redv[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(redv[0], redv[1]), fmaxf(redv[2], redv[3]));
  const float ref = m == -INFINITY ? 0.f : m;
  float s = 0.f, t = 0.f;
  for (int j = tid; j < vocab; j += kThreads) {
    const float d = cvt<float, S>(z[j]) - ref;
    const float e = expf(d);
    s += e;
    t += fmaxf(d, -1e30f) * e;  // 0, not NaN, for an entry that is not allowed
  }
  s = sum(s);
  t = sum(t);
  const float ls = logf(s);
  const float lse = ref + ls;
  if (tid == 0) {
    lse_out[r] = lse;
    if (entropy) entropy[r] = s == 0.f ? 0.f : ls - t / s;
    if (logp) {
      const int64_t tg = targets[r];
      float v = 0.f;
      if (tg >= 0 && tg < vocab) v = s == 0.f ? -INFINITY : (cvt<float, S>(z[tg]) - ref) - ls;
      logp[r] = v;
    }
  }
  float pv = INFINITY;  // the last alternative found
  int pi = -1;
  bool none = false;
  for (int a = 0; a < k; ++a) {
    float bv = -INFINITY;
    int bi = INT32_MAX;
    if (!none && s == s) {
      for (int j = tid; j < vocab; j += kThreads) {
        const float v = cvt<float, S>(z[j]);
        if (better(pv, pi, v, j) && better(v, j, bv, bi)) bv = v, bi = j;
      }
      for (int o = 32; o > 0; o >>= 1) {
        const float v = __shfl_xor(bv, o, 64);
        const int i = __shfl_xor(bi, o, 64);
        if (better(v, i, bv, bi)) bv = v, bi = i;
      }
    }
    __syncthreads();
    if (lane == 0) redv[wave] = bv, redi[wave] = bi;
    __syncthreads();
    for (int w = 0; w < kThreads / 64; ++w)
      if (better(redv[w], redi[w], bv, bi)) bv = redv[w], bi = redi[w];
    none = none || bv == -INFINITY;
    if (tid == 0) {
      top_ids[r * k + a] = none ? -1 : bi;
      top_logp[r * k + a] = s != s ? NAN : none ? -INFINITY : (bv - ref) - ls;
    }
    pv = bv;
    pi = bi;
  }
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
