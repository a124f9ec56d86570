// Device kernels of the 8-bit activation checkpoints: encode (with the
// activation), decode, activation gradient.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "logprobs.hpp"
#include "shampoo.h"
#include "tile_mfma.hpp"

namespace shp {

constexpr int kActGroup = 32;  // columns that share one scale

// Where the codes and scale bytes of a rows x cols checkpoint lie.
struct ActCkpt {
  int64_t ldq;    // codes per row: cols rounded up to 32
  int64_t scales; // byte offset of the scale bytes
  int64_t bytes;
};
__host__ __device__ __forceinline__ ActCkpt act_ckpt(int64_t rows, int64_t cols) {
  ActCkpt c;
  c.ldq = (cols + kActGroup - 1) / kActGroup * kActGroup;
  c.scales = (rows * c.ldq + 255) / 256 * 256;
  c.bytes = c.scales + (rows * (c.ldq / kActGroup) + 255) / 256 * 256;
  return c;
}

// Scale byte of a group whose largest |x| has these bits: the exponent of the
// largest x less 6, one more when its multiple of 2^e would round to 128
// (significand at or above 127.5 / 64: the addition carries), at most 121
// (2^128 would not be finite); 255 for infinities and NaN.
__device__ __forceinline__ uint32_t act_scale_byte(uint32_t bits) {
  if (bits >= 0x7f800000u) return 255u;
  const int s = (int)((bits + 0x10000u) >> 23) - 6;
  return (uint32_t)min(max(s, 1), 248);
}
// 2^(s - 127); infinity for s = 255, whose codes are 0: 0 times infinity is
// the NaN that such a group stands for.
__device__ __forceinline__ float act_scale(uint32_t s) { return __uint_as_float(s << 23); }
// 2^-(s - 127), s <= 248.
__device__ __forceinline__ float act_unscale(uint32_t s) { return __uint_as_float((254u - s) << 23); }

// The normal distribution's lower tail Phi(-|x|) = R e, e = exp(-x^2 / 2): R, with
// e beside it.  gelu and its slope are formed from it without the cancellation of
// 1 + erf, so that their negative tails keep all bits.  FAST: R is a polynomial in
// 1 / (1 + p |x|) that was fitted for the least relative error, 4e-6 for |x| up to
// 14 (where Phi leaves fp32's normal range).
template <bool FAST>
__device__ __forceinline__ float normal_tail(float x, float& e) {
  if constexpr (!FAST) {
    e = expf(-0.5f * x * x);
    return 0.5f * erfcxf(fabsf(x) * 0.70710678f);
  }
  const float t = __builtin_amdgcn_rcpf(fmaf(0.30815624f, fabsf(x), 1.f));
  e = __builtin_amdgcn_exp2f(x * x * -0.72134752f);
  float h = fmaf(-0.0753979f, t, 0.18913349f);
  h = fmaf(h, t, 0.00769323f);
  h = fmaf(h, t, 0.13641141f);
  h = fmaf(h, t, 0.11897507f);
  h = fmaf(h, t, 0.12318278f);
  return h * t;
}
__device__ __forceinline__ float fast_sigmoid(float x) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.44269504f));
}

// FAST: for results kept in bf16 (relative errors of at most 2^-15 down to -9), where the
// library functions' 20 to 40 instructions a value would bound the pass; fp32
// passes move twice the bytes and call them.
template <int ACT, bool FAST>
__device__ __forceinline__ float act_value(float x) {
  if constexpr (ACT == SHAMPOO_ACT_RELU) return x < 0.f ? 0.f : x;
  if constexpr (ACT == SHAMPOO_ACT_GELU) {
    float e;
    const float p = normal_tail<FAST>(x, e) * e;
    return x * (x < 0.f ? p : 1.f - p);
  }
  if constexpr (ACT == SHAMPOO_ACT_GELU_TANH) {
    const float w = 1.59576912f * (x + 0.044715f * x * x * x);
    return FAST ? x * fast_sigmoid(w) : x / (1.f + expf(-w));
  }
  if constexpr (ACT == SHAMPOO_ACT_SILU) return FAST ? x * fast_sigmoid(x) : x / (1.f + expf(-x));
  return x;
}

template <int ACT, bool FAST>
__device__ __forceinline__ float act_slope(float x) {
  if constexpr (ACT == SHAMPOO_ACT_RELU) return x > 0.f ? 1.f : (x != x ? x : 0.f);
  if constexpr (ACT == SHAMPOO_ACT_GELU) {
    // Phi(x) + x phi(x), at -|x|; the slopes at x and -x add up to 1
    float e;
    const float p = fmaf(-0.39894228f, fabsf(x), normal_tail<FAST>(x, e)) * e;
    return x < 0.f ? p : 1.f - p;
  }
  if constexpr (ACT == SHAMPOO_ACT_GELU_TANH) {
    const float w = 1.59576912f * (x + 0.044715f * x * x * x);
    const float p = FAST ? fast_sigmoid(w) : 1.f / (1.f + expf(-w));
    // beyond 20 the second term is below 2^-24 and its factors overflow
    return fabsf(x) > 20.f ? p : p + x * p * (1.f - p) * (1.59576912f + 0.21406445f * x * x);
  }
  if constexpr (ACT == SHAMPOO_ACT_SILU) {
    const float p = FAST ? fast_sigmoid(x) : 1.f / (1.f + expf(-x));
    return p + x * p * (1.f - p);
  }
  return 1.f;
}

// ---------------------------------------------------------------- passes
// All passes move units of 8 columns, one to a lane in row order: 16 or 32 bytes
// of a tensor, 8 of the codes; the 4 lanes of a group agree on its scale.  Bound
// by memory: 16384 x 4096 in bf16, activation with both checkpoints and their
// values in 142 us (5.7 TB/s), gelu's gradient in 59 us (5.7 TB/s); the activation alone
// with both checkpoints 69 to 73 us whichever it is (fp32 116, gelu 131: erfcx and
// exp), the gradients 57 to 61 (fp32 105, gelu 117).  Two or four units to a lane were
// 6 and 16% slower; rows of 4095 take 167 and 66 us.
struct ActShape {
  int64_t row0, units;   // first row, and units of the launch (below 2^31)
  int cols, upr;         // columns, and units of a row (ldq / 8)
  uint32_t magic, shift; // n / upr = (t + (n - t) / 2) >> shift, t the upper half of n magic
};

// Calls f(row, unit, in) for the unit of the lane; `in` is false past the tensor
// (the lanes of a group are in or out together).
template <typename F>
__device__ __forceinline__ void act_units_of(const ActShape& h, uint32_t block, F&& f) {
  const uint32_t n = block * kThreads + threadIdx.x;
  const uint32_t t = __umulhi(n, h.magic), row = (t + ((n - t) >> 1)) >> h.shift;
  f(h.row0 + row, (int)(n - row * h.upr), n < h.units);
}
template <typename F>
__device__ __forceinline__ void act_units(const ActShape& h, F&& f) {
  act_units_of(h, blockIdx.x, f);
}

// (at element alignment)
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(2)));

// 8 elements of a tensor.
template <typename S>
struct ActVec {
  u32x4u raw[sizeof(S) / 2];

  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(S) == 4) return __uint_as_float(raw[i / 4][i % 4]);
    return __uint_as_float(i & 1 ? raw[0][i / 2] & 0xffff0000u : raw[0][i / 2] << 16);
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(S) == 4) {
        raw[0][i] = __float_as_uint(v[i]);
        raw[1][i] = __float_as_uint(v[4 + i]);
      } else {
        raw[0][i] = pack_bf16(v[2 * i], v[2 * i + 1]);
      }
    }
  }
  // n of the 8 lie in the row; the others are zeros.  A part is 4, 2 and 1
  // elements (one by one, the last unit of a row of 4095 made the activation
  // gradient take 84 us instead of 65).
  __device__ __forceinline__ void load(const S* p, int n) {
    if (n >= 8) {
#pragma unroll
      for (int h = 0; h < (int)sizeof(S) / 2; ++h) raw[h] = gload<u32x4u>(p + 4 * h);
      return;
    }
    const bool four = n > 0 && n & 4, two = n > 0 && n & 2, one = n > 0 && n & 1;
    const S* p2 = p + (four ? 4 : 0);
    const S* p1 = p2 + (two ? 2 : 0);
    if constexpr (sizeof(S) == 4) {
      u32x4u a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
      if (four) a = gload<u32x4u>(p);
      if (two) {
        const u32x2u w = gload<u32x2u>(p2);
        b[0] = w[0], b[1] = w[1];
      }
      if (one) {
        const uint32_t w = gload<uint32_t>(p1);
        if (two) b[2] = w;
        else b[0] = w;
      }
      raw[0] = four ? a : b;
      raw[1] = four ? b : a;
    } else {
      u32x2u a = {0, 0};
      uint32_t b = 0, c = 0;
      if (four) a = gload<u32x2u>(p);
      if (two) b = gload<u32u>(p2);
      if (one) c = gload<uint16_t>(p1);
      const uint32_t lo = two ? b : c, hi = two ? c : 0;
      raw[0] = four ? u32x4u{a[0], a[1], lo, hi} : u32x4u{lo, hi, 0, 0};
    }
  }
  __device__ __forceinline__ void store(S* p, int n) const {
    if (n >= 8) {
#pragma unroll
      for (int h = 0; h < (int)sizeof(S) / 2; ++h) gstore<u32x4u>(p + 4 * h, raw[h]);
      return;
    }
    const bool four = n > 0 && n & 4, two = n > 0 && n & 2, one = n > 0 && n & 1;
    S* p2 = p + (four ? 4 : 0);
    S* p1 = p2 + (two ? 2 : 0);
    if constexpr (sizeof(S) == 4) {
      if (four) gstore<u32x4u>(p, raw[0]);
      const u32x4u b = four ? raw[1] : raw[0];
      if (two) gstore<u32x2u>(p2, u32x2u{b[0], b[1]});
      if (one) gstore<uint32_t>(p1, two ? b[2] : b[0]);
    } else {
      if (four) gstore<u32x2u>(p, u32x2u{raw[0][0], raw[0][1]});
      const uint32_t b = four ? raw[0][2] : raw[0][0], c = four ? raw[0][3] : raw[0][1];
      if (two) gstore<u32u>(p2, b);
      if (one) gstore<uint16_t>(p1, (uint16_t)(two ? c : b));
    }
  }
};

// Codes and scale byte of a lane's unit, with its 3 neighbours of the group.
// x 2^-e + 1.5 2^23 rounds to the nearest even integer, whose low byte is the code.
__device__ __forceinline__ uint32_t act_quantize(const float (&v)[8], u32x2& codes) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xb1, 0xf, 0xf, true));  // lane ^ 1
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4e, 0xf, 0xf, true));  // lane ^ 2
  const uint32_t s = act_scale_byte(top);
  const float us = act_unscale(s);
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(fmaf(v[i], us, 12582912.f));
  if (__builtin_expect(__any(s >= 248u), 0)) {  // the largest scale, where 128 becomes 127, and NaN
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (s == 248u) b[i] = __float_as_uint(fminf(fmaxf(v[i] * us, -127.f), 127.f) + 12582912.f);
      if (s == 255u) b[i] = 0;
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
    codes[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[4 * h + 3], b[4 * h + 2], 0x0c0c0400u),
                                     __builtin_amdgcn_perm(b[4 * h + 1], b[4 * h], 0x0c0c0400u), 0x05040100u);
  return s;
}

// The 8 values of a unit.
__device__ __forceinline__ void act_expand(u32x2 codes, uint32_t s, float (&v)[8]) {
  const float scale = act_scale(s);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)(int8_t)(codes[i / 4] >> (8 * (i % 4))) * scale;
}

struct ActCkptPtr {
  char* codes;  // NULL: no checkpoint
  uint8_t* scales;
};

// X and Y may be the same buffer.
template <typename S, int ACT>
__global__ __launch_bounds__(kThreads) void act_encode_kernel(ActShape h, const S* X, int64_t ld_x, S* Y, int64_t ld_y,
                                                             ActCkptPtr cx, ActCkptPtr cy) {
  act_units(h, [&](int64_t row, int unit, bool in) {
    ActVec<S> x;
    x.load(X + row * ld_x + unit * 8, in ? h.cols - unit * 8 : 0);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x.at(i);
    auto keep = [&](const ActCkptPtr& c) {
      u32x2 q;
      const uint32_t s = act_quantize(v, q);
      const int64_t at = row * h.upr + unit;
      if (in) gstore<u32x2>(c.codes + at * 8, q);
      if (in && (unit & 3) == 0) gstore<uint8_t>(c.scales + at / 4, (uint8_t)s);
    };
    if (cx.codes) keep(cx);
    if (!Y && !cy.codes) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = act_value<ACT, sizeof(S) == 2>(v[i]);
    ActVec<S> y;
    y.set(v);
    if (Y && in) y.store(Y + row * ld_y + unit * 8, h.cols - unit * 8);
    if (cy.codes) {  // of y as stored
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = y.at(i);
      keep(cy);
    }
  });
}

template <typename S>
__global__ __launch_bounds__(kThreads) void act_decode_kernel(ActShape h, ActCkptPtr c, S* __restrict__ X,
                                                             int64_t ld_x) {
  act_units(h, [&](int64_t row, int unit, bool in) {
    if (!in) return;
    const int64_t at = row * h.upr + unit;
    float v[8];
    act_expand(gload<u32x2>(c.codes + at * 8), gload<uint8_t>(c.scales + at / 4), v);
    ActVec<S> x;
    x.set(v);
    x.store(X + row * ld_x + unit * 8, h.cols - unit * 8);
  });
}

// dX may be dY.
template <typename S, int ACT>
__global__ __launch_bounds__(kThreads) void act_grad_kernel(ActShape h, ActCkptPtr c, const S* dY, int64_t ld_dy,
                                                           S* dX, int64_t ld_dx) {
  act_units(h, [&](int64_t row, int unit, bool in) {
    if (!in) return;
    const int64_t at = row * h.upr + unit;
    const u32x2 q = gload<u32x2>(c.codes + at * 8);
    const uint32_t s = gload<uint8_t>(c.scales + at / 4);
    ActVec<S> d;
    d.load(dY + row * ld_dy + unit * 8, h.cols - unit * 8);
    float v[8];
    act_expand(q, s, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = d.at(i) * act_slope<ACT, sizeof(S) == 2>(v[i]);
    d.set(v);
    d.store(dX + row * ld_dx + unit * 8, h.cols - unit * 8);
  });
}

}  // namespace shp
