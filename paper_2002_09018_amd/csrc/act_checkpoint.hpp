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

template <int ACT>
__device__ __forceinline__ float act_value(float x) {
  if constexpr (ACT == SHAMPOO_ACT_RELU) return x > 0.f ? x : (x != x ? x : 0.f);
  if constexpr (ACT == SHAMPOO_ACT_GELU) return 0.5f * x * (1.f + erff(x * 0.70710678f));
  if constexpr (ACT == SHAMPOO_ACT_GELU_TANH)
    return x / (1.f + expf(-1.59576912f * (x + 0.044715f * x * x * x)));
  if constexpr (ACT == SHAMPOO_ACT_SILU) return x / (1.f + expf(-x));
  return x;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float x) {
  if constexpr (ACT == SHAMPOO_ACT_RELU) return x > 0.f ? 1.f : (x != x ? x : 0.f);
  if constexpr (ACT == SHAMPOO_ACT_GELU)
    return 0.5f * (1.f + erff(x * 0.70710678f)) + x * (0.39894228f * expf(-0.5f * x * x));
  if constexpr (ACT == SHAMPOO_ACT_GELU_TANH) {
    const float p = 1.f / (1.f + expf(-1.59576912f * (x + 0.044715f * x * x * x)));
    // beyond 20 the second term is below 2^-24 and its factors overflow
    return fabsf(x) > 20.f ? p : p + x * p * (1.f - p) * (1.59576912f + 0.21406659f * x * x);
  }
  if constexpr (ACT == SHAMPOO_ACT_SILU) {
    const float p = 1.f / (1.f + expf(-x));
    return p + x * p * (1.f - p);
  }
  return 1.f;
}

// Codes and scale of one group of up to 32 values.
__device__ __forceinline__ void act_encode_group(const float* v, char* ckpt, const ActCkpt& c, int64_t r, int64_t g) {
  uint32_t top = 0;
  for (int i = 0; i < kActGroup; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  const uint32_t s = act_scale_byte(top);
  int8_t* q = reinterpret_cast<int8_t*>(ckpt) + r * c.ldq + g * kActGroup;
  for (int i = 0; i < kActGroup; ++i) q[i] = s == 255u ? 0 : (int8_t)fminf(fmaxf(rintf(v[i] * act_unscale(s)), -127.f), 127.f);
  reinterpret_cast<uint8_t*>(ckpt)[c.scales + r * (c.ldq / kActGroup) + g] = (uint8_t)s;
}

// One thread per group of 32 columns.  X and Y may be the same buffer.
template <typename S, int ACT>
__global__ __launch_bounds__(kThreads) void act_encode_kernel(const S* X, int64_t ld_x, int64_t rows, int64_t cols,
                                                             S* Y, int64_t ld_y, char* ckpt_x, char* ckpt_y) {
  const ActCkpt c = act_ckpt(rows, cols);
  const int64_t ng = c.ldq / kActGroup;
  const int64_t step = (int64_t)gridDim.x * kThreads;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * ng; i += step) {
    const int64_t r = i / ng, g = i % ng;
    float v[kActGroup];
    for (int j = 0; j < kActGroup; ++j)
      v[j] = g * kActGroup + j < cols ? cvt<float, S>(X[r * ld_x + g * kActGroup + j]) : 0.f;
    if (ckpt_x) act_encode_group(v, ckpt_x, c, r, g);
    if (!Y && !ckpt_y) continue;
    for (int j = 0; j < kActGroup; ++j) {
      const S y = from_f32<S>(act_value<ACT>(v[j]));
      if (Y && g * kActGroup + j < cols) Y[r * ld_y + g * kActGroup + j] = y;
      v[j] = g * kActGroup + j < cols ? cvt<float, S>(y) : 0.f;
    }
    if (ckpt_y) act_encode_group(v, ckpt_y, c, r, g);
  }
}

__device__ __forceinline__ float act_load(const char* ckpt, const ActCkpt& c, int64_t r, int64_t j) {
  const float q = (float)reinterpret_cast<const int8_t*>(ckpt)[r * c.ldq + j];
  return q * act_scale(reinterpret_cast<const uint8_t*>(ckpt)[c.scales + r * (c.ldq / kActGroup) + j / kActGroup]);
}

template <typename S>
__global__ __launch_bounds__(kThreads) void act_decode_kernel(const char* __restrict__ ckpt, int64_t rows,
                                                             int64_t cols, S* __restrict__ X, int64_t ld_x) {
  const ActCkpt c = act_ckpt(rows, cols);
  const int64_t step = (int64_t)gridDim.x * kThreads;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * cols; i += step) {
    const int64_t r = i / cols, j = i % cols;
    X[r * ld_x + j] = from_f32<S>(act_load(ckpt, c, r, j));
  }
}

// dX may be dY.
template <typename S, int ACT>
__global__ __launch_bounds__(kThreads) void act_grad_kernel(const char* __restrict__ ckpt, int64_t rows, int64_t cols,
                                                           const S* dY, int64_t ld_dy, S* dX, int64_t ld_dx) {
  const ActCkpt c = act_ckpt(rows, cols);
  const int64_t step = (int64_t)gridDim.x * kThreads;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < rows * cols; i += step) {
    const int64_t r = i / cols, j = i % cols;
    dX[r * ld_dx + j] = from_f32<S>(cvt<float, S>(dY[r * ld_dy + j]) * act_slope<ACT>(act_load(ckpt, c, r, j)));
  }
}

}  // namespace shp
