// Weight gradient G = beta G + X^^T dY from an 8-bit activation checkpoint.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "act_checkpoint.hpp"
#include "tile_mfma.hpp"

namespace shp {

// One workgroup per 16 x 16 tile of G: 16 tokens at a time through LDS, fp32.
template <typename S, typename SG>
__global__ __launch_bounds__(256) void weight_grad_kernel(const char* __restrict__ ckpt, int64_t rows, int64_t cols,
                                                         const S* __restrict__ dY, int64_t out, int64_t ld_dy,
                                                         SG* __restrict__ G, int64_t ld_g, float beta) {
  __shared__ float a[16][17], b[16][17];
  const ActCkpt c = act_ckpt(rows, cols);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int64_t tiles_n = (out + 15) / 16;
  const int64_t m0 = blockIdx.x / tiles_n * 16, n0 = blockIdx.x % tiles_n * 16;
  float acc = 0.f;
  for (int64_t k0 = 0; k0 < rows; k0 += 16) {
    const int64_t r = k0 + ty;
    a[ty][tx] = r < rows && m0 + tx < cols ? act_load(ckpt, c, r, m0 + tx) : 0.f;
    b[ty][tx] = r < rows && n0 + tx < out ? cvt<float, S>(dY[r * ld_dy + n0 + tx]) : 0.f;
    __syncthreads();
    for (int k = 0; k < 16; ++k) acc += a[k][ty] * b[k][tx];
    __syncthreads();
  }
  if (m0 + ty < cols && n0 + tx < out) {
    SG* g = G + (m0 + ty) * ld_g + n0 + tx;
    *g = from_f32<SG>(beta == 0.f ? acc : beta * cvt<float, SG>(*g) + acc);
  }
}

}  // namespace shp
