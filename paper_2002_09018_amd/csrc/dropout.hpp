// Device kernel of dropout, its mask from a counter-based generator: Philox 4x32 with
// 10 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2,
// 3", 2011).  Each 8 columns of a row are one counter (column / 8, row, offset), whose
// 128 bits decide them by 16 each; the mask depends on nothing else, so a gradient
// forms it again.
//
// Bound by memory: 16384 x 4096 in bf16 with a residual 69 us = 5.8 TB/s (a plain copy
// 5.0), the generator's 20 wide multiplications for 8 elements beside it (43% of vector
// issue).  A few rows: one launch, 2.4 us (a call 7.0, the host's side).
#pragma once

#include "stream_mma.hpp"

namespace shp {

struct DropoutArgs {
  uint32_t key[2], offset[2];
  uint32_t least;  // elements whose 16 bits are at or above it stay
  float scale;
};

__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p = (uint64_t)0xD2511F53u * c[0], q = (uint64_t)0xCD9E8D57u * c[2];
    c[0] = (uint32_t)(q >> 32) ^ c[1] ^ k0;
    c[1] = (uint32_t)q;
    c[2] = (uint32_t)(p >> 32) ^ c[3] ^ k1;
    c[3] = (uint32_t)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

// Y = R + scale (kept X); Y may be X or R.  An element that does not stay leaves no
// trace, whatever it holds.
template <typename S>
__global__ __launch_bounds__(kThreads) void dropout_kernel(ActShape h, DropoutArgs q, const S* X, int64_t ld_x,
                                                          const S* R, int64_t ld_r, S* Y, int64_t ld_y) {
  act_units(h, [&](int64_t row, int unit, bool in) {
    const int n = h.cols - unit * 8;
    if (!in || n <= 0) return;
    ActVec<S> x, r;
    x.load(X + row * ld_x + unit * 8, n);
    if (R) r.load(R + row * ld_r + unit * 8, n);
    uint32_t c[4] = {(uint32_t)unit, (uint32_t)row, q.offset[0], q.offset[1]};
    philox(c, q.key[0], q.key[1]);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t bits = i & 1 ? c[i / 2] >> 16 : c[i / 2] & 0xffffu;
      const bool stays = bits >= q.least;
      const float y = stays ? x.at(i) * q.scale : 0.f;
      v[i] = R ? r.at(i) + y : y;
    }
    x.set(v);
    x.store(Y + row * ld_y + unit * 8, n);
  });
}

}  // namespace shp
