// Device kernels of the gated feed-forward block: H = act(G) o U of G = X Wg and U = X
// Wu, and its gradients.  One tile holds the same columns of G and U (a pair), so the
// activation and the product are the epilogue of both projections, and of the
// backward pass where they were not kept.
//
// What bounds them.  16 rows of 1024 x 4096 in bf16: 17 MB of weights and latency, 7.1 us
// (a call 8-9, the host's side).  16384 rows with G and U kept: 296-306 us, 275 GFLOP at
// 0.9 PFLOP/s and 400 MB of stores, which a tile's 16 stages hide in part (without G and
// U 280; with 64 stages to a tile 1.2 PFLOP/s).  Two workgroups of 128 x 256 on a compute
// unit take 342 us, and 277 without G and U.  Their gradient: the elementwise pass 111 us (671 MB, 6.1 TB/s), dX
// 236 and dWg with dWu 241 + 13 (1.15 PFLOP/s); dG and dU in the products' loads instead
// of a pass would form each of them once per tile that reads it.
#pragma once

#include "stream_mma.hpp"

namespace shp {

// f with the activation as a compile-time constant (a uniform branch).
template <typename F>
__device__ __forceinline__ void act_switch(int act, F&& f) {
  switch (act) {
    case SHAMPOO_ACT_RELU: f(std::integral_constant<int, SHAMPOO_ACT_RELU>()); break;
    case SHAMPOO_ACT_GELU: f(std::integral_constant<int, SHAMPOO_ACT_GELU>()); break;
    case SHAMPOO_ACT_GELU_TANH: f(std::integral_constant<int, SHAMPOO_ACT_GELU_TANH>()); break;
    case SHAMPOO_ACT_SILU: f(std::integral_constant<int, SHAMPOO_ACT_SILU>()); break;
    default: f(std::integral_constant<int, SHAMPOO_ACT_NONE>()); break;
  }
}

// H, and G and U where they are kept (rounded for themselves: H is of the sums).
template <typename S>
struct GatedEpilogue : UnitEpilogue<GatedEpilogue<S>> {
  static constexpr bool kPair = true;
  int act, N;
  S *H, *G, *U;
  int64_t ld_h, ld_g, ld_u;

  GatedEpilogue(int a, int n, S* h, S* g, S* u, int64_t lh, int64_t lg, int64_t lu)
      : act(a), N(n), H(h), G(g), U(u), ld_h(lh), ld_g(lg), ld_u(lu) {}
  __device__ __forceinline__ void operator()(int row, const f32x4&, int col, float (&g)[8], float (&u)[8]) const {
    ActVec<S> v;
    if (G) {
      v.set(g);
      v.store(G + row * ld_g + col, N - col);
      v.set(u);
      v.store(U + row * ld_u + col, N - col);
    }
    act_switch(act, [&](auto a) {
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = act_value<decltype(a)::value, sizeof(S) == 2>(g[i]) * u[i];
    });
    v.set(g);
    v.store(H + row * ld_h + col, N - col);
  }
};

// dG = dH o U o act'(G) and dU = dH o act(G), in P = one or three bf16 terms with zeros up
// to a multiple of 8 columns.  One term (of bf16 inputs with bf16 gradients) rounds each
// once to bf16, as a tensor of that type between the layers would (results are 0.0023 of
// the norm off, 0.0017 by their own rounding), and takes the activations' short forms, whose
// errors are 2^-7 of that rounding; fp32 gradients take three, exact, of the activations as
// exact as fp32 passes have them.
template <typename S, int P>
struct GatedGradEpilogue : UnitEpilogue<GatedGradEpilogue<S, P>> {
  static constexpr bool kPair = true;
  int act, N;
  const S* dH;
  int64_t ld_dh;
  uint16_t *dG, *dU;  // M x ld
  int64_t ld, plane;

  GatedGradEpilogue(int a, int n, const S* h, int64_t lh, uint16_t* g, uint16_t* u, int64_t l, int64_t pl)
      : act(a), N(n), dH(h), ld_dh(lh), dG(g), dU(u), ld(l), plane(pl) {}
  __device__ __forceinline__ void put(uint16_t* d, const float (&x)[8]) const {
    if constexpr (P == 1) {
      ActVec<uint16_t> v;
      v.set(x);
      gstore<u32x4u>(d, v.raw[0]);
    } else {
      u32x4u p[3];
      planes_of(x, p);
#pragma unroll
      for (int s = 0; s < 3; ++s) gstore<u32x4u>(d + s * plane, p[s]);
    }
  }
  __device__ __forceinline__ void operator()(int row, const f32x4&, int col, float (&g)[8], float (&u)[8]) const {
    ActVec<S> d;
    d.load(dH + row * ld_dh + col, N - col);
    act_switch(act, [&](auto a) {
      constexpr int kAct = decltype(a)::value;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool in = col + i < N;
        const float h = d.at(i), slope = act_slope<kAct, P == 1>(g[i]);
        const float value = act_value<kAct, P == 1>(g[i]);
        g[i] = in ? h * u[i] * slope : 0.f;
        u[i] = in ? h * value : 0.f;
      }
    });
    put(dG + row * ld + col, g);
    put(dU + row * ld + col, u);
  }
};

// The same from projections that were kept.
template <typename S, int P>
__global__ __launch_bounds__(kThreads) void gated_grad_kernel(ActShape h, const S* __restrict__ G, int64_t ld_g,
                                                             const S* __restrict__ U, int64_t ld_u,
                                                             GatedGradEpilogue<S, P> e) {
  act_units(h, [&](int64_t row, int unit, bool in) {
    const int n = h.cols - unit * 8;
    if (!in || n <= 0) return;
    ActVec<S> g, u;
    g.load(G + row * ld_g + unit * 8, n);
    u.load(U + row * ld_u + unit * 8, n);
    float x[8], y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = g.at(i), y[i] = u.at(i);
    e((int)row, f32x4{0.f, 0.f, 0.f, 0.f}, unit * 8, x, y);
  });
}

}  // namespace shp
