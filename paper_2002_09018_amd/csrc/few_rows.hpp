// Products of few rows with a matrix that stream_mma.hpp cannot read as it lies: fp32, or
// bf16 at any address and stride.  Copied into planes first, such a matrix goes through
// memory four times (fp32: read, three planes written, three read) or three (bf16); here
// its elements pass from memory through registers to the matrix cores once.
//
// A tile is 32 rows x 64 columns of C (a pair: 32 of each) for eight waves, each with a
// share of the contraction, no barrier among them, their sums added in order at the end
// as stream_mma.hpp's tiles of few rows do.  A wave holds the loads of the next kDepth
// steps of 16 contraction indices in registers.  A lane of B's fragment is 8 indices of
// one column: 8 neighbours where the contraction lies along B's rows, else 8 loads that
// the 32 lanes beside it make whole rows of.  An fp32 fragment is split into its three
// planes in registers; A comes in planes (it is small, and stays in the caches).
//
// What bounds it.  Contraction along columns: memory and latency (16 rows through weights
// of 1024 x 8192 in fp32, 34 MB, 17 us a call with the copy of X; copies of the weights
// made it 33).  Along rows every lane's 16 bytes are in a line of their own, and a compute
// unit serves 9-12 B/ns of such (bf16 at odd addresses, fp32), the chip 2.1-3.3 TB/s: 5
// rows over 40960 x 2589 in fp32 167 us (132 with rows at 16 bytes; 330 with copies).
// Aligned bf16 stays with stream_mma.hpp's tiles (16 rows of the block 8.1 us, 12.6 here).
#pragma once

#include "stream_mma.hpp"
#include "stream_plans.hpp"

namespace shp {

struct FewShape {
  static constexpr int TM = 32, TN = 64, WM = 32, WN = 64, kSolo = 8, kThr = 64 * kSolo, kBm = 1, kBn = 2;
  static constexpr int kPitch = WN * 4 + 16, kRingB = 32 * kPitch, kLdsB = kSolo * kRingB, kStateB = TM * 16;
};

struct FewSeg {
  const uint16_t* a;  // planes
  int64_t plane_a;
  int lda;
  const void *b, *b2;  // b2: the second matrix of a pair
  int64_t ldb, ldb2;
};
struct FewArgs {
  MmaArgs q;  // without its segments; stages are FewStage's
  FewSeg seg[kMostSegs];
  int k;      // contraction indices of a segment
};

// Steps of 16 indices that a lane loads together.  Along rows a lane takes 64 bytes of its
// row, so that two lanes use a 128-byte line at once: half h of the lanes has the indices
// h 8 kTogether + t 8 .. + 7 of a stage in step t, of A too (the order of a sum is free).
template <typename S, int LB>
struct FewStage {
  static constexpr int kTogether = LB == kLayoutRow ? 8 / (int)sizeof(S) : 1;
  static constexpr int kBk = 16 * kTogether, kDepth = LB == kLayoutRow ? 2 : sizeof(S) == 2 ? 4 : 2;
};

// What a lane loads for one stage: P planes of B, PA of A (more than B's one of a gradient in
// terms).
template <typename S, int LB, int PA_>
struct FewLoads {
  static constexpr int P = sizeof(S) == 2 ? 1 : 3, PA = PA_, T = FewStage<S, LB>::kTogether;
  static_assert(PA >= P, "");
  u32x4 a[T][PA];
  ActVec<S> row[LB == kLayoutRow ? 2 : 1][T];
  S col[LB == kLayoutRow ? 1 : 2][8];

  // Block j's fragment of step t in planes.
  __device__ __forceinline__ void planes(int j, int t, bf16x8 (&f)[P]) const {
    if constexpr (sizeof(S) == 2) {
      if constexpr (LB == kLayoutRow) {
        f[0] = __builtin_bit_cast(bf16x8, row[j][t].raw[0]);
      } else {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (uint32_t)col[j][2 * i] | (uint32_t)col[j][2 * i + 1] << 16;
        f[0] = __builtin_bit_cast(bf16x8, v);
      }
    } else {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = LB == kLayoutRow ? row[j][t].at(i) : col[j][i];
      u32x4u p[3];
      planes_of(x, p);
#pragma unroll
      for (int s = 0; s < 3; ++s) f[s] = __builtin_bit_cast(bf16x8, p[s]);
    }
  }
};

struct FewCore {
  wg_acc acc[1][2];
  static constexpr int wm = 0, wn = 0;
};

template <typename S, int LB, bool PAIR, int PA>
__device__ __forceinline__ void few_run(const FewArgs& w, FewCore& core, int m0, int n0, int split) {
  using L = FewLoads<S, LB, PA>;
  constexpr int P = L::P, T = L::T, kDepth = FewStage<S, LB>::kDepth, kBk = FewStage<S, LB>::kBk;
  const MmaArgs& q = w.q;
  const int lane = threadIdx.x & 63, half = (lane >> 5) * 8 * T;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int from = split * q.per_split, stages = min(q.per_split, q.segs * q.seg_stages - from);
  const int first = from + stages * wave / FewShape::kSolo;
  int left = stages * (wave + 1) / FewShape::kSolo - stages * wave / FewShape::kSolo;
  const int turns = left;
  int seg = left > 0 ? first / q.seg_stages : 0, k0 = left > 0 ? first % q.seg_stages * kBk : 0;
  // rows and columns past the last are read as the last: what they give is not stored
  const int row = min(m0 + (lane & 31), q.M - 1);
  const int c0 = min(n0 + (lane & 31), q.N - 1), c1 = min(n0 + (PAIR ? 0 : 32) + (lane & 31), q.N - 1);

  const uint16_t* pa;
  const S* pb[2];
  int64_t ldb[2], plane;
  auto open = [&] {
    const FewSeg& s = w.seg[seg];
    pa = s.a + (int64_t)row * s.lda + half;
    plane = s.plane_a;
    ldb[0] = s.ldb;
    ldb[1] = PAIR ? s.ldb2 : s.ldb;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const S* b = static_cast<const S*>(PAIR && j ? s.b2 : s.b);
      const int c = j ? c1 : c0;
      pb[j] = LB == kLayoutRow ? b + c * ldb[j] + half : b + half * ldb[j] + c;
    }
  };
  open();
  // The next stage, zeros past the last index (A's planes are zeros there up to a multiple
  // of 8) and past the last stage.
  auto load = [&](L& l) {
    const bool some = left > 0;
    const int n = some ? w.k - k0 - half : 0;  // indices of this lane that are left
    if (some && k0 + kBk <= w.k) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if constexpr (LB == kLayoutRow) {
#pragma unroll
          for (int t = 0; t < T; ++t) l.row[j][t].load(pb[j] + k0 + t * 8, 8);
        } else {
          const S* at = pb[j] + k0 * ldb[j];
#pragma unroll
          for (int i = 0; i < 8; ++i) l.col[j][i] = at[i * ldb[j]];
        }
      }
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int p = 0; p < PA; ++p) l.a[t][p] = *reinterpret_cast<const u32x4*>(pa + p * plane + k0 + t * 8);
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if constexpr (LB == kLayoutRow) {
#pragma unroll
          for (int t = 0; t < T; ++t) l.row[j][t].load(pb[j] + k0 + t * 8, n - t * 8);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            l.col[j][i] = S(0);
            if (i < n) l.col[j][i] = (pb[j] + k0 * ldb[j])[i * ldb[j]];
          }
        }
      }
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int p = 0; p < PA; ++p) {
          l.a[t][p] = u32x4{0, 0, 0, 0};
          if (t * 8 < n) l.a[t][p] = *reinterpret_cast<const u32x4*>(pa + p * plane + k0 + t * 8);
        }
    }
    --left;
    k0 += kBk;
    if (k0 >= q.seg_stages * kBk && left > 0) {
      ++seg;
      k0 = 0;
      open();
    }
  };

  constexpr bool kTwo = PA > 1;  // sums of the small pairs of planes
  wg_acc small[kTwo ? 2 : 1];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int v = 0; v < 16; ++v) core.acc[0][j][v] = 0.f;
#pragma unroll
  for (int j = 0; j < (kTwo ? 2 : 1); ++j) small[j] = core.acc[0][j];
  L l[kDepth];
#pragma unroll
  for (int d = 0; d < kDepth; ++d) load(l[d]);
#pragma unroll 1
  for (int s = 0; s < turns; s += kDepth) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
#pragma unroll
      for (int t = 0; t < T; ++t) {
        bf16x8 fa[PA], fb[2][P];
#pragma unroll
        for (int p = 0; p < PA; ++p) fa[p] = __builtin_bit_cast(bf16x8, l[d].a[t][p]);
#pragma unroll
        for (int j = 0; j < 2; ++j) l[d].planes(j, t, fb[j]);
        // pairs of planes by size, the smallest first and in a sum of their own
#pragma unroll
        for (int r = PA - 1; r >= 0; --r)
#pragma unroll
          for (int p = 0; p <= r; ++p) {
            if (r - p >= P) continue;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              wg_acc& c = kTwo && r > 0 ? small[kTwo ? j : 0] : core.acc[0][j];
              c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j][r - p], fa[p], c, 0, 0, 0);
            }
          }
      }
      load(l[d]);
    }
  }
  if constexpr (kTwo) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) core.acc[0][j][v] += small[j][v];
  }
}

template <typename S, int LB, typename E>
__global__ __launch_bounds__(FewShape::kThr, sizeof(S) == 2 && LB == kLayoutK && E::kTerms == 1 ? 4 : 2) void few_kernel(
    FewArgs w, E e) {
  extern __shared__ __align__(16) char lds_bytes[];
  using T = FewShape;
  lds_char* lds = (lds_char*)lds_bytes;
  const MmaArgs& q = w.q;
  // (tiles of the same columns run on the same XCD)
  const int tiles = q.tiles_m * q.tiles_n, l = xcd_remap(blockIdx.x, gridDim.x), split = l / tiles, t = l % tiles;
  const int m0 = t % q.tiles_m * T::TM, tn = t / q.tiles_m, n0 = tn * (E::kPair ? T::TN / 2 : T::TN);
  lds_char* state = lds + T::kLdsB;
  if constexpr (E::kState) {
    for (int r = threadIdx.x; r < T::TM; r += T::kThr)
      *(lds_f32x4*)(state + r * 16) = m0 + r < q.M ? e.state(m0 + r) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
  FewCore core;
  few_run<S, LB, E::kPair, sizeof(S) == 4 ? 3 : E::kTerms>(w, core, m0, n0, split);
  if constexpr (E::kWhole) {
    if (!q.part) {
      e.template few<T>(q, core, lds, m0, n0, tn);
      return;
    }
  }
  mma_units<T>(q, core, lds, state, m0, n0, split, e);
}

}  // namespace shp
