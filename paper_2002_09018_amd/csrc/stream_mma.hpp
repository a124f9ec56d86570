// Products of bf16 matrices on the matrix cores (v_mfma_f32_32x32x16_bf16), with what
// follows them applied to the tile: the core of the loss from the last activations
// and of the gated feed-forward block.
//
// Operands.  An operand lies with its contraction index along its rows (kLayoutRow)
// or along its columns (kLayoutK), in bf16, 16-byte aligned with strides that are
// multiples of 8.  An fp32 matrix is three bf16 matrices ("planes", x = p0 + p1 +
// p2 exactly); a stage holds all planes of both operands, and each 16 contraction
// indices are multiplied for the pairs of planes that count (six of nine, or three
// where the other operand has one), the smallest first.  A sum of two products (dG
// Wg^T + dU Wu^T) is two segments of one long contraction.  Two terms of A with a B of one
// plane (a gradient's, before bf16 matrices) go beside each other through small tiles, which
// the bytes of B bound, and through larger ones in two rounds of the contraction, the
// smaller first: a stage of both would leave one workgroup to a compute unit (128 x 128: 1021
// x 333 x 50001 400 -> 412 us, 48 to 128 rows 5-8% less).
//
// Staging.  Stages of kBk = 64 or 32 contraction indices go from memory to LDS
// without passing registers (buffer_load ... lds, 1 KB a wave and instruction), into a
// ring of kBufs buffers: kBufs - 1 stages are in flight.  Lanes whose row, column or
// contraction index lies outside the operand have an offset outside the buffer's
// range and receive zeros, so that no size needs other code.
//   kLayoutRow: [row][kBk], its 16-byte chunks stored at chunk ^ (row >> 1 & 7) (rows
//               of 128 bytes) or ^ (row >> 2 & 3) (of 64); a fragment (8 k of a row) is
//               one 16-byte read.  64 bytes of a row cost the memory path what its whole
//               128-byte line does (a compute unit streams 41-70 B/ns against 98-136), so
//               bf16 tiles take 64 indices to a stage: 16384 x 1024 x 8192 331 -> 310 us.
//               Three planes of two operands leave room for 32.
//   kLayoutK:   panels of [k][128 or 64 columns], 32-byte pieces stored at piece ^
//               swizzle(k), read with the transposing read (ds_read_b64_tr_b16).  Where
//               both operands lie so, three stages of 32 are faster than two of 64 (217 us
//               and 228 for 16384 x 1024 x 8192).
// The destination of a load is fixed (1 KB in lane order), so the swizzle is in
// the addresses that the lanes load from; conflicts take 0-2% of LDS cycles in the loop.
//
// Loop.  One barrier per stage, before its last 16 indices are multiplied: all
// fragments of the stage are in registers then, its buffer is free for the stage
// kBufs further on, and the first fragments of the next stage are read beside the
// last products.  Reads and loads go out between the matrix instructions (in blocks
// before them: 6559 -> 6277 us for the gradients of 8192 x 1024 x 131072).
//
// Few rows.  A product of up to 32 rows is bound by the other operand's bytes and by
// latency: 32 x 64 tiles whose waves (eight; four of three planes) each have a ring and a
// share of the contraction, no barrier among them, summed at the end (16 x 1024 x 8192:
// 13.1 -> 10.4 us against 32 x 128 tiles of two waves in parts).
//
// What bounds it.  256 x 256 tiles in bf16 run at 1.15-1.24 PFLOP/s, where a library's
// 8192^3 product reaches 1.3 on the same card: the clock falls under both, and the same
// instructions on small gradients instead of random numbers take 5% less time.  With an
// epilogue that stores more than the tile (the logits' gradient, the block with its projections)
// they run at 0.91-0.94: one workgroup to a compute unit has nothing of its next tile in flight
// while a tile leaves, 55-70 us of each launch of 275 GFLOP (294-301 us, the plain products
// 221-238).  Neither two workgroups of half the tile on a compute unit (7 and 13% slower)
// nor starting workgroups apart nor skipped LDS reads (4%) lift it; loads of the next tile
// ahead of this one's stores were not tried.
// fp32 products reach 190-200 TFLOP/s, six bf16 products each.
//
// The instruction's first operand is B and its second A, so that a lane holds one
// row of C (lane % 32) and runs of four columns: sums along a row are formed in the
// lane.  Results leave through LDS, 32 rows of a wave at a time, as units of 8
// neighbouring columns.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "act_checkpoint.hpp"
#include "layer_plans.hpp"
#include "split_mfma.hpp"
#include "stream_plans.hpp"
#include "tile_mfma.hpp"
#include "weight_grad.hpp"

namespace shp {

// One product of the sum.
struct MmaSeg {
  const uint16_t *a, *b, *b2;          // b2: the second matrix of a pair (columns of the tile's other half)
  int64_t plane_a, plane_b, plane_b2;  // elements from one plane to the next
  int lda, ldb, ldb2;
};
constexpr int kMostSegs = 2;

struct MmaArgs {
  MmaSeg seg[kMostSegs];
  int segs;
  int M, N;            // of C; of a pair: of each of the two
  int ka, kb;          // contraction indices of A and B (rounded up to 8 where they lie along rows)
  int seg_stages;      // stages of a segment
  int tiles_m, tiles_n;
  int splits, per_split;  // parts of the contraction, and their stages
  float* part;         // parts of C (splits x M x ld_part, a pair's second matrix at ld_part / 2), or NULL
  int64_t ld_part;
  int part_add;        // added to what `part` holds
};

// Tiles of TM x TN, waves of WM x WN.  SOLO: so many waves that each hold the whole tile
// and a share of the contraction, with a ring of their own and no barrier; their sums
// are added in order at the end.
template <int TM_, int TN_, int WM_, int WN_, int BUFS_, int PA_ = 1, int PB_ = 1, int SOLO_ = 0,
          int BK_ = 32>
struct MmaShape {
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, kBufs = BUFS_, PA = PA_, PB = PB_, kSolo = SOLO_;
  static constexpr int kBk = BK_, kSteps = kBk / 16;  // contraction indices of a stage, 16 to a step
  static constexpr int kWavesN = TN / WN, kWaves = (TM / WM) * kWavesN;  // that share a stage
  static constexpr int kThr = 64 * kWaves * (kSolo ? kSolo : 1);
  static constexpr int kBytesA = TM * kBk * 2, kBytesB = TN * kBk * 2;  // of one plane
  static constexpr int kStageB = PA * kBytesA + PB * kBytesB;
  static constexpr int kLoadsA = kBytesA / 1024 / kWaves, kLoadsB = kBytesB / 1024 / kWaves;
  static constexpr int kLoads = PA * kLoadsA + PB * kLoadsB;
  static constexpr int kBm = WM / 32, kBn = WN / 32;
  static constexpr int kPitch = WN * 4 + 16;          // bytes of a row on its way out
  static constexpr int kRingB = kBufs * kStageB;
  static constexpr int kOutB = kThr / 64 * 32 * kPitch;
  // the rings or what leaves, then 16 bytes a row for an epilogue's state
  static constexpr int kLdsB = kSolo ? kRingB * kSolo : kRingB > kOutB ? kRingB : kOutB;
  static constexpr int kStateB = TM * 16;
  static_assert(kLoadsA * kWaves * 1024 == kBytesA && kLoadsB * kWaves * 1024 == kBytesB, "");
  static_assert(kSolo == 0 || (kWaves == 1 && kBm == 1 && 32 * kPitch <= kRingB && kThr >= TN * 4), "");
};

// An offset outside every buffer's range.
constexpr uint32_t kOutside = 0x80000000u;

// What a row's 16-byte chunks are exchanged by: the 16 lanes that LDS serves at a time read
// one chunk of 16 rows, and 256 bytes hold 2 or 4 rows.
template <int BK>
__device__ __forceinline__ int mma_row_swz(int row) {
  return BK == 64 ? (row >> 1) & 7 : (row >> 2) & 3;
}
template <int W>
__device__ __forceinline__ int mma_swz(int k) {
  return W == 128 ? wg_swz(k) : W == 64 ? ((k >> 1) & 1) << 1 : 0;
}

// One lane's share of an operand's staging: the offsets it loads from and their
// contraction indices within a stage.
template <int LAYOUT, int W, int BK, int LOADS, int WAVES>
struct MmaLoader {
  static constexpr int kPerPanel = W * BK * 2 / 1024;  // loads of a panel of W columns (kLayoutK)
  uint32_t off[LOADS];
  int kl[LOADS];

  // Panels of a pair take their columns from n0 each (PAIR), others go on.
  template <bool PAIR>
  __device__ __forceinline__ void init(int i0, int end, int ld, int wave, int lane) {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int idx = j * WAVES + wave;
      if constexpr (LAYOUT == kLayoutRow) {
        constexpr int kChunks = BK / 8;  // of a row
        const int row = idx * (64 / kChunks) + lane / kChunks, c = (lane % kChunks) ^ mma_row_swz<BK>(row);
        kl[j] = c * 8;
        off[j] = i0 + row < end ? (uint32_t)row * (uint32_t)ld * 2u + c * 16u : kOutside;
      } else {
        const int in = idx % kPerPanel, panel = idx / kPerPanel;
        const int k = in * (512 / W) + lane / (W / 8);
        const int piece = ((lane >> 1) & (W / 16 - 1)) ^ mma_swz<W>(k);
        const int col = (PAIR ? 0 : panel * W) + piece * 16 + (lane & 1) * 8;
        kl[j] = k;
        off[j] = i0 + col < end ? ((uint32_t)k * (uint32_t)ld + (uint32_t)col) * 2u : kOutside;
      }
    }
  }
};

// 1 KB from the lanes' offsets to LDS, in lane order.  In asm, as the compiler would
// have every later transposing read wait for all loads in flight; mma_wait and
// mma_barrier are what orders them.  (The instruction writes no
// register.  The wait states are those that M0, and the scalar registers of the range
// if the vector unit wrote them, need before it.  M0 is a reserved register, which the compiler
// warns of; it uses it for nothing else in this code.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void mma_dma(const char* base, uint32_t off, lds_char* to) {
  const uint64_t at = reinterpret_cast<uint64_t>(base);
  const u32x4 rsrc = {(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               ::"s"((uint32_t)(uintptr_t)to), "v"(off), "s"(rsrc)
               : "memory", "m0");
}
#pragma clang diagnostic pop

template <int N>
__device__ __forceinline__ void mma_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// All of this wave's LDS reads have arrived; then the barrier of the waves that share
// its stages.
template <bool SHARED>
__device__ __forceinline__ void mma_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  if (SHARED) __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Logical tile of a workgroup: groups of 8 tile rows, within them column by column,
// so that the workgroups that run at once on an XCD share few operand panels.
__device__ __forceinline__ void mma_tile(int t, int tiles_m, int tiles_n, int& tm, int& tn) {
  constexpr int kGroup = 8;
  const int64_t whole = (int64_t)kGroup * tiles_n;
  const int g = (int)(t / whole), in = (int)(t % whole);
  const int rows = min(kGroup, tiles_m - g * kGroup);
  tm = g * kGroup + in % rows;
  tn = in / rows;
}

// The accumulators of one wave after all stages of its part, in ROUNDS rounds over the planes
// of an A that is read as if it had one.
template <typename T, int LA, int LB, bool PAIR, int ROUNDS = 1>
struct MmaCore {
  static_assert(ROUNDS == 1 || T::PA + T::PB == 2, "");
  static constexpr int kWa = T::TM < 128 ? T::TM : 128, kWb = PAIR ? T::TN / 2 : T::TN < 128 ? T::TN : 128;
  wg_acc acc[T::kBm][T::kBn];
  int wm, wn;  // first row of the wave in the tile, and number of its column strip

  // Column of the tile where block j of the wave begins.
  __device__ __forceinline__ int block_col(int j) const {
    return PAIR ? j * (T::TN / 2) + wn * 32 * (T::kBn / 2) : wn * T::WN + j * 32;
  }

  template <int LAYOUT, int W>
  static __device__ __forceinline__ int frag_at(int first, int lane) {
    if constexpr (LAYOUT == kLayoutRow)
      return (first + (lane & 31)) * (T::kBk * 2) + ((lane >> 5) ^ mma_row_swz<T::kBk>(lane & 31)) * 16;
    const int k = (lane >> 5) * 8 + ((lane >> 2) & 3), side = (lane >> 4) & 1;
    return first / W * (W * T::kBk * 2) + k * (W * 2) + ((first % W / 16 + side) ^ mma_swz<W>(k)) * 32 +
           (lane & 3) * 8;
  }
  template <int LAYOUT, int W>
  static __device__ __forceinline__ bf16x8 frag(lds_char* stage, int at, int step) {
    if constexpr (LAYOUT == kLayoutRow)
      return __builtin_bit_cast(bf16x8, *(lds_u32x4*)(stage + (at ^ (step * 32))));
    else
      return wg_frag<W * 2>(stage + at + step * 16 * W * 2);
  }

  // `between` runs while the first stages are on their way.
  template <typename F>
  __device__ __forceinline__ void run(const MmaArgs& q, lds_char* lds, int m0, int n0, int split, F&& between) {
    static_assert(T::kBn == 2 || !PAIR, "");
    const int lane = threadIdx.x & 63;
    const int all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = T::kSolo ? 0 : all;
    wm = wave / T::kWavesN * T::WM;
    wn = wave % T::kWavesN;
    int first = split * q.per_split;
    int stages = min(q.per_split, q.segs * q.seg_stages - first);
    if constexpr (T::kSolo > 0) {
      const int from = stages * all / T::kSolo, to = stages * (all + 1) / T::kSolo;
      first = from < to ? first + from : 0;
      stages = to - from;
      lds += all * T::kRingB;
    }
    constexpr bool kShared = T::kSolo == 0;

    // where the next stage to be loaded lies
    int seg = first / q.seg_stages, at = first % q.seg_stages, left = stages * ROUNDS;
    [[maybe_unused]] int in_round = stages, term = ROUNDS - 1;
    const char *pa, *pb, *pb2;
    int64_t step_a, step_b, step_b2, plane_a, plane_b, plane_b2;  // bytes
    MmaLoader<LA, kWa, T::kBk, T::kLoadsA, T::kWaves> la;
    MmaLoader<LB, kWb, T::kBk, T::kLoadsB, T::kWaves> lb;
    // whether load j of B is of a pair's second panel
    auto second = [&](int j) { return PAIR && (j * T::kWaves + wave) * 2 >= T::kLoadsB * T::kWaves; };
    auto open = [&] {
      const MmaSeg& s = q.seg[seg];
      step_a = LA == kLayoutRow ? T::kBk * 2 : (int64_t)s.lda * T::kBk * 2;
      step_b = LB == kLayoutRow ? T::kBk * 2 : (int64_t)s.ldb * T::kBk * 2;
      plane_a = 2 * s.plane_a;
      plane_b = 2 * s.plane_b;
      plane_b2 = 2 * s.plane_b2;
      step_b2 = PAIR ? (int64_t)s.ldb2 * T::kBk * 2 : 0;
      pa = reinterpret_cast<const char*>(s.a) + (LA == kLayoutRow ? (int64_t)m0 * s.lda : m0) * 2 + at * step_a;
      pb = reinterpret_cast<const char*>(s.b) + (LB == kLayoutRow ? (int64_t)n0 * s.ldb : n0) * 2 + at * step_b;
      if (PAIR) pb2 = reinterpret_cast<const char*>(s.b2) + (int64_t)n0 * 2 + at * step_b2;
      if constexpr (ROUNDS > 1) pa += term * plane_a;
      la.template init<false>(m0, q.M, s.lda, wave, lane);
      lb.template init<PAIR>(n0, q.N, s.ldb, wave, lane);
      if (PAIR && s.ldb2 != s.ldb) {
        MmaLoader<LB, kWb, T::kBk, T::kLoadsB, T::kWaves> l2;
        l2.template init<PAIR>(n0, q.N, s.ldb2, wave, lane);
#pragma unroll
        for (int j = 0; j < T::kLoadsB; ++j)
          if (second(j)) lb.off[j] = l2.off[j];
      }
    };
    open();
    // Load n of the next stage's kLoads into the buffer (zeros past the last stage), and
    // the step to the stage after it.
    auto load = [&](lds_char* to, int n) {
      if (n < T::PA * T::kLoadsA) {
        const int p = n / T::kLoadsA, j = n % T::kLoadsA, left_k = left > 0 ? q.ka - at * T::kBk : 0;
        mma_dma(pa + p * plane_a, la.kl[j] < left_k ? la.off[j] : kOutside,
                to + p * T::kBytesA + (j * T::kWaves + wave) * 1024);
      } else {
        const int m = n - T::PA * T::kLoadsA, p = m / T::kLoadsB, j = m % T::kLoadsB;
        const int left_k = left > 0 ? q.kb - at * T::kBk : 0;
        mma_dma(second(j) ? pb2 + p * plane_b2 : pb + p * plane_b,
                lb.kl[j] < left_k ? lb.off[j] : kOutside,
                to + T::PA * T::kBytesA + p * T::kBytesB + (j * T::kWaves + wave) * 1024);
      }
    };
    auto advance = [&] {
      --left;
      if constexpr (ROUNDS > 1) {
        if (--in_round == 0 && left > 0) {  // the next round
          seg = first / q.seg_stages;
          at = first % q.seg_stages;
          in_round = stages;
          --term;
          open();
          return;
        }
      }
      if (++at == q.seg_stages && left > 0) {
        ++seg;
        at = 0;
        open();
      } else {
        pa += step_a;
        pb += step_b;
        if (PAIR) pb2 += step_b2;
      }
    };
    auto issue = [&](lds_char* to) {
#pragma unroll
      for (int n = 0; n < T::kLoads; ++n) load(to, n);
      advance();
    };

    int oa[T::kBm], ob[T::kBn];
#pragma unroll
    for (int i = 0; i < T::kBm; ++i) oa[i] = frag_at<LA, kWa>(wm + i * 32, lane);
#pragma unroll
    for (int j = 0; j < T::kBn; ++j) ob[j] = frag_at<LB, kWb>(block_col(j), lane);
#pragma unroll
    for (int i = 0; i < T::kBm; ++i)
#pragma unroll
      for (int j = 0; j < T::kBn; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    // Products of planes that are not both the first are sums of their own: they are 2^-8
    // of the others, so that these are rounded at the size of the sum once in 16 indices,
    // not six times.
    constexpr bool kTwo = T::PA + T::PB > 2;
    wg_acc small[kTwo ? T::kBm : 1][kTwo ? T::kBn : 1];
    if constexpr (kTwo) {
#pragma unroll
      for (int i = 0; i < T::kBm; ++i)
#pragma unroll
        for (int j = 0; j < T::kBn; ++j) small[i][j] = acc[i][j];
    }

    bf16x8 fa[2][T::PA][T::kBm], fb[2][T::PB][T::kBn];
    constexpr int kFrags = T::PA * T::kBm + T::PB * T::kBn;
    auto read_one = [&](lds_char* stage, int step, int n) {
      if (n < T::PB * T::kBn) {
        const int p = n / T::kBn, j = n % T::kBn;
        fb[step & 1][p][j] = frag<LB, kWb>(stage + T::PA * T::kBytesA + p * T::kBytesB, ob[j], step);
      } else {
        const int m = n - T::PB * T::kBn, p = m / T::kBm, i = m % T::kBm;
        fa[step & 1][p][i] = frag<LA, kWa>(stage + p * T::kBytesA, oa[i], step);
      }
    };
    // The products of a step, pairs of planes by size, the smallest first.  beside(n)
    // puts what else the wave issues behind product n: a product keeps the matrix unit
    // busy for 32 cycles, in which a few other instructions go out.
    constexpr int kPairs = T::PA + T::PB < 6 ? T::PA + T::PB - 1 : 6;
    constexpr int kProducts = kPairs * T::kBm * T::kBn;
    auto multiply = [&](int step, auto&& beside) {
      int n = 0;
#pragma unroll
      for (int s = kPairs > 1 ? 2 : 0; s >= 0; --s)
#pragma unroll
        for (int p = 0; p < T::PA; ++p) {
          const int r = s - p;
          if (r < 0 || r >= T::PB) continue;
#pragma unroll
          for (int i = 0; i < T::kBm; ++i)
#pragma unroll
            for (int j = 0; j < T::kBn; ++j) {
              wg_acc& c = kTwo && s > 0 ? small[kTwo ? i : 0][kTwo ? j : 0] : acc[i][j];
              c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[step & 1][r][j], fa[step & 1][p][i], c, 0, 0, 0);
              beside(n++);
              __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    // The fragments of a step go out behind the first three quarters of the products
    // before it, the loads of a stage behind all of them.
    constexpr int kEarly = kProducts >= 4 ? kProducts * 3 / 4 : kProducts;
    auto read_beside = [&](lds_char* stage, int step, int n) {
#pragma unroll
      for (int k = 0; k < kFrags; ++k)
        if (k * kEarly / kFrags == n) read_one(stage, step, k);
    };

#pragma unroll
    for (int b = 0; b < T::kBufs - 1; ++b) issue(lds + b * T::kStageB);
    between();
    mma_wait<(T::kBufs - 2) * T::kLoads>();
    mma_barrier<kShared>();
    int cur = 0;
#pragma unroll
    for (int k = 0; k < kFrags; ++k) read_one(lds, 0, k);
    issue(lds + (T::kBufs - 1) * T::kStageB);
#pragma unroll 1
    for (int s = 0; s < stages * ROUNDS; ++s) {
      lds_char* now = lds + cur;
      cur = cur == (T::kBufs - 1) * T::kStageB ? 0 : cur + T::kStageB;
#pragma unroll
      for (int t = 0; t < T::kSteps - 1; ++t) multiply(t, [&](int n) { read_beside(now, t + 1, n); });
      mma_wait<(T::kBufs - 2) * T::kLoads>();
      mma_barrier<kShared>();
      multiply(T::kSteps - 1, [&](int n) {
        read_beside(lds + cur, 0, n);
#pragma unroll
        for (int k = 0; k < T::kLoads; ++k)
          if (k * kProducts / T::kLoads == n) load(now, k);
      });
      advance();
    }
    if constexpr (kTwo) {
#pragma unroll
      for (int i = 0; i < T::kBm; ++i)
#pragma unroll
        for (int j = 0; j < T::kBn; ++j)
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[i][j][v] += small[i][j][v];
    }
    mma_wait<0>();
    mma_barrier<kShared>();
  }
};

typedef __attribute__((address_space(3))) f32x4 lds_f32x4;

// Blocks j of a wave's 32 rows to LDS, [row][column].
template <typename T>
__device__ __forceinline__ void mma_rows_out(const wg_acc (&acc)[T::kBn], lds_char* own, int lane) {
#pragma unroll
  for (int j = 0; j < T::kBn; ++j)
#pragma unroll
    for (int v = 0; v < 4; ++v)
      *(lds_f32x4*)(own + (lane & 31) * T::kPitch + (j * 32 + v * 8 + (lane >> 5) * 4) * 4) =
          f32x4{acc[j][4 * v], acc[j][4 * v + 1], acc[j][4 * v + 2], acc[j][4 * v + 3]};
}
__device__ __forceinline__ void lds_add8(float (&w)[8], lds_char* p) {
  const f32x4 lo = *(lds_f32x4*)p, hi = *(lds_f32x4*)(p + 16);
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] += lo[k], w[4 + k] += hi[k];
}
// Units to the part of C that this split forms.
template <bool PAIR>
__device__ __forceinline__ void mma_part(const MmaArgs& q, int split, int row, int col, const float (&x)[8],
                                         const float (&y)[8]) {
  auto put = [&](const float (&w)[8], float* p) {
    f32x4 lo = {w[0], w[1], w[2], w[3]}, hi = {w[4], w[5], w[6], w[7]};
    if (q.part_add) {
      lo += *reinterpret_cast<f32x4*>(p);
      hi += *reinterpret_cast<f32x4*>(p + 4);
    }
    *reinterpret_cast<f32x4*>(p) = lo;
    *reinterpret_cast<f32x4*>(p + 4) = hi;
  };
  float* p = q.part + ((int64_t)split * q.M + row) * q.ld_part + col;
  put(x, p);
  if (PAIR) put(y, p + q.ld_part / 2);
}

// The wave's results in units of 8 columns, written to part or given to e(row, its
// state, column, first values, second values of a pair).  The units of 32 rows are
// read together, so that their ways through LDS and the epilogue overlap (one unit
// after another, the logits' gradient took 17 us of a 256 x 256 tile's 45).
template <typename T, typename Core, typename E>
__device__ __forceinline__ void mma_units(const MmaArgs& q, const Core& core, lds_char* lds, lds_char* state, int m0,
                                          int n0, int split, const E& e) {
  constexpr bool PAIR = E::kPair;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int kUnits = PAIR ? T::WN / 16 : T::WN / 8;  // of a row
  if constexpr (T::kSolo > 0) {
    mma_rows_out<T>(core.acc[0], lds + wave * T::kRingB, lane);
    __syncthreads();
    const int r = threadIdx.x / kUnits, c = threadIdx.x % kUnits * 8, row = m0 + r, col = n0 + c;
    if (r >= 32 || row >= q.M || col >= q.N) return;
    float x[1][8] = {}, y[1][8] = {};
    f32x4 st[1];
#pragma unroll
    for (int w = 0; w < T::kSolo; ++w) {
      lds_add8(x[0], lds + w * T::kRingB + r * T::kPitch + c * 4);
      if (PAIR) lds_add8(y[0], lds + w * T::kRingB + r * T::kPitch + (T::WN / 2 + c) * 4);
    }
    if (E::kState) st[0] = *(lds_f32x4*)(state + r * 16);
    if (q.part) mma_part<PAIR>(q, split, row, col, x[0], y[0]);
    else e.template units<1>(row, 0, q.M, st, col, x, y);
    return;
  } else {
    lds_char* own = lds + wave * 32 * T::kPitch;
    constexpr int kTurns = 32 * kUnits / 64;
    const int col = n0 + (PAIR ? core.wn * (T::WN / 2) : core.wn * T::WN) + lane % kUnits * 8;
#pragma unroll 1
    for (int i = 0; i < T::kBm; ++i) {
#pragma unroll
      for (int b = 0; b < T::kBm; ++b)
        if (b == i) mma_rows_out<T>(core.acc[b], own, lane);
      wave_lds_order();
      float x[kTurns][8] = {}, y[kTurns][8] = {};
      f32x4 st[kTurns];
#pragma unroll
      for (int t = 0; t < kTurns; ++t) {
        const int r = t * (64 / kUnits) + lane / kUnits;
        lds_add8(x[t], own + r * T::kPitch + lane % kUnits * 32);
        if (PAIR) lds_add8(y[t], own + r * T::kPitch + T::WN * 2 + lane % kUnits * 32);
        if (E::kState) st[t] = *(lds_f32x4*)(state + (core.wm + i * 32 + r) * 16);
      }
      wave_lds_order();
      const int row = m0 + core.wm + i * 32 + lane / kUnits;
      if (q.part) {
#pragma unroll
        for (int t = 0; t < kTurns; ++t)
          if (row + t * (64 / kUnits) < q.M && col < q.N) mma_part<PAIR>(q, split, row + t * (64 / kUnits), col, x[t], y[t]);
      } else {
        e.template units<kTurns>(row, 64 / kUnits, q.M, st, col, x, y);
      }
    }
  }
}

// What epilogues have in common: units go to E's operator one by one, unless it takes
// them together.
template <typename E>
struct UnitEpilogue {
  static constexpr bool kPair = false, kWhole = false, kState = false;
  static constexpr int kTerms = 1;  // planes of A that count, where B has one
  template <int N>
  __device__ __forceinline__ void units(int row, int step, int M, const f32x4 (&st)[N], int col, float (&x)[N][8],
                                        float (&y)[N][8]) const {
    const E& e = *static_cast<const E*>(this);
    if (col >= e.N) return;
#pragma unroll
    for (int t = 0; t < N; ++t)
      if (row + t * step < M) e(row + t * step, st[t], col, x[t], y[t]);
  }
};

// C, each unit handed to the epilogue E.  ld_part holds whole units.
template <typename T, int LA, int LB, typename E>
__device__ __forceinline__ void mma_body(const MmaArgs& q, const E& e, lds_char* lds, int block, int blocks) {
  const int tiles = q.tiles_m * q.tiles_n;
  const int l = xcd_remap(block, blocks);
  const int split = l / tiles;
  int tm, tn;
  mma_tile(l % tiles, q.tiles_m, q.tiles_n, tm, tn);
  const int m0 = tm * T::TM, n0 = tn * (E::kPair ? T::TN / 2 : T::TN);
  lds_char* state = lds + T::kLdsB;
  // what the epilogue needs of each row, loaded behind the first stages
  auto states = [&] {
    if constexpr (E::kState) {
      for (int r = threadIdx.x; r < T::TM; r += T::kThr)
        *(lds_f32x4*)(state + r * 16) = m0 + r < q.M ? e.state(m0 + r) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  MmaCore<T, LA, LB, E::kPair, T::PA == 1 ? E::kTerms : 1> core;
  core.run(q, lds, m0, n0, split, states);
  if constexpr (E::kWhole && T::kSolo == 0) {
    if (!q.part) {
      e.template whole<T>(q, core, lds, m0, n0, tn);
      return;
    }
  }
  mma_units<T>(q, core, lds, state, m0, n0, split, e);
}

template <typename T, int LA, int LB, typename E>
__global__ __launch_bounds__(T::kThr, 2) void mma_kernel(MmaArgs q, E e) {
  extern __shared__ __align__(16) char lds_bytes[];
  mma_body<T, LA, LB>(q, e, (lds_char*)lds_bytes, blockIdx.x, gridDim.x);
}

// Two products that hang on nothing of each other in one launch, the first's workgroups
// before the second's (whose contraction runs along the columns of both operands).
// What it gains stands at its rule, two_plan.
template <typename T, int LB, typename E>
__global__ __launch_bounds__(T::kThr, 2) void mma_two_kernel(MmaArgs q, E e, MmaArgs q2, E e2, int first) {
  extern __shared__ __align__(16) char lds_bytes[];
  if ((int)blockIdx.x < first) mma_body<T, kLayoutRow, LB>(q, e, (lds_char*)lds_bytes, blockIdx.x, first);
  else mma_body<T, kLayoutK, kLayoutK>(q2, e2, (lds_char*)lds_bytes, blockIdx.x - first, gridDim.x - first);
}

// The epilogue of a product whose contraction was cut: parts added in order.  One
// unit of 8 columns to a thread.
template <typename E>
__device__ __forceinline__ void mma_join(const MmaArgs& q, const E& e, int block, int blocks) {
  const int units = (q.N + 7) / 8;
  const int64_t n = (int64_t)q.M * units, step = (int64_t)blocks * kThreads;
  for (int64_t i = (int64_t)block * kThreads + threadIdx.x; i < n; i += step) {
    const int row = (int)(i / units), col = (int)(i % units) * 8;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto add = [&](float (&w)[8], const float* p) {
      const f32x4 lo = *reinterpret_cast<const f32x4*>(p), hi = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] += lo[k], w[4 + k] += hi[k];
    };
#pragma unroll 4
    for (int s = 0; s < q.splits; ++s) {
      const float* p = q.part + ((int64_t)s * q.M + row) * q.ld_part + col;
      add(x, p);
      if (E::kPair) add(y, p + q.ld_part / 2);
    }
    f32x4 st = {0.f, 0.f, 0.f, 0.f};
    if constexpr (E::kState) st = e.state(row);
    e(row, st, col, x, y);
  }
}
template <typename E>
__global__ __launch_bounds__(kThreads) void mma_join_kernel(MmaArgs q, E e) {
  mma_join(q, e, blockIdx.x, gridDim.x);
}
template <typename E>
__global__ __launch_bounds__(kThreads) void mma_join_two_kernel(MmaArgs q, E e, MmaArgs q2, E e2, int first) {
  if ((int)blockIdx.x < first) mma_join(q, e, blockIdx.x, first);
  else mma_join(q2, e2, blockIdx.x - first, gridDim.x - first);
}

// x = p0 + p1 + p2 in bf16, each to nearest even: 8 bits apiece, exact from 2^-110 in
// size on.  A value whose p0 is not finite (infinities, NaN, and what rounds up to
// an infinity) is p0 alone.
__device__ __forceinline__ void planes_of(const float (&x)[8], u32x4u (&p)[3]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
    for (int t = 0; t < 3; ++t) {
      p[t][i] = pack_bf16(a, b);
      const float ha = __uint_as_float(p[t][i] << 16), hb = __uint_as_float(p[t][i] & 0xffff0000u);
      a = finite_f32(ha) ? a - ha : 0.f;
      b = finite_f32(hb) ? b - hb : 0.f;
    }
  }
}

// Matrices into bf16 planes with rows of 8 upr elements, zeros from `cols` on; one launch
// for those of a call.  Bound by memory: one read, one write (three of half the size
// for fp32).
struct PackJob {
  ActShape h;
  const void* X;
  int64_t ld;
  uint16_t* out;
  int64_t plane;
  uint32_t first;  // workgroup
};
constexpr int kMostPacks = 3;
struct PackArgs {
  PackJob job[kMostPacks];
  int jobs;
};

template <typename S>
__global__ __launch_bounds__(kThreads) void pack_kernel(PackArgs q) {
  int i = 0;
  while (i + 1 < q.jobs && blockIdx.x >= q.job[i + 1].first) ++i;
  const PackJob& j = q.job[i];
  act_units_of(j.h, blockIdx.x - j.first, [&](int64_t row, int unit, bool in) {
    if (!in) return;
    ActVec<S> x;
    x.load(static_cast<const S*>(j.X) + row * j.ld + unit * 8, j.h.cols - unit * 8);
    uint16_t* d = j.out + (row * j.h.upr + unit) * 8;
    if constexpr (sizeof(S) == 2) {
      gstore<u32x4u>(d, x.raw[0]);
    } else {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = x.at(k);
      u32x4u p[3];
      planes_of(v, p);
#pragma unroll
      for (int t = 0; t < 3; ++t) gstore<u32x4u>(d + t * j.plane, p[t]);
    }
  });
}

// C = beta C + the product, in either type.  With `second`, the product's columns from
// there on are another matrix.
struct OutEpilogue : UnitEpilogue<OutEpilogue> {
  void* C[2];
  int64_t ld[2];
  int second, Nc, N;  // where the second begins, columns of one, of the product
  int bf16;
  float beta;

  template <typename S>
  __device__ __forceinline__ void put(int64_t row, int col, float (&x)[8]) const {
    const bool b = second && col >= second;
    if (b) col -= second;
    S* p = static_cast<S*>(b ? C[1] : C[0]) + row * (b ? ld[1] : ld[0]) + col;
    ActVec<S> v;
    if (beta != 0.f) {
      v.load(p, Nc - col);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fmaf(beta, v.at(i), x[i]);
    }
    v.set(x);
    v.store(p, Nc - col);
  }
  OutEpilogue(void* c0, int64_t ld0, void* c1, int64_t ld1, int cols, int n, int n_all, int b, float be)
      : C{c0, c1}, ld{ld0, ld1}, second(cols), Nc(n), N(n_all), bf16(b), beta(be) {}
  __device__ __forceinline__ void operator()(int row, const f32x4&, int col, float (&x)[8], float (&)[8]) const {
    if (bf16) put<uint16_t>(row, col, x);
    else put<float>(row, col, x);
  }
};

// The same of several of A's terms.
struct OutTermsEpilogue : OutEpilogue {
  static constexpr int kTerms = kDxTerms;
  explicit OutTermsEpilogue(const OutEpilogue& e) : OutEpilogue(e) {}
};

// C = beta C.
template <typename S>
__global__ __launch_bounds__(kThreads) void scale_kernel(S* C, int64_t rows, int64_t cols, int64_t ld, float beta) {
  const int64_t n = rows * cols, step = (int64_t)gridDim.x * kThreads;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += step) {
    S* p = C + i / cols * ld + i % cols;
    *p = from_f32<S>(beta == 0.f ? 0.f : beta * cvt<float, S>(*p));
  }
}

}  // namespace shp
