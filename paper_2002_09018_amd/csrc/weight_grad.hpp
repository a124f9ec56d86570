// Weight gradient G = beta G + X^^T dY from an 8-bit activation checkpoint, on
// the bf16 matrix cores (v_mfma_f32_32x32x16_bf16).
//
// A code times its power of two has at most 7 significant bits, so x^ is exact
// in bf16, and so is a bf16 gradient: their products are exact, and one
// instruction per 16 tokens forms them.  An fp32 gradient is cut into three
// bf16 terms, y = p0 + p1 + p2 (truncated: 8 bits each, every difference exact;
// p0 keeps the sign of an infinity and never rounds up to one), which takes
// three.  (Below 2^-110 the last term ends below bf16's smallest step: it is cut off at
// multiples of 2^-133 then.)
//
// Both operands lie token by token, and the contraction runs over tokens.  A
// stage of kBk tokens of both is copied into LDS as it lies,
//   [operand][term][token][column],
// and the fragments, 8 tokens of one column for each lane, are read with the
// transposing read (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16 columns and
// receive 4 tokens of one column each).  A row of 16 columns is 32 bytes; the
// 32-byte pieces of a row are stored at piece ^ swz(token), which puts the four
// tokens of such a read, and its neighbour's, on different banks.
//
// While stage s is multiplied, the registers loaded during stage s - 1 are
// written as stage s + 1 (codes converted on the way) and the loads of stage
// s + 2 are issued; one barrier per stage, before the last 16 tokens of it, so
// that the first fragments of the next stage are read while those are
// multiplied.
//
// 65536 x 1024 x 4096 with bf16 gradients: 473 to 495 us (1110 to 1160 TFLOP/s; a
// library product of the same size, of bf16 operands, 674 us), where the chip
// lowers its clock.  32768 x 512 x 512: 29 us, 24 of them the products of 24 parts
// of the tokens (matrix cores and LDS busy in 23% of the cycles each; a second
// stage of loads in flight gained nothing), the rest the sum of the parts.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "act_checkpoint.hpp"
#include "split_mfma.hpp"
#include "tile_mfma.hpp"

namespace shp {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float wg_acc __attribute__((ext_vector_type(16)));

struct WgradArgs {
  const char* codes;     // rows x ldq
  const uint8_t* scales; // rows x ldq / 32
  int64_t ldq;
  const void* dY;        // rows x out
  int64_t ld_dy;
  int64_t rows;
  int cols, out;
  void* G;
  int64_t ld_g;
  float beta;
  float* part;           // partial tiles of a split launch, or NULL
  int splits;
  int64_t per_split;     // tokens of one split, a multiple of the stage
  int tiles_m, tiles_n;
};

// TM x TN tiles of G; waves of WM x WN.  Tiles of 128 x 128, which mostly have a
// compute unit to themselves, take eight waves of 64 x 32, so that a wave stages
// while another multiplies, and stages of 64 tokens: four waves of 64 x 64 (fp32:
// stages of 32) took 4096 x 256 x 512 in bf16 15.1 us (now 12.5), 405 x 3117 x 320 in
// fp32 19.7 (15.1).
template <typename S, int TM, int TN, int WM, int WN>
struct WgradTile {
  static constexpr int kTerms = sizeof(S) == 2 ? 1 : 3;
  static constexpr int kBk = sizeof(S) == 2 || TM == 128 ? 64 : 32;  // tokens of a stage
  static constexpr int kWavesN = TN / WN;
  static constexpr int kThr = (TM / WM) * (TN / WN) * 64;
  static constexpr int kRowA = 2 * TM, kRowB = 2 * TN;  // bytes of one token
  static constexpr int kPlaneA = kBk * kRowA, kPlaneB = kBk * kRowB;
  static constexpr int kUsedB = kPlaneA + kTerms * kPlaneB;
  // the buffers are one address bit apart
  static constexpr int kStageB = kUsedB <= 32768 ? 32768 : 65536;
  static constexpr int kLdsB = kStageB + kUsedB;
  static constexpr int kBm = WM / 32, kBn = WN / 32;
  static constexpr int kUa = kBk * (TM / 16) / kThr;  // 16-code units of a thread
  static constexpr int kUb = kBk * (TN / 8) / kThr;   // 8-column units of a thread
  static constexpr int kTa = kThr / (TM / 16), kTb = kThr / (TN / 8);  // tokens between a thread's units
  static constexpr int kSteps = kBk / 16;
  static_assert(kUsedB <= kStageB && kSteps % 2 == 0 && kTa % 4 == 0 && kTb % 4 == 0 && kUa * kTa == kBk &&
                    kUb * kTb == kBk, "");
};

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

__device__ __forceinline__ int wg_swz(int token) { return (token & 3) ^ ((token & 1) << 2); }

// The bf16 of two values that are exact in it (or NaN), x in the low half.
__device__ __forceinline__ uint32_t wg_pack(float x, float y) {
  return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
}

// The share of a thread in staging: kUa units of 16 codes and kUb units of 8
// gradients, each kind in one column range at tokens kTa and kTb apart.
template <typename S, int TM, int TN, int WM, int WN>
struct WgradLoader {
  using L = WgradTile<S, TM, TN, WM, WN>;
  static constexpr int kV = sizeof(S) / 2;  // 16-byte loads of a gradient unit
  const char* pa;
  const uint8_t* ps;
  const S* pb;
  int la, lb;  // LDS offsets of the first units
  u32x4 a[L::kUa];
  uint32_t sc[L::kUa];
  u32x4u b[L::kUb][kV];

  __device__ __forceinline__ void init(const WgradArgs& q, int m0, int n0, int tid) {
    const int ta = tid / (TM / 16), piece = tid % (TM / 16);
    la = ta * L::kRowA + (piece ^ wg_swz(ta)) * 32;
    const int tb = tid / (TN / 8), c8 = tid % (TN / 8);
    lb = L::kPlaneA + tb * L::kRowB + ((c8 >> 1) ^ wg_swz(tb)) * 32 + (c8 & 1) * 16;
    // codes past a row's end and gradients past `out` only feed elements of G
    // that are not stored: any column does, and a unit may run into the next row
    int m = m0 + piece * 16, n = n0 + c8 * 8;
    if (m >= q.ldq) m = 0;
    if (n >= q.out) n = 0;
    pa = q.codes + ta * q.ldq + m;
    ps = q.scales + ta * (q.ldq / kActGroup) + m / kActGroup;
    pb = static_cast<const S*>(q.dY) + tb * q.ld_dy + n;
  }

  __device__ __forceinline__ void load_a(const WgradArgs& q, int64_t k0, int u) {
    a[u] = gload<u32x4>(pa + (k0 + u * L::kTa) * q.ldq);
    sc[u] = gload<uint8_t>(ps + (k0 + u * L::kTa) * (q.ldq / kActGroup));
  }
  __device__ __forceinline__ void load_b(const WgradArgs& q, int64_t k0, int u) {
#pragma unroll
    for (int h = 0; h < kV; ++h) b[u][h] = gload<u32x4u>(pb + (k0 + u * L::kTb) * q.ld_dy + 4 * h);
  }

  __device__ __forceinline__ void store_a(lds_char* stage, int u) {
    const float s = act_scale(sc[u]);
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t x = a[u][i / 2] >> (16 * (i & 1));
      w[i] = wg_pack((float)(int8_t)(x & 0xff) * s, (float)(int8_t)((x >> 8) & 0xff) * s);
    }
    lds_u32x4* d = (lds_u32x4*)(stage + la + u * L::kTa * L::kRowA);
    d[0] = u32x4{w[0], w[1], w[2], w[3]};
    d[1] = u32x4{w[4], w[5], w[6], w[7]};
  }

  // One unit of gradients, in its terms.
  static __device__ __forceinline__ void put_b(lds_char* d, const u32x4u (&v)[kV]) {
    if constexpr (sizeof(S) == 2) {
      *(lds_u32x4*)d = u32x4{v[0][0], v[0][1], v[0][2], v[0][3]};
    } else {
      uint32_t p[3][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x[3][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          // a NaN is made quiet, so that its upper half is one too
          const float y = __builtin_canonicalizef(__uint_as_float(v[i / 2][2 * (i % 2) + h]));
          x[0][h] = y;
          // infinities and NaN are the first term alone
          const float r = finite_f32(y) ? y - __uint_as_float(__float_as_uint(y) & 0xffff0000u) : 0.f;
          x[1][h] = r;
          x[2][h] = r - __uint_as_float(__float_as_uint(r) & 0xffff0000u);
        }
#pragma unroll
        for (int t = 0; t < 3; ++t) p[t][i] = wg_pack(x[t][0], x[t][1]);
      }
#pragma unroll
      for (int t = 0; t < 3; ++t) *(lds_u32x4*)(d + t * L::kPlaneB) = u32x4{p[t][0], p[t][1], p[t][2], p[t][3]};
    }
  }
  __device__ __forceinline__ void store_b(lds_char* stage, int u) {
    put_b(stage + lb + u * L::kTb * L::kRowB, b[u]);
  }

  // Part g of `parts` of the stage in the registers: to LDS, and (LOAD) the
  // same units of the stage at token k0 into their place.
  template <bool LOAD>
  __device__ __forceinline__ void pass_on(const WgradArgs& q, lds_char* stage, int64_t k0, int g, int parts) {
    constexpr int kU = L::kUa + L::kUb;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      if (u * parts / kU != g) continue;
      if (u < L::kUa) {
        store_a(stage, u);
        if (LOAD) load_a(q, k0, u);
      } else {
        store_b(stage, u - L::kUa);
        if (LOAD) load_b(q, k0, u - L::kUa);
      }
    }
  }

  // A stage that reaches past the split's or the tensor's end, straight to LDS:
  // tokens at or past k_end are zeros, columns at or past `out` zeros too.
  __device__ __forceinline__ void tail(const WgradArgs& q, lds_char* stage, int64_t k0, int64_t k_end, int n0,
                                       int tid) {
    const int left = (int)(k_end - k0), ta = tid / (TM / 16), tb = tid / (TN / 8), n = n0 + tid % (TN / 8) * 8;
#pragma unroll
    for (int u = 0; u < L::kUa; ++u) {
      a[u] = u32x4{0, 0, 0, 0};
      sc[u] = 0;
      if (ta + u * L::kTa < left) load_a(q, k0, u);
      store_a(stage, u);
    }
#pragma unroll 1
    for (int u = 0; u < L::kUb; ++u) {
      const int have = tb + u * L::kTb < left ? q.out - n : 0;
      const S* p = pb + (k0 + u * L::kTb) * q.ld_dy;
      u32x4u v[kV];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(S) == 4) {
          v[i / 4][i % 4] = i < have ? gload<uint32_t>(p + i) : 0u;
        } else {
          const uint32_t w = i < have ? (uint32_t)gload<uint16_t>(p + i) : 0u;
          v[0][i / 2] = i & 1 ? v[0][i / 2] | w << 16 : w;
        }
      }
      put_b(stage + lb + u * L::kTb * L::kRowB, v);
    }
  }
};

// The 8 tokens of a lane: two transposing reads, 4 rows apart.
template <int ROW_B>
__device__ __forceinline__ bf16x8 wg_frag(lds_char* p) {
  const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p);
  const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p + 4 * ROW_B));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Four rows of one column of G, rounded once.
template <typename SG>
__device__ __forceinline__ void wg_store4(const WgradArgs& q, int m, int n, f32x4 v) {
  if (n >= q.out) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (m + i >= q.cols) continue;
    SG* g = static_cast<SG*>(q.G) + (int64_t)(m + i) * q.ld_g + n;
    const float x = q.beta == 0.f ? v[i] : fmaf(q.beta, cvt<float, SG>(*g), v[i]);
    *g = from_f32<SG>(x);
  }
}

template <typename S, typename SG, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__((WgradTile<S, TM, TN, WM, WN>::kThr), 2) void weight_grad_kernel(WgradArgs q) {
  using L = WgradTile<S, TM, TN, WM, WN>;
  extern __shared__ __align__(16) char lds_bytes[];
  lds_char* lds = (lds_char*)lds_bytes;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tiles = q.tiles_m * q.tiles_n;
  const int l = xcd_remap(blockIdx.x, gridDim.x);
  const int split = l / tiles, t = l % tiles;
  const int tm = t % q.tiles_m, tn = t / q.tiles_m;
  const int m0 = tm * TM, n0 = tn * TN;
  const int64_t kb = split * q.per_split, ke = min(q.rows, kb + q.per_split);
  // Stages from the front that lie whole in the split and whose units of
  // gradients are all readable: where a row's last unit runs past `out`, it
  // must not be the tensor's last row (last 8 rows when rows are closer than
  // a unit).  The one or two others go first.
  const int64_t safe = q.out % 8 == 0 ? q.rows : q.rows - (q.ld_dy >= 8 ? 1 : 8);
  const int stages = (int)((ke - kb + L::kBk - 1) / L::kBk);
  const int plain = max(0, (int)((min(ke, safe) - kb) / L::kBk));

  WgradLoader<S, TM, TN, WM, WN> ld;
  ld.init(q, m0, n0, tid);

  // fragment offsets: 16-lane group g reads columns 16 (g & 1).., tokens 8 (g >> 1)..
  const int wm = wave / L::kWavesN * WM, wn = wave % L::kWavesN * WN;
  const int token = (lane >> 5) * 8 + ((lane >> 2) & 3), side = (lane >> 4) & 1;
  int oa[L::kBm], ob[L::kBn];
#pragma unroll
  for (int i = 0; i < L::kBm; ++i)
    oa[i] = token * L::kRowA + ((wm / 16 + 2 * i + side) ^ wg_swz(token)) * 32 + (lane & 3) * 8;
#pragma unroll
  for (int j = 0; j < L::kBn; ++j)
    ob[j] = L::kPlaneA + token * L::kRowB + ((wn / 16 + 2 * j + side) ^ wg_swz(token)) * 32 + (lane & 3) * 8;

  wg_acc acc[L::kBm][L::kBn];
#pragma unroll
  for (int i = 0; i < L::kBm; ++i)
#pragma unroll
    for (int j = 0; j < L::kBn; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

  bf16x8 fa[L::kBm], fb[2][L::kTerms][L::kBn];
  auto read_a = [&](lds_char* stage, int step, int i) { fa[i] = wg_frag<L::kRowA>(stage + oa[i] + step * 16 * L::kRowA); };
  auto read_b = [&](lds_char* stage, int step, int set) {
#pragma unroll
    for (int p = 0; p < L::kTerms; ++p)
#pragma unroll
      for (int j = 0; j < L::kBn; ++j)
        fb[set][p][j] = wg_frag<L::kRowB>(stage + ob[j] + p * L::kPlaneB + step * 16 * L::kRowB);
  };
  auto read_first = [&](lds_char* stage) {
    read_b(stage, 0, 0);
#pragma unroll
    for (int i = 0; i < L::kBm; ++i) read_a(stage, 0, i);
  };

  // The products of one staged stage.  STORE: the stage in the registers is
  // written to the other buffer beside the products of all steps but the last,
  // and the last step reads the first fragments of it; LOAD: the registers are
  // filled with the stage at token k0.  A row block's fragment is read again as
  // soon as its products are issued; the scheduler may move the conversion
  // between products, but not the reads (left free it reads a whole stage's
  // fragments first and spills).
  auto stage = [&](lds_char* cur, int64_t k0, auto store, auto load) {
    lds_char* nxt = lds + ((int)(cur - lds) ^ L::kStageB);
#pragma unroll
    for (int step = 0; step < L::kSteps; ++step) {
      const bool last = step == L::kSteps - 1;
      if (last && decltype(store)::value) __syncthreads();
      if (!last) read_b(cur, step + 1, (step + 1) & 1);
      else if (decltype(store)::value) read_b(nxt, 0, 0);
#pragma unroll
      for (int i = 0; i < L::kBm; ++i) {
#pragma unroll
        for (int p = L::kTerms - 1; p >= 0; --p)  // the smallest terms first
#pragma unroll
          for (int j = 0; j < L::kBn; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[step & 1][p][j], acc[i][j], 0, 0, 0);
        if (!last) read_a(cur, step + 1, i);
        else if (decltype(store)::value) read_a(nxt, 0, i);
        if (!last && decltype(store)::value)
          ld.template pass_on<decltype(load)::value>(q, nxt, k0, step * L::kBm + i, (L::kSteps - 1) * L::kBm);
        __builtin_amdgcn_sched_barrier(0x2);
      }
    }
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};

  lds_char* cur = lds;
  auto flip = [&] { cur = lds + ((int)(cur - lds) ^ L::kStageB); };
  int next = 0;  // the plain stage that goes to the registers next
  for (int s = stages - 1; s >= plain; --s) {
    if (s < stages - 1) {
      __syncthreads();
      read_first(cur);
      stage(cur, 0, no, no);
      flip();
    }
    ld.tail(q, cur, kb + (int64_t)s * L::kBk, ke, n0, tid);
  }
  auto fill = [&](int64_t k0) {
#pragma unroll
    for (int u = 0; u < L::kUa; ++u) ld.load_a(q, k0, u);
#pragma unroll
    for (int u = 0; u < L::kUb; ++u) ld.load_b(q, k0, u);
  };
  if (stages == plain) {
    fill(kb);
#pragma unroll
    for (int u = 0; u < L::kUa; ++u) ld.store_a(cur, u);
#pragma unroll
    for (int u = 0; u < L::kUb; ++u) ld.store_b(cur, u);
    next = 1;
  }
  if (next < plain) fill(kb + (int64_t)next * L::kBk);
  __syncthreads();
  read_first(cur);
  for (; next + 1 < plain; ++next) {
    stage(cur, kb + (int64_t)(next + 1) * L::kBk, yes, yes);
    flip();
  }
  if (next < plain) {
    stage(cur, 0, yes, no);
    flip();
  }
  stage(cur, 0, no, no);

  if (q.part) {
    // partial tiles in accumulator order: 16 bytes a lane
    f32x4* d = reinterpret_cast<f32x4*>(q.part) + (((int64_t)split * tiles + t) * (L::kThr / 64) + wave) *
                                                      (L::kBm * L::kBn * 4 * 64) + lane;
#pragma unroll
    for (int i = 0; i < L::kBm; ++i)
#pragma unroll
      for (int j = 0; j < L::kBn; ++j)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          d[((i * L::kBn + j) * 4 + v) * 64] =
              f32x4{acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]};
    return;
  }
#pragma unroll
  for (int i = 0; i < L::kBm; ++i)
#pragma unroll
    for (int j = 0; j < L::kBn; ++j)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        wg_store4<SG>(q, m0 + wm + i * 32 + v * 8 + (lane >> 5) * 4, n0 + wn + j * 32 + (lane & 31),
                      f32x4{acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]});
}

// G from the partial tiles, added in split order: one wave per 4 accumulator
// elements of a 32 x 32 block.
template <typename SG, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(kThreads) void weight_grad_sum_kernel(WgradArgs q) {
  constexpr int kPerTile = (TM / 32) * (TN / 32) * 4;  // 64-lane pieces of a tile
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int tiles = q.tiles_m * q.tiles_n;
  if (w >= (int64_t)tiles * kPerTile) return;
  const int t = (int)(w / kPerTile), piece = (int)(w % kPerTile);
  const int v = piece & 3, blk = piece >> 2;
  constexpr int kBm = WM / 32, kBn = WN / 32;
  const int wave = blk / (kBm * kBn), i = blk % (kBm * kBn) / kBn, j = blk % kBn;
  const int m = t % q.tiles_m * TM + wave / (TN / WN) * WM + i * 32 + v * 8 + (lane >> 5) * 4;
  const int n = t / q.tiles_m * TN + wave % (TN / WN) * WN + j * 32 + (lane & 31);
  const f32x4* d = reinterpret_cast<const f32x4*>(q.part) + w * 64 + lane;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < q.splits; ++s) sum += d[(int64_t)s * tiles * kPerTile * 64];
  wg_store4<SG>(q, m, n, sum);
}

// No tokens: G = beta G.
template <typename SG>
__global__ __launch_bounds__(kThreads) void weight_grad_scale_kernel(WgradArgs q) {
  const int64_t n = (int64_t)q.cols * q.out, step = (int64_t)gridDim.x * kThreads;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += step) {
    SG* g = static_cast<SG*>(q.G) + i / q.out * q.ld_g + i % q.out;
    *g = from_f32<SG>(q.beta == 0.f ? 0.f : q.beta * cvt<float, SG>(*g));
  }
}

}  // namespace shp
