// Host check of the rules in stream_plans.hpp.  Reads lines
//   vocab ROWS DIM VOCAB DTYPE PACK | vgrad ROWS DIM VOCAB DTYPE GDTYPE PACK
//   ffn ROWS DIM WIDTH DTYPE PACK | fgrad ROWS DIM WIDTH DTYPE GDTYPE PACK
// and prints the shape and the parts of each product (pieces first for vocab and
// vgrad; of a gradient last whether dX and the weights' gradient may share a launch,
// and their parts there); every plan, and those of a sweep of sizes, must cover its
// product once, and its buffers must lie apart.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cmath>
#include <cstring>
#include <random>

#include "stream_plans.hpp"

using namespace shp;
typedef long long ll;

static void require(bool ok, const char* what, ll a, ll b, ll c, ll d) {
  if (ok) return;
  printf("%s: %lld %lld %lld %lld\n", what, a, b, c, d);
  exit(1);
}

static void product(const MmaPlan& p, ll M, ll N, ll K, const MmaCost* cost, int segs, bool pair, int least,
                    bool along_rows = false) {
  require(p.shape == kShapeDirect ? M <= 64 : p.shape >= least && p.shape <= kShapeBig, "shape", M, N, K, p.shape);
  const MmaCost t = p.shape == kShapeDirect ? few_tile(cost == kCost1 ? 1 : 3, along_rows) : cost[p.shape];
  const ll n = pair ? t.n / 2 : t.n;
  require((p.tiles_m - 1) * t.m < M && M <= p.tiles_m * t.m && (p.tiles_n - 1) * n < N && N <= p.tiles_n * n, "tiles", M,
          N, K, p.shape);
  require((p.seg_stages - 1) * t.bk < K && K <= p.seg_stages * t.bk, "stages", M, N, K, p.shape);
  const ll stages = p.seg_stages * segs;
  require((ll)(p.splits - 1) * p.per_split < stages && stages <= (ll)p.splits * p.per_split, "parts", M, N, K, p.splits);
  require(p.ld_part % 8 == 0 && p.ld_part >= (pair ? 2 : 1) * N, "rows of parts", M, N, K, p.ld_part);
  require(p.splits == 1 || p.part > 0, "room of parts", M, N, K, p.splits);
  require(p.part == 0 || p.part == (size_t)(p.splits * M * p.ld_part) * 4, "bytes of parts", M, N, K, p.splits);
}

// Two products of one launch: the same tiles and planes, and numbers that a launch holds.
static void two(const MmaPlan& x, ll Mx, ll Nx, ll Kx, int segs, const MmaPlan& w, ll Mw, ll Nw, ll Kw, int planes,
                int dtype) {
  require(planes == (dtype == SHAMPOO_F32 ? 3 : 1), "planes of two products", Mx, Nx, Kx, planes);
  require(x.shape == kShapeMid && w.shape == kShapeMid, "tiles of two products", Mx, Nx, Kx, w.shape);
  product(x, Mx, Nx, Kx, mma_cost(planes), segs, false, kShapeMid);
  product(w, Mw, Nw, Kw, weight_cost(planes, planes), 1, false, kShapeMid);
  require(fits(x) && fits(w), "launch of two products", Mx, Nx, Kx, x.splits);
}

// Buffers in the order they were taken: each begins at or past the end of the one before.
struct Layout {
  size_t end = 0;
  void put(size_t at, size_t bytes, const char* what) {
    if (bytes == 0) return;
    require(at >= end && at % 256 == 0, what, at, end, bytes, 0);
    end = at + bytes;
  }
};

// The room that a call asks for holds its plan, and hangs on sizes alone.
static void rooms(size_t need, size_t bytes, size_t whole, bool alike, ll a, ll b, ll c) {
  require(bytes <= whole, "room", a, b, c, bytes);
  if (alike) require(need == whole, "room of every call", a, b, c, need);
}

static VocabPlan vocab(ll rows, ll dim, ll v, int dtype, bool px, bool pw) {
  const VocabPlan p = vocab_plan(rows, dim, v, dtype, px, pw);
  const MmaCost* cost = mma_cost(dtype == SHAMPOO_F32 ? 3 : 1);
  const ll last = v - (p.pieces - 1) * p.piece;
  require(p.pieces >= 1 && last >= 1 && last <= p.piece && ((pw && !p.direct) || p.pieces == 1), "pieces", rows, dim, v,
          p.piece);
  require(p.direct == (pw && few_direct(rows, v * dim, dtype, true, false)) && p.direct == (p.mma[0].shape == kShapeDirect), "direct", rows, dim, v,
          p.direct);
  product(p.mma[0], rows, p.piece, dim, cost, 1, false, kShapeFew, true);
  product(p.mma[1], rows, last, dim, cost, 1, false, kShapeFew, true);
  require(p.entries == (p.pieces - 1) * vocab_entries(p.mma[0], p.piece) + vocab_entries(p.mma[1], last), "entries",
          rows, dim, v, p.entries);
  Layout l;
  l.put(p.at_x, px ? p.x.bytes : 0, "x");
  l.put(p.at_w, pw && !p.direct ? p.w.bytes : 0, "w");
  l.put(p.at_stat, (size_t)(rows * p.entries) * 8, "statistics");
  l.put(p.at_target, (size_t)rows * 4, "targets");
  l.put(p.at_part, std::max(p.mma[0].part, p.mma[1].part), "parts");
  const size_t whole = std::max(vocab_plan(rows, dim, v, dtype, true, true).bytes,
                                dtype == SHAMPOO_F32 ? 0 : vocab_plan(rows, dim, v, dtype, true, false).bytes);
  if (dtype == SHAMPOO_BF16 || (px && pw)) rooms(p.need, p.bytes, whole, vocab_alike(rows, dim, v, dtype), rows, dim, v);
  require(l.end <= p.bytes, "bytes", rows, dim, v, p.bytes);
  return p;
}

static VocabGradPlan vgrad(ll rows, ll dim, ll v, int dtype, int g, bool px, bool pw) {
  const VocabGradPlan p = vocab_grad_plan(rows, dim, v, dtype, g, px, pw);
  const MmaCost* cost = mma_cost(dtype == SHAMPOO_F32 ? 3 : 1);
  const ll last = v - (p.pieces - 1) * p.piece;
  require(p.pieces >= 1 && last >= 1 && last <= p.piece && p.ld_dz >= p.piece && p.ld_dz % 64 == 0, "pieces", rows, dim,
          v, p.piece);
  require(p.planes == (dtype == SHAMPOO_F32 || g == SHAMPOO_F32 ? 3 : 1), "terms", rows, dim, v, p.planes);
  for (int i = 0; i < 2; ++i) {
    const ll n = i ? last : p.piece;
    product(p.z[i], rows, n, dim, cost, 1, false, kShapeSolo, true);
    product(p.dx[i], rows, dim, n, cost, 1, false, kShapeSolo);
    product(p.dw[i], n, dim, rows, weight_cost(dtype == SHAMPOO_F32 ? 3 : 1, p.planes), 1, false, kShapeFew);
  }
  // the last piece adds to parts that the first ones wrote
  require(p.dx[1].splits <= p.dx[0].splits && p.dx[1].ld_part == p.dx[0].ld_part && !p.dx[1].part == !p.dx[0].part &&
              (p.pieces == 1 || p.dx[0].part > 0), "parts of dX", rows, dim, v, p.dx[1].splits);
  Layout l;
  l.put(p.at_x, px ? p.x.bytes : 0, "x");
  l.put(p.at_w, pw && !p.direct ? p.w.bytes : 0, "w");
  l.put(p.at_dz, (size_t)(rows * p.ld_dz * p.planes) * 2, "dz");
  l.put(p.at_dx, std::max(p.dx[0].part, p.two_dx.part), "dX");
  l.put(p.at_part, std::max({p.z[0].part, p.z[1].part, p.dw[0].part, p.dw[1].part, p.two_dw.part}), "parts");
  const size_t whole = std::max(vocab_grad_plan(rows, dim, v, dtype, g, true, true).bytes,
                                dtype == SHAMPOO_F32 ? 0 : vocab_grad_plan(rows, dim, v, dtype, g, true, false).bytes);
  if (dtype == SHAMPOO_BF16 || (px && pw))
    rooms(p.need, p.bytes, whole, vocab_grad_alike(rows, dim, v, dtype, p.planes), rows, dim, v);
  if (p.two) {
    require(p.pieces == 1, "one launch of two products", rows, dim, v, p.pieces);
    two(p.two_dx, rows, dim, v, 1, p.two_dw, v, dim, rows, p.planes, dtype);
  }
  require(l.end <= p.bytes, "bytes", rows, dim, v, p.bytes);
  return p;
}

static FfnPlan ffn(ll rows, ll dim, ll width, int dtype, bool pack) {
  const FfnPlan p = ffn_plan(rows, dim, width, dtype, true, pack, pack);
  require(p.direct == ((pack || dtype == SHAMPOO_F32) && few_direct(rows, 2 * dim * width, dtype, false, false)), "direct", rows, dim, width, p.direct);
  product(p.mma, rows, width, dim, mma_cost(dtype == SHAMPOO_F32 ? 3 : 1), 1, true, kShapeSolo);
  Layout l;
  l.put(p.at_x, p.x.bytes, "x");
  l.put(p.at_wg, pack && !p.direct ? p.wg.bytes : 0, "wg");
  l.put(p.at_wu, pack && !p.direct ? p.wu.bytes : 0, "wu");
  l.put(p.at_part, p.mma.part, "parts");
  require(l.end <= p.bytes, "bytes", rows, dim, width, p.bytes);
  const size_t whole = std::max(ffn_plan(rows, dim, width, dtype, true, true, true).bytes,
                                dtype == SHAMPOO_F32 ? 0 : ffn_plan(rows, dim, width, dtype, true, false, false).bytes);
  for (int i = 0; i < 8; ++i) {
    const FfnPlan o = ffn_plan(rows, dim, width, dtype, i & 1, i & 2, i & 4);
    rooms(o.need, o.bytes, whole, ffn_alike(rows, dim, width, dtype, false), rows, dim, width);
  }
  return p;
}

static FfnGradPlan fgrad(ll rows, ll dim, ll width, int dtype, int g, bool pack) {
  const FfnGradPlan p = ffn_grad_plan(rows, dim, width, dtype, g, true, pack, pack);
  require(p.direct == ((pack || dtype == SHAMPOO_F32) && few_direct(rows, 2 * dim * width, dtype, true, true)) &&
              !(p.direct && p.two), "direct", rows, dim, width, p.direct);
  const MmaCost* cost = mma_cost(dtype == SHAMPOO_F32 ? 3 : 1);
  product(p.gu, rows, width, dim, cost, 1, true, kShapeSolo);
  product(p.dx, rows, dim, width, cost, 2, false, kShapeSolo, true);
  product(p.dw, dim, 2 * p.ld_d, rows, weight_cost(dtype == SHAMPOO_F32 ? 3 : 1, p.planes), 1, false, kShapeFew);
  Layout l;
  l.put(p.at_x, p.x.bytes, "x");
  l.put(p.at_wg, pack && !p.direct ? p.wg.bytes : 0, "wg");
  l.put(p.at_wu, pack && !p.direct ? p.wu.bytes : 0, "wu");
  l.put(p.at_d, (size_t)(rows * 2 * p.ld_d * p.planes) * 2, "d");
  l.put(p.at_part, std::max({p.gu.part, p.dx.part, p.dw.part, p.two_dw.part}), "parts");
  l.put(p.at_dx, p.two_dx.part, "parts of dX");
  const size_t whole =
      std::max(ffn_grad_plan(rows, dim, width, dtype, g, true, true, true).bytes,
               dtype == SHAMPOO_F32 ? 0 : ffn_grad_plan(rows, dim, width, dtype, g, true, false, false).bytes);
  for (int i = 0; i < 8; ++i) {
    const FfnGradPlan o = ffn_grad_plan(rows, dim, width, dtype, g, i & 1, i & 2, i & 4);
    rooms(o.need, o.bytes, whole, ffn_alike(rows, dim, width, dtype, true), rows, dim, width);
  }
  if (p.two) two(p.two_dx, rows, dim, width, 2, p.two_dw, dim, 2 * p.ld_d, rows, p.planes, dtype);
  require(l.end <= p.bytes && p.ld_d >= width && p.ld_d % 64 == 0, "bytes", rows, dim, width, p.bytes);
  return p;
}

static void print(const MmaPlan& p) { printf(" %d %d", p.shape, p.splits); }

int main() {
  char kind[16];
  ll a, b, c;
  int d, e, f;
  char line[256];
  while (fgets(line, sizeof line, stdin)) {
    if (sscanf(line, "vocab %lld %lld %lld %d %d", &a, &b, &c, &d, &e) == 5) {
      const VocabPlan p = vocab(a, b, c, d, e, e);
      printf("%lld", (ll)p.pieces);
      print(p.mma[0]);
      print(p.mma[1]);
    } else if (sscanf(line, "vgrad %lld %lld %lld %d %d %d", &a, &b, &c, &d, &e, &f) == 6) {
      const VocabGradPlan p = vgrad(a, b, c, d, e, f, f);
      printf("%lld", (ll)p.pieces);
      for (int i = 0; i < 2; ++i) print(p.z[i]), print(p.dx[i]), print(p.dw[i]);
      printf(" %d %d %d", p.two, p.two_dx.splits, p.two_dw.splits);
    } else if (sscanf(line, "ffn %lld %lld %lld %d %d", &a, &b, &c, &d, &e) == 5) {
      print(ffn(a, b, c, d, e).mma);
    } else if (sscanf(line, "fgrad %lld %lld %lld %d %d %d", &a, &b, &c, &d, &e, &f) == 6) {
      const FfnGradPlan p = fgrad(a, b, c, d, e, f);
      print(p.gu), print(p.dx), print(p.dw);
      printf(" %d %d %d", p.two, p.two_dx.splits, p.two_dw.splits);
    } else {
      sscanf(line, "%15s", kind);
      printf("unknown %s", kind);
      return 1;
    }
    printf("\n");
  }
  std::mt19937_64 r(1);
  auto size = [&](double hi) { return (ll)std::exp(std::uniform_real_distribution<>(0, std::log(hi))(r)); };
  for (int i = 0; i < 20000; ++i) {
    const ll rows = size(1 << 20), dim = size(1 << 14), v = size(1 << 20);
    const int dt = r() & 1, g = r() & 1;
    vocab(rows, dim, v, dt, r() & 1, dt == SHAMPOO_F32 || r() & 1);
    vgrad(rows, dim, v, dt, g, r() & 1, dt == SHAMPOO_F32 || r() & 1);
    ffn(rows, dim, size(1 << 16), dt, dt == SHAMPOO_F32 || r() & 1);
    fgrad(rows, dim, size(1 << 16), dt, g, dt == SHAMPOO_F32 || r() & 1);
  }
  // the largest: past what a launch holds, but no number overflows
  for (int dt = 0; dt < 2; ++dt) {
    require(!fits(vocab(INT32_MAX, 1 << 20, 1 << 30, dt, true, true).mma[0]), "largest", 0, 0, 0, dt);
    require(!fits(vgrad(INT32_MAX, 1 << 20, 1 << 30, dt, 0, true, true).z[0]), "largest", 0, 0, 0, dt);
    require(!fits(ffn(INT32_MAX, 1 << 20, 1 << 19, dt, true).mma), "largest", 0, 0, 0, dt);
    require(!fits(fgrad(INT32_MAX, 1 << 20, 1 << 19, dt, 0, true).dx), "largest", 0, 0, 0, dt);
  }
  puts("ok");
}
