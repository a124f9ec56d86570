// Host check of the dispatch rules in layer_plans.hpp.  Reads lines
//   logprobs ROWS VOCAB K DTYPE | grad ROWS VOCAB DTYPE | wgrad ROWS COLS OUT DTYPE
// and prints what each size takes; every plan, and those of a sweep of sizes,
// must cover its rows, entries and tokens once.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "layer_plans.hpp"

using namespace shp;
typedef long long ll;

static void require(bool ok, const char* what, ll a, ll b, ll c, ll d) {
  if (ok) return;
  printf("%s: %lld %lld %lld %lld\n", what, a, b, c, d);
  exit(1);
}

static LogprobPlan logprobs(ll rows, ll vocab, int k, int dtype) {
  const LogprobPlan p = logprob_plan(rows, vocab, k, dtype);
  const ll block = kLogitBlockB / (dtype == SHAMPOO_BF16 ? 2 : 4);
  require(p.waves == 1 || p.waves == 2 || p.waves == 4 || p.waves == 8, "waves", rows, vocab, k, dtype);
  require(p.parts >= 1 && p.parts <= 64 && (p.parts == 1 || (rows < 256 && p.waves == 4)), "parts", rows, vocab, k, dtype);
  require((ll)(p.parts - 1) * p.per_part < vocab && (ll)p.parts * p.per_part >= vocab, "entries", rows, vocab, k, dtype);
  require(p.parts == 1 || p.per_part % (p.waves * block) == 0, "blocks", rows, vocab, k, dtype);
  require(p.ws == (p.parts == 1 ? 0 : (size_t)(rows * p.parts * logprob_record(k)) * 4), "workspace", rows, vocab, k, dtype);
  return p;
}

static LossGradPlan grad(ll rows, ll vocab, int dtype) {
  const LossGradPlan p = loss_grad_plan(rows, vocab, dtype);
  const ll block = kLogitBlockB / (dtype == SHAMPOO_BF16 ? 2 : 4);
  require(p.per >= 1 && p.per <= 2 && (ll)p.segs * p.per * block >= vocab + 7, "gradient", rows, vocab, dtype, 0);
  return p;
}

static WgradPlan wgrad(ll rows, ll cols, ll out, int dtype) {
  const WgradPlan p = wgrad_plan(rows, cols, out, dtype);
  require((p.tile_m == 256 && p.tile_n == 256) || (p.tile_m == 128 && p.tile_n == 128) ||
              (p.tile_m == 128 && p.tile_n == 256 && dtype == SHAMPOO_BF16), "tile", rows, cols, out, dtype);
  require(p.tiles_m * p.tile_m >= cols && (p.tiles_m - 1) * p.tile_m < cols && p.tiles_n * p.tile_n >= out &&
              (p.tiles_n - 1) * p.tile_n < out, "tiles", rows, cols, out, dtype);
  require(p.per_split % 32 == 0 && p.splits * p.per_split >= rows && (rows == 0 || (p.splits - 1) * p.per_split < rows),
          "tokens", rows, cols, out, dtype);
  require(p.ws == (p.splits == 1 ? 0 : (size_t)(p.splits * p.tiles_m * p.tiles_n) * p.tile_m * p.tile_n * 4), "workspace",
          rows, cols, out, dtype);
  return p;
}

// apart() against the bytes themselves: exact for one row, or rows of one pitch
// away from each other's ends, and never true for buffers that share a byte.
static void spans() {
  for (int rows_a = 1; rows_a <= 3; ++rows_a)
    for (int rows_b = 1; rows_b <= 3; ++rows_b)
      for (int a = 1; a <= 4; ++a)
        for (int b = 1; b <= 4; ++b)
          for (int pa = a; pa <= 9; ++pa)
            for (int pb = b; pb <= 9; ++pb)
              for (int off = -40; off <= 40; ++off) {
                const Span x = {1000, rows_a, a, pa}, y = {(uintptr_t)(1000 + off), rows_b, b, pb};
                bool hit = false, inside = false;
                for (int i = 0; i < rows_a; ++i)
                  for (int j = 0; j < rows_b; ++j) {
                    const int s = i * pa, t = off + j * pb;
                    hit |= s < t + b && t < s + a;
                    inside |= i > 0 && (s - pa + a <= t && t + b <= s);  // y's row between two of x's
                  }
                require(!(hit && apart(x, y)) && apart(x, y) == apart(y, x), "spans", rows_a, rows_b, off, pa * 100 + pb);
                if (!hit && inside && (rows_b == 1 || pa == pb)) require(apart(x, y), "gap", rows_a, rows_b, off, pa * 100 + pb);
              }
  require(apart(span(nullptr, 8), span(nullptr, 8)) && apart({8, 0, 4, 4}, {8, 1, 4, 4}), "empty", 0, 0, 0, 0);
}

int main() {
  spans();
  char kind[16];
  ll a, b, c;
  int d;
  while (scanf("%15s", kind) == 1) {
    if (!strcmp(kind, "logprobs") && scanf("%lld %lld %lld %d", &a, &b, &c, &d) == 4) {
      const LogprobPlan p = logprobs(a, b, (int)c, d);
      printf("%d %d %d\n", p.waves, p.parts, p.per_part);
    } else if (!strcmp(kind, "grad") && scanf("%lld %lld %d", &a, &b, &d) == 3) {
      const LossGradPlan p = grad(a, b, d);
      printf("%d %d\n", p.per, p.segs);
    } else if (!strcmp(kind, "wgrad") && scanf("%lld %lld %lld %d", &a, &b, &c, &d) == 4) {
      const WgradPlan p = wgrad(a, b, c, d);
      printf("%d %d %d\n", p.tile_m, p.tile_n, p.splits);
    } else {
      return 1;
    }
  }
  unsigned seed = 1;
  auto size = [&](int bits) {  // about as many of each length in bits
    seed = seed * 1664525u + 1013904223u;
    const int n = (int)(seed >> 8) % (bits + 1);
    seed = seed * 1664525u + 1013904223u;
    return (ll)1 << n | ((ll)(seed >> 2) & (((ll)1 << n) - 1));
  };
  for (int i = 0; i < 200000; ++i) {
    const int dtype = i & 1 ? SHAMPOO_BF16 : SHAMPOO_F32;
    const ll rows = size(29), vocab = size(29), k = size(6) - 1, cols = size(19), out = size(19);
    logprobs(rows, vocab, (int)(k > 64 ? 64 : k), dtype);
    grad(rows, vocab, dtype);
    wgrad(rows, cols, out, dtype);
  }
  printf("ok\n");
}
