// Host check of what a call of the loss refuses (stream_plans.hpp).  Reads lines
//   ROWS DIM VOCAB DTYPE PACK
// and prints whether its products fit launches, its pieces, and the most parts of one; the
// statistics of logits that were formed in parts must fit a launch for every size.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "stream_plans.hpp"

using namespace shp;
typedef long long ll;

static VocabPlan plan(ll rows, ll dim, ll vocab, int dtype, bool pack) {
  const VocabPlan p = vocab_plan(rows, dim, vocab, dtype, dtype == SHAMPOO_F32 || pack, dtype == SHAMPOO_F32 || pack);
  const ll last = vocab - (p.pieces - 1) * p.piece;
  for (int i = 0; i < 2; ++i)
    if (p.mma[i].part && stat_groups(rows, i ? last : p.piece) >= kMostTiles) {
      printf("statistics: %lld %lld %lld %d\n", rows, dim, vocab, dtype);
      exit(1);
    }
  return p;
}

int main() {
  ll a, b, c;
  int d, e;
  while (scanf("%lld %lld %lld %d %d", &a, &b, &c, &d, &e) == 5) {
    const VocabPlan p = plan(a, b, c, d, e);
    printf("%d %lld %d\n", fits(p.mma[0]) && fits(p.mma[1]), (ll)p.pieces, std::max(p.mma[0].splits, p.mma[1].splits));
  }
  std::mt19937_64 r(1);
  auto size = [&](double hi) { return (ll)std::exp(std::uniform_real_distribution<>(0, std::log(hi))(r)); };
  for (int i = 0; i < 200000; ++i) plan(size(INT32_MAX), size(1 << 20), size(1 << 30), r() & 1, r() & 1);
  for (int i = 0; i < 4; ++i) plan(INT32_MAX, 1 << 20, 1 << 30, i & 1, i >> 1);
  puts("ok");
}
