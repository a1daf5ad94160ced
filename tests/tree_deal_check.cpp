// Host check of how the cache attention's units are counted (tree_deal.h): the
// largest tiles that the cache's limits allow, in every combination that may
// pass 31 bits, against sums in 64 bits.
#include <cstdio>
#include <initializer_list>

#include "tree_deal.h"

using namespace mv;

template <int W>
static int check(int kmax) {
  uint32_t units[W];
  int64_t sum = 0;
  for (int w = 0; w < W; ++w) {
    units[w] = 0;
    for (int i = 0; i < 64; ++i) units[w] += uint32_t(units_of(kmax));
    int64_t before, all;
    for (int x = w + 1; x < W; ++x) units[x] = 0;
    add_waves<W>(units, w, before, all);
    if (before != sum) return std::printf("kmax %d: before wave %d: %lld\n", kmax, w, (long long)before);
    sum += 64 * ((int64_t(kmax) + 63) / 64);
    if (all != sum) return std::printf("kmax %d: of %d waves: %lld\n", kmax, w + 1, (long long)all);
  }
  return 0;
}

int main() {
  for (int kmax : {0, 1, 63, 64, 65, (1 << 29) - 64, 1 << 29, (1 << 29) + 1, 1 << 30, 2147483584,
                   2147483585, 2147483632}) {
    if (int64_t(units_of(kmax)) != (int64_t(kmax) + 63) / 64) {
      std::printf("kmax %d: %d units\n", kmax, units_of(kmax));
      return 1;
    }
    if (check<2>(kmax) || check<4>(kmax)) return 1;
  }
  return 0;
}
