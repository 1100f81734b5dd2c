// Host-only check of the records and tickets of vp_attend_new's tensor-core
// kernels (vp_attend.h): over every line of items cut for any number of CTAs, an
// item joined by ticket has its ticket, and each CTA's record of it, for itself.
// Prints one line per violation and exits non-zero if there was any.
#include <cstdio>
#include <random>
#include <vector>

#include "vp_attend.h"

int main() {
  using namespace vp;
  std::mt19937 rng(11);
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  int fails = 0;
  auto once = [&](int uses, const char* what, int at, int cta, int rows) {
    if (uses > 1 && ++fails <= 20) std::printf("FAIL %s: %d at CTA %d, %d rows\n", what, at, cta, rows);
  };
  for (int trial = 0; trial < 3000; ++trial) {
    const int G = pick(1, 16), n_new = pick(0, 2) ? pick(1, 16) : pick(1, 400), R = n_new * G;
    const int block = R > kTcTile ? 2 * kTcTile : R, nqt = (R + block - 1) / block;
    const int fixed = (R <= kDecRows ? 1 : 2) * kTileUnits, ctas = pick(0, 1) ? 152 : pick(1, 320);
    const int B = pick(1, 70), Hkv = pick(1, 8), window = pick(0, 1) ? -1 : pick(0, 2000), longest = pick(0, 1) ? 600 : 9000;
    std::vector<AttItem> items;
    int total = 0;
    for (int b = 0; b < B; ++b) {
      const int len = pick(0, 5) ? pick(0, longest) : 0, n = len < n_new ? len : n_new;
      for (int qt = 0; qt < nqt; ++qt) {
        items.push_back(att_item(len, n, G, block, qt, window, 4));
        total += items.back().cost(fixed);
      }
    }
    const LineCut lc(total * Hkv, ctas);
    std::vector<int> tickets(lc.nc, 0), records(2 * lc.nc, 0);
    int begin = 0;
    for (int g = 0; g < Hkv; ++g)
      for (const AttItem& it : items) {
        if (it.tl.n > 0) {
          const int first = lc.owner(begin + fixed), last = lc.owner(begin + fixed + (it.tl.n - 1) * it.unit());
          if (by_ticket(last - first + 1)) {
            once(++tickets[first], "a ticket of two items", first, first, it.rows);
            for (int c = first; c <= last; ++c) once(++records[record_of(c, first)], "a record of two items", record_of(c, first), c, it.rows);
          }
        }
        begin += it.cost(fixed);
      }
  }
  std::printf("%d violations\n", fails);
  return fails != 0;
}
