// Host-only check of the records and tickets of vp_attend_new's tensor-core
// kernels (vp_attend.h): over every line of items cut for any number of CTAs, an
// item joined by ticket has its ticket, and each CTA's record of it, for itself;
// the workspace has room for all of them and for no more.
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
  // The workspace holds every kernel's records and tickets, and grows with the
  // batch and the weights by the logits and the log-sum-exps alone.
  for (int sms : {1, 148, 152})
    for (int D : {64, 128}) {
      const NewLayout one = new_layout(1, 32, 4, D, 4096, 256, 0, sms), many = new_layout(64, 32, 4, D, 4096, 256, 16, sms);
      const size_t rows = (many.o_z - many.o_o) / (D * sizeof(float)), tickets = (many.o_lse - many.o_tk) / sizeof(unsigned);
      if (many.o_z - many.o_o != one.o_z - one.o_o || many.o_o - many.o_st != one.o_o - one.o_st)
        ++fails, std::printf("FAIL records that grow: %zu, %zu bytes\n", one.o_z - one.o_o, many.o_z - many.o_o);
      const size_t most = 4u * sms * kTcTile;  // 2 per CTA, 2 groups of 128 rows, a CTA per SM
      if (rows < most || rows < 2u * 2 * sms * 16 || rows < 2u * sms * kDecRows || rows < 8u * sms * kAnyRows ||
          tickets < 2u * sms * kDecRows / 32 || tickets < 4u * sms || (many.o_o - many.o_st) / 8 < rows)
        ++fails, std::printf("FAIL room for records and tickets: %zu %zu\n", rows, tickets);
    }
  std::printf("%d violations\n", fails);
  return fails != 0;
}
