// Host-only check of how vp_attend_new cuts its work (vp_attend.h): the tiles of
// a row block cover the tokens its rows see and no tile comes twice; a line of
// items cut for any number of CTAs gives every tile to one CTA, and every CTA
// between the first and the last of an item one of its tiles; items with CTAs
// of their own get a tile per share; the splits of k_att_any stay within the
// workspace.  Prints one line per violation and exits non-zero if there was any.
#include <cstdio>
#include <random>
#include <vector>

#include "vp_attend.h"

namespace {

using namespace vp;

int fails = 0;
void check(bool ok, const char* what, long a = 0, long b = 0, long c = 0, long d = 0) {
  if (ok) return;
  if (++fails <= 20) std::printf("FAIL %s: %ld %ld %ld %ld\n", what, a, b, c, d);
}

void check_tiles(std::mt19937& rng) {
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  for (int trial = 0; trial < 20000; ++trial) {
    const int t0 = pick(0, 600), t1 = t0 + pick(0, 40), rows = trial % 2 ? 32 : 128;
    const int window = pick(0, 3) ? pick(0, 300) : (pick(0, 1) ? -1 : 2147483647);
    const int sinks = pick(0, 2) ? pick(0, 200) : (pick(0, 1) ? 0 : 2147483647);
    const SeenRange sr = seen_range(t0, t1, window, sinks);
    const TileList tl = tile_list(sr, rows);
    std::vector<int> times(t1 / rows + 3, 0);
    for (int u = 0; u < tl.n; ++u) {
      const int tile = tl.tile(u);
      check(tile >= 0 && tile < (int)times.size(), "tile index", t0, t1, window, sinks);
      if (tile >= 0 && tile < (int)times.size()) ++times[tile];
    }
    for (int j = 0; j <= t1 + rows; ++j) {
      bool seen = false;
      for (int t = t0; t <= t1 && !seen; ++t) seen = sees(j, t, window, sinks);
      const bool in = j < sr.s_end || (j >= sr.lo && j < sr.hi);
      if (seen) check(in && times[j / rows] == 1, "a seen token without a tile", j, t0, window, sinks);
      if (in) check(j <= t1, "a token behind the last row", j, t0, window, sinks);
    }
    for (int x : times) check(x <= 1, "a tile twice", t0, t1, window, sinks);
  }
}

// The tiles [u0, u1) of an item that the part [off, off + take) of it does.
struct Tiles {
  int u0, u1;
};
Tiles tiles_of(const AttItem& it, int off, int take, int fixed) {
  const int cost = it.cost(fixed), end = off + take < cost ? off + take : cost;
  return {it.tiles_before(off, fixed), it.tiles_before(end, fixed)};
}

void check_lines(std::mt19937& rng) {
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  for (int trial = 0; trial < 4000; ++trial) {
    const int G = 1 << pick(0, 3), n_new = pick(0, 2) ? pick(1, 8) : pick(1, 700);
    const int R = n_new * G, dec = R <= kDecRows;
    const int block = R > kTcTile ? 2 * kTcTile : R, nqt = (R + block - 1) / block;
    const int B = pick(1, 20), Hkv = pick(1, 8), fixed = (dec ? 1 : 2) * kTileUnits;
    const int ctas = pick(0, 1) ? 152 : pick(1, 320);
    const int window = pick(0, 1) ? -1 : pick(0, 3000), sinks = pick(0, 40);
    std::vector<AttItem> items;
    std::vector<int> costs;
    int total = 0;
    for (int b = 0; b < B; ++b) {
      const int len = pick(0, 3) ? pick(0, 9000) : 0, n = len < n_new ? len : pick(0, n_new);
      for (int qt = 0; qt < nqt; ++qt) {
        items.push_back(att_item(len, n, G, block, qt, window, sinks));
        costs.push_back(items.back().cost(fixed));
        total += costs.back();
      }
    }
    const int pairs = (int)items.size();
    if (pairs * Hkv <= ctas / 4) {
      const int all = total * Hkv, low = (all + ctas - 1) / ctas;
      const int high = (all + ctas - pairs * Hkv - 1) / (ctas - pairs * Hkv);
      bool found = false;
      for (int t = 0; t < 4 && !found; ++t) {
        const int per = min_share(fixed) > low + (high - low) * t / 3 ? min_share(fixed) : low + (high - low) * t / 3;
        int shares = 0;
        for (int c : costs) shares += share_count(c, per);
        if (shares * Hkv > ctas) continue;
        found = true;
        for (int i = 0; i < pairs; ++i) {
          const int m = share_count(costs[i], per);
          check(m >= 1, "an item without a share", i, m, per);
          int done = 0;
          for (int k = 0; k < m; ++k) {
            const int off = (int)((long long)costs[i] * k / m), end = (int)((long long)costs[i] * (k + 1) / m);
            const Tiles q = tiles_of(items[i], off, end - off, fixed);
            check(q.u0 == done, "shares leave a gap", i, k, q.u0, done);
            check(q.u1 > q.u0 || m == 1, "a share without a tile", costs[i], m, k, per);
            done = q.u1;
          }
          check(done == items[i].tl.n, "shares end early", i, done, items[i].tl.n);
        }
      }
      check(found, "no share fits", pairs, Hkv, ctas, total);
      continue;
    }
    const LineCut lc(total * Hkv, ctas);
    check(lc.nc >= 1 && lc.nc <= ctas && lc.start(lc.nc) == total * Hkv, "line ends", lc.nc, ctas, total, Hkv);
    int cta = 0, pos = 0;
    for (int g = 0; g < Hkv; ++g) {
      for (int i = 0; i < pairs; ++i) {
        const int begin = pos, cost = costs[i];
        const AttItem& it = items[i];
        while (lc.start(cta + 1) <= begin) ++cta;
        int done = 0, first = -1, last = -1, owners = 0;
        for (int c = cta; c < lc.nc && lc.start(c) < begin + cost; ++c) {
          const int off = lc.start(c) > begin ? lc.start(c) - begin : 0;
          const Tiles q = tiles_of(it, off, lc.start(c + 1) - begin - off, fixed);
          owners += off == 0;
          check(q.u0 == done, "the line leaves a gap", g, i, q.u0, done);
          done = q.u1;
          if (q.u1 > q.u0) {
            if (first < 0) first = c;
            check(last < 0 || last == c - 1, "a CTA between without a tile", c, first, cost, lc.per);
            last = c;
          }
        }
        check(owners == 1, "owners of an item", g, i, owners);
        check(done == it.tl.n, "the line ends early", g, i, done, it.tl.n);
        if (it.tl.n > 0) {
          const int at = begin + fixed;
          check(lc.owner(at) == first, "CTA of the first tile", lc.owner(at), first, g, i);
          check(lc.owner(at + (it.tl.n - 1) * it.unit()) == last, "CTA of the last tile", last, g, i);
        }
        pos += cost;
      }
    }
  }
}

void check_splits() {
  for (int sms : {1, 132, 152})
    for (int B : {1, 2, 7, 64, 700})
      for (int Hkv : {1, 4, 32})
        for (int R : {1, 4, 5, 8, 9, 64, 128, 5000})
          for (int window : {-1, 0, 100, 4000})
            for (int seq : {1, 31, 33, 700, 20000, 1 << 20}) {
              const int rows = any_rows(R), ns = any_splits(B, Hkv, R, rows, R, window, 4, seq, sms);
              const long units = (long)B * Hkv * ((R + rows - 1) / rows);
              check(ns >= 1 && (ns == 1 || units * ns <= 8L * sms), "splits within the records", B, Hkv, R, ns);
              check(ns == 1 || units <= 4L * sms, "splits within the tickets", B, Hkv, R, ns);
              check(ns == 1 || ns <= (seq + kAnyTile - 1) / kAnyTile, "splits without a tile", B, seq, R, ns);
            }
  for (int max_new : {1, 17, 4096})
    for (int wn : {0, 1, 16}) {
      if (wn > max_new) continue;
      const NewLayout w = new_layout(8, 32, 4, 128, 5000, max_new, wn, 152);
      check(w.o_tk % 16 == 0 && w.o_lse % 16 == 0 && w.o_st % 16 == 0 && w.o_o % 16 == 0 && w.o_z % 16 == 0,
            "workspace alignment", max_new, wn);
      check(w.o_lse - w.o_tk >= 4u * 152 * 4, "tickets", max_new, wn);
      check(w.o_o - w.o_st >= 8u * 152 * kAnyRows * 8, "records' sums", max_new, wn);
      check(w.o_z - w.o_o >= 8u * 152 * kAnyRows * 128 * 4, "records' outputs", max_new, wn);
      check(w.z_row >= 5000 && w.total - w.o_z >= (size_t)8 * 4 * wn * 8 * w.z_row * 4, "logits", max_new, wn);
    }
}

}  // namespace

int main() {
  std::mt19937 rng(7);
  check_tiles(rng);
  check_lines(rng);
  check_splits();
  std::printf("%d violations\n", fails);
  return fails != 0;
}
