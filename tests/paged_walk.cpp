// Walks random launches of df_paged_attn as its kernels do, on the host (df_paged_walk.h is the kernels' own), and compares with a walk key by
// key: every row sees each of its keys in exactly one piece, tiles that are taken without a look at single keys hold only keys that all
// rows see, tiles begin at keys that are there, and pieces of cut units form chains that the second kernel finds.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "df_paged_walk.h"

using namespace df;

static std::mt19937 rng;
static int pick(int lo, int hi) { return lo + int(rng() % uint32_t(hi - lo + 1)); }
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s (seed %d)\n", __LINE__, #x, seed); std::exit(1); } } while (0)

struct Launch {
  int B, Hkv, G, block, max_new, total, page_log2;
  bool keys;
  std::vector<int> len, cu, sink, win;
};

static Launch draw(int seed) {
  Launch l;
  rng.seed(seed);
  l.B = pick(1, 4);
  l.Hkv = pick(1, 3);
  l.G = (int[]){1, 1, 2, 4, 7, 64}[pick(0, 5)];
  l.page_log2 = pick(4, 7);
  l.keys = pick(0, 5) != 0;
  const bool single = pick(0, 2) == 0;
  l.cu = {pick(0, 3)};
  l.max_new = 1;
  const int most_new = l.G >= 7 ? 40 : 300;
  for (int b = 0; b < l.B; ++b) {
    const int n = single ? pick(0, 1) : pick(0, 3) == 0 ? pick(0, 8) : pick(0, most_new);
    l.cu.push_back(l.cu.back() + n);
    l.max_new = most(l.max_new, n);
    l.len.push_back(pick(0, 4) == 0 ? 0 : pick(0, 3) == 0 ? pick(1, 3000) : pick(1, 700));
    for (int h = 0; h < l.Hkv; ++h) {
      const int kind = pick(0, 6);
      l.sink.push_back(kind == 0 || kind == 3 ? 0 : kind == 5 ? pick(1, 2000) : pick(1, 200));
      l.win.push_back(kind <= 1 ? (kind ? pick(0, 3) * 0 : 0) : kind == 2 ? kMaxLen : pick(1, 500));
    }
  }
  l.total = l.cu.back() + pick(0, 2);
  l.block = (int[]){1, 1, 2, 33, 64, 100, 1 << 30}[pick(0, 6)];
  return l;
}

// KT keys a tile, ROWS rows of WAVES waves (WAVES = 1: waves share the tiles of a piece out instead), `turned` rounds
template <int KT, int ROWS, int WAVES>
static void walk(const Launch &l, int seed, int workgroups, bool turned) {
  const int row_tiles = (l.max_new * l.G + ROWS - 1) / ROWS, units = l.B * l.Hkv * row_tiles;
  const Rules rules{Divider::by(l.G), Divider::by(l.block), l.keys};
  const Divider by_tiles = Divider::by(row_tiles), by_heads = Divider::by(l.Hkv);
  auto request = [&](int b, int h) {
    return make_request(l.cu[b], l.cu[b + 1], l.len[b], l.sink[b * l.Hkv + h], l.win[b * l.Hkv + h], l.total, l.max_new, int64_t(1) << 40);
  };
  std::vector<int64_t> cost(units), at(units + 1, 0);
  for (int u = 0; u < units; ++u) {
    const Unit un = unit_of(u, by_tiles, by_heads, ROWS);
    const Request r = request(un.b, un.h);
    cost[u] = un.row0 >= r.n * l.G ? 0 : kUnitCost + tiles_of<KT>(r, row_range(r, rules, un.row0, ROWS), l.keys).count();
    at[u + 1] = at[u] + cost[u];
  }
  const Line line = Line::of(at[units], workgroups);
  CHECK((line.all > 0) == (line.count > 0) && line.count <= workgroups);
  // seen[u][tile]: times taken; owner: pieces of cut units in span order
  std::vector<std::vector<int>> seen(units);
  std::vector<int> tail(line.count, -1), head(line.count, 0), head_unit(line.count, -1), whole(units, 0);
  for (int sp = 0; sp < line.count; ++sp) {
    const int64_t begin = line.begin_of(sp), end = line.begin_of(sp + 1);
    CHECK(begin == line.all * sp / line.count && end == line.all * (sp + 1) / line.count);
    CHECK(end > begin);
    for (int u = 0; u < units && at[u] < end; ++u) {
      if (at[u + 1] <= begin && !(at[u + 1] == at[u])) continue;
      if (cost[u] == 0) continue;
      const Unit un = unit_of(u, by_tiles, by_heads, ROWS);
      const Request r = request(un.b, un.h);
      const RowRange x = row_range(r, rules, un.row0, ROWS);
      const Tiles<KT> tl = tiles_of<KT>(r, x, l.keys);
      const int T = tl.count();
      CHECK(T + kUnitCost == cost[u]);
      const Piece pc = piece_of(line, begin, end, at[u], T, turned);
      if (!pc.is) continue;
      CHECK(pc.t0 >= 0 && pc.t0 < most(T, 1) && pc.t1 >= pc.t0 && pc.t1 - pc.t0 <= T);
      if (seen[u].empty()) seen[u].assign(T, 0);
      if (pc.begins && pc.ends) ++whole[u];
      if (pc.begins && !pc.ends) { CHECK(tail[sp] == -1); tail[sp] = u; }
      if (!pc.begins) { CHECK(head[sp] == 0); head[sp] = pc.ends ? 2 : 1; head_unit[sp] = u; }
      for (int t = pc.t0; t < pc.t1; ++t) {
        const Place pl = place_of(r, tl, t);
        ++seen[u][t >= T ? t - T : t];
        CHECK(pl.k0 % KT == 0 && pl.k0 >= 0 && pl.k0 < pl.limit);
      }
      // waves: what is taken as seen by all is, of what is skipped nothing is, and where only the tail is missing all that is there is seen
      for (int wave = 0; wave < WAVES; ++wave) {
        const int rows = ROWS / WAVES, row0 = un.row0 + rows * wave, last = r.n * l.G;
        if (row0 >= last) continue;
        const RowRange mine = WAVES > 1 ? row_range(r, rules, row0, rows) : x;
        const RangeKeys rk = range_keys(r, mine);
        for (int t = pc.t0; t < pc.t1; ++t) {
          const Place pl = place_of(r, tl, t);
          const Seen what = seen_of(pl, KT, rk);
          if (what == kSomeHidden) continue;
          for (int row = row0; row < least(row0 + rows, last); ++row) {
            const Keys s = pl.is_new ? row_fresh(r, rules, rules.first_of(row)) : row_slots(r, rules.first_of(row));
            for (int k = pl.k0; k < pl.k0 + KT; ++k)
              CHECK(s.sees(k) == (what == kAllSeen || (what == kTailMissing && k < pl.limit)));
          }
        }
      }
    }
  }
  // the chains of the second kernel
  std::vector<int> chains(units, 0);
  for (int sp = 0; sp < line.count; ++sp)
    if (tail[sp] >= 0) {
      int w = sp + 1;
      for (;; ++w) {
        CHECK(w < line.count && head[w] != 0 && head_unit[w] == tail[sp]);
        if (head[w] == 2) break;
      }
      ++chains[tail[sp]];
    }
  for (int u = 0; u < units; ++u) {
    CHECK(whole[u] + chains[u] == (cost[u] > 0));
    for (int n : seen[u]) CHECK(n == 1);
    if (!cost[u]) continue;
    // by definition: row by row, position by position
    const Unit un = unit_of(u, by_tiles, by_heads, ROWS);
    const Request r = request(un.b, un.h);
    const Tiles<KT> tl = tiles_of<KT>(r, row_range(r, rules, un.row0, ROWS), l.keys);
    const int T = tl.count(), n = l.cu[un.b + 1] - l.cu[un.b], L = l.len[un.b], s = r.s, w = r.w;
    std::vector<char> slot_in(r.held, 0), new_in(n, 0);
    for (int t = 0; t < T; ++t) {
      const Place pl = place_of(r, tl, t);
      for (int k = pl.k0; k < least(pl.k0 + KT, pl.limit); ++k) ++(pl.is_new ? new_in : slot_in)[k];
    }
    for (char c : slot_in) CHECK(c <= 1);
    for (char c : new_in) CHECK(c <= 1);
    CHECK(n == r.n);
    for (int row = un.row0; row < least(un.row0 + ROWS, n * l.G); row += pick(1, 9)) {
      const int i = row / l.G, first = int(int64_t(i) / l.block * l.block);
      const int64_t last = int64_t(first) + l.block < n ? int64_t(first) + l.block : n;
      const Keys hist = row_slots(r, rules.first_of(row)), fresh = row_fresh(r, rules, rules.first_of(row));
      for (const Keys &x : {hist, fresh})
        for (int k = 0; k < most(r.held, n) + 8; k += 8) {
          unsigned bits = 0;
          for (int i = 0; i < 8; ++i) bits |= unsigned(x.sees(k + i)) << i;
          CHECK(eight_keys(x, k) == bits);
        }
      int held = 0;
      for (int j = 0; j < L; ++j) {
        if (!(j < s || (w > 0 && j >= L - w))) continue;    // not kept
        ++held;
        const int slot = slot_of(j, s, w);
        CHECK(slot < r.held);
        const bool sees = j < s || j >= L + first - w;
        CHECK(hist.sees(slot) == sees);
        if (sees) CHECK(slot_in[slot] == 1);
      }
      CHECK(held == r.held);
      for (int k = r.held; k < r.held + KT; ++k) CHECK(!hist.sees(k));
      for (int t = 0; t < n + KT; ++t) {
        const bool sees = t < last && (t >= first - w || L + t < s);
        CHECK(fresh.sees(t) == sees);
        if (sees && l.keys) CHECK(new_in[t] == 1);
      }
    }
  }
}

int main(int argc, char **argv) {
  for (int seed = 0, i = 0; i < 200000; ++i) {
    const unsigned d = i < 300 ? i + 1 : 1 + rng() % (i % 3 ? 5000u : 0x7fffffffu);
    const int x = i % 5 ? int(rng() >> (1 + rng() % 30)) : 0x7fffffff - int(rng() % 3);
    CHECK(Divider::by(d).of(x) == int(unsigned(x) / d));
  }
  const int from = std::atoi(argv[1]), to = std::atoi(argv[2]);
  for (int seed = from; seed < to; ++seed) {
    const Launch l = draw(seed);
    const int rows = l.max_new * l.G, wg = (int[]){1, 3, 8, 64, 512}[pick(0, 4)];
    if (rows <= 16) walk<32, 16, 1>(l, seed, wg, false);
    if (rows <= 32) walk<32, 32, 1>(l, seed, wg, false);
    walk<64, 128, 4>(l, seed, wg, true);
  }
  std::printf("ok\n");
  return 0;
}
