// The walk of df_paged_attn: what a row sees of its keys, which tiles of keys a tile of rows needs, and how all of that is shared out over
// workgroups.  Whole numbers only, the same code on the device and on the host (where tests/test_paged_walk.py checks it against
// a walk key by key).
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define DF_WALK __host__ __device__ __forceinline__
#else
#define DF_WALK inline
#endif

namespace df {

constexpr int kMaxLen = 1 << 30;       // bound of lengths, sinks and windows

// One of two values.  (A conditional expression between two members is one between their addresses: it keeps the compiler from taking their structure
// apart.  One left in memory comes to lie in LDS, for its place there every wave reads the launch's packet from the host, and a launch takes 13 us longer.)
DF_WALK int pick(bool first, int a, int b) { return first ? a : b; }
DF_WALK int least(int a, int b) { return a < b ? a : b; }
DF_WALK int most(int a, int b) { return a > b ? a : b; }
DF_WALK int clamp_int(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// Division of whole numbers >= 0 by one that the host knows (2^32 / d rounded up, with the bit above the 32 added by hand).
struct Divider {
  unsigned d, m;
  int shift;
  static Divider by(unsigned d) {
    int l = 0;
    while (l < 32 && (uint64_t(1) << l) < d) ++l;
    return Divider{d, unsigned(((uint64_t(1) << 32) * ((uint64_t(1) << l) - d)) / d + 1), l - 1};
  }
  DF_WALK int of(int x) const {
    if (d == 1) return x;
    const unsigned t = unsigned((uint64_t(m) * unsigned(x)) >> 32);
    return int((t + ((unsigned(x) - t) >> 1)) >> shift);
  }
};

// What all requests of a launch have in common.
struct Rules {
  Divider G, block;          // query heads to a key head, tokens of a causal block
  bool keys;                 // new tokens have keys
  // First token of the causal block that row `row` belongs to.
  DF_WALK int first_of(int row) const { return block.of(G.of(row)) * int(block.d); }
};

// Filled slots after `len` tokens: min(len, sink + win), whose sum may not fit into 32 bits.
DF_WALK int filled_slots(int len, int sink, int win) { return len < sink || len - sink < win ? len : sink + win; }
// Slot of position j in a head with a window, and of a sink position in any.
DF_WALK int slot_of(int j, int sink, int win) { return j < sink ? j : sink + (j - sink) % win; }

// A request as one key head sees it.
struct Request {
  int n, q0;                 // new tokens and the first one's row
  int L, s, w, held;         // tokens in the cache, sink, window, filled slots
  bool bad;                  // more slots than the table has entries for
};
// c0, c1: rows of the request; `room`: slots that the table has entries for.  Whatever the numbers are, the result is inside all buffers.
DF_WALK Request make_request(int c0, int c1, int len, int sink, int win, int total, int max_new, int64_t room) {
  Request r;
  c0 = clamp_int(c0, 0, total);
  r.q0 = c0;
  r.n = least(clamp_int(c1, c0, total) - c0, max_new);
  r.L = clamp_int(len, 0, kMaxLen);
  r.s = clamp_int(sink, 0, kMaxLen);
  r.w = clamp_int(win, 0, kMaxLen);
  r.held = filled_slots(r.L, r.s, r.w);
  r.bad = r.held > room;
  if (r.bad) r.held = int(room);
  return r;
}

// Slots that a causal block beginning at new token `first` sees: [0, a1) and [b0, b1).  Behind the sink they are a ring; what the
// block does not see of it are the `first` oldest tokens (or, before the ring is full, those older than the window).
struct Visible { int a1, b0, b1; };
DF_WALK Visible visible_slots(const Request &r, int first) {
  Visible v;
  const int sink = least(r.held, r.s), turn = r.L - r.s;
  if (first >= r.w || turn <= 0) {
    v.a1 = v.b0 = v.b1 = sink;
  } else if (turn <= r.w) {
    const int lo = r.L + first - r.w;
    v.a1 = lo <= r.s ? r.held : sink;
    v.b0 = lo <= r.s ? r.held : least(lo, r.held);
    v.b1 = r.held;
  } else if (first == 0) {
    v.a1 = v.b0 = v.b1 = r.held;
  } else {
    const int at = turn % r.w;
    const bool wraps = at > r.w - first;
    v.a1 = least(r.held, wraps ? r.s : r.s + at);
    v.b0 = least(r.held, wraps ? r.s + (at - (r.w - first)) : r.s + at + first);
    v.b1 = least(r.held, wraps ? r.s + at : r.s + r.w);
  }
  return v;
}

// The causal blocks of a range of rows (row r is new token r / G).
struct RowRange {
  int first0, first1;        // first tokens of the first and the last row's causal blocks
  int end0, end1;            // and their ends
};
DF_WALK RowRange row_range(const Request &r, const Rules &u, int row0, int rows) {
  RowRange x;
  x.first0 = u.first_of(row0);
  x.first1 = u.first_of(least(r.n * int(u.G.d) - 1, row0 + rows - 1));
  // (a sum only where a block is shorter than the request, else it may not fit into 32 bits)
  x.end0 = int(u.block.d) < r.n ? least(x.first0 + int(u.block.d), r.n) : r.n;
  x.end1 = int(u.block.d) < r.n ? least(x.first1 + int(u.block.d), r.n) : r.n;
  return x;
}

// The key tiles of one unit (request, key head, tile of rows): slots first, new tokens behind them, each in up to two runs of tiles.
template <int KT>
struct Tiles {
  int nA, nB, nC, nD;        // tiles of the four runs
  int firstB, firstD;        // first tile of the second runs (the first ones begin at 0)
  DF_WALK int count() const { return nA + nB + nC + nD; }
};
template <int KT>
DF_WALK Tiles<KT> tiles_of(const Request &r, const RowRange &x, bool keys) {
  Tiles<KT> t;
  const Visible v = visible_slots(r, x.first0);
  t.nA = (v.a1 + KT - 1) / KT;
  t.firstB = most(v.b0 / KT, t.nA);
  t.nB = v.b1 > v.b0 ? most(0, (v.b1 + KT - 1) / KT - t.firstB) : 0;
  t.nC = t.nD = t.firstD = 0;
  if (keys) {
    const int c1 = clamp_int(r.s - r.L, 0, x.end1), d0 = most(0, x.first0 - r.w);
    t.nC = (c1 + KT - 1) / KT;
    t.firstD = most(d0 / KT, t.nC);
    t.nD = most(0, (x.end1 + KT - 1) / KT - t.firstD);
  }
  return t;
}

// Where tile t of a unit lies (from the last on round again).
struct Place {
  bool is_new;               // new tokens, or slots
  int k0;                    // first key
  int limit;                 // keys that are there
};
template <int KT>
DF_WALK Place place_of(const Request &r, const Tiles<KT> &tl, int t) {
  const int hist = tl.nA + tl.nB, all = tl.count(), at = t >= all ? t - all : t, i = at - hist;
  Place x;
  x.is_new = at >= hist;
  x.k0 = KT * (x.is_new ? (i < tl.nC ? i : tl.firstD + i - tl.nC) : (at < tl.nA ? at : tl.firstB + at - tl.nA));
  x.limit = pick(x.is_new, r.n, r.held);
  return x;
}

// Keys that the rows of a range see of the cache (`hist`) and of the new tokens (`fresh`): [0, a) and [b, c), `all` of them or `some`.
struct Keys {
  int a, b, c;
  DF_WALK bool sees(int key) const { return (key < a) | ((key >= b) & (key < c)); }
};
DF_WALK Keys pick(bool first, const Keys &x, const Keys &y) { return Keys{pick(first, x.a, y.a), pick(first, x.b, y.b), pick(first, x.c, y.c)}; }
struct RangeKeys {
  Keys all_hist, all_fresh, some_hist, some_fresh;
};
DF_WALK RangeKeys range_keys(const Request &r, const RowRange &x) {
  RangeKeys k;
  Visible v = visible_slots(r, x.first1);
  k.all_hist = Keys{v.a1, v.b0, v.b1};
  k.all_fresh = Keys{clamp_int(r.s - r.L, 0, x.end0), most(0, x.first1 - r.w), x.end0};
  v = visible_slots(r, x.first0);
  k.some_hist = Keys{v.a1, v.b0, v.b1};
  k.some_fresh = Keys{clamp_int(r.s - r.L, 0, x.end1), most(0, x.first0 - r.w), x.end1};
  return k;
}
// What the rows see of a tile: all of its keys, all that are there (the rows behind the last key are zeros), only some, or none.
enum Seen { kAllSeen, kTailMissing, kSomeHidden, kNoneSeen };
DF_WALK Seen seen_of(const Place &x, int KT, const RangeKeys &k) {
  const Keys all = pick(x.is_new, k.all_fresh, k.all_hist), some = pick(x.is_new, k.some_fresh, k.some_hist);
  const int until = x.k0 < all.a ? all.a : x.k0 >= all.b ? all.c : x.k0;      // seen by all without a gap from k0 to here
  if (x.k0 >= some.a && (x.k0 >= some.c || x.k0 + KT <= some.b)) return kNoneSeen;
  return x.k0 + KT <= until ? kAllSeen : least(x.k0 + KT, x.limit) <= until ? kTailMissing : kSomeHidden;
}

// What one row sees, whose causal block begins at token `first`: slots, and new tokens.
DF_WALK Keys row_slots(const Request &r, int first) {
  const Visible v = visible_slots(r, first);
  return Keys{v.a1, v.b0, v.b1};
}
DF_WALK Keys row_fresh(const Request &r, const Rules &u, int first) {
  const int end = int(u.block.d) < r.n ? least(first + int(u.block.d), r.n) : r.n;
  return Keys{clamp_int(r.s - r.L, 0, end), most(0, first - r.w), end};
}
// Which of the keys k .. k + 7 they are: a bit for each.
DF_WALK unsigned below8(int n) { return (1u << clamp_int(n, 0, 8)) - 1u; }
DF_WALK unsigned eight_keys(const Keys &x, int k) { return below8(x.a - k) | (below8(x.c - k) & ~below8(x.b - k)); }

// ---- sharing out -------------------------------------------------------------------------------------------------------------
// The units' costs (tiles + a constant) form a line, requests outermost, then key heads, then tiles of rows (neighbours read the same keys); it is
// cut into equal spans.
// Cost of a unit besides its tiles, in tiles: its request, pages and queries are fetched one after the other, and its hidden tiles take longer than
// others.  When it was set, 4, 10, 16, 24: single tokens 236, 206, 204, 206 us, prompt pieces 506, 471, 462, 495, 390-token frames 87, 77, 80, 79,
// 480p chunks 640, 634, 643, 654; since then 13 and 16 make no difference to 60 drawn cases (0.2 %).
constexpr int kUnitCost = 10;
constexpr int kSnap = 3;               // no piece of a cut unit has fewer tiles ...
constexpr int kMinSpan = 8;            // ... than fit into the shortest span; units of up to kMinSpan tiles are not cut
static_assert(2 * kSnap < kMinSpan, "a span inside a unit is a piece");

struct Unit { int b, h, row0; };
DF_WALK Unit unit_of(int u, const Divider &row_tiles, const Divider &Hkv, int rows) {
  const int e = row_tiles.of(u), b = Hkv.of(e);
  return Unit{b, e - b * int(Hkv.d), (u - e * int(row_tiles.d)) * rows};
}

// Tile at which position x of a unit's part of the line (its first kUnitCost positions are no tiles) cuts its T tiles.
DF_WALK int cut_at(int64_t x, int T) {
  if (T <= kMinSpan) return x <= 0 ? 0 : T;
  const int64_t t = x - kUnitCost;
  return t < kSnap ? 0 : t > T - kSnap ? T : int(t);
}

struct Line {
  int64_t all;               // its length
  int count;                 // spans: as many as there are workgroups, fewer on a line shorter than kMinSpan each
  int64_t each;              // all = each * count + rest
  int rest;
  DF_WALK static Line of(int64_t all, int workgroups) {
    const int64_t n = all / kMinSpan;
    Line x{all, int(n < 1 ? (all > 0) : n > workgroups ? workgroups : n), 0, 0};
    // (a division in 64 bits takes a wave half a microsecond)
    if (x.count == 0) return x;
    if ((x.count & (x.count - 1)) == 0) x.each = all >> __builtin_ctz(x.count);
    else x.each = all <= UINT32_MAX ? unsigned(all) / unsigned(x.count) : all / x.count;
    x.rest = int(all - x.each * x.count);
    return x;
  }
  // Where a span begins (of the one behind the last: the line's end).
  DF_WALK int64_t begin_of(int i) const {
    const unsigned r = unsigned(rest) * unsigned(i), c = unsigned(count);
    return each * i + ((c & (c - 1)) == 0 ? r >> __builtin_ctz(c) : r / c);
  }
  // How far into its span position x lies.
  DF_WALK int64_t into_span(int64_t x) const {
    int i = clamp_int(int(float(x) * (float(count) / float(all))), 0, count - 1);
    while (begin_of(i) > x) --i;
    while (begin_of(i + 1) <= x) ++i;
    return x - begin_of(i);
  }
};

// A span's part of a unit of T tiles that begins at `at` on the line.
struct Piece {
  int t0, t1;                // tiles; with `turn`, in the order of the round that begins at the tile of the workgroup's time
  bool begins, ends;         // whether the unit's first and last part is in it
  bool is;                   // there is something to do
};
DF_WALK Piece piece_of(const Line &line, int64_t begin, int64_t end, int64_t at, int T, bool turned) {
  Piece x;
  x.t0 = cut_at(begin - at, T);
  x.t1 = at + kUnitCost + T <= end ? T : cut_at(end - at, T);
  x.begins = x.t0 == 0;
  x.ends = x.t1 == T;
  x.is = x.t0 < x.t1 || (T == 0 && begin <= at);
  if (turned && T > 0 && x.is) {
    const int64_t into = line.into_span(at);
    const int turn = into <= INT32_MAX ? int(unsigned(into) % unsigned(T)) : int(into % T);
    x.t0 += turn;
    x.t1 += turn;
    if (x.t0 >= T) {
      x.t0 -= T;
      x.t1 -= T;
    }
  }
  return x;
}

}  // namespace df
