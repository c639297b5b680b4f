// df_paged_attn: attention of the new tokens of a batch of requests over paged caches and over themselves.
//
// Mathematics.  Per row out = sum_k 2^(c s_k - c m) v_k / sum_k 2^(c s_k - c m), c = scale log2(e), in one pass over the keys: m
// is a reference that follows the running maximum of s, and sum and output are rescaled where it moves.  Sums, maxima and
// outputs are held in 32 bits; the weights are rounded to the tensors' type for the second product (the matrix core takes both
// operands in 16 bits), the sum takes them unrounded.
//
// Layout.  The query heads of a key head are taken together: row r of a (request, key head) is query r / G of head
// r % G, so the keys are read once for all of them and a single token of G heads is one tile of rows.  Scores are
// computed transposed, S^T = K Q^T with v_mfma_f32_16x16x32: a lane owns one row (lane % 16) and, because the rows of K are
// dealt to the operand's rows as key_of_operand_row says, its scores are already the second product's operand P^T of
// O^T += V^T P^T.  V^T is read from row-major tiles in LDS with ds_read_b64_tr_b16.
//
// Two kernels.  Few rows (up to 32: single tokens, drafted tokens) are bound by HBM: every wave streams tiles of its own
// through a private ring in LDS and never meets the others until the end.  Many rows are bound by the matrix core: four
// waves of 32 rows share tiles of 64 keys.
//
// Sharing out.  Rows of the same key head read the same keys.  Where these are more than an XCD's L2 holds, its workgroups should read the same
// tiles at about the same time: a workgroup of the second kernel that comes to a unit t tiles after its start begins it at tile t (modulo
// their number) and goes round, and where its span ends within the unit the next workgroup does the rest of the round.  All of them start
// at the same tile, so at any time two places are read, by the workgroups on their first unit and by those past it.  1280x720 chunk: 21 GB
// fetched past the L2s without this, 1.4 GB with it; 2990 -> 2620 us when it came (2230 to 2340 since).  Keys that fit are better read from the first to the last
// (fewer runs of tiles: 390-token frames took 85 us, 89 with turned rounds, before they came down to 68).
//
// Lengths are on the device, so the launch is, too: all workgroups add up the cost of all units (request, key
// head, tile of rows; cost = tiles of keys + a constant), and workgroup w takes the w-th of equal spans of that line.  A
// unit that a span's end cuts leaves partial sums in the workspace; a second kernel puts them together.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "df_paged.h"

namespace df {

typedef unsigned short u16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef u16 u16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) s16x8 lds_s16x8;
typedef const __attribute__((address_space(4))) int const_int;

struct Bf16 {
  static constexpr u16 kExponent = 0x7f80;
  static __device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ unsigned pack(float a, float b) {
    return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{a, b}), bf16x2));
  }
};
struct Fp16 {
  static constexpr u16 kExponent = 0x7c00;
  static __device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ unsigned pack(float a, float b) {
    return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{a, b}), f16x2));
  }
};

struct PagedParams {
  const char *q, *k_cur, *v_cur, *k_pages, *v_pages;
  char *out;
  float *lse;
  const_int *table, *len, *cu, *sink, *win;        // read only: where the index is uniform, with scalar loads
  int64_t q_tok, q_head, kc_head, o_tok, o_head;   // bytes
  int64_t cap_stride;
  unsigned kc_tok;           // bytes
  int B, Hkv, Hq, G;
  Rules rules;
  Divider by_tiles, by_heads;
  int page_log2, n_pages, max_pages;
  int total, max_new;
  int row_tiles;             // tiles of rows of max_new tokens
  int units;                 // B * Hkv * row_tiles
  float c;                   // scale * log2(e)
  float ln_unit;             // natural logarithm of one unit of c * score
  char *ws;
  int whole;                 // 1: no unit is ever cut, there is no second kernel
};

constexpr int kThreads = 256;
__device__ __forceinline__ Request request_of(const PagedParams &p, int b, int h) {
  const int64_t cap = b * p.cap_stride + h;
  return make_request(p.cu[b], p.cu[b + 1], p.len[b], p.sink[cap], p.win[cap], p.total, p.max_new, int64_t(p.max_pages) << p.page_log2);
}

struct Span {
  Line line;
  int index;                 // number of the span
  int64_t begin, end;        // on the line
  int unit;                  // the unit that `begin` lies in, -1: there is no span for this workgroup
  int64_t unit_at;           // where that unit begins
};

__device__ __forceinline__ int64_t least64(int64_t a, int64_t b) { return a < b ? a : b; }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return int64_t(unsigned(__builtin_amdgcn_readfirstlane(int(x)))) | int64_t(__builtin_amdgcn_readfirstlane(int(x >> 32))) << 32;
}

// This workgroup's span.  Every workgroup adds up all units; `lds` is kStaged * 16 bytes of LDS and `scratch` kThreads / 64 + 2 words.  What a unit costs depends on
// four numbers of its (request, key head), which are brought to LDS first, all in one trip to memory: read unit by unit, a thousand units took
// 10 us, and 2500 25.
constexpr int kStaged = 2048;
struct Entry { int n, L, s, w; };
template <int KT, int ROWS>
__device__ __forceinline__ Span my_span(const PagedParams &p, Entry *lds, int64_t *scratch) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int entries = p.B * p.Hkv;
  const bool staged = entries <= kStaged;
  auto load = [&](int e) {
    const int b = p.by_heads.of(e);
    const Request r = request_of(p, b, e - b * p.Hkv);
    return Entry{r.n, r.L, r.s, r.w};
  };
  if (staged) {
#pragma unroll 4
    for (int e = tid; e < entries; e += kThreads) lds[e] = load(e);
    __syncthreads();
  }
  auto cost = [&](int u) {
    if (u >= p.units) return 0;
    const int e = p.by_tiles.of(u), row0 = (u - e * p.row_tiles) * ROWS;
    const Entry x = staged ? lds[e] : load(e);
    if (row0 >= x.n * p.G) return 0;
    Request r;
    r.n = x.n;
    r.L = x.L;
    r.s = x.s;
    r.w = x.w;
    r.held = int(least64(filled_slots(x.L, x.s, x.w), int64_t(p.max_pages) << p.page_log2));
    return kUnitCost + tiles_of<KT>(r, row_range(r, p.rules, row0, ROWS), p.rules.keys).count();
  };
  const int per = (p.units + kThreads - 1) / kThreads;
  int64_t mine = 0;
  for (int i = 0; i < per; ++i) mine += cost(tid * per + i);
  int64_t incl = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(incl, d);
    if (lane >= d) incl += y;
  }
  if (lane == 63) scratch[wave] = incl;
  __syncthreads();
  int64_t base = incl - mine, all = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    const int64_t s = scratch[w];
    if (w < wave) base += s;
    all += s;
  }
  const int wgs = gridDim.x;
  Span sp;
  sp.line = Line::of(uniform(all), wgs);
  const int count = sp.line.count;
  // Workgroups are dealt to the eight XCDs in turn: with a full launch an XCD takes neighbouring spans, which read the same keys.
  sp.index = count == wgs && wgs % 8 == 0 ? int(blockIdx.x % 8) * (wgs / 8) + int(blockIdx.x / 8) : int(blockIdx.x);
  sp.begin = sp.end = sp.unit_at = 0;
  sp.unit = -1;
  if (sp.index >= count) return sp;
  sp.begin = sp.line.begin_of(sp.index);
  sp.end = sp.line.begin_of(sp.index + 1);
  // whose units hold it ...
  if (mine > 0 && sp.begin >= base && sp.begin < base + mine) {
    scratch[kThreads / 64] = tid;
    scratch[kThreads / 64 + 1] = base;
  }
  __syncthreads();
  // ... and which of them, a unit to a lane
  const int u0 = __builtin_amdgcn_readfirstlane(int(scratch[kThreads / 64])) * per;
  int64_t at = uniform(scratch[kThreads / 64 + 1]);
  for (int i = 0; i < per; i += 64) {
    const int c = i + lane < per ? cost(u0 + i + lane) : 0;
    int upto = c;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(upto, d);
      if (lane >= d) upto += y;
    }
    const uint64_t in = __builtin_amdgcn_ballot_w64(c > 0 && sp.begin >= at + upto - c && sp.begin < at + upto);
    if (in) {
      const int l = __builtin_ctzll(in);
      sp.unit = u0 + i + l;
      sp.unit_at = at + __builtin_amdgcn_readlane(upto - c, l);
      break;
    }
    at += __builtin_amdgcn_readlane(upto, 63);
  }
  __syncthreads();                       // the numbers in LDS make room for tiles
  return sp;
}

// Workspace: per span a note of its pieces of cut units, and behind the notes two slots of partial sums each.
struct Note {
  int tail_unit;             // the unit that the span begins and does not end, or -1 (its sums: slot 1)
  int head;                  // piece of a unit that an earlier span begins: 0 none, 1 not its last, 2 its last (slot 0)
};
constexpr int kMaxSpans = 1024;
constexpr size_t kNotesBytes = kMaxSpans * sizeof(Note);

template <int ROWS, int D>
struct PartialSlot {
  static constexpr size_t kFloats = size_t(ROWS) * (D + 2);      // rows of O, then m, then l
  __device__ static float *of(char *ws, int span, int which) {
    return reinterpret_cast<float *>(ws + kNotesBytes) + (size_t(span) * 2 + which) * kFloats;
  }
};

// ---- tiles in LDS ------------------------------------------------------------------------------------------------------------
// A row's 16-byte chunks are stored at places that depend on the row, so that the reads of the operands meet no bank twice: the
// hardware takes the lanes of a ds_read_b128 in groups of 16, {0-3, 12-15, 20-27} and so on, and 256 bytes a cycle.  K: chunk c
// of the row that operand row m reads is at place c ^ m (D = 128, a row is all banks) or c ^ (m >> 1) (D = 64, two rows are).  V:
// the 32 bytes of 16 output columns stay together, and move by the row's place among the eight that one pass reads.
template <int D>
struct Layout {
  static constexpr int ROWB = 2 * D;
  static constexpr int CH = D / 8;                       // chunks of a row
  static constexpr int RPL = 1024 / ROWB;                // rows that one wave's load brings
  static constexpr int LPG = 16 / RPL;                   // loads per group of 16 rows
  __device__ static int k_turn(int row) {
    const int m = (row & 3) | ((row >> 3) & 3) << 2;
    return D == 128 ? m : m >> 1;
  }
  __device__ static int v_turn(int row) {
    const int x = D == 128 ? (row & 3) | ((row >> 3) & 1) << 2 : ((row >> 1) & 1) | ((row >> 3) & 1) << 1;
    return 2 * x;
  }
};
// Key (of 32) that operand row m of block u (of two) holds; the block's scores 4 g + v, u = 0, 1 are then keys 8 g + 4 u + v.
__device__ __forceinline__ int key_of_operand_row(int m, int u) { return 8 * (m >> 2) + 4 * u + (m & 3); }

// The lane, as a value that the compiler does not know from before: what is derived from it is worked out where it is used.  Left to itself the
// compiler works everything out once, keeps more than there are registers, and what it reloads from scratch memory waits for all
// loads on their way, the next tile's among them.
__device__ __forceinline__ int lane_here() {
  int x = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0));
  asm volatile("" : "+v"(x));
  return x;
}

// Workgroup barrier that waits for this wave's LDS traffic only: stores of finished rows stay on their way (with a wait for them a piece took 3 us longer).
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ unsigned lds_address(const void *ptr) { return unsigned(reinterpret_cast<uintptr_t>(ptr)); }

__device__ __forceinline__ unsigned scalar(unsigned x) { return unsigned(__builtin_amdgcn_readfirstlane(int(x))); }

// Where a group of 16 rows comes from (uniform).
struct RowSource {
  const char *k, *v;         // first row
  unsigned bytes;            // addressable bytes (0: none; loads past them write zeros)
};

// 16 rows of K and V into LDS, asynchronously: LPG loads each.  `at` is the LDS address of the K rows, the V rows lie `v_off` behind them.
// The statement is not one of the compiler's loads, so the reads of older tiles do not wait for it; whoever reads the rows waits for
// them by count.  It begins with the wait states that a descriptor written by v_readlane needs, and keeps one instruction
// between a write of m0 and the load that uses it.
template <int D>
__device__ __forceinline__ void load_group(const RowSource &src, const unsigned (&koff)[Layout<D>::LPG], const unsigned (&voff)[Layout<D>::LPG],
                                           unsigned at, unsigned v_at) {
  const uint64_t ka = reinterpret_cast<uint64_t>(src.k), va = reinterpret_cast<uint64_t>(src.v);
  const unsigned bytes = scalar(src.bytes);
  const u32x4 dk = {scalar(unsigned(ka)), scalar(unsigned(ka >> 32) & 0xffffu), bytes, 0x00020000u};
  const u32x4 dv = {scalar(unsigned(va)), scalar(unsigned(va >> 32) & 0xffffu), bytes, 0x00020000u};
  at = scalar(at);
  v_at = scalar(v_at);
  if constexpr (D == 128) {
    asm volatile(
        "s_nop 4\n\t"
        "s_mov_b32 m0, %[at]\n\ts_nop 0\n\tbuffer_load_dwordx4 %[k0], %[dk], 0 offen lds\n\t"
        "s_add_u32 m0, %[at], 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %[k1], %[dk], 0 offen lds\n\t"
        "s_add_u32 m0, %[at], 0x800\n\ts_nop 0\n\tbuffer_load_dwordx4 %[k2], %[dk], 0 offen lds\n\t"
        "s_add_u32 m0, %[at], 0xc00\n\ts_nop 0\n\tbuffer_load_dwordx4 %[k3], %[dk], 0 offen lds\n\t"
        "s_mov_b32 m0, %[vt]\n\ts_nop 0\n\tbuffer_load_dwordx4 %[v0], %[dv], 0 offen lds\n\t"
        "s_add_u32 m0, %[vt], 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %[v1], %[dv], 0 offen lds\n\t"
        "s_add_u32 m0, %[vt], 0x800\n\ts_nop 0\n\tbuffer_load_dwordx4 %[v2], %[dv], 0 offen lds\n\t"
        "s_add_u32 m0, %[vt], 0xc00\n\ts_nop 0\n\tbuffer_load_dwordx4 %[v3], %[dv], 0 offen lds"
        ::[at] "s"(at), [vt] "s"(v_at), [dk] "s"(dk), [dv] "s"(dv), [k0] "v"(koff[0]), [k1] "v"(koff[1]), [k2] "v"(koff[2]),
        [k3] "v"(koff[3]), [v0] "v"(voff[0]), [v1] "v"(voff[1]), [v2] "v"(voff[2]), [v3] "v"(voff[3])
        : "memory", "scc");
  } else {
    asm volatile(
        "s_nop 4\n\t"
        "s_mov_b32 m0, %[at]\n\ts_nop 0\n\tbuffer_load_dwordx4 %[k0], %[dk], 0 offen lds\n\t"
        "s_add_u32 m0, %[at], 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %[k1], %[dk], 0 offen lds\n\t"
        "s_mov_b32 m0, %[vt]\n\ts_nop 0\n\tbuffer_load_dwordx4 %[v0], %[dv], 0 offen lds\n\t"
        "s_add_u32 m0, %[vt], 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 %[v1], %[dv], 0 offen lds"
        ::[at] "s"(at), [vt] "s"(v_at), [dk] "s"(dk), [dv] "s"(dv), [k0] "v"(koff[0]), [k1] "v"(koff[1]), [v0] "v"(voff[0]), [v1] "v"(voff[1])
        : "memory", "scc");
  }
}

// Brings the tiles of a piece to LDS, every STEP-th of them.  Everything about the next 64 of them is worked out at once, a tile to a lane (look_ahead): where its
// rows lie, and what the wave's rows see of it.  A step then reads a lane and shifts some masks.
template <int D, int KT, int GROUPS, int STEP>           // GROUPS of 16 rows that the wave brings of a tile, from its group `grp0` on
struct Feed {
  using L = Layout<D>;
  const PagedParams &p;
  const Request &r;
  const Tiles<KT> &tl;
  const RangeKeys &seen;
  const bool live;           // the wave has rows
  const int grp0, end;       // tile behind the piece's last
  const_int *pages;          // the head's row of the block table
  const int64_t cur;         // byte offset of the request's first new token of the head
  int t, lane;               // the tile that is brought next, and its lane
  unsigned slots[GROUPS];    // per lane: first row of the tile's group, among the head's pages or the request's new tokens
  int keys;                  // per lane: the tile's first key
  uint64_t fresh, whole, seen1, seen2;                   // tiles of new tokens, with all rows, and what is seen of them (two bits)
  bool bad;                  // per lane: a page was no page of the pool

  __device__ __forceinline__ Feed(const PagedParams &p_, const Request &r_, const Tiles<KT> &tl_, const RangeKeys &seen_, bool live_, int b, int h, int grp0_,
                                  int begin, int end_)
      : p(p_), r(r_), tl(tl_), seen(seen_), live(live_), grp0(grp0_), end(end_), pages(p_.table + (int64_t(b) * p_.Hkv + h) * p_.max_pages),
        cur(int64_t(r_.q0) * p_.kc_tok + h * p_.kc_head), t(begin), bad(r_.bad) {
    look_ahead();
  }
  __device__ __forceinline__ void look_ahead() {
    const int mine = t + STEP * lane_here();
    const Place x = place_of(r, tl, mine);
    const bool is = mine < end;
    const int what = live ? int(seen_of(x, KT, seen)) : int(kNoneSeen);
    keys = x.k0;
    fresh = __builtin_amdgcn_ballot_w64(x.is_new);
    whole = __builtin_amdgcn_ballot_w64(is && x.k0 + KT <= x.limit);
    seen1 = __builtin_amdgcn_ballot_w64(what & 1);
    seen2 = __builtin_amdgcn_ballot_w64(what & 2);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int row = x.k0 + 16 * (grp0 + g);
      slots[g] = x.is_new ? row : 0;
      if (is && !x.is_new && row < x.limit) {
        const int page = pages[row >> p.page_log2];
        const bool is_page = unsigned(page) < unsigned(p.n_pages);
        bad |= !is_page;
        slots[g] = is_page ? (unsigned(page) << p.page_log2) + unsigned(row & ((1 << p.page_log2) - 1)) : 0;
      }
    }
    lane = 0;
  }
  __device__ __forceinline__ bool next_is_new() const { return fresh >> lane & 1; }
  __device__ __forceinline__ const char *k_base(bool is_new) const { return is_new ? p.k_cur + cur : p.k_pages; }
  __device__ __forceinline__ const char *v_base(bool is_new) const { return is_new ? p.v_cur + cur : p.v_pages; }
  __device__ __forceinline__ unsigned stride(bool is_new) const { return is_new ? p.kc_tok : unsigned(L::ROWB); }
  // Where the lane's 16 bytes of every load of group g lie behind the group's first row, of rows `stride` bytes apart.
  __device__ __forceinline__ void aim(int g, unsigned stride, unsigned (&ko)[L::LPG], unsigned (&vo)[L::LPG]) const {
    const int me = lane_here();
#pragma unroll
    for (int i = 0; i < L::LPG; ++i) {
      const int in_group = i * L::RPL + me / L::CH, place = (grp0 + g) * 16 + in_group;
      ko[i] = unsigned(in_group) * stride + 16u * unsigned((me % L::CH) ^ L::k_turn(place));
      vo[i] = unsigned(in_group) * stride + 16u * unsigned((me % L::CH) ^ L::v_turn(place));
    }
  }
  // A tile that is under way.
  struct Coming {
    int k0, seen;
    bool is_new;
  };
  __device__ __forceinline__ Coming coming(int at) const {
    return Coming{__builtin_amdgcn_readlane(keys, at), int(seen1 >> at & 1) | int(seen2 >> at & 1) << 1, bool(fresh >> at & 1)};
  }
  // The next tile's rows to LDS, K rows of the tile at `k_to` and V rows at `v_to`; then on to the one behind it.
  __device__ __forceinline__ Coming bring(unsigned k_to, unsigned v_to) {
    const Coming c = coming(lane);
    const char *kb = k_base(c.is_new), *vb = v_base(c.is_new);
    const unsigned apart = stride(c.is_new);
    const int limit = pick(c.is_new, r.n, r.held);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int rows = clamp_int(limit - (c.k0 + 16 * (grp0 + g)), 0, 16);
      const uint64_t at = uint64_t(unsigned(__builtin_amdgcn_readlane(int(slots[g]), lane))) * apart;
      const unsigned bytes = rows > 0 ? unsigned(rows - 1) * apart + L::ROWB : 0;
      unsigned ko[L::LPG], vo[L::LPG];
      aim(g, apart, ko, vo);
      load_group<D>(RowSource{kb + at, vb + at, bytes}, ko, vo, k_to + (grp0 + g) * 16 * L::ROWB, v_to + (grp0 + g) * 16 * L::ROWB);
    }
    on(1);
    return c;
  }
  __device__ __forceinline__ void on(int steps) {
    t += STEP * steps;
    lane += steps;
    if (__builtin_expect(lane == 64 && t < end, 0)) look_ahead();
  }
  // How many steps can be taken, from the tile under way on, in which the tile is one that all rows see and the one behind it, of the kind of the
  // next, has all of its rows.
  __device__ __forceinline__ int steps(const Coming &now) const {
    if (lane == 64) return 0;
    const uint64_t all = ~(seen1 | seen2) << 1, here = uint64_t(1) << lane;
    uint64_t x = (now.seen == kAllSeen ? all | here : all & ~here) & whole & (next_is_new() ? fresh : ~fresh);
    x = ~(x >> lane);
    return x ? __builtin_ctzll(x) : 64;
  }
  // Whether a page of the wave's was none, in any lane.
  __device__ __forceinline__ bool met_bad() const { return __builtin_amdgcn_ballot_w64(bad) != 0; }
};

// ---- one tile of keys against a wave's rows -------------------------------------------------------------------------------------

// What each of a wave's rows sees of the slots (0) and of the new tokens (1), worked out once a piece, in LDS.
template <int ROWS>
struct RowNotes {
  Keys of[2][ROWS];
  __device__ __forceinline__ void fill(const PagedParams &p, const Request &r, int row0) {
    const int lane = threadIdx.x & 63;
    if (lane < ROWS) {
      const int first = p.rules.first_of(min(row0 + lane, r.n * p.G - 1));
      of[0][lane] = row_slots(r, first);
      of[1][lane] = row_fresh(r, p.rules, first);
    }
  }
  __device__ __forceinline__ Keys row(int qb, bool is_new) const { return of[is_new][16 * qb + (lane_here() & 15)]; }
};
// The products of a tile of 64 keys and 32 rows, each as one asm statement (df_paged_tiles.inc; operands on their way from LDS as in the loop over
// tiles): S^T from the lane's first K operand on, O^T from its first V^T operand on.
template <class T, int D>
__device__ __forceinline__ void scores_of(unsigned first, const s16x8 (&q)[D / 32][2], f32x4 (&s)[4][2]);
template <class T, int D>
__device__ __forceinline__ void values_of(unsigned first, const s16x8 (&w)[2][2], f32x4 (&o)[D / 16][2]);

template <class T, int D, int KB, int QB>      // KB blocks of 16 keys, QB blocks of 16 rows
struct Rows {
  static constexpr int KS = D / 32, DB = D / 16;
  static constexpr float kMost = 32768.f;
  static constexpr int kAhead = 4;             // operands on their way from LDS
  s16x8 q[KS][QB];
  f32x4 o[DB][QB];
  float m[QB], minus_mc[QB], l[QB];
  bool all_set;              // every row of the wave has a reference (uniform)

  __device__ __forceinline__ void clear() {
    all_set = false;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      m[qb] = -INFINITY;
      minus_mc[qb] = l[qb] = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // The lane's share of rows row0 + 16 qb + lane % 16; rows behind the request's last repeat it and are not stored.
  __device__ __forceinline__ void load_q(const PagedParams &p, const Request &r, int h, int row0) {
    const int lane = threadIdx.x & 63, g = lane >> 4;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int row = min(row0 + 16 * qb + (lane & 15), r.n * p.G - 1);
      const int i = p.rules.G.of(row), head = h * p.G + row - i * p.G;
      const char *src = p.q + int64_t(r.q0 + i) * p.q_tok + head * p.q_head + 16 * g;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) q[ks][qb] = *reinterpret_cast<const s16x8 *>(src + 64 * ks);
    }
  }

  // Waits for the queries here, so that no wait for them is left in the loop over tiles (where it would also wait for tiles).
  __device__ __forceinline__ void settle() {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) asm volatile("" : "+v"(q[ks][qb]));
  }

  // Where the lane reads K of a tile at `k`: chunk 4 ks + lane / 16 of its operand row, for ks = 0.  (Tiles begin at multiples of 1 KB, so
  // ks turns bits of the address.)
  __device__ __forceinline__ static unsigned k_first(unsigned k) {
    const int lane = lane_here(), row = key_of_operand_row(lane & 15, 0);
    return k + unsigned(row * Layout<D>::ROWB + 16 * ((lane >> 4) ^ Layout<D>::k_turn(row)));
  }

  // S^T: scores of keys 32 (kb / 2) + 8 g + 4 (kb % 2) + v of the lane's quarter g.  kAhead operands are on their way from LDS while
  // the matrix core works: left to itself the compiler reads each right before its use and waits out the latency.
  __device__ __forceinline__ void scores(unsigned k, f32x4 (&s)[KB][QB]) const {
    using L = Layout<D>;
    const unsigned first = k_first(k);
    if constexpr (KB == 4 && QB == 2) return scores_of<T, D>(first, q, s);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const unsigned at = first ^ unsigned(64 * ks);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const s16x8 a = *(const lds_s16x8 *)(uintptr_t)(at + (32 * (kb >> 1) + 4 * (kb & 1)) * L::ROWB);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
          s[kb][qb] = T::mfma(a, q[ks][qb], ks ? s[kb][qb] : f32x4{0.f, 0.f, 0.f, 0.f});
      }
    }
    // the order: kAhead reads, then a read behind every operand's products
    constexpr int OPS = KS * KB, A = OPS < kAhead ? OPS : kAhead;
    __builtin_amdgcn_sched_group_barrier(0x100, A, 0);
#pragma unroll
    for (int i = 0; i < OPS - A; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x8, QB, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x8, A * QB, 0);
  }

  // Scores of keys that a row does not see, and of those before `from`, become minus infinity.  A lane's keys are runs of eight: three bounds make eight bits
  // of them, and a bit takes two instructions.  (With a comparison of every key with every bound, 365 instructions, 390-token frames took 78 us where
  // they take 69; with a branch per key, 112.)
  __device__ __forceinline__ static void hide(const RowNotes<16 * QB> &notes, int k0, bool is_new, int from, f32x4 (&s)[KB][QB]) {
    const int g = lane_here() >> 4;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const Keys x = notes.row(qb, is_new);
#pragma unroll
      for (int ts = 0; ts < KB / 2; ++ts) {
        const int k = k0 + 32 * ts + 8 * g;
        const unsigned bits = eight_keys(x, k) & ~below8(from - k);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const unsigned seen = unsigned(int(bits << (31 - i)) >> 31);
          const float y = s[2 * ts + i / 4][qb][i % 4];  // (a bit_cast of an element itself takes the first one's bits)
          s[2 * ts + i / 4][qb][i % 4] = __builtin_bit_cast(float, (__builtin_bit_cast(unsigned, y) & seen) | (0xff800000u & ~seen));
        }
      }
    }
  }

  // Weights 2^(c s - c m) of row block qb, packed as the second product's operand, and their sum over the lane's keys.
  __device__ __forceinline__ float weigh(const PagedParams &p, const f32x4 (&s)[KB][QB], int qb, s16x8 (&w)[KB / 2][QB]) const {
    f32x4 sum;
#pragma unroll
    for (int ts = 0; ts < KB / 2; ++ts) {
      u32x4 x;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x4 e;
#pragma unroll
        for (int v = 0; v < 4; ++v) e[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * ts + u][qb][v], p.c, minus_mc[qb]));
        sum = ts + u == 0 ? e : sum + e;
        x[2 * u] = T::pack(e[0], e[1]);
        x[2 * u + 1] = T::pack(e[2], e[3]);
      }
      w[ts][qb] = __builtin_bit_cast(s16x8, x);
    }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
  }

  // The reference goes up to the largest score so far.
  __device__ __forceinline__ void raise(const PagedParams &p, const f32x4 (&s)[KB][QB]) {
    bool none = false;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      float t = s[0][qb][0];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int v = 0; v < 4; ++v) t = fmaxf(t, s[kb][qb][v]);
      t = fmaxf(t, __shfl_xor(t, 16));
      t = fmaxf(t, __shfl_xor(t, 32));
      t = fmaxf(t, m[qb]);
      // no score yet: the reference stays, and nothing is scaled by the NaN of inf - inf
      const float scale = t == m[qb] ? 1.f : __builtin_amdgcn_exp2f((m[qb] - t) * p.c);
      m[qb] = t;
      minus_mc[qb] = t == -INFINITY ? 0.f : -(t * p.c);
      l[qb] *= scale;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db][qb] *= scale;
      none |= t == -INFINITY;
    }
    all_set = !__builtin_amdgcn_ballot_w64(none);
  }

  // One tile, or what of it begins at key `from`; `seen` says whether all rows see all of its keys (kAllSeen), all that are there (the rows behind the last
  // key are zeros), or not.  The reference m of a row is the largest score of the tiles up to some tile, not of all: a weight may pass one.  Only where a
  // lane's weights add up to more than 2^15 (fp16 holds weights to 2^16, and sums and outputs stay far from the largest number
  // in 32 bits), and where a row has no reference yet, the wave looks for the maximum, brings what it has to the new reference
  // and weighs the tile again.  That leaves the common tile without a maximum, a comparison per score or a product of the outputs.
  __device__ __forceinline__ void tile(const PagedParams &p, const RowNotes<16 * QB> &notes, unsigned k, unsigned v, int k0, bool is_new, int from, int seen) {
    f32x4 s[KB][QB];
    s16x8 w[KB / 2][QB];
    float sum[QB];
    scores(k, s);
    if (__builtin_expect(seen != kAllSeen, 0)) hide(notes, k0, is_new, from, s);
    constexpr bool kAsm = KB == 4 && QB == 2;
    Values x;
    if constexpr (!kAsm) x = begin_values(v);
    bool over = false;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      sum[qb] = weigh(p, s, qb, w);
      over |= !(sum[qb] <= kMost);
    }
    if (__builtin_expect(!all_set || __builtin_amdgcn_ballot_w64(over), 0)) {
      raise(p, s);
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) sum[qb] = weigh(p, s, qb, w);
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) l[qb] += sum[qb];
    if (__builtin_expect(seen == kSomeHidden && odd_values(v), 0)) odd_products(notes, v, k0, is_new, w);
    else if constexpr (kAsm) values_of<T, D>(v_first(v), w, o);
    else values(x, w);
  }

  // Where the lane reads V^T of a tile at `v`: columns 16 db + lane % 16 of keys 8 g .. 8 g + 3 and, four rows on, the next four.
  __device__ __forceinline__ static unsigned v_first(unsigned v) {
    using L = Layout<D>;
    const int lane = lane_here(), g = lane >> 4, j = lane & 15, row = 8 * g + (j >> 2);
    return v + unsigned(row * L::ROWB + 16 * L::v_turn(row) + 8 * (j & 3));
  }
  __device__ __forceinline__ static s16x8 v_operand(unsigned first, int ts, int db) {
    using L = Layout<D>;
    const unsigned at = (first ^ unsigned(32 * db)) + 32 * ts * L::ROWB;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(at));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(at + 4 * L::ROWB));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }

  // O^T += V^T P^T.  The first kAhead operands may be read before the weights are there (begin), the others follow as many operands ahead of
  // their products.  (The order is the statements': the compiler does not move these reads.)
  static constexpr int kValueOps = KB / 2 * DB, kValuesAhead = kValueOps < kAhead ? kValueOps : kAhead;
  struct Values {
    unsigned first;
    s16x8 a[kValuesAhead];
  };
  __device__ __forceinline__ static Values begin_values(unsigned v) {
    Values x;
    x.first = v_first(v);
#pragma unroll
    for (int i = 0; i < kValuesAhead; ++i) x.a[i] = v_operand(x.first, i / DB, i % DB);
    return x;
  }
  __device__ __forceinline__ void values(Values &x, const s16x8 (&w)[KB / 2][QB]) {
#pragma unroll
    for (int i = 0; i < kValueOps; ++i) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) o[i % DB][qb] = T::mfma(x.a[i % kValuesAhead], w[i / DB][qb], o[i % DB][qb]);
      if (i + kValuesAhead < kValueOps) x.a[i % kValuesAhead] = v_operand(x.first, (i + kValuesAhead) / DB, (i + kValuesAhead) % DB);
    }
  }

  // A weight of zero does not hide an infinity or a NaN from the product.  Where some rows do not see all of a tile (only there) the wave
  // looks for them among the values.  If there are any, the product takes zeros in their place, and each is added to the outputs of the rows that see
  // its key: what an infinity or a NaN times a weight adds.
  __device__ __forceinline__ static bool odd_values(unsigned v) {
    typedef u16 u16x8 __attribute__((ext_vector_type(8)));
    const unsigned first = v + 16u * unsigned(lane_here());
    u16x8 top = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16 * KB * Layout<D>::ROWB / 1024; ++i) {
      const s16x8 x = *(const lds_s16x8 *)(uintptr_t)(first + 1024 * i);
      top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x8, x) & u16(0x7fff));
    }
    u16 most = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) most = most > top[k] ? most : top[k];
    return __builtin_amdgcn_ballot_w64(most >= T::kExponent) != 0;
  }
  __device__ __forceinline__ void odd_products(const RowNotes<16 * QB> &notes, unsigned v, int k0, bool is_new, const s16x8 (&w)[KB / 2][QB]) {
    using L = Layout<D>;
    const unsigned first = v_first(v);
#pragma unroll
    for (int i = 0; i < kValueOps; ++i) {
      s16x8 a = v_operand(first, i / DB, i % DB);
#pragma unroll
      for (int k = 0; k < 8; ++k) a[k] = (u16(a[k]) & T::kExponent) == T::kExponent ? short(0) : a[k];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) o[i % DB][qb] = T::mfma(a, w[i / DB][qb], o[i % DB][qb]);
    }
    const int g = lane_here() >> 4;
    Keys row_sees[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) row_sees[qb] = notes.row(qb, is_new);
#pragma unroll 1
    for (int key = 0; key < 16 * KB; ++key) {
      const unsigned row = v + unsigned(key * L::ROWB);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        // columns 16 db + 4 g .. + 3 of the key's row: half of chunk 2 db + g / 2
        const s16x4 x = *(const lds_s16x4 *)(uintptr_t)(row + 16u * unsigned((2 * db + (g >> 1)) ^ L::v_turn(key)) + 8u * unsigned(g & 1));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool odd = (u16(x[i]) & T::kExponent) == T::kExponent;
          const float f = odd ? ((u16(x[i]) & ~(T::kExponent | 0x8000u)) ? NAN : (u16(x[i]) & 0x8000u) ? -INFINITY : INFINITY) : 0.f;
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) o[db][qb][i] += row_sees[qb].sees(k0 + key) ? f : 0.f;
        }
      }
    }
  }
};

template <class T>
__device__ __forceinline__ void store_row4(const PagedParams &p, const Request &r, int h, int row, int col, f32x4 x) {
  const int i = p.rules.G.of(row), head = h * p.G + row - i * p.G;
  char *dst = p.out + int64_t(r.q0 + i) * p.o_tok + head * p.o_head + 2 * col;
  uint2 y;
  y.x = T::pack(x[0], x[1]);
  y.y = T::pack(x[2], x[3]);
  *reinterpret_cast<uint2 *>(dst) = y;
}
// m and l of a finished row: l = 0 where the row sees nothing.
__device__ __forceinline__ void store_lse(const PagedParams &p, const Request &r, int h, int row, float m, float l) {
  const int i = p.rules.G.of(row), head = h * p.G + row - i * p.G;
  const float log2_sum = m * p.c + __builtin_amdgcn_logf(l);
  p.lse[int64_t(head) * p.total + r.q0 + i] = l == 0.f ? -INFINITY : log2_sum * p.ln_unit;
}

// ---- many rows: four waves of 32 share tiles of 64 keys ---------------------------------------------------------------------------

constexpr int kManyRows = 128, kManyKeys = 64;
constexpr int kL2 = 4 << 20;           // bytes of an XCD's L2

// What the loop over whole tiles that all rows of the wave see needs besides the queries.
template <int D>
struct SeenTiles {
  unsigned k[D / 32], v[D / 16];                         // per lane: LDS addresses of the operands in buffer 0
  unsigned ko[D / 32], vo[D / 32], slots;                // per lane, as in Feed
  unsigned klo, khi, vlo, vhi, stride, bytes;            // row 0 of the run, bytes between rows, bytes of 16 rows
  unsigned to;                                           // LDS address of the wave's K rows in buffer 0
  int buf;                                               // buffer of the first tile
  float c, most;
  __device__ __forceinline__ void place(unsigned lds0, int buf_, int wave, float c_) {
    constexpr int TILE = kManyKeys * Layout<D>::ROWB;
    using R = Rows<Bf16, D, 4, 2>;                       // (the addresses do not depend on the type)
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) k[ks] = R::k_first(lds0) ^ unsigned(64 * ks);
#pragma unroll
    for (int db = 0; db < D / 16; ++db) v[db] = R::v_first(lds0 + TILE) ^ unsigned(32 * db);
    to = scalar(lds0 + wave * 16 * Layout<D>::ROWB);
    buf = scalar(buf_);
    c = c_;
    most = R::kMost;
  }
  template <class F>
  __device__ __forceinline__ void rows_of(const F &f) {
    const bool is_new = f.next_is_new();
    const uint64_t ka = reinterpret_cast<uint64_t>(f.k_base(is_new)), va = reinterpret_cast<uint64_t>(f.v_base(is_new));
    klo = scalar(unsigned(ka));
    khi = scalar(unsigned(ka >> 32));
    vlo = scalar(unsigned(va));
    vhi = scalar(unsigned(va >> 32));
    stride = scalar(f.stride(is_new));
    bytes = scalar(15 * f.stride(is_new) + Layout<D>::ROWB);
    slots = f.slots[0];
    f.aim(0, f.stride(is_new), ko, vo);
  }
};
// Up to n tiles from the one that is on its way to buffer a.buf, each as Rows::tile does it; lane i of a.slots is the tile behind the first.  Returns 0, or
// 1 (2) where the tile of the last step, or its second half, is left to Rows::tile because its weights are too large.
template <class T, int D>
__device__ __forceinline__ int seen_tiles(const SeenTiles<D> &a, const s16x8 (&q)[D / 32][2], f32x4 (&o)[D / 16][2], float (&l)[2], const float (&nm)[2],
                                          int &i, int n);
#include "df_paged_tiles.inc"

template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void df_paged_many_kernel(const PagedParams p) {
  using L = Layout<D>;
  constexpr int KT = kManyKeys, ROWS = kManyRows, TILE = KT * L::ROWB;
  static_assert(kStaged * sizeof(Entry) <= 4 * TILE, "the line's numbers lie where tiles will");
  __shared__ __attribute__((aligned(1024))) char tiles[4 * TILE];      // two buffers of K and V
  __shared__ int64_t scratch[kThreads / 64 + 2];
  __shared__ RowNotes<32> notes[kThreads / 64];
  __shared__ int poison;                 // the last unit of which a page was none
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (tid == 0) poison = -1;
  const Span sp = my_span<KT, ROWS>(p, reinterpret_cast<Entry *>(tiles), scratch);
  Note note{-1, 0};
  const unsigned lds0 = lds_address(tiles);
  int64_t at = sp.unit_at;
  for (int u = max(sp.unit, 0); u < p.units && at < sp.end; ++u) {
    const Unit un = unit_of(u, p.by_tiles, p.by_heads, ROWS);
    const Request r = request_of(p, un.b, un.h);
    if (un.row0 >= r.n * p.G) continue;
    const RowRange x = row_range(r, p.rules, un.row0, ROWS);
    const Tiles<KT> tl = tiles_of<KT>(r, x, p.rules.keys);
    const int nt = tl.count();
    const Piece pc = piece_of(sp.line, sp.begin, sp.end, at, nt, int64_t(nt) * 2 * TILE > kL2);
    const int t0 = pc.t0, t1 = pc.t1;
    at += kUnitCost + nt;
    if (!pc.is) continue;

    Rows<T, D, KT / 16, 2> rows;
    rows.clear();
    const int row0 = un.row0 + 32 * wave;
    if (t0 < t1) {
      const RowRange mine = row_range(r, p.rules, min(row0, r.n * p.G - 1), 32);
      const RangeKeys seen = range_keys(r, mine);
      Feed<D, KT, 1, 1> ld(p, r, tl, seen, row0 < r.n * p.G, un.b, un.h, wave, t0, t1);
      rows.load_q(p, r, un.h, row0);
      auto now = ld.bring(lds0, lds0 + TILE);
      notes[wave].fill(p, r, row0);
      rows.settle();
      unsigned buf = lds0;
      for (int t = t0; t < t1; ++t) {
        unsigned other = buf == lds0 ? lds0 + 2 * TILE : lds0;
        const int n = rows.all_set ? ld.steps(now) : 0;
        int due = 0;
        auto next = now;
        if (n > 0) {
          SeenTiles<D> a;
          a.place(lds0, buf == lds0 ? 0 : 1, wave, p.c);
          a.rows_of(ld);
          int lane_at = scalar(ld.lane);
          due = seen_tiles<T, D>(a, rows.q, rows.o, rows.l, rows.minus_mc, lane_at, scalar(n));
          const int begun = lane_at - ld.lane, done = begun - (due != 0);
          // the tile under way, or the one that is left to be done and the one that is under way behind it
          next = ld.coming(lane_at - 1);
          if (done > 0) now = ld.coming(lane_at - 1 - (due != 0));
          ld.on(begun);
          t += done;
          if (done & 1) {
            buf = other;
            other = buf == lds0 ? lds0 + 2 * TILE : lds0;
          }
        }
        if (!due) {
          // the wave's rows of this tile have landed, and every wave is done with the tile before
          asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
          if (t + 1 < t1) next = ld.bring(other, other + TILE);
        }
        if (now.seen != kNoneSeen)
          rows.tile(p, notes[wave], buf, buf + TILE, now.k0, now.is_new, due == 2 ? now.k0 + KT / 2 : now.k0, due == 2 ? int(kSomeHidden) : now.seen);
        now = next;
        buf = other;
      }
      if (ld.met_bad()) poison = u;
    } else if (r.bad) {
      poison = u;
    }
    lds_barrier();                       // all waves are done with the tiles and have said what pages they met
    const bool nan = poison == u;
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
      float l = rows.l[qb];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      if (nan) l = NAN;
      const int row = row0 + 16 * qb + (lane & 15), g = lane >> 4;
      if (pc.begins && pc.ends) {
        if (row < r.n * p.G) {
          const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
          for (int db = 0; db < L::CH / 2; ++db) store_row4<T>(p, r, un.h, row, 16 * db + 4 * g, rows.o[db][qb] * inv);
          if (p.lse && g == 0) store_lse(p, r, un.h, row, rows.m[qb], l);
        }
      } else {
        float *slot = PartialSlot<ROWS, D>::of(p.ws, sp.index, pc.begins);
        const int in_unit = row - un.row0;
#pragma unroll
        for (int db = 0; db < L::CH / 2; ++db) *reinterpret_cast<f32x4 *>(slot + in_unit * D + 16 * db + 4 * g) = rows.o[db][qb];
        if (g == 0) {
          slot[ROWS * D + in_unit] = rows.m[qb];
          slot[ROWS * (D + 1) + in_unit] = l;
        }
      }
    }
    if (pc.begins && !pc.ends) note.tail_unit = u;
    if (!pc.begins) note.head = pc.ends ? 2 : 1;
    lds_barrier();                       // the poison of this piece has been read, the tiles may be loaded again
  }
  if (!p.whole && tid == 0) reinterpret_cast<Note *>(p.ws)[sp.index] = note;
}

// ---- few rows: every wave streams tiles of its own ----------------------------------------------------------------------------------

constexpr int kFewKeys = 32, kFewWaves = 4;

template <class T, int D, int QB>
__global__ __launch_bounds__(kThreads) void df_paged_few_kernel(const PagedParams p) {
  using L = Layout<D>;
  constexpr int KT = kFewKeys, ROWS = 16 * QB, TILE = KT * L::ROWB, RING = 2;
  constexpr int LOADS = 4 * L::LPG;                                    // loads of a tile, K and V
  __shared__ __attribute__((aligned(1024))) char tiles[kFewWaves][RING][2][TILE];
  __shared__ int64_t scratch[kThreads / 64 + 2];
  __shared__ float stats[kFewWaves][2][ROWS];
  __shared__ RowNotes<ROWS> notes[kFewWaves];
  __shared__ int poison;                 // the last unit of which a page was none
  static_assert(kStaged * sizeof(Entry) <= sizeof(tiles), "the line's numbers lie where tiles will");
  static_assert(sizeof(float) * ROWS * D <= sizeof(tiles[0]), "a wave's sums pass through its tiles");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (tid == 0) poison = -1;
  const Span sp = my_span<KT, ROWS>(p, reinterpret_cast<Entry *>(tiles), scratch);
  Note note{-1, 0};
  const unsigned lds0 = lds_address(&tiles[wave][0][0][0]);
  int64_t at = sp.unit_at;
  for (int u = max(sp.unit, 0); u < p.units && at < sp.end; ++u) {
    const Unit un = unit_of(u, p.by_tiles, p.by_heads, ROWS);
    const Request r = request_of(p, un.b, un.h);
    if (un.row0 >= r.n * p.G) continue;
    const RowRange x = row_range(r, p.rules, un.row0, ROWS);
    const Tiles<KT> tl = tiles_of<KT>(r, x, p.rules.keys);
    const int nt = tl.count();
    const Piece pc = piece_of(sp.line, sp.begin, sp.end, at, nt, false);
    const int t0 = pc.t0, t1 = pc.t1;
    at += kUnitCost + nt;
    if (!pc.is) continue;

    Rows<T, D, 2, QB> rows;
    rows.clear();
    int t = t0 + wave;
    if (t < t1) {
      const RangeKeys seen = range_keys(r, x);
      Feed<D, KT, 2, kFewWaves> ld(p, r, tl, seen, true, un.b, un.h, 0, t, t1);
      rows.load_q(p, r, un.h, un.row0);
      notes[wave].fill(p, r, un.row0);
      auto now = ld.bring(lds0, lds0 + TILE), next = now;
      if (t + kFewWaves < t1) next = ld.bring(lds0 + 2 * TILE, lds0 + 3 * TILE);
      rows.settle();
      for (unsigned buf = lds0; t < t1; t += kFewWaves) {
        // this tile has landed, the next one may still be on its way
        if (t + kFewWaves < t1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (now.seen != kNoneSeen) rows.tile(p, notes[wave], buf, buf + TILE, now.k0, now.is_new, now.k0, now.seen);
        now = next;
        if (t + 2 * kFewWaves < t1) {
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // the reads of this buffer are done
          next = ld.bring(buf, buf + TILE);
        }
        buf = buf == lds0 ? lds0 + 2 * TILE : lds0;
      }
      if (ld.met_bad()) poison = u;
    } else if (r.bad) {
      poison = u;
    }
    // the four waves' sums meet in LDS: references, row sums, outputs
    float *mine = reinterpret_cast<float *>(&tiles[wave][0][0][0]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      float l = rows.l[qb];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      const int row = 16 * qb + (lane & 15), g = lane >> 4;
#pragma unroll
      for (int db = 0; db < L::CH / 2; ++db) *reinterpret_cast<f32x4 *>(mine + row * D + 16 * db + 4 * g) = rows.o[db][qb];
      if (g == 0) {
        stats[wave][0][row] = rows.m[qb];
        stats[wave][1][row] = l;
      }
    }
    lds_barrier();
    const bool nan = poison == u, whole = pc.begins && pc.ends;
    float *slot = PartialSlot<ROWS, D>::of(p.ws, sp.index, pc.begins);
    for (int i = tid; i < ROWS * D / 4; i += kThreads) {
      const int in_unit = i / (D / 4), col = 4 * (i % (D / 4)), row = un.row0 + in_unit;
      if (row >= r.n * p.G) continue;
      float m = stats[0][0][in_unit];
#pragma unroll
      for (int w = 1; w < kFewWaves; ++w) m = fmaxf(m, stats[w][0][in_unit]);
      float l = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) {
        const float mw = stats[w][0][in_unit];
        const float f = mw == m ? 1.f : __builtin_amdgcn_exp2f((mw - m) * p.c);
        l += f * stats[w][1][in_unit];
        o += f * *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(&tiles[w][0][0][0]) + in_unit * D + col);
      }
      if (nan) l = NAN;
      if (whole) {
        store_row4<T>(p, r, un.h, row, col, o * (l == 0.f ? 0.f : 1.f / l));
        if (p.lse && col == 0) store_lse(p, r, un.h, row, m, l);
      } else {
        *reinterpret_cast<f32x4 *>(slot + in_unit * D + col) = o;
        if (col == 0) {
          slot[ROWS * D + in_unit] = m;
          slot[ROWS * (D + 1) + in_unit] = l;
        }
      }
    }
    if (pc.begins && !pc.ends) note.tail_unit = u;
    if (!pc.begins) note.head = pc.ends ? 2 : 1;
    lds_barrier();                       // the tiles may be loaded again
  }
  if (!p.whole && tid == 0) reinterpret_cast<Note *>(p.ws)[sp.index] = note;
}

// ---- cut units ------------------------------------------------------------------------------------------------------------------------

// Workgroup (w, y): if span w begins a unit that it does not end, rows y * RPB ... of it are put together from its slot 1 and slot 0
// of the spans behind it, up to the one that holds the unit's end.  Bound by trips to memory: the end is looked for by 64 lanes at once, and the pieces' references
// and sums are read several at a time, first all references (their largest is the unit's), then the sums.  A piece after the other, one token of 32
// pieces took 12 us.
constexpr int kMergeThreads = 256;

template <class T, int D, int ROWS, int KT>
__global__ __launch_bounds__(kMergeThreads) void df_paged_merge_kernel(const PagedParams p, int spans) {
  constexpr int V = D / 4, RPB = kMergeThreads / V;      // four columns a thread, rows of a workgroup
  const Note *notes = reinterpret_cast<const Note *>(p.ws);
  const int w0 = blockIdx.x, u = notes[w0].tail_unit;
  if (u < 0 || u >= p.units) return;
  int last = w0;
  for (bool found = false; !found && last + 1 < spans;) {
    const int w = last + 1 + (threadIdx.x & 63);
    const uint64_t ends = __builtin_amdgcn_ballot_w64(w < spans && notes[min(w, spans - 1)].head != 1);
    found = ends != 0;
    last = min(last + (found ? 1 + __builtin_ctzll(ends) : 64), spans - 1);
  }
  const Unit un = unit_of(u, p.by_tiles, p.by_heads, ROWS);
  const Request r = request_of(p, un.b, un.h);
  const int in_unit = blockIdx.y * RPB + threadIdx.x / V, row = un.row0 + in_unit, col = 4 * (threadIdx.x % V);
  if (row >= r.n * p.G) return;
  const float *slot = PartialSlot<ROWS, D>::of(p.ws, w0, 1), *head = PartialSlot<ROWS, D>::of(p.ws, 0, 0);
  constexpr size_t kApart = 2 * PartialSlot<ROWS, D>::kFloats;
  const float m0 = slot[ROWS * D + in_unit], l0 = slot[ROWS * (D + 1) + in_unit];
  const f32x4 o0 = *reinterpret_cast<const f32x4 *>(slot + in_unit * D + col);
  float m = m0, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  // REFS references and SUMS pieces of sums are read at once (behind the last: the last again, not counted).
  const auto fold = [&](auto refs, auto sums) {
    constexpr int REFS = decltype(refs)::value, SUMS = decltype(sums)::value;
    for (int w = w0 + 1; w <= last; w += REFS) {
      float x[REFS];
#pragma unroll
      for (int i = 0; i < REFS; ++i) x[i] = head[min(w + i, last) * kApart + ROWS * D + in_unit];
#pragma unroll
      for (int i = 0; i < REFS; ++i) m = fmaxf(m, x[i]);
    }
    const auto share = [&](float x) { return x == m ? 1.f : __builtin_amdgcn_exp2f((x - m) * p.c); };    // (minus infinity: no NaN)
    l = share(m0) * l0;
    o = share(m0) * o0;
    for (int w = w0 + 1; w <= last; w += SUMS) {
      float x[SUMS], l1[SUMS];
      f32x4 o1[SUMS];
#pragma unroll
      for (int i = 0; i < SUMS; ++i) {
        slot = head + min(w + i, last) * kApart;
        x[i] = slot[ROWS * D + in_unit];
        l1[i] = slot[ROWS * (D + 1) + in_unit];
        o1[i] = *reinterpret_cast<const f32x4 *>(slot + in_unit * D + col);
      }
#pragma unroll
      for (int i = 0; i < SUMS; ++i) {
        const bool is = w + i <= last;
        const float f = share(x[i]);
        l = is ? l + f * l1[i] : l;
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = is ? o[k] + f * o1[i][k] : o[k];
      }
    }
  };
  // Units of many rows mostly have two or three pieces, a long history of few rows has dozens (one token of 131072 keys: 14 us with 8 at a
  // time, 7 with these; for a batch of single tokens, which has up to 8 pieces, the larger numbers cost 2 us more than they save).
  if (ROWS != kManyRows && last - w0 > 8) fold(std::integral_constant<int, 32>(), std::integral_constant<int, 16>());
  else fold(std::integral_constant<int, ROWS == kManyRows ? 4 : 8>(), std::integral_constant<int, ROWS == kManyRows ? 4 : 8>());
  store_row4<T>(p, r, un.h, row, col, o * (l == 0.f ? 0.f : 1.f / l));
  if (p.lse && col == 0) store_lse(p, r, un.h, row, m, l);
}

}  // namespace df

using namespace df;

// Which kernel: the rows that max_new tokens make of a key head's query heads decide.  Up to 32 rows the tile of rows is
// one wave's, and streaming the keys bounds the call; beyond, four waves share them.
namespace {
struct Shape {
  int rows, keys;            // of a tile
  int spans;                 // most spans
};
const_int *as_const(const int32_t *x) { return (const_int *)(uintptr_t)x; }
Shape shape_of(int64_t rows) {
  if (rows <= 16) return {16, kFewKeys, 256};
  if (rows <= 32) return {32, kFewKeys, 256};
  return {kManyRows, kManyKeys, 512};
}
bool sizes_ok(int64_t H_q, int64_t H_kv, int64_t d, int64_t max_new) {
  return H_kv > 0 && H_kv <= kMaxHeads && H_q > 0 && H_q % H_kv == 0 && H_q / H_kv <= 64 && (d == 64 || d == 128) && max_new > 0 &&
         max_new * (H_q / H_kv) <= kMaxLen;
}
}  // namespace

extern "C" size_t df_paged_workspace_bytes(int32_t H_q, int32_t H_kv, int32_t d, int32_t max_new) {
  if (!sizes_ok(H_q, H_kv, d, max_new)) return 0;
  const Shape s = shape_of(int64_t(max_new) * (H_q / H_kv));
  return kNotesBytes + size_t(s.spans) * 2 * s.rows * (d + 2) * sizeof(float);
}

namespace {
template <class T, int D>
df_status launch_attn(const PagedParams &p, const Shape &s, hipStream_t stream) {
  const dim3 threads(kThreads);
  if (s.rows == 16)
    hipLaunchKernelGGL((df_paged_few_kernel<T, D, 1>), dim3(s.spans), threads, 0, stream, p);
  else if (s.rows == 32)
    hipLaunchKernelGGL((df_paged_few_kernel<T, D, 2>), dim3(s.spans), threads, 0, stream, p);
  else
    hipLaunchKernelGGL((df_paged_many_kernel<T, D>), dim3(s.spans), threads, 0, stream, p);
  if (df_status st = launch_status()) return st;
  if (p.whole) return DF_OK;
  const int per = kMergeThreads / (D / 4);
  const int rows = int(std::min<int64_t>(s.rows, int64_t(p.max_new) * p.G));
  const dim3 grid(s.spans, (rows + per - 1) / per);
  if (s.rows == 16)
    hipLaunchKernelGGL((df_paged_merge_kernel<T, D, 16, kFewKeys>), grid, dim3(kMergeThreads), 0, stream, p, s.spans);
  else if (s.rows == 32)
    hipLaunchKernelGGL((df_paged_merge_kernel<T, D, 32, kFewKeys>), grid, dim3(kMergeThreads), 0, stream, p, s.spans);
  else
    hipLaunchKernelGGL((df_paged_merge_kernel<T, D, kManyRows, kManyKeys>), grid, dim3(kMergeThreads), 0, stream, p, s.spans);
  return launch_status();
}
}  // namespace

extern "C" df_status df_paged_attn(const df_paged_attn_args *a, void *stream) {
  if (!a) return DF_ERR_NULL;
  if (df_status s = check_paged_cache(a->cache)) return s;
  const df_paged_cache *c = a->cache;
  if (!a->q || !a->out || !a->cu_new || !a->k_cur != !a->v_cur) return DF_ERR_NULL;
  if (a->H_q <= 0 || a->total_new <= 0 || a->max_new <= 0 || a->block <= 0 || a->H_q % c->H_kv) return DF_ERR_SHAPE;
  if (a->H_q / c->H_kv > 64) return DF_ERR_UNSUPPORTED;
  if (a->max_new > a->total_new) return DF_ERR_SHAPE;
  if (!(a->softmax_scale > 0.f) || !std::isfinite(a->softmax_scale * 1.4426950408889634f)) return DF_ERR_RANGE;
  if (a->total_new > kMaxLen || !sizes_ok(a->H_q, c->H_kv, c->d, a->max_new)) return DF_ERR_RANGE;
  if (!aligned16(a->q) || !aligned16(a->out) || !stride_ok(a->q_stride_tok) || !stride_ok(a->o_stride_tok) ||
      (a->H_q > 1 && (!stride_ok(a->q_stride_head) || !stride_ok(a->o_stride_head))))
    return DF_ERR_ALIGN;
  if (a->k_cur && (!aligned16(a->k_cur) || !aligned16(a->v_cur) || !stride_ok(a->kc_stride_tok) ||
                   (c->H_kv > 1 && !stride_ok(a->kc_stride_head))))
    return DF_ERR_ALIGN;
  if (a->k_cur && a->kc_stride_tok > (1 << 26)) return DF_ERR_RANGE;       // 16 rows are addressed by 32 bits
  const int G = a->H_q / c->H_kv;
  const int64_t rows = int64_t(a->max_new) * G;
  const Shape s = shape_of(rows);
  const int64_t row_tiles = (rows + s.rows - 1) / s.rows, units = row_tiles * c->B * c->H_kv;
  if (units > kMaxLen) return DF_ERR_RANGE;
  if (!a->workspace || a->workspace_bytes < df_paged_workspace_bytes(a->H_q, c->H_kv, c->d, a->max_new)) return DF_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(a->workspace) & 255u) return DF_ERR_ALIGN;

  PagedParams p{};
  p.q = static_cast<const char *>(a->q);
  p.k_cur = static_cast<const char *>(a->k_cur);
  p.v_cur = static_cast<const char *>(a->v_cur);
  p.k_pages = static_cast<const char *>(c->k_pages);
  p.v_pages = static_cast<const char *>(c->v_pages);
  p.out = static_cast<char *>(a->out);
  p.lse = a->lse_out;
  p.table = as_const(c->block_table); p.len = as_const(c->len); p.cu = as_const(a->cu_new);
  p.sink = as_const(c->sink_cap); p.win = as_const(c->win_cap);
  p.q_tok = 2 * a->q_stride_tok; p.q_head = 2 * a->q_stride_head;
  p.o_tok = 2 * a->o_stride_tok; p.o_head = 2 * a->o_stride_head;
  p.kc_tok = unsigned(2 * a->kc_stride_tok); p.kc_head = 2 * a->kc_stride_head;
  p.cap_stride = c->cap_stride;
  p.B = c->B; p.Hkv = c->H_kv; p.Hq = a->H_q; p.G = G;
  p.page_log2 = log2_of(c->page_tokens); p.n_pages = c->n_pages; p.max_pages = c->max_pages;
  p.total = a->total_new; p.max_new = a->max_new;
  p.rules = Rules{Divider::by(G), Divider::by(a->block), a->k_cur != nullptr};
  p.row_tiles = int(row_tiles);
  p.units = int(units);
  p.by_tiles = Divider::by(p.row_tiles);
  p.by_heads = Divider::by(c->H_kv);
  p.c = a->softmax_scale * 1.4426950408889634f;
  p.ln_unit = float(double(a->softmax_scale) / double(p.c));
  p.ws = static_cast<char *>(a->workspace);
  // the most tiles that a unit can have: its slots and its new tokens, each in two runs
  const int64_t slots = int64_t(c->max_pages) * c->page_tokens;
  const int64_t most = (slots + s.keys - 1) / s.keys + 1 + (a->k_cur ? (int64_t(a->max_new) + s.keys - 1) / s.keys + 1 : 0);
  p.whole = most <= kMinSpan;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (c->dtype == DF_BF16) return c->d == 128 ? launch_attn<Bf16, 128>(p, s, st) : launch_attn<Bf16, 64>(p, s, st);
  return c->d == 128 ? launch_attn<Fp16, 128>(p, s, st) : launch_attn<Fp16, 64>(p, s, st);
}
