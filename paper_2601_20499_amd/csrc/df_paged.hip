// df_page_map / df_paged_append: pages, block tables and slots of a batch of requests, all from lengths in device
// memory, and the rows that go into them.
//
// df_page_map.  need(b, h) = pages after the step - pages before it; an exclusive sum over (request, head) says which
// free pages a head takes.  Latency bounds it: a few KB are read, and the sum, the check of the whole step (all or
// nothing) and the writes depend on each other, so one workgroup does all of it between barriers, and no other
// workgroup or launch has to agree on anything (64 requests of 8 heads: 6.3 us, of which an empty launch is 2.4).
// Only the slot map (8 bytes per token and head) can be large; from kFusedSlots entries on a second kernel writes it
// with the whole device, below that the same workgroup does.
//
// df_paged_append.  A row mover like df_rows_kernel, bound by HBM; destinations come from the slot map.
#include "df_paged.h"

namespace df {

constexpr int kMapThreads = 1024;
constexpr int kMapWaves = kMapThreads / 64;
constexpr int kFusedSlots = 8192;
constexpr int kCuInLds = 4096;           // requests whose offsets are bisected in LDS

struct MapParams {
  int *table;
  const int *len, *sink, *win, *cu;
  const unsigned char *release;
  int *free_pages;
  const int *n_free;
  int64_t *slots;
  int *len_out, *n_free_out, *status;
  int64_t cap_stride;
  int B, H, n_pages, max_pages, page_log2, total;
  int fused;                 // 1: the slot map is this kernel's as well
};

struct HeadPages {
  int before, after;         // pages held before and after the step (a released request: 0 before)
  int released;              // pages a released request gives back
  bool bad;
};

__device__ __forceinline__ HeadPages head_pages(const MapParams &p, int e) {
  const int b = e / p.H, h = e - b * p.H;
  const int64_t cap = b * p.cap_stride + h;
  const int len = p.len[b], sink = p.sink[cap], win = p.win[cap];
  const int c0 = p.cu[b], c1 = p.cu[b + 1];
  const bool rel = p.release && p.release[b];
  HeadPages r{0, 0, 0, false};
  r.bad = unsigned(len) >= unsigned(kMaxLen) || unsigned(sink) > unsigned(kMaxLen) || unsigned(win) > unsigned(kMaxLen) || c0 < 0 ||
          c1 < c0 || c1 > p.total;
  if (r.bad) return r;
  const int n = c1 - c0, from = rel ? 0 : len;
  if (n >= kMaxLen - from) { r.bad = true; return r; }
  // round up in 32 unsigned bits: at most 2^31 slots
  const unsigned up = (1u << p.page_log2) - 1u;
  const int held = int((unsigned(filled_slots(len, sink, win)) + up) >> p.page_log2);
  r.released = rel ? held : 0;
  r.before = rel ? 0 : held;
  r.after = int((unsigned(filled_slots(from + n, sink, win)) + up) >> p.page_log2);
  r.bad = held > p.max_pages || r.after > p.max_pages;
  return r;
}

// Exclusive sum over the workgroup, and the total (in 64 bits: only once they are checked do the sums fit into 32).
__device__ __forceinline__ int64_t exclusive_sum(int64_t x, int64_t *wave_sums, int64_t &total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t incl = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(incl, d);
    if (lane >= d) incl += y;
  }
  __syncthreads();                       // the last use of wave_sums is over
  if (lane == 63) wave_sums[wave] = incl;
  __syncthreads();
  int64_t base = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kMapWaves; ++w) {
    const int64_t s = wave_sums[w];
    if (w < wave) base += s;
    total += s;
  }
  return base + incl - x;
}

// Slot of (token t of the batch, head h): the request by bisection of cu, which lies in LDS or in memory.
template <class Cu>
__device__ __forceinline__ int64_t slot_for(const MapParams &p, const Cu &cu, int t, int h, bool len_is_new) {
  if (t < cu[0] || t >= cu[p.B]) return -1;
  int lo = 0, hi = p.B;                  // cu[lo] <= t < cu[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= t) lo = mid; else hi = mid;
  }
  const int b = lo, c0 = cu[b], n = cu[b + 1] - c0;
  // len_out holds the new lengths by now, and may be the array that held the old ones
  const int after = len_is_new ? p.len_out[b] : p.len[b] + n;
  const int64_t cap = b * p.cap_stride + h;
  const int sink = p.sink[cap], win = p.win[cap], j = after - n + (t - c0);
  if (j >= sink && (win == 0 || j < after - win)) return -1;
  const int slot = slot_of(j, sink, win);
  const int page = p.table[(int64_t(b) * p.H + h) * p.max_pages + (slot >> p.page_log2)];
  return (int64_t(page) << p.page_log2) + (slot & ((1 << p.page_log2) - 1));
}

// First what all entries (request, head) need is added up, and whether the step can be done; then pages are handed out,
// kMapThreads entries at a time.  Their pages form a line, cut where the exclusive sums in LDS say, and the threads take
// the line's positions one after the other, so that one head that grows by thousands of pages costs no more than
// thousands that grow by one.
__global__ __launch_bounds__(kMapThreads) void df_page_map_kernel(const MapParams p) {
  __shared__ int64_t wave_sums[kMapWaves];
  __shared__ int line[kMapThreads + 1], first_new[kMapThreads];
  __shared__ int bad_flag, cu_lds[kCuInLds + 1];
  const int tid = threadIdx.x, E = p.B * p.H;
  const bool in_lds = p.fused && p.B <= kCuInLds;        // (read below, behind barriers)
  if (in_lds)
    for (int b = tid; b <= p.B; b += kMapThreads) cu_lds[b] = p.cu[b];
  const int have = *p.n_free;
  if (tid == 0) bad_flag = 0;
  bool bad = have < 0 || have > p.n_pages || p.cu[0] < 0;
  int64_t need = 0, back = 0;
  HeadPages mine{0, 0, 0, false};
  for (int e = tid; e < E; e += kMapThreads) {
    mine = head_pages(p, e);
    bad |= mine.bad;
    need += mine.after > mine.before ? mine.after - mine.before : 0;
    back += mine.released;
  }
  int64_t need_all, back_all = 0;
  const int64_t need_before = exclusive_sum(need, wave_sums, need_all);
  if (p.release) exclusive_sum(back, wave_sums, back_all);
  bad |= need_all > have + back_all || have + back_all > p.n_pages;
  // what is taken from the stack as it is has to be pages
  if (!bad)
    for (int64_t i = max(have + back_all - need_all, int64_t(0)) + tid; i < have; i += kMapThreads)
      bad |= unsigned(p.free_pages[i]) >= unsigned(p.n_pages);
  if (bad) bad_flag = 1;
  __syncthreads();
  bool ok = !bad_flag;

  // kCheck: what is given back has to be pages; kGive: it goes onto the stack; kTake: pages off the stack into the table
  enum { kCheck, kGive, kTake, kDone };
  const int top = have + int(back_all);
  for (int pass = !ok ? kDone : back_all ? kCheck : kTake; pass != kDone;) {
    for (int e0 = 0, base = 0; e0 < E; e0 += kMapThreads) {
      const int e = e0 + tid;
      HeadPages hp{0, 0, 0, false};
      if (e < E) hp = E <= kMapThreads ? mine : head_pages(p, e);
      int64_t count = need_all;
      const int n = pass != kTake ? hp.released : hp.after > hp.before ? hp.after - hp.before : 0;
      line[tid] = int(pass == kTake && E <= kMapThreads ? need_before : exclusive_sum(n, wave_sums, count));
      first_new[tid] = hp.before;
      if (tid == 0) line[kMapThreads] = int(count);
      __syncthreads();
      for (int i = tid; i < int(count); i += kMapThreads) {
        int lo = 0, hi = kMapThreads;    // line[lo] <= i < line[hi], the last such lo: entries of no pages are passed over
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (line[mid] <= i) lo = mid; else hi = mid;
        }
        const int k = i - line[lo];
        int *row = p.table + int64_t(e0 + lo) * p.max_pages;
        if (pass == kCheck) {
          if (unsigned(row[k]) >= unsigned(p.n_pages)) bad_flag = 1;
        } else if (pass == kGive) {
          p.free_pages[have + base + i] = row[k];
        } else {
          row[first_new[lo] + k] = p.free_pages[top - 1 - (base + i)];
        }
      }
      base += int(count);
      __syncthreads();                   // other threads read what was written; the line is written again
    }
    if (pass == kCheck && bad_flag) { ok = false; break; }
    ++pass;
  }
  // old lengths and the old count are read for the last time before any new one is written (the arrays may be the same)
  __syncthreads();
  for (int b = tid; b < p.B; b += kMapThreads) {
    const int len = p.len[b];
    p.len_out[b] = ok ? (p.release && p.release[b] ? 0 : len) + p.cu[b + 1] - p.cu[b] : len;
  }
  if (tid == 0) {
    *p.n_free_out = ok ? int(have + back_all - need_all) : have;
    *p.status = ok ? DF_OK : DF_ERR_RANGE;
  }
  if (!p.fused) return;
  __syncthreads();
  for (int i = tid; i < p.total * p.H; i += kMapThreads) {
    const int t = i / p.H, h = i - t * p.H;
    p.slots[i] = !ok ? -1 : in_lds ? slot_for(p, cu_lds, t, h, true) : slot_for(p, p.cu, t, h, true);
  }
}

constexpr int kSlotThreads = 256;
constexpr int kSlotsPerBlock = 1024;

__global__ __launch_bounds__(kSlotThreads) void df_slot_kernel(const MapParams p) {
  __shared__ int cu_lds[kCuInLds + 1];
  const bool ok = *p.status == DF_OK, in_lds = p.B <= kCuInLds;
  if (in_lds)
    for (int b = threadIdx.x; b <= p.B; b += kSlotThreads) cu_lds[b] = p.cu[b];
  __syncthreads();
  const int64_t all = int64_t(p.total) * p.H;
#pragma unroll
  for (int it = 0; it < kSlotsPerBlock / kSlotThreads; ++it) {
    const int64_t i = int64_t(blockIdx.x) * kSlotsPerBlock + it * kSlotThreads + threadIdx.x;
    if (i < all) {
      const int t = int(i / p.H), h = int(i - int64_t(t) * p.H);
      p.slots[i] = !ok ? -1 : in_lds ? slot_for(p, cu_lds, t, h, true) : slot_for(p, p.cu, t, h, true);
    }
  }
}

typedef unsigned vec16 __attribute__((ext_vector_type(4)));   // one 128-bit access

struct PutParams {
  const vec16 *src_k, *src_v;
  vec16 *dst_k, *dst_v;
  int64_t stride_tok, stride_head;       // in 16-byte units
  const int64_t *slots;
  int64_t n_slots;                       // of the pool
  int64_t n_vec;                         // 16-byte vectors of the batch's keys
  int H;
};

constexpr int kPutThreads = 256;
constexpr int kPutVecs = 2;              // per thread, of the keys and of the values

template <int RV>                        // 16-byte vectors per row
__global__ __launch_bounds__(kPutThreads) void df_put_kernel(const PutParams p) {
  const vec16 *__restrict__ src = blockIdx.y ? p.src_v : p.src_k;
  vec16 *__restrict__ dst = blockIdx.y ? p.dst_v : p.dst_k;
  vec16 val[kPutVecs];
  int64_t to[kPutVecs];
#pragma unroll
  for (int it = 0; it < kPutVecs; ++it) {
    const int64_t v = int64_t(blockIdx.x) * (kPutThreads * kPutVecs) + it * kPutThreads + threadIdx.x;
    const int64_t row = v / RV;
    const int col = int(v - row * RV);
    to[it] = -1;
    if (v < p.n_vec) {
      const int64_t slot = p.slots[row];
      if (uint64_t(slot) < uint64_t(p.n_slots)) {
        const int64_t t = row / p.H;
        val[it] = src[t * p.stride_tok + (row - t * p.H) * p.stride_head + col];
        to[it] = slot * RV + col;
      }
    }
  }
#pragma unroll
  for (int it = 0; it < kPutVecs; ++it)
    if (to[it] >= 0) __builtin_nontemporal_store(val[it], &dst[to[it]]);
}

}  // namespace df

using namespace df;

extern "C" df_status df_page_map(const df_page_map_args *a, void *stream) {
  if (!a) return DF_ERR_NULL;
  if (df_status s = check_paged_cache(a->cache)) return s;
  const df_paged_cache *c = a->cache;
  if (a->total_new < 0) return DF_ERR_SHAPE;
  if (!c->free_pages || !c->n_free || !a->cu_new || !a->len_out || !a->n_free_out || !a->status) return DF_ERR_NULL;
  if (a->total_new > 0 && !a->slot_map) return DF_ERR_NULL;
  if (a->total_new > kMaxLen) return DF_ERR_RANGE;
  MapParams p{};
  p.table = c->block_table;
  p.len = c->len; p.sink = c->sink_cap; p.win = c->win_cap; p.cu = a->cu_new;
  p.release = a->release;
  p.free_pages = c->free_pages; p.n_free = c->n_free;
  p.slots = a->slot_map;
  p.len_out = a->len_out; p.n_free_out = a->n_free_out; p.status = a->status;
  p.cap_stride = c->cap_stride;
  p.B = c->B; p.H = c->H_kv; p.n_pages = c->n_pages; p.max_pages = c->max_pages;
  p.page_log2 = log2_of(c->page_tokens);
  p.total = a->total_new;
  const int64_t slots = int64_t(a->total_new) * c->H_kv, blocks = (slots + kSlotsPerBlock - 1) / kSlotsPerBlock;
  if (blocks * kSlotThreads > UINT32_MAX) return DF_ERR_RANGE;             // before anything is launched
  p.fused = slots < kFusedSlots;
  hipLaunchKernelGGL(df_page_map_kernel, dim3(1), dim3(kMapThreads), 0, static_cast<hipStream_t>(stream), p);
  if (df_status s = launch_status()) return s;
  if (!p.fused) {
    hipLaunchKernelGGL(df_slot_kernel, dim3(unsigned(blocks)), dim3(kSlotThreads), 0,
                       static_cast<hipStream_t>(stream), p);
    return launch_status();
  }
  return DF_OK;
}

extern "C" df_status df_paged_append(const df_paged_append_args *a, void *stream) {
  if (!a) return DF_ERR_NULL;
  if (df_status s = check_paged_cache(a->cache)) return s;
  const df_paged_cache *c = a->cache;
  if (a->total_new < 0) return DF_ERR_SHAPE;
  if (a->total_new == 0) return DF_OK;
  if (!a->k_new || !a->v_new || !a->slot_map) return DF_ERR_NULL;
  if (!aligned16(a->k_new) || !aligned16(a->v_new) || !stride_ok(a->stride_tok) || (c->H_kv > 1 && !stride_ok(a->stride_head)))
    return DF_ERR_ALIGN;
  PutParams p{};
  p.src_k = static_cast<const vec16 *>(a->k_new);
  p.src_v = static_cast<const vec16 *>(a->v_new);
  p.dst_k = static_cast<vec16 *>(c->k_pages);
  p.dst_v = static_cast<vec16 *>(c->v_pages);
  p.stride_tok = a->stride_tok / 8;
  p.stride_head = a->stride_head / 8;
  p.slots = a->slot_map;
  p.n_slots = int64_t(c->n_pages) * c->page_tokens;
  p.H = c->H_kv;
  p.n_vec = int64_t(a->total_new) * c->H_kv * (c->d / 8);
  const int64_t blocks = (p.n_vec + kPutThreads * kPutVecs - 1) / (kPutThreads * kPutVecs);
  if (blocks * kPutThreads > UINT32_MAX) return DF_ERR_RANGE;              // a launch counts its threads in 32 bits
  const dim3 grid(unsigned(blocks), 2);
  if (c->d == 128)
    hipLaunchKernelGGL((df_put_kernel<16>), grid, dim3(kPutThreads), 0, static_cast<hipStream_t>(stream), p);
  else
    hipLaunchKernelGGL((df_put_kernel<8>), grid, dim3(kPutThreads), 0, static_cast<hipStream_t>(stream), p);
  return launch_status();
}
