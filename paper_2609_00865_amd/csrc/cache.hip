// The page operators of a live view's cache: room for new rows, forks,
// compaction after an edit, release.  The state (page table, lengths, the
// number of holders of each page) lives on the device, so a call is one or
// two launches and no copy to or from the host.
//
// Which pages a call takes must not depend on timing: the new pages are the
// lowest-numbered free ones in entry order, found by one block that scans the
// holder counts from a hint (no page below it is free) with prefix sums.
// Everything that grows with the data (rows moved, tables copied, holders
// counted up or down) runs over many blocks; the counts are integers, so the
// order of their atomics does not show.
//
// The move is bound by memory (16 spans out of 32768 rows of 8 layers, 4 heads
// of 128: 620 MB in 110 to 127 us, at or above a large copy's 4.9 TB/s), the others are
// chains of dependent reads and barriers: reserve 6.8 us (16 sequences), plan 6.2
// (32 forks) and 5.1 (the edit above), release 4.8 (32 sequences) and 7.1 (one of
// 2048 pages), move 5.2 (the part-filled pages of 32 forks).  These are of pools
// of a round or two of the search (4096 pages each): with the free pages behind
// 65536 or 250000 held ones a reservation takes 19 or 53 us.  A wave fills the
// slots of an entry, so a prompt's 32768 rows take 71 us, and a row that moves
// walks its entry's spans, so many of one row each cost more than the bytes (the
// edit above into a branch: 0.21 ms with 16, 4.3 ms with 4096).
#include "mv_cache_dev.h"

namespace mv {

constexpr int kPlan = 1024;   // threads of the planning blocks
constexpr int kMaxSeqs = MV_CACHE_MAX_SEQS;
constexpr int kTogether = 16;  // entries up to which a plan's threads share each one's pages

__global__ __launch_bounds__(256) void cache_reset_kernel(CacheDev a) {
  const int64_t n = int64_t(a.n_seqs) * a.max_pages;
  const int64_t step = int64_t(gridDim.x) * 256;
  const int64_t i0 = int64_t(blockIdx.x) * 256 + threadIdx.x;
  for (int64_t i = i0; i < n; i += step) a.table[i] = -1;
  for (int64_t i = i0; i < a.n_pages; i += step) a.refs[i] = 0;
  for (int64_t i = i0; i < a.n_seqs; i += step) a.len[i] = 0;
  if (i0 < 4) a.ctl[i0] = 0;
}

// ctl[kCtlFree] = free pages (one block)
__global__ __launch_bounds__(kPlan) void cache_count_kernel(CacheDev a) {
  __shared__ int tmp[kPlan / 64 + 1];
  int c = 0, total;
  for (int64_t i = threadIdx.x; i < a.n_pages; i += kPlan) c += a.refs[i] == 0;
  block_scan<kPlan>(c, tmp, total);
  if (threadIdx.x == 0) a.ctl[kCtlFree] = total;
}

__global__ void cache_clear_counts_kernel(CacheDev a) {
  a.ctl[kCtlNoPages] = 0;
  a.ctl[kCtlBad] = 0;
}

// The holder counts of 4 pages per thread from `base` on (1 past the pool).
__device__ __forceinline__ int4 refs_at(const CacheDev& a, int64_t base) {
  const int64_t p = base + 4 * threadIdx.x;
  if (p + 3 < a.n_pages) return *reinterpret_cast<const int4*>(a.refs + p);
  int4 r = make_int4(1, 1, 1, 1);
  if (p < a.n_pages) r.x = a.refs[p];
  if (p + 1 < a.n_pages) r.y = a.refs[p + 1];
  if (p + 2 < a.n_pages) r.z = a.refs[p + 2];
  return r;
}

// Where the search for free pages begins, and what it sees first: read when a
// block starts, so that these loads wait beside those of the entries.
struct Search {
  int64_t base;
  int4 refs;
  __device__ __forceinline__ explicit Search(const CacheDev& a)
      : base(max(0, a.ctl[kCtlHint]) & ~3), refs(refs_at(a, base)) {}
  // Waits for them: where they are used the wait would also be for every store
  // made by then.
  __device__ __forceinline__ void settle() {
    asm volatile("" : "+v"(refs.x), "+v"(refs.y), "+v"(refs.z), "+v"(refs.w));
  }
};

// The last e with pre[e] <= q, of n >= 1 ascending prefix sums (pre[0] = 0),
// for four q at a time: their look-ups in LDS are unconditional, so they wait
// together (by themselves, a plan of 32 forks took 0.3 us longer).
__device__ __forceinline__ void entries_of(const int* pre, int n, const int (&q)[4],
                                           int (&e)[4]) {
#pragma unroll
  for (int u = 0; u < 4; ++u) e[u] = 0;
  for (int step = 1 << (31 - __clz(n)); step; step >>= 1) {
    int p[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) p[u] = pre[min(e[u] + step, n)];   // (pre[n] is the sum: past any q)
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (e[u] + step < n && p[u] <= q[u]) e[u] += step;
  }
}

// Deals the lowest `need` free pages to the n entries that pre divides:
// take(q, entry, page) for q = 0, 1, ...; returns how many there were (at most
// need).  Every thread of the block calls it; the hint is moved past the last
// page dealt.  (What take() stores is not waited for.)
template <typename F>
__device__ __forceinline__ int deal_pages(const CacheDev& a, const int* pre, int n, int need,
                                          const Search& from, int* tmp, F take) {
  int found = 0;
  int64_t base = from.base;
  int4 r = from.refs;
  while (found < need && base < a.n_pages) {
    const int f[4] = {r.x == 0, r.y == 0, r.z == 0, r.w == 0};
    int total;
    int q[4], e[4];
    q[0] = found + block_scan<kPlan>(f[0] + f[1] + f[2] + f[3], tmp, total);
#pragma unroll
    for (int u = 1; u < 4; ++u) q[u] = q[u - 1] + f[u - 1];
    if (q[0] < need && (f[0] | f[1] | f[2] | f[3])) {
      entries_of(pre, n, q, e);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (!f[u] || q[u] >= need) continue;
        const int page = int(base) + 4 * threadIdx.x + u;
        take(q[u], e[u], page);
        if (q[u] == need - 1) a.ctl[kCtlHint] = page + 1;
      }
    }
    found = min(need, found + total);
    base += 4 * kPlan;
    if (found < need && base < a.n_pages) r = refs_at(a, base);
  }
  if (found < need && threadIdx.x == 0) a.ctl[kCtlHint] = a.n_pages;
  return found;
}

// --------------------------------------------------------------------------
// reserve: one block
// --------------------------------------------------------------------------
struct Grow {   // what entry e asks for
  int s, rows, len, have, need, r0;
  bool bad, over;   // malformed; more rows than the table can hold
};

// Entry e's words and its sequence's length, as read
struct GrowIn {
  int s, r0, r1, len;
  GrowIn() = default;
  __device__ __forceinline__ GrowIn(const CacheDev& a, const int32_t* ids, const int32_t* ptr,
                                    int e)
      : s(ids[e]), r0(ptr[e]), r1(ptr[e + 1]),
        len(unsigned(s) < unsigned(a.n_seqs) ? a.length(s) : 0) {}
};

__device__ __forceinline__ Grow grow_of(const CacheDev& a, const GrowIn& in, int n_new,
                                        const int* claim, int e) {
  Grow g{};
  g.s = in.s;
  g.r0 = in.r0;
  const bool inside = unsigned(g.s) < unsigned(a.n_seqs);
  g.bad = in.r0 < 0 || in.r1 < in.r0 || in.r1 > n_new || (!inside && g.s != -1) ||
          (inside && claim[g.s] != e);
  if (g.bad || !inside) return g;
  g.rows = in.r1 - in.r0;
  g.len = in.len;
  g.have = a.pages_of(g.len);
  const int64_t want = (int64_t(g.len) + g.rows + (1 << a.psl) - 1) >> a.psl;
  g.over = want > a.max_pages;
  if (g.over) g.rows = 0;
  g.need = g.over ? 0 : int(want) - g.have;
  return g;
}

__global__ __launch_bounds__(kPlan) void cache_reserve_kernel(CacheDev a, int n,
                                                              const int32_t* __restrict__ ids,
                                                              const int32_t* __restrict__ ptr,
                                                              int n_new, int32_t* __restrict__ slot,
                                                              int32_t* __restrict__ pos) {
  __shared__ int claim[kMaxSeqs];
  __shared__ int pre[kMaxSeqs + 1];
  __shared__ Grow grow[kPlan];          // of the kPlan entries at hand
  __shared__ int tmp[kPlan / 64 + 1];
  __shared__ int cnt[2], cut_e;
  const int tid = threadIdx.x;
  const GrowIn in = n > 0 ? GrowIn(a, ids, ptr, min(tid, n - 1)) : GrowIn{};
  Search from(a);
  for (int64_t t = tid; t < n_new; t += kPlan) {
    slot[t] = -1;
    if (pos) pos[t] = -1;
  }
  for (int s = tid; s < a.n_seqs; s += kPlan) claim[s] = n;
  if (tid == 0) cnt[0] = cnt[1] = 0, cut_e = -1;
  lds_barrier();
  for (int e = tid; e < n; e += kPlan) {
    const int x = e == tid ? in.s : ids[e];
    if (unsigned(x) < unsigned(a.n_seqs)) atomicMin(&claim[x], e);
  }
  lds_barrier();
  from.settle();
  int need = 0;
  for (int e0 = 0; e0 < n; e0 += kPlan) {
    const int e = e0 + tid;
    Grow g{};
    int total;
    if (e < n) {
      g = grow_of(a, e0 == 0 ? in : GrowIn(a, ids, ptr, e), n_new, claim, e);
      if (g.bad) atomicAdd(&cnt[1], 1);
      if (g.over) atomicAdd(&cnt[0], 1);
    }
    if (e0 == 0) grow[tid] = g;
    const int before = need + block_scan<kPlan>(g.need, tmp, total);
    if (e < n) pre[e] = before;
    need += total;   // at most the table's entries: sequences are named once
  }
  if (tid == 0) pre[n] = need;
  lds_barrier();
  const int found = deal_pages(a, pre, n, need, from, tmp, [&](int q, int e, int page) {
    const int s = e < kPlan ? grow[e].s : ids[e];
    const int have = e < kPlan ? grow[e].have : a.pages_of(a.length(s));
    a.table[int64_t(s) * a.max_pages + have + q - pre[e]] = page;
    a.refs[page] = 1;
  });
  __syncthreads();   // table entries dealt, slots cleared
  if (found < need) {
    // the one entry that some but not all of its pages were dealt to
    for (int e = tid; e < n; e += kPlan) {
      if (pre[e + 1] > found && pre[e + 1] > pre[e]) {
        atomicAdd(&cnt[0], 1);
        if (pre[e] < found) cut_e = e;
      }
    }
    __syncthreads();
    if (cut_e >= 0) {
      const int s = ids[cut_e];
      int32_t* row = a.table + int64_t(s) * a.max_pages + a.pages_of(a.length(s));
      for (int j = tid; j < found - pre[cut_e]; j += kPlan) {
        if (j == 0) a.ctl[kCtlHint] = row[0];
        a.refs[row[j]] = 0;
        row[j] = -1;
      }
    }
    __syncthreads();
  }
  // the rows and new lengths of accepted entries, a wave to an entry
  const int lane = tid & 63, mask = (1 << a.psl) - 1;
  for (int e0 = 0; e0 < n; e0 += kPlan) {
    if (e0 > 0) {
      __syncthreads();
      if (e0 + tid < n)
        grow[tid] = grow_of(a, GrowIn(a, ids, ptr, e0 + tid), n_new, claim, e0 + tid);
      __syncthreads();
    }
    for (int e = e0 + (tid >> 6); e < min(n, e0 + kPlan); e += kPlan / 64) {
      const Grow g = grow[e - e0];
      if (g.rows == 0 || (g.need > 0 && pre[e + 1] > found)) continue;
      for (int i = lane; i < g.rows; i += 64) {
        const int r = g.len + i;
        slot[g.r0 + i] = (a.page(g.s, r >> a.psl) << a.psl) + (r & mask);
        if (pos) pos[g.r0 + i] = r;
      }
      if (lane == 0) a.len[g.s] = g.len + g.rows;
    }
  }
  if (tid == 0) {
    a.ctl[kCtlNoPages] += cnt[0];
    a.ctl[kCtlBad] += cnt[1];
  }
}

// --------------------------------------------------------------------------
// fork and compact: a plan by one block, then moves and table updates by many
// --------------------------------------------------------------------------
struct MoveRec {   // entry e, as planned
  int src, dst;
  int ok;          // 0: refused
  int len, new_len;
  int keep;        // pages that stay (dst == src) or are shared
  int n_new;       // new pages behind them
  int span0, n_spans;
  int old_pages;   // pages of src
};

struct MoveWs {
  int* head;       // [4]: new pages dealt
  MoveRec* rec;    // [n]
  int* off;        // [n]: its new pages' first place in the list of them
  int2* fresh;     // [min(n * max_pages, n_pages)] (page, entry)
  int* old;        // [n * max_pages]: pages from `keep` on of a source compacted in place
};

static size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

static size_t move_ws(const mv_cache_shape& s, int n, char* base, MoveWs* w) {
  const size_t tables = size_t(n) * s.max_pages;
  const size_t fresh = std::min(tables, size_t(s.n_pages));
  size_t at = 0;
  auto put = [&](size_t bytes) {
    char* p = base + at;
    at += up256(bytes);
    return p;
  };
  MoveWs t;
  t.head = reinterpret_cast<int*>(put(16));
  t.rec = reinterpret_cast<MoveRec*>(put(sizeof(MoveRec) * n));
  t.off = reinterpret_cast<int*>(put(sizeof(int) * n));
  t.fresh = reinterpret_cast<int2*>(put(sizeof(int2) * fresh));
  t.old = reinterpret_cast<int*>(put(sizeof(int) * tables));
  if (w) *w = t;
  return at;
}

size_t cache_move_ws_bytes(const mv_cache_shape& s, int n) {
  return move_ws(s, n, nullptr, nullptr);
}

// Entry e's words, the lengths of its sequences and a span, as read
struct MoveIn {
  int src, dst, span0, span1, len, dst_len;
  mv_span span;    // of lane `lane`
  int prev;        // the end of the one before
  __device__ __forceinline__ MoveIn(const CacheDev& a, const int32_t* s, const int32_t* d,
                                    const int32_t* span_ptr, const mv_span* spans, int n_spans,
                                    int e, int lane)
      : src(s[e]), dst(d[e]), span0(span_ptr ? span_ptr[e] : 0),
        span1(span_ptr ? span_ptr[e + 1] : 0) {
    len = unsigned(src) < unsigned(a.n_seqs) ? a.length(src) : 0;
    dst_len = unsigned(dst) < unsigned(a.n_seqs) ? a.len[dst] : 0;
    read(spans, n_spans, lane);
  }
  __device__ __forceinline__ void read(const mv_span* spans, int n_spans, int lane) {
    const int64_t j = int64_t(span0) + lane;
    const bool in = j >= 0 && j < n_spans;
    span = in ? spans[j] : mv_span{0, 0};
    prev = in && lane > 0 ? spans[j - 1].end : 0;
  }
};

// over groups of gs lanes (a power of two)
__device__ __forceinline__ int group_sum(int x, int gs) {
  for (int o = gs >> 1; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ int group_min(int x, int gs) {
  for (int o = gs >> 1; o; o >>= 1) x = min(x, __shfl_xor(x, o));
  return x;
}

__global__ __launch_bounds__(kPlan) void cache_plan_kernel(CacheDev a, int n,
                                                           const int32_t* __restrict__ src,
                                                           const int32_t* __restrict__ dst,
                                                           const int32_t* __restrict__ span_ptr,
                                                           const mv_span* __restrict__ spans,
                                                           int n_spans, int share, MoveWs w) {
  __shared__ int claim[kMaxSeqs];
  __shared__ int pre[kMaxSeqs + 1];
  __shared__ uint32_t inplace[kMaxSeqs / 32];
  __shared__ int2 old_of[kTogether];   // first and past the last page a source in place may lose
  __shared__ int tmp[kPlan / 64 + 1];
  __shared__ int cnt[2], cut;
  const int tid = threadIdx.x;
  // A wave to an entry, or a lane if there are no spans to read.  What the first
  // entries read is asked for before anything waits.
  const int gs = span_ptr ? 64 : 1, lane = tid & (gs - 1);
  const MoveIn ahead(a, src, dst, span_ptr, spans, n_spans, min(tid / gs, n - 1), lane);   // (n >= 1)
  Search from(a);
  for (int s = tid; s < a.n_seqs; s += kPlan) claim[s] = n;
  for (int s = tid; s < kMaxSeqs / 32; s += kPlan) inplace[s] = 0;
  if (tid == 0) cnt[0] = cnt[1] = 0, cut = INT32_MAX;
  lds_barrier();
  for (int e = tid; e < n; e += kPlan) {
    const int s = src[e], t = dst[e];
    if (unsigned(t) < unsigned(a.n_seqs)) {
      atomicMin(&claim[t], e);
      if (s == t && span_ptr) atomicOr(&inplace[t >> 5], 1u << (t & 31));
    }
  }
  lds_barrier();
  from.settle();
  // an entry's spans, and what becomes of its pages
  const int mask = (1 << a.psl) - 1;
  for (int e = tid / gs; e < n; e += kPlan / gs) {
    MoveIn in = e == tid / gs ? ahead : MoveIn(a, src, dst, span_ptr, spans, n_spans, e, lane);
    MoveRec r{};
    r.src = in.src;
    r.dst = in.dst;
    bool ok = unsigned(r.src) < unsigned(a.n_seqs) && unsigned(r.dst) < unsigned(a.n_seqs);
    ok = ok && claim[r.dst] == e;
    if (ok && r.src != r.dst)
      ok = in.dst_len == 0 && !(inplace[r.src >> 5] >> (r.src & 31) & 1);
    if (!span_ptr) {
      ok = ok && r.src != r.dst;   // a fork
    } else {
      r.span0 = in.span0;
      r.n_spans = in.span1 - in.span0;
      ok = ok && r.span0 >= 0 && r.n_spans >= 0 && r.span0 <= n_spans - r.n_spans;
    }
    if (ok) {   // (the same in every lane of the group)
      r.len = in.len;
      int gone = 0, first = INT32_MAX, bad = 0;
      for (int j = lane; j < r.n_spans; j += gs) {
        if (j != lane) in.read(spans, n_spans, j);
        bad |= in.span.begin < in.prev || in.span.end < in.span.begin;
        const int b = min(in.span.begin, r.len), t = min(in.span.end, r.len);
        gone += t - b;
        if (t > b) first = min(first, b);
      }
      bad = group_sum(bad, gs);
      gone = group_sum(gone, gs);
      first = min(group_min(first, gs), r.len);
      ok = bad == 0;
      r.new_len = r.len - gone;
      r.old_pages = a.pages_of(r.len);
      r.keep = share || r.src == r.dst ? first >> a.psl : 0;
      // rows cut off at the end alone: a part-filled last page stays if no
      // one else holds it
      if (ok && r.src == r.dst && first == r.new_len && (first & mask) != 0 &&
          a.refs[a.page(r.src, r.keep)] == 1)
        r.keep += 1;
      r.n_new = a.pages_of(r.new_len) - r.keep;
      if (ok && r.src == r.dst && n > kTogether)
        for (int j = r.keep + lane; j < r.old_pages; j += gs)
          w.old[int64_t(e) * a.max_pages + j - r.keep] = a.page(r.src, j);
    }
    if (!ok) r.n_new = 0;
    r.ok = ok;
    if (lane == 0) {
      w.rec[e] = r;
      pre[e] = r.n_new;
      if (!ok) atomicAdd(&cnt[1], 1);
      if (n <= kTogether) old_of[e] = make_int2(r.keep, ok && r.src == r.dst ? r.old_pages : 0);
    }
  }
  lds_barrier();
  // The pages that sequences compacted in place are about to lose, all threads
  // on one sequence if there are few (32768 rows in pages of 16: 6 us by a wave)
  for (int e = 0; e < min(n, kTogether); ++e)
    if (n <= kTogether)
      for (int j = old_of[e].x + tid; j < old_of[e].y; j += kPlan)
        w.old[int64_t(e) * a.max_pages + j - old_of[e].x] = a.page(src[e], j);
  int need = 0;
  for (int e0 = 0; e0 < n; e0 += kPlan) {
    const int e = e0 + tid;
    int total;
    const int before = need + block_scan<kPlan>(e < n ? pre[e] : 0, tmp, total);
    if (e < n) {
      pre[e] = before;
      w.off[e] = before;
    }
    need += total;   // at most the table's entries: destinations are named once
  }
  if (tid == 0) pre[n] = need;
  lds_barrier();
  const int found = deal_pages(a, pre, n, need, from, tmp, [&](int q, int e, int page) {
    w.fresh[q] = make_int2(page, e);
    a.refs[page] = 1;
  });
  if (found < need) {
    __syncthreads();   // what was dealt is read back
    for (int e = tid; e < n; e += kPlan) {
      if (pre[e + 1] > found && pre[e + 1] > pre[e]) {
        w.rec[e].ok = 0;
        atomicAdd(&cnt[0], 1);
        atomicMin(&cut, pre[e]);
      }
    }
    __syncthreads();
    for (int q = cut + tid; q < found; q += kPlan) {
      if (q == cut) a.ctl[kCtlHint] = w.fresh[q].x;
      a.refs[w.fresh[q].x] = 0;
    }
  }
  if (tid == 0) {
    w.head[0] = min(found, cut);
    a.ctl[kCtlNoPages] += cnt[0];
    a.ctl[kCtlBad] += cnt[1];
  }
}

// Blocks [0, n): entry b's table, length and holders.  The others: a new page
// of one layer at a time, its rows gathered from the source's old pages.
__global__ __launch_bounds__(256) void cache_move_kernel(CacheDev a, int n,
                                                         const mv_span* __restrict__ spans,
                                                         MoveWs w) {
  const int tid = threadIdx.x;
  if (int(blockIdx.x) < n) {
    __shared__ int low;
    const MoveRec r = w.rec[blockIdx.x];
    if (!r.ok) return;
    if (tid == 0) low = INT32_MAX;
    __syncthreads();
    int32_t* row = a.table + int64_t(r.dst) * a.max_pages;
    const bool same = r.src == r.dst;
    if (!same)
      for (int j = tid; j < r.keep; j += 256) {
        const int p = a.page(r.src, j);
        row[j] = p;
        atomicAdd(&a.refs[p], 1);
      }
    const int off = w.off[blockIdx.x];
    for (int j = tid; j < r.n_new; j += 256) row[r.keep + j] = w.fresh[off + j].x;
    if (same) {
      const int* old = w.old + int64_t(blockIdx.x) * a.max_pages;
      int mine = INT32_MAX;
      for (int j = r.keep + tid; j < r.old_pages; j += 256) {
        const int p = old[j - r.keep];
        if (j >= r.keep + r.n_new) row[j] = -1;
        if (atomicSub(&a.refs[p], 1) == 1) mine = min(mine, p);
      }
      if (mine != INT32_MAX) atomicMin(&low, mine);
      __syncthreads();
      if (tid == 0 && low != INT32_MAX) atomicMin(&a.ctl[kCtlHint], low);
    }
    if (tid == 0) a.len[r.dst] = r.new_len;
    return;
  }
  __shared__ int64_t from[256];   // element offset, within a layer, of head 0's row
  const int64_t tasks = int64_t(w.head[0]) * a.n_layers;
  const int P = 1 << a.psl, CH = a.D / 8;
  const int64_t hs = int64_t(a.D) << a.psl;            // from one head to the next
  const int64_t ls = hs * a.Hkv * a.n_pages;           // from one layer to the next
  for (int64_t x = blockIdx.x - n; x < tasks; x += gridDim.x - n) {
    const int q = int(x / a.n_layers), layer = int(x - int64_t(q) * a.n_layers);
    const int2 f = w.fresh[q];
    const MoveRec r = w.rec[f.y];
    const int i0 = (r.keep + q - w.off[f.y]) << a.psl;   // first new row of the page
    const int cnt = min(P, r.new_len - i0);
    __syncthreads();
    if (tid < cnt) {
      int at = i0 + tid;
      for (int j = 0; j < r.n_spans; ++j) {
        const mv_span s = spans[r.span0 + j];
        const int b = min(s.begin, r.len), t = min(s.end, r.len);
        if (b > at) break;
        at += t - b;
      }
      const int j = at >> a.psl;
      const int p = r.src == r.dst && j >= r.keep
                        ? w.old[int64_t(f.y) * a.max_pages + j - r.keep]
                        : a.page(r.src, j);
      from[tid] = int64_t(p) * a.Hkv * hs + int64_t(at & (P - 1)) * a.D;
    }
    __syncthreads();
    // a thread to a 16-byte chunk of a row, four heads' K and V at a time
    const int64_t to = int64_t(f.x) * a.Hkv * hs;
    u16* k = a.k + layer * ls;
    u16* v = a.v + layer * ls;
    const int c = (tid & (CH - 1)) * 8;
    for (int i = tid / CH; i < cnt; i += 256 / CH) {
      const int64_t s = from[i] + c, t = to + int64_t(i) * a.D + c;
      for (int h = 0; h < a.Hkv; h += 4) {
        uint4 kk[4], vv[4];
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (h + x < a.Hkv) {
            kk[x] = ld16(k + s + (h + x) * hs);
            vv[x] = ld16(v + s + (h + x) * hs);
          }
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (h + x < a.Hkv) {
            st16(k + t + (h + x) * hs, kk[x]);
            st16(v + t + (h + x) * hs, vv[x]);
          }
      }
    }
  }
}

// A block to an entry, of many threads: a page is a chain of a table entry and
// an atomic that returns, 1250 of them took 9.6 us by 256 threads.
__global__ __launch_bounds__(kPlan) void cache_free_kernel(CacheDev a, int n,
                                                         const int32_t* __restrict__ ids) {
  __shared__ int low, seen;
  const int e = blockIdx.x, tid = threadIdx.x, s = ids[e];
  if (unsigned(s) >= unsigned(a.n_seqs)) {
    if (s != -1 && tid == 0) atomicAdd(&a.ctl[kCtlBad], 1);
    return;
  }
  if (tid == 0) low = INT32_MAX, seen = 0;
  __syncthreads();
  for (int j = tid; j < e; j += kPlan)
    if (ids[j] == s) seen = 1;
  __syncthreads();
  if (seen) return;   // an earlier entry frees it
  const int pages = a.pages_of(a.length(s));
  __syncthreads();    // the length is read before it is cleared
  int32_t* row = a.table + int64_t(s) * a.max_pages;
  int mine = INT32_MAX;
  for (int j = tid; j < pages; j += kPlan) {
    const int p = a.page(s, j);
    row[j] = -1;
    if (atomicSub(&a.refs[p], 1) == 1) mine = min(mine, p);
  }
  if (mine != INT32_MAX) atomicMin(&low, mine);
  __syncthreads();
  if (tid == 0) {
    a.len[s] = 0;
    if (low != INT32_MAX) atomicMin(&a.ctl[kCtlHint], low);
  }
}

// --------------------------------------------------------------------------
// launches
// --------------------------------------------------------------------------
hipError_t launch_cache_reset(const CacheDev& a, hipStream_t stream) {
  hipLaunchKernelGGL(cache_reset_kernel, dim3(4 * kNumCu), dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_cache_count(const CacheDev& a, hipStream_t stream) {
  hipLaunchKernelGGL(cache_count_kernel, dim3(1), dim3(kPlan), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_cache_clear_counts(const CacheDev& a, hipStream_t stream) {
  hipLaunchKernelGGL(cache_clear_counts_kernel, dim3(1), dim3(1), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_cache_reserve(const CacheDev& a, int n, const int32_t* ids, const int32_t* ptr,
                                int n_new, int32_t* slot, int32_t* pos, hipStream_t stream) {
  ProfScope prof("cache_reserve", stream);
  hipLaunchKernelGGL(cache_reserve_kernel, dim3(1), dim3(kPlan), 0, stream, a, n, ids, ptr, n_new,
                     slot, pos);
  return hipGetLastError();
}

hipError_t launch_cache_move(const mv_cache_shape& shape, const CacheDev& a, int n,
                             const int32_t* src, const int32_t* dst, const int32_t* span_ptr,
                             const mv_span* spans, int n_spans, bool share, void* ws,
                             hipStream_t stream) {
  MoveWs w;
  move_ws(shape, n, static_cast<char*>(ws), &w);
  {
    ProfScope prof("cache_plan", stream);
    hipLaunchKernelGGL(cache_plan_kernel, dim3(1), dim3(kPlan), 0, stream, a, n, src, dst,
                       span_ptr, spans, n_spans, share ? 1 : 0, w);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  // A fork that shares moves at most one page of each entry; otherwise as
  // many as the tables and the pool hold.
  const int64_t pages = share && span_ptr == nullptr
                            ? n : std::min(int64_t(n) * a.max_pages, int64_t(a.n_pages));
  const int64_t movers = std::min(pages * a.n_layers, int64_t(16) * kNumCu);
  ProfScope prof("cache_move", stream);
  hipLaunchKernelGGL(cache_move_kernel, dim3(unsigned(n + movers)), dim3(256), 0, stream, a, n,
                     spans, w);
  return hipGetLastError();
}

hipError_t launch_cache_free(const CacheDev& a, int n, const int32_t* ids, hipStream_t stream) {
  ProfScope prof("cache_free", stream);
  hipLaunchKernelGGL(cache_free_kernel, dim3(n), dim3(kPlan), 0, stream, a, n, ids);
  return hipGetLastError();
}

}  // namespace mv
