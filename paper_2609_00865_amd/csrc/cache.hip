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
#include "mv_cache_dev.h"

namespace mv {

constexpr int kPlan = 1024;   // threads of the planning blocks
constexpr int kMaxSeqs = MV_CACHE_MAX_SEQS;

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

// Deals the lowest `need` free pages: take(q, page) for q = 0, 1, ...;
// returns how many there were (at most need).  Every thread of the block
// calls it; the hint is moved past the last page dealt.
template <typename F>
__device__ __forceinline__ int deal_pages(const CacheDev& a, int need, int* tmp, F take) {
  int found = 0;
  int64_t base = max(0, a.ctl[kCtlHint]) & ~3;
  __syncthreads();   // the hint is read before it is moved
  for (; found < need && base < a.n_pages; base += 4 * kPlan) {
    const int64_t p = base + 4 * threadIdx.x;
    int4 r = make_int4(1, 1, 1, 1);
    if (p + 3 < a.n_pages) {
      r = *reinterpret_cast<const int4*>(a.refs + p);
    } else {
      if (p < a.n_pages) r.x = a.refs[p];
      if (p + 1 < a.n_pages) r.y = a.refs[p + 1];
      if (p + 2 < a.n_pages) r.z = a.refs[p + 2];
    }
    const int f[4] = {r.x == 0, r.y == 0, r.z == 0, r.w == 0};
    int total;
    int q = found + block_scan<kPlan>(f[0] + f[1] + f[2] + f[3], tmp, total);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (f[u] && q < need) {
        take(q, int(p) + u);
        if (q == need - 1) a.ctl[kCtlHint] = int(p) + u + 1;
      }
      q += f[u];
    }
    found = min(need, found + total);
  }
  if (found < need && threadIdx.x == 0) a.ctl[kCtlHint] = a.n_pages;
  __syncthreads();
  return found;
}

// The last e with pre[e] <= q, of n >= 1 ascending prefix sums (pre[0] = 0).
__device__ __forceinline__ int entry_of(const int* pre, int n, int q) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= q) lo = mid; else hi = mid;
  }
  return lo;
}

// --------------------------------------------------------------------------
// reserve: one block
// --------------------------------------------------------------------------
struct Grow {   // what entry e asks for
  int s, rows, len, have, need, r0;
  bool bad, over;   // malformed; more rows than the table can hold
};

__device__ __forceinline__ Grow grow_of(const CacheDev& a, const int32_t* ids, const int32_t* ptr,
                                        int n_new, const int* claim, int e) {
  Grow g{};
  g.s = ids[e];
  g.r0 = ptr[e];
  const int r1 = ptr[e + 1];
  const bool in = unsigned(g.s) < unsigned(a.n_seqs);
  g.bad = g.r0 < 0 || r1 < g.r0 || r1 > n_new || (!in && g.s != -1) || (in && claim[g.s] != e);
  if (g.bad || !in) return g;
  g.rows = r1 - g.r0;
  g.len = a.length(g.s);
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
  __shared__ int tmp[kPlan / 64 + 1];
  __shared__ int cnt[2], cut_e;
  const int tid = threadIdx.x;
  for (int t = tid; t < n_new; t += kPlan) {
    slot[t] = -1;
    if (pos) pos[t] = -1;
  }
  for (int s = tid; s < a.n_seqs; s += kPlan) claim[s] = n;
  if (tid == 0) cnt[0] = cnt[1] = 0, cut_e = -1;
  __syncthreads();
  for (int e = tid; e < n; e += kPlan)
    if (unsigned(ids[e]) < unsigned(a.n_seqs)) atomicMin(&claim[ids[e]], e);
  __syncthreads();
  int need = 0;
  for (int e0 = 0; e0 < n; e0 += kPlan) {
    const int e = e0 + tid;
    int want = 0, total;
    if (e < n) {
      const Grow g = grow_of(a, ids, ptr, n_new, claim, e);
      want = g.need;
      if (g.bad) atomicAdd(&cnt[1], 1);
      if (g.over) atomicAdd(&cnt[0], 1);
    }
    const int before = need + block_scan<kPlan>(want, tmp, total);
    if (e < n) pre[e] = before;
    need += total;   // at most the table's entries: sequences are named once
  }
  if (tid == 0) pre[n] = need;
  __syncthreads();
  const int found = deal_pages(a, need, tmp, [&](int q, int page) {
    const int e = entry_of(pre, n, q), s = ids[e];
    a.table[int64_t(s) * a.max_pages + a.pages_of(a.length(s)) + q - pre[e]] = page;
    a.refs[page] = 1;
  });
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
  // rows of an accepted entry, a wave to an entry
  const int lane = tid & 63, mask = (1 << a.psl) - 1;
  for (int e = tid >> 6; e < n; e += kPlan / 64) {
    const Grow g = grow_of(a, ids, ptr, n_new, claim, e);
    if (g.need > 0 && pre[e + 1] > found) continue;
    for (int i = lane; i < g.rows; i += 64) {
      const int r = g.len + i;
      slot[g.r0 + i] = (a.page(g.s, r >> a.psl) << a.psl) + (r & mask);
      if (pos) pos[g.r0 + i] = r;
    }
  }
  __syncthreads();
  for (int e = tid; e < n; e += kPlan) {
    const Grow g = grow_of(a, ids, ptr, n_new, claim, e);
    if (g.rows > 0 && (g.need == 0 || pre[e + 1] <= found)) a.len[g.s] = g.len + g.rows;
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
  int off;         // their first place in the list of new pages
  int span0, n_spans;
  int old_pages;   // pages of src
  int pad;
};

struct MoveWs {
  int* head;       // [4]: new pages dealt
  MoveRec* rec;    // [n]
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
  t.fresh = reinterpret_cast<int2*>(put(sizeof(int2) * fresh));
  t.old = reinterpret_cast<int*>(put(sizeof(int) * tables));
  if (w) *w = t;
  return at;
}

size_t cache_move_ws_bytes(const mv_cache_shape& s, int n) {
  return move_ws(s, n, nullptr, nullptr);
}

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x = min(x, __shfl_xor(x, o));
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
  __shared__ int tmp[kPlan / 64 + 1];
  __shared__ int cnt[2], cut;
  const int tid = threadIdx.x, lane = tid & 63;
  for (int s = tid; s < a.n_seqs; s += kPlan) claim[s] = n;
  for (int s = tid; s < kMaxSeqs / 32; s += kPlan) inplace[s] = 0;
  if (tid == 0) cnt[0] = cnt[1] = 0, cut = INT32_MAX;
  __syncthreads();
  for (int e = tid; e < n; e += kPlan) {
    const int s = src[e], t = dst[e];
    if (unsigned(t) < unsigned(a.n_seqs)) {
      atomicMin(&claim[t], e);
      if (s == t && span_ptr) atomicOr(&inplace[t >> 5], 1u << (t & 31));
    }
  }
  __syncthreads();
  // a wave to an entry: its spans, and what becomes of its pages
  const int mask = (1 << a.psl) - 1;
  for (int e = tid >> 6; e < n; e += kPlan / 64) {
    MoveRec r{};
    r.src = src[e];
    r.dst = dst[e];
    bool ok = unsigned(r.src) < unsigned(a.n_seqs) && unsigned(r.dst) < unsigned(a.n_seqs);
    ok = ok && claim[r.dst] == e;
    if (ok && r.src != r.dst)
      ok = a.len[r.dst] == 0 && !(inplace[r.src >> 5] >> (r.src & 31) & 1);
    if (!span_ptr) {
      ok = ok && r.src != r.dst;   // a fork
    } else {
      r.span0 = span_ptr[e];
      r.n_spans = span_ptr[e + 1] - r.span0;
      ok = ok && r.span0 >= 0 && r.n_spans >= 0 && r.span0 <= n_spans - r.n_spans;
    }
    if (ok) {
      r.len = a.length(r.src);
      int gone = 0, first = INT32_MAX, bad = 0;
      for (int j = lane; j < r.n_spans; j += 64) {
        const mv_span x = spans[r.span0 + j];
        const int prev = j > 0 ? spans[r.span0 + j - 1].end : 0;
        bad |= x.begin < prev || x.end < x.begin;
        const int b = min(x.begin, r.len), t = min(x.end, r.len);
        gone += t - b;
        if (t > b) first = min(first, b);
      }
      bad = wave_sum(bad);
      gone = wave_sum(gone);
      first = min(wave_min(first), r.len);
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
      if (ok && r.src == r.dst)
        for (int j = r.keep + lane; j < r.old_pages; j += 64)
          w.old[int64_t(e) * a.max_pages + j - r.keep] = a.page(r.src, j);
    }
    if (!ok) r.n_new = 0;
    r.ok = ok;
    if (lane == 0) {
      w.rec[e] = r;
      if (!ok) atomicAdd(&cnt[1], 1);
    }
  }
  __syncthreads();
  int need = 0;
  for (int e0 = 0; e0 < n; e0 += kPlan) {
    const int e = e0 + tid;
    int total;
    const int before = need + block_scan<kPlan>(e < n ? w.rec[e].n_new : 0, tmp, total);
    if (e < n) {
      pre[e] = before;
      w.rec[e].off = before;
    }
    need += total;   // at most the table's entries: destinations are named once
  }
  if (tid == 0) pre[n] = need;
  __syncthreads();
  const int found = deal_pages(a, need, tmp, [&](int q, int page) {
    w.fresh[q] = make_int2(page, entry_of(pre, n, q));
    a.refs[page] = 1;
  });
  if (found < need) {
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
    for (int j = tid; j < r.n_new; j += 256) row[r.keep + j] = w.fresh[r.off + j].x;
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
    const int i0 = (r.keep + q - r.off) << a.psl;      // first new row of the page
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
    const int64_t to = int64_t(f.x) * a.Hkv * hs;
    const u16* k = a.k + layer * ls;
    const u16* v = a.v + layer * ls;
    const int chunks = a.Hkv * cnt * CH;
#pragma unroll 4
    for (int y = tid; y < chunks; y += 256) {
      const int c = y % CH, i = y / CH % cnt, h = y / CH / cnt;
      const int64_t s = from[i] + h * hs + c * 8, t = to + h * hs + int64_t(i) * a.D + c * 8;
      const uint4 kk = ld16(k + s), vv = ld16(v + s);
      st16(a.k + layer * ls + t, kk);
      st16(a.v + layer * ls + t, vv);
    }
  }
}

// A block to an entry.
__global__ __launch_bounds__(256) void cache_free_kernel(CacheDev a, int n,
                                                         const int32_t* __restrict__ ids) {
  __shared__ int low, seen;
  const int e = blockIdx.x, tid = threadIdx.x, s = ids[e];
  if (unsigned(s) >= unsigned(a.n_seqs)) {
    if (s != -1 && tid == 0) atomicAdd(&a.ctl[kCtlBad], 1);
    return;
  }
  if (tid == 0) low = INT32_MAX, seen = 0;
  __syncthreads();
  for (int j = tid; j < e; j += 256)
    if (ids[j] == s) seen = 1;
  __syncthreads();
  if (seen) return;   // an earlier entry frees it
  const int pages = a.pages_of(a.length(s));
  __syncthreads();    // the length is read before it is cleared
  int32_t* row = a.table + int64_t(s) * a.max_pages;
  int mine = INT32_MAX;
  for (int j = tid; j < pages; j += 256) {
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
  hipLaunchKernelGGL(cache_free_kernel, dim3(n), dim3(256), 0, stream, a, n, ids);
  return hipGetLastError();
}

}  // namespace mv
