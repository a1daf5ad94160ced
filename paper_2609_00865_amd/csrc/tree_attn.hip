// Attention of a sequence's newest rows (one decoded token, a tree of drafted
// ones, a chunk of a prompt) over its rows in a paged cache, on gfx950.
//
// A tile is R (query row, query head) pairs of one KV head, which read the
// same keys; 64 keys of a tile are a unit of work.  The units of all tiles and
// KV heads, one after another, are dealt to the workgroups in equal runs,
// from the sequences' lengths as the device holds them: the workgroups do
// equal work however uneven the batch is, with no copy to the host.  A run is
// a few segments, each of one tile; a segment that is not its whole tile
// leaves an unnormalised O with its maximum and sum, and a second pass joins
// those of a tile in order.
//
// Two kernels take a segment.  For few pairs (tree_few_kernel, R = 32) the
// time is the reading of K and V: each wave streams 32-key tiles of its own
// through its own LDS buffers, no barrier between waves, and the waves'
// results meet in LDS at the end.  (Few pairs of sequences known not to be long
// are not dealt: a workgroup takes a tile whole.)  For many pairs (tree_many_kernel, R = 128)
// the products count: four waves of 32 pairs share 64-key tiles, and the
// scores of a tile are computed while the vector ALU turns those of the one
// before into probabilities.  Both compute S^T = K Q^T and O^T += V^T P^T with
// bf16 MFMA (a query per lane: the softmax statistics stay in a lane pair)
// and keep maximum, sum and O in fp32.
#include <type_traits>

#include "mv_cache_dev.h"
#include "tree_deal.h"

namespace mv {

struct TreeArgs {
  const u16* q;
  const u16* k;        // of the layer
  const u16* v;
  u16* o;
  float* lse;
  float* part_o;       // [2 * groups][R][D] unnormalised
  float* part_ml;      // [2 * groups][R][2] maximum (base 2, scaled), sum
  struct TreeJoin* join;   // [tiles][Hkv]
  const int32_t* table;
  const int32_t* len;
  const int32_t* ids;
  const int32_t* ptr;
  const uint32_t* tree;
  int words;
  int B, N, Hq, Hkv, G, n_pages, n_seqs, max_pages, psl;
  int tiles;           // tile places: at least as many as there are tiles
  int groups;          // workgroups
  float scale_log2;
  uint32_t g_mul;      // for by_heads
  int g_shift;
};

// x / G for 0 <= x < 2^31 by a product: g_mul = ceil(2^g_shift / G) with
// 2^(g_shift - 31) >= G, so that what it is too large by adds less than 1 / G.
__device__ __forceinline__ int by_heads(const TreeArgs& a, int x) {
  return int(uint64_t(uint32_t(x)) * a.g_mul >> a.g_shift);
}

// What is to be joined of a tile place and KV head: the tile's first segment,
// of run `run`, is at `slot`, that of run r > run at 2 r.
struct TreeJoin {
  int rows;            // pairs of the tile; 0: no tile, or it was written whole
  int m0, r0;          // first pair, the entry's first row of q
  int run, slot, runs;
  int pad[2];
};

// Entries whose sizes are held in LDS; those of more are read from memory (single
// tokens over 16 rows each: 512 of them 39 us, 513 50).
constexpr int kPlanB = 512;
constexpr int kChunks = 256;    // blocks of tile places whose first unit is held in LDS

// One tile: the entry, its first pair, and the keys any of its rows may see.
struct Tile {
  int b, n, c;      // entry, its rows, its context rows (negative: absent rows)
  int r0;           // its first row of q
  int m0, rows;     // first pair and pairs of the tile (0: no such tile)
  int kmax;         // keys [0, kmax)
  // a tile without keys is one unit: its rows are still written
  __device__ __forceinline__ int units() const {
    return rows ? max(1, units_of(kmax)) : 0;
  }
};

struct TreeShared {
  int ptr[kPlanB + 1];
  int id[kPlanB], len[kPlanB];
  uint32_t unit_tmp[4];         // of each wave's tiles
  int tile_tmp[4];
  int64_t units[kChunks], tiles[kChunks];   // before each BLOCK of places
  Tile tile;                    // where a run begins
  int at;
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return int64_t(uint64_t(uint32_t(uniform(int(x >> 32)))) << 32 | uint32_t(uniform(int(x))));
}

// Entry b's first tile place: places of entries never overlap, because
// ceil(n G / R) <= floor((r + n) G / R) - floor(r G / R) + 1.
template <int R>
__device__ __forceinline__ int first_place(int64_t r, int b, int G) {
  return int(r * G / R) + b;
}

__device__ __forceinline__ int entry_len(const TreeArgs& a, int id) {
  return unsigned(id) < unsigned(a.n_seqs)
             ? int(min(int64_t(max(a.len[id], 0)), int64_t(a.max_pages) << a.psl)) : 0;
}

__device__ __forceinline__ uint32_t read_lane(uint32_t x, int lane) {
  return uint32_t(__builtin_amdgcn_readlane(int(x), lane));
}

// A value that is worked out here, not before a loop and held in registers.
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// A value read from LDS here and now: a choice between it and one from memory
// would otherwise become one load by a generic address, which waits for both.
__device__ __forceinline__ int from_lds(const int& x) { return here(x); }

__device__ __forceinline__ int first_row(const TreeArgs& a, const TreeShared& s, int b) {
  if (a.B <= kPlanB) return from_lds(s.ptr[b]);
  return min(max(a.ptr[b], 0), a.N);
}

__device__ __forceinline__ int entry_id(const TreeArgs& a, const TreeShared& s, int b) {
  if (a.B <= kPlanB) return from_lds(s.id[b]);
  return a.ids[b];
}

// The tile of entry b whose first pair is m0.
template <int R>
__device__ __forceinline__ Tile tile_at(const TreeArgs& a, const TreeShared& s, int b, int m0) {
  Tile t;
  t.b = b;
  t.r0 = first_row(a, s, b);
  t.n = max(0, first_row(a, s, b + 1) - t.r0);
  t.m0 = m0;
  t.rows = m0 >= 0 ? max(0, min(R, t.n * a.G - m0)) : 0;
  t.kmax = t.c = 0;
  if (t.rows == 0) return t;
  const int L = a.B <= kPlanB ? from_lds(s.len[b]) : entry_len(a, a.ids[b]);
  t.c = L - t.n;
  const int last = by_heads(a, m0 + t.rows - 1);
  t.kmax = a.tree ? L : max(0, t.c + last + 1);
  return t;
}

// The tile of place u (no rows: there is none).
template <int R>
__device__ __forceinline__ Tile tile_of(const TreeArgs& a, const TreeShared& s, int u) {
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first_place<R>(first_row(a, s, mid), mid, a.G) <= u) lo = mid; else hi = mid;
  }
  return tile_at<R>(a, s, lo, (u - first_place<R>(first_row(a, s, lo), lo, a.G)) * R);
}

// A tile's fields are the same in every lane: held in scalar registers.
__device__ __forceinline__ Tile uniform(const Tile& t) {
  return {uniform(t.b), uniform(t.n), uniform(t.c), uniform(t.r0), uniform(t.m0), uniform(t.rows),
          uniform(t.kmax)};
}

// The kernel's arguments read again from where they were passed: outside the
// loops over keys, so that they do not take scalar registers inside them.
__device__ __forceinline__ const TreeArgs& again() {
  typedef __attribute__((address_space(4))) const TreeArgs args;
  uint64_t p = reinterpret_cast<uint64_t>((const args*)__builtin_amdgcn_kernarg_segment_ptr());
  asm volatile("" : "+s"(p));
  return *(const TreeArgs*)(const args*)p;
}

__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {   // of what mostly fits 32 bits
  if (((x | y) >> 32) == 0) return uint32_t(x) / uint32_t(y);
  return x / y;
}

// The deal: every workgroup works out the same one from the lengths, and
// walks its own run of it, segment by segment.  To begin and end a tile takes
// as long as several units (the first keys' way from memory, masked units, the
// result's way back), so where runs are long a tile counts for that many more:
// without it runs of many short tiles were the last to end (us, counting a tile
// for 0 / 2 / 4 / 6 more: 4000 rows of a prompt over no context, 28/4 heads,
// 234 / 187 / 168 / 155; 64 rollouts' decode over 257 to 16384 keys
// 111 / 103 / 101 / 102; 128 over 250 to 1000 keys - / 37.3 / 37.9 / 41.1).
// AGAIN: behind the constructor the arguments are read from where they were
// passed each time (the kernel has no scalar registers to hold them in).
constexpr int kTileCostMany = 6, kTileCostFew = 4, kLongRun = 8;

template <int R, int BLOCK, bool AGAIN>
struct Deal {
  const TreeArgs& direct;
  TreeShared& s;
  int extra;           // what a tile counts for beside its units
  int64_t total;       // of one KV head: units and extras
  int64_t per;         // of a run
  int64_t begin, end;  // this run, over all KV heads
  // the segment: where it begins among all and what it counts for; its tile and
  // KV head, where the tile begins, first unit, units of the segment and the tile
  int64_t p, tile_p;
  Tile t;
  int len, hk, unit, n, of;
  int run, seg;

  __device__ __forceinline__ const TreeArgs& args() const {
    if constexpr (AGAIN) return again();
    return direct;
  }

  // The tiles of places [j BLOCK, (j + 1) BLOCK): units and tiles before each
  struct Before {
    int64_t units;
    int tiles;
  };
  __device__ __forceinline__ void scan(int j, Tile& mine, Before& before, Before& sum) {
    const TreeArgs& a = direct;
    const int u = j * BLOCK + threadIdx.x;
    mine = Tile{};
    if (u < a.tiles) mine = tile_of<R>(a, s, u);
    if (blockIdx.x == 0 && u < a.tiles && mine.rows == 0)   // no run comes by here
      for (int h = 0; h < a.Hkv; ++h) a.join[int64_t(u) * a.Hkv + h].rows = 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t units = mine.units(), x = wave_scan(units);
    const uint64_t is = __ballot(mine.rows > 0);
    lds_barrier();   // what an earlier block of places left is read
    if (lane == 63) {
      s.unit_tmp[wave] = x;
      s.tile_tmp[wave] = __popcll(is);
    }
    lds_barrier();
    add_waves<BLOCK / 64>(s.unit_tmp, wave, before.units, sum.units);
    before.units += x - units;
    before.tiles = __popcll(is & ((uint64_t(1) << lane) - 1));
    sum.tiles = 0;
#pragma unroll
    for (int w = 0; w < BLOCK / 64; ++w) {
      const int n = s.tile_tmp[w];
      before.tiles += w < wave ? n : 0;
      sum.tiles += n;
    }
  }

  __device__ __forceinline__ Deal(const TreeArgs& a0, TreeShared& sh, int r)
      : direct(a0), s(sh), run(r), seg(0) {
    const TreeArgs& a = direct;
    if (a.B <= kPlanB) {
      for (int b = threadIdx.x; b <= a.B; b += BLOCK) {
        s.ptr[b] = min(max(a.ptr[b], 0), a.N);
        if (b < a.B) {
          s.id[b] = a.ids[b];
          s.len[b] = entry_len(a, s.id[b]);
        }
      }
    }
    __syncthreads();
    const int chunks = (a.tiles + BLOCK - 1) / BLOCK;
    Tile mine;
    Before before{}, sum;
    int64_t units = 0, tiles = 0;
    for (int j = 0; j < chunks; ++j) {
      scan(j, mine, before, sum);
      if (threadIdx.x == 0) {
        s.units[j] = units;
        s.tiles[j] = tiles;
      }
      units += sum.units;
      tiles += sum.tiles;
    }
    units = uniform(units);
    tiles = uniform(tiles);
    extra = units * a.Hkv >= int64_t(kLongRun) * a.groups
                ? (R == 128 ? kTileCostMany : kTileCostFew) : 0;
    total = units + extra * tiles;
    per = max(int64_t(1), quotient(total * a.Hkv + a.groups - 1, a.groups));
    begin = run * per;
    end = min(begin + per, total * a.Hkv);
    p = begin;
    if (p >= end) return;
    hk = uniform(int(quotient(p, total)));
    int64_t x = p - hk * total;
    if (chunks > 1) {
      lds_barrier();
      int lo = 0, hi = chunks;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s.units[mid] + extra * s.tiles[mid] <= x) lo = mid; else hi = mid;
      }
      lo = uniform(lo);
      x -= s.units[lo] + extra * s.tiles[lo];
      scan(lo, mine, before, sum);
    }
    const int64_t first = before.units + extra * before.tiles;
    if (mine.rows > 0 && x >= first && x < first + mine.units() + extra) {
      s.tile = mine;
      s.at = int(x) - first;
    }
    lds_barrier();
    t = uniform(s.tile);
    enter(uniform(s.at));
    if (n == 0) next();
  }

  // the run's part of the tile from place `at` of it on
  __device__ __forceinline__ void enter(int at) {
    of = t.units();
    tile_p = p - at;
    len = int(min(int64_t(of + extra - at), end - p));
    unit = max(0, at - extra);
    n = max(0, at + len - extra) - unit;
  }

  __device__ __forceinline__ bool done() const { return p >= end; }

  // On to the next tile: of the entry, of the next entry that has rows, of the
  // next KV head.  (A run that ends before a tile's first unit leaves it.)
  __device__ __forceinline__ void next() {
    if (n > 0) ++seg;
    p += len;
    if (p >= end) return;
    const TreeArgs& a = args();
    int b = t.b, m0 = t.m0 + R;
    if (m0 >= t.n * a.G) {
      m0 = 0;
      do {
        if (++b == a.B) {
          b = 0;
          if (++hk == a.Hkv) {   // (row_ptr not as it should be)
            p = end;
            return;
          }
        }
      } while (uniform(first_row(a, s, b + 1)) <= uniform(first_row(a, s, b)));
    }
    t = uniform(tile_at<R>(a, s, b, m0));
    enter(0);
    if (n == 0) p = end;
  }

  __device__ __forceinline__ bool whole() const { return n == of; }
  // where the segment's partial result goes
  __device__ __forceinline__ int64_t slot() const { return 2 * int64_t(run) + (seg != 0); }

  __device__ __forceinline__ const int32_t* pages() const {   // the sequence's row of the table
    const TreeArgs& a = args();
    return a.table + int64_t(uniform(entry_id(a, s, t.b))) * a.max_pages;
  }

  // For the join: by the segment that a tile begins with
  __device__ __forceinline__ void note() const {
    if (unit != 0 || threadIdx.x != 0) return;
    const TreeArgs& a = args();
    const int place = first_place<R>(t.r0, t.b, a.G) + t.m0 / R;
    TreeJoin j{};
    if (!whole()) {
      j.rows = t.rows;
      j.m0 = t.m0;
      j.r0 = t.r0;
      j.run = run;
      j.slot = int(slot());
      j.runs = int(quotient(tile_p + extra + of - 1, per)) - run + 1;
    }
    a.join[int64_t(place) * a.Hkv + hk] = j;
  }
};

// Instead of a deal: a workgroup to a tile place and KV head, all of the tile's
// keys, no partial results.
struct WholeShared {
  Tile tile;
  int id, first;
};

template <int R, int BLOCK>
struct Whole {
  const TreeArgs& a;
  Tile t;
  int hk, unit, n, id;
  bool over;

  __device__ __forceinline__ Whole(const TreeArgs& args, WholeShared& s)
      : a(args), unit(0), over(true) {
    const int u = blockIdx.x / a.Hkv;
    hk = blockIdx.x - u * a.Hkv;
    if (threadIdx.x == 0) s.first = INT32_MAX;
    lds_barrier();
    // Each thread looks at entries of its own: the place is in one of them (if
    // row_ptr is not as it should be, in the first)
    int b = INT32_MAX, my_id = -1;
    Tile mine{};
    for (int e = threadIdx.x; e < a.B; e += BLOCK) {
      const int r0 = min(max(a.ptr[e], 0), a.N), r1 = min(max(a.ptr[e + 1], 0), a.N);
      const int e_id = a.ids[e];
      const int64_t m0 = int64_t(u - first_place<R>(r0, e, a.G)) * R;
      if (b != INT32_MAX || r1 <= r0 || m0 < 0 || m0 >= int64_t(r1 - r0) * a.G) continue;
      b = e;
      my_id = e_id;
      mine.b = e;
      mine.r0 = r0;
      mine.n = r1 - r0;
      mine.m0 = int(m0);
      mine.rows = min(R, mine.n * a.G - mine.m0);
      const int L = entry_len(a, e_id);
      mine.c = L - mine.n;
      mine.kmax = a.tree ? L : max(0, mine.c + by_heads(a, mine.m0 + mine.rows - 1) + 1);
      atomicMin(&s.first, e);
    }
    lds_barrier();
    if (s.first == INT32_MAX) return;   // block-uniform: no tile
    if (b == s.first) {
      s.tile = mine;
      s.id = my_id;
    }
    lds_barrier();
    t = uniform(s.tile);
    id = uniform(s.id);
    n = t.units();
    over = false;
  }
  __device__ __forceinline__ bool done() const { return over; }
  __device__ __forceinline__ void next() { over = true; }
  __device__ __forceinline__ bool whole() const { return true; }
  __device__ __forceinline__ int64_t slot() const { return 0; }
  __device__ __forceinline__ void note() const {}
  __device__ __forceinline__ const int32_t* pages() const {
    return a.table + int64_t(id) * a.max_pages;
  }
};

// Workgroups of an XCD (dealt to them in turn) take neighbouring runs: tiles
// of one sequence and KV head meet in its L2.
__device__ __forceinline__ int run_of_block(int groups) {
  int xcd, local;
  xcd_split(xcd, local);
  const int full = groups / kNumXcd, more = groups % kNumXcd;
  return xcd * full + min(xcd, more) + local;
}

// What a partial result with maximum m counts for beside maximum M.  Without
// a maximum it holds nothing (or only NaN, which has to stay).
__device__ __forceinline__ float weight(float m, float M) {
  return m == -INFINITY ? 1.f : fast_exp2(m - M);
}

// lse from a maximum (base 2) and the sum beside it.  The sum's exponent and the
// maximum are added in 64 bits: in 32 their sum would be off by as much as all
// before it.  What is left of the sum has a logarithm in [-1, 0].
__device__ __forceinline__ float lse_of(float M, float l) {
  if (l == 0.f) return -INFINITY;
  const double log2_l = double(__builtin_amdgcn_frexp_expf(l)) +
                        double(__builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(l)));
  return float((double(M) + log2_l) * 0.6931471805599453);
}

// The keys of [key0, key0 + 32) that new row i of a tile's entry sees, as
// bits; row: its row of q.
__device__ __forceinline__ uint32_t seen32(const TreeArgs& a, const Tile& t, int64_t row, int i,
                                           int key0) {
  auto low = [](int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; };
  if (!a.tree) return low(t.c + i + 1 - key0);
  const uint32_t* w = a.tree + row * a.words;
  const int a0 = key0 - t.c;   // new row that key0 is
  uint32_t bits = 0;
  if (a0 >= 0) {
    const int x = a0 >> 5, sh = a0 & 31;
    if (x < a.words) bits = w[x] >> sh;
    if (sh && x + 1 < a.words) bits |= w[x + 1] << (32 - sh);
  } else if (a0 > -32) {
    if (a.words > 0) bits = w[0] << -a0;
  }
  bits &= low(t.c + t.n - key0);                 // new rows there are
  return bits | low(t.c - key0);                 // and the context
}

// Page ids of the keys ahead, per wave: 64 at a time into two LDS slots by
// direct loads that land in order with those of the keys.
struct PageRing {
  const int32_t* row;   // the sequence's table
  uint32_t lds;         // slot 0 (slot 1 is 256 bytes behind)
  const int* slots;
  int window;           // the last window asked for
  int n_pages, psl;
  __device__ __forceinline__ void load(int w, int last_page) {
    // lanes past the last page read it again
    const int lane = threadIdx.x & 63;
    lds_load4(row + min(w * 64 + lane, last_page), lds + uint32_t(w & 1) * 256);
    window = w;
  }
  // 4 bytes per lane from global memory into LDS (lane l at lds + 4 l)
  static __device__ __forceinline__ void lds_load4(const void* src, uint32_t lds) {
    uint32_t saved;
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\t"
        "global_load_lds_dword %1, off\n\ts_mov_b32 m0, %0"
        : "=&s"(saved)
        : "v"(src), "s"(__builtin_amdgcn_readfirstlane(lds))
        : "memory");
  }
  // The windows of keys [key0, ..): call with the first key of the segment,
  // and wait for the loads before get().
  __device__ __forceinline__ void start(int key0, int last) {
    const int w = (key0 >> psl) >> 6;
    load(w, last >> psl);
    load(w + 1, last >> psl);
  }
  // before the keys of page index j are asked for: the window behind j's is in flight
  __device__ __forceinline__ void ahead(int j, int last) {
    if ((j >> 6) == window) load(window + 1, last >> psl);
  }
  // The row of the layer's pool (from the KV head's first) that holds a key, a
  // page having page_rows; a key past the last is read from the last one's page.
  // (Each lane its own: the look-ups of a tile are one, their results read by lane.)
  __device__ __forceinline__ uint32_t row_of(int key, int last, uint32_t page_rows) const {
    const int j = min(key, last) >> psl;
    const unsigned p = slots[j & 127];
    return (p < unsigned(n_pages) ? p : 0) * page_rows + (key & ((1 << psl) - 1));
  }
};

// 16 rows of a page (N KiB) into LDS by direct loads of 1 KiB: lane l's 16 bytes
// of load j from base + voff[j] + j KiB to lds + j KiB + 16 l.  The instruction's
// offset moves both addresses, so the LDS address is set once; it is read a state
// after it is written.
template <int N>
__device__ __forceinline__ void load_rows16(const void* base, const uint32_t (&voff)[N],
                                            uint32_t lds) {
  static_assert(N == 4 || N == 2, "rows of 128 or 64 elements");
  uint32_t saved;
  if constexpr (N == 4)
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %6\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %5\n\tglobal_load_lds_dwordx4 %2, %5 offset:1024\n\t"
        "global_load_lds_dwordx4 %3, %5 offset:2048\n\t"
        "global_load_lds_dwordx4 %4, %5 offset:3072\n\ts_mov_b32 m0, %0"
        : "=&s"(saved)
        : "v"(voff[0]), "v"(voff[1]), "v"(voff[2]), "v"(voff[3]), "s"(base), "s"(lds)
        : "memory");
  else
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %4\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %3\n\tglobal_load_lds_dwordx4 %2, %3 offset:1024\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "v"(voff[0]), "v"(voff[1]), "s"(base), "s"(lds)
        : "memory");
}

// The offsets per lane of loads of 16 rows: load j's lane has chunk c ^ kv_swz of
// its row, which repeats every 16 rows.
template <int D>
__device__ __forceinline__ void row_offsets(int lane, uint32_t (&voff)[D / 32]) {
  const int r = lane / (D / 8);
#pragma unroll
  for (int j = 0; j < D / 32; ++j)
    voff[j] = uint32_t(r * D * 2 + ((lane % (D / 8) ^ kv_swz<D>(j * (512 / D) + r)) << 4));
}

template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// Operands loaded before a loop are waited for here: left to itself the compiler
// waits at their first use inside it, for every load in flight, each time round.
template <int N>
__device__ __forceinline__ void settle(bf16x8 (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

__device__ __forceinline__ bool odd_bf16x2(uint32_t w) {   // one of two is not finite
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}

// Rows of 1 KiB loads of a V tile from 16-byte place x on: are all finite / made 0 where not
__device__ __forceinline__ bool odd16(const char* p) {
  const uint4 x = ld16(p);
  return odd_bf16x2(x.x) || odd_bf16x2(x.y) || odd_bf16x2(x.z) || odd_bf16x2(x.w);
}
__device__ __forceinline__ void clear_odd16(char* p) {
  const uint4 x = ld16(p);
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if ((w[e] & 0x7f80u) == 0x7f80u) w[e] &= 0xffff0000u;
    if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] &= 0xffffu;
  }
  st16(p, make_uint4(w[0], w[1], w[2], w[3]));
}

// Adds what the elements of V row `key` that are not finite give to the
// queries that see it (p: this lane's query's probability of the key).
template <int D>
__device__ __forceinline__ void add_odd_row(const char* sV, int key, float p, bool sees,
                                            f32x16 (&oacc)[D / 32]) {
  const int g = (threadIdx.x & 63) >> 5;
  const char* row = sV + key * (D * 2) + g * 8;
  const int swz = kv_swz<D>(key) << 4;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {   // dims db * 32 + q4 * 8 + g * 4 .. + 4
      const uint2 x = *reinterpret_cast<const uint2*>(row + (((db * 4 + q4) << 4) ^ swz));
      const uint32_t w[4] = {x.x & 0xffffu, x.x >> 16, x.y & 0xffffu, x.y >> 16};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if ((w[e] & 0x7f80u) == 0x7f80u && sees)
          oacc[db][q4 * 4 + e] += p * bf16_to_f32(uint16_t(w[e]));
      asm volatile("" ::: "memory");   // (a row at a time: this path is rare, registers are not)
    }
}

// Pair m of a tile: its row of q and its head
struct Pair {
  int i, h;
  int64_t row;
  __device__ __forceinline__ Pair(const TreeArgs& a, const Tile& t, int hk, int m) {
    i = by_heads(a, m);
    h = hk * a.G + m - i * a.G;
    row = int64_t(t.r0) + i;
  }
};

// --------------------------------------------------------------------------
// few pairs: NW waves, each with two K and two V tiles of 32 keys, a run of the
// deal; or (WHOLE) with one of each, all keys of one tile: K of a wave's next tile
// is asked for when K of this one is used up, V likewise.
//
// Bound by the reading of K and V; a wave has a tile's 16 KiB (head_dim 128) in
// flight while it works on another.  64 single tokens over 257 to 16384 rows,
// 28/4 heads of 128: 522 MB in 100 us, 5.2 TB/s; 6 over 65536 to 131071 rows,
// 64/8 heads: 2.47 GB in 415 us, 5.9 TB/s.  One token over 777 rows is a chain
// of waits: dealt 8.4 us (about 0.5 for the lengths, 0.7 for the deal and 0.7 for
// finding the run in it, 1.0 for page ids, 0.9 for the first keys, 1.1 for a tile
// and 0.9 for the waves' joint result, the launch the rest) and 3.4 for the join;
// whole 11.1, of one launch.
// Two waves to a workgroup and two workgroups to a CU (us: 101 and 413; four
// waves and one workgroup 102 and 413, short runs 0 to 8 % slower; one wave and
// four workgroups 128 and 488).  64 or 128 pairs to a wave were no faster.
// --------------------------------------------------------------------------
template <int D, int NW, bool WHOLE>
__global__ __launch_bounds__(NW * 64) void tree_few_kernel(TreeArgs a) {
  constexpr int R = 32, BLOCK = NW * 64, NB = WHOLE ? 1 : 2;
  constexpr int KS = D / 16, DB = D / 32;
  constexpr int TB = 32 * D * 2;             // bytes of a tile
  constexpr int NI = TB / 1024;              // 1 KiB loads of a tile
  constexpr int LR = 512 / D;                // rows of a load
  // floats of a row of O where the waves meet; its 16-byte chunks are permuted by
  // row where there is no room to set rows apart
  constexpr int OS = WHOLE ? D : D + 4;
  static_assert(R * OS * 4 <= 2 * NB * TB, "a wave's O fits its tiles");
  auto chunk_at = [](int r, int ch) { return r * OS + (WHOLE ? ch ^ (r & (D / 4 - 1)) : ch) * 4; };
  __shared__ __align__(1024) char buf[NW][2 * NB * TB];   // K's, V's
  __shared__ __align__(16) int pg[NW][128];
  __shared__ std::conditional_t<WHOLE, WholeShared, TreeShared> sh;
  __shared__ float sm[NW][R], sl[NW][R];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int c = lane & 31, g = lane >> 5;
  auto deal = [&] {
    if constexpr (WHOLE) return Whole<R, BLOCK>(a, sh);
    else return Deal<R, BLOCK, false>(a, sh, run_of_block(a.groups));
  }();
  const int ps = 1 << a.psl;
  constexpr int NO = 16 / LR;                // loads of 16 rows, which lie in one page
  uint32_t voff[NO];
  row_offsets<D>(lane, voff);
  const int wv = uniform(wave);
  const uint32_t lds0 = uniform(int(lds_addr(&buf[0][0]) + wv * 2 * NB * TB));

  for (; !deal.done(); deal.next()) {
    const Tile& t = deal.t;
    const int hk = deal.hk;

    // Q^T as the B operand: lane holds pair c, dims ks*16 + g*8 .. + 8
    // (loaded below; lanes past the tile's pairs hold its first, and store nothing)
    const Pair mine(a, t, hk, t.m0 + (c < t.rows ? c : 0));
    bf16x8 qf[KS];
    f32x16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;

    // this segment's keys; wave w takes 32-key tiles w, w + NW, ...
    const int k_begin = deal.unit * kUnit;
    const int k_end = int(min(int64_t(t.kmax), int64_t(deal.unit + deal.n) * kUnit));
    const int nt = k_end > k_begin ? (k_end - k_begin + 31) / 32 : 0;
    const int todo = nt > wv ? (nt - wv + NW - 1) / NW : 0;
    auto key_of = [&](int x) { return k_begin + (wv + x * NW) * 32; };
    const int last = t.kmax - 1;
    const uint32_t page_rows = uint32_t(a.Hkv) * ps;   // (a pool of 2^32 rows is past any memory)
    const char* kb = reinterpret_cast<const char*>(a.k) + int64_t(hk) * ps * D * 2;
    const char* vb = reinterpret_cast<const char*>(a.v) + int64_t(hk) * ps * D * 2;
    PageRing pages{nullptr, lds_addr(&pg[wave][0]), &pg[wave][0], 0, a.n_pages, a.psl};
    if (todo > 0) {
      pages.row = deal.pages();
      pages.start(key_of(0), last);
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      qf[ks] = as_bf16x8(ld16(a.q + (mine.row * a.Hq + mine.h) * D + ks * 16 + g * 8));
    wait_loads<KS>();   // the page ids have landed, Q may be on its way
    // Tile x of this wave into buffer x % NB.  Rows past the last key are read
    // from the last key's page (what they hold is masked).
    uint32_t at;   // where 16 rows at a time are, of the tile last asked for
    auto issue = [&](const char* base, uint32_t lds) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        load_rows16(base + uint64_t(read_lane(at, j)) * (D * 2), voff, lds + j * NO * 1024);
    };
    auto issue_k = [&](int x) {
      const int key0 = key_of(x);
      pages.ahead(key0 >> a.psl, last);
      at = pages.row_of(key0 + (lane & 1) * 16, last, page_rows);
      issue(kb, lds0 + uint32_t(x % NB) * TB);
    };
    auto issue_v = [&](int x) { issue(vb, lds0 + uint32_t(NB + x % NB) * TB); };
    if (todo > 0) {
      issue_k(0);
      issue_v(0);
    }
    wait_loads<0>();
    settle(qf);
    if (!WHOLE && todo > 1) {
      issue_k(1);
      issue_v(1);
    }
    const int clear = a.tree ? t.c : t.c + by_heads(a, t.m0) + 1;   // keys every row of the tile sees
    for (int x = 0; x < todo; ++x) {
      // K of the tile has landed, and with two buffers V too (behind them may be
      // in flight: V; the next tile)
      if (WHOLE)
        wait_loads<NI>();
      else if (x + 1 < todo)
        wait_loads<2 * NI>();
      else
        wait_loads<0>();
      const char* sK = &buf[wave][(x % NB) * TB];
      char* sV = &buf[wave][(NB + x % NB) * TB];
      f32x16 sc = {};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) sc = mfma32(ld_row_swz<D>(sK, c, ks * 2 + g), qf[ks], sc);
      if (WHOLE && x + 1 < todo) {
        wait_lds();   // K's reads are done
        issue_k(x + 1);
      }
      const int key0 = key_of(x);
      uint32_t see = ~0u;
      const bool masked = key0 + 32 > min(clear, k_end);   // wave-uniform
      if (masked) {
        const int n = k_end - key0;
        see = seen32(a, t, mine.row, mine.i, key0) & (n >= 32 ? ~0u : (1u << n) - 1u);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          sc[r] = (see >> ((r >> 2) * 8 + g * 4 + (r & 3))) & 1u ? sc[r] : -INFINITY;
      }
      float mx = sc[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sc[r]);
      mx = max_halves(mx) * a.scale_log2;
      if (__any(mx > m_run)) {
        const float m_new = fmaxf(m_run, mx);
        const float alpha = m_run == -INFINITY ? 0.f : fast_exp2(m_run - m_new);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[db][r] *= alpha;
      }
      const float mu = m_run == -INFINITY ? 0.f : m_run;
      // P in bf16 for the product (its sum is taken before the rounding): half
      // an ulp of each, 2^-8 relative, averaged over the row
      float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sc[r] = fast_exp2(fmaf(sc[r], a.scale_log2, -mu));
        part[r & 3] += sc[r];
      }
      l_run += (part[0] + part[1]) + (part[2] + part[3]);
      if (WHOLE) {   // V has landed (the next K may be in flight)
        if (x + 1 < todo)
          wait_loads<NI>();
        else
          wait_loads<0>();
      }
      if (masked) {
        // A value that is not finite in a row that some query does not see
        // would reach it as 0 * inf: such elements are taken out of the tile
        // and added, query by query, where they are seen.
        bool odd = false;
#pragma unroll
        for (int j = 0; j < NI; ++j) odd |= odd16(sV + j * 1024 + lane * 16);
        if (__any(odd)) {
#pragma nounroll
          for (int key = 0; key < 32; ++key) {
            const int rr = (key >> 3) * 4 + (key & 3), hh = (key >> 2) & 1;
            float pk = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) pk = r == rr ? sc[r] : pk;
            pk = __shfl(pk, c + 32 * hh);
            add_odd_row<D>(sV, key, pk, (see >> key) & 1u, oacc);
          }
          wait_lds();
#pragma unroll
          for (int j = 0; j < NI; ++j) clear_odd16(sV + j * 1024 + lane * 16);
          wait_lds();
        }
      }
      const bf16x8 pf[2] = {to_operand(sc, 0), to_operand(sc, 8)};
#pragma unroll
      for (int st = 0; st < 2 * DB; ++st)
        oacc[st % DB] = mfma32(ld_tr_swz<D>(sV, (st / DB) * 16, (st % DB) * 32), pf[st / DB],
                               oacc[st % DB]);
      if (x + NB < todo) {
        wait_lds();   // the buffer's reads are done
        if (!WHOLE) issue_k(x + NB);
        issue_v(x + NB);
      }
    }
    l_run += __shfl_xor(l_run, 32);

    // the waves' results meet: each scales its own to the common maximum
    if (g == 0) {
      sm[wave][c] = m_run;
      sl[wave][c] = l_run;
    }
    __syncthreads();
    float M = sm[0][c];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, sm[w][c]);
    const float f = weight(m_run, M);
    float* so = reinterpret_cast<float*>(&buf[wave][0]);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<float4*>(so + chunk_at(c, db * 8 + q4 * 2 + g)) =
            make_float4(oacc[db][q4 * 4 + 0] * f, oacc[db][q4 * 4 + 1] * f,
                        oacc[db][q4 * 4 + 2] * f, oacc[db][q4 * 4 + 3] * f);
    __syncthreads();
    const int64_t slot = deal.slot();
    for (int x = tid; x < t.rows * (D / 8); x += BLOCK) {
      const int r = x / (D / 8), d0 = (x % (D / 8)) * 8;
      float Mr = sm[0][r], l = 0.f;
#pragma unroll
      for (int w = 1; w < NW; ++w) Mr = fmaxf(Mr, sm[w][r]);
#pragma unroll
      for (int w = 0; w < NW; ++w) l += sl[w][r] * weight(sm[w][r], Mr);
      float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float* q = reinterpret_cast<const float*>(&buf[w][0]);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] += q[chunk_at(r, d0 / 4 + e / 4) + e % 4];
      }
      if (deal.whole()) {
        const Pair pr(a, t, hk, t.m0 + r);
        const float inv = l == 0.f ? 0.f : 1.f / l;   // l is 0 where no key was seen
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= inv;
        store_v<8>(a.o + (pr.row * a.Hq + pr.h) * D + d0, y);
        if (d0 == 0)
          a.lse[int64_t(pr.h) * a.N + pr.row] = lse_of(Mr, l);
      } else {
        float* q = a.part_o + (slot * R + r) * D + d0;
        *reinterpret_cast<float4*>(q) = make_float4(y[0], y[1], y[2], y[3]);
        *reinterpret_cast<float4*>(q + 4) = make_float4(y[4], y[5], y[6], y[7]);
        if (d0 == 0) {
          a.part_ml[(slot * R + r) * 2] = Mr;
          a.part_ml[(slot * R + r) * 2 + 1] = l;
        }
      }
    }
    deal.note();
    __syncthreads();
  }
}

// --------------------------------------------------------------------------
// many pairs: four waves of 32 pairs on shared tiles of 64 keys, K and V in two
// buffers each, two workgroups to a CU
//
// Where contexts are read once (24 trees of 8 to 61 tokens over 301 to 8192
// rows, 28/4 heads of 128: 181 MB of keys and Q, 30 MB of partial results, 42
// us, 5.0 TB/s) it is bound by memory; where rows are many (two chunks of 1531
// to 2048 rows over 4099 to 8192, 420 GFLOP: 394 to 450 us with the chip's clock,
// 0.93 to 1.06 PFLOP/s) by the matrix pipe, 58 % busy, and the six vector
// instructions beside each MFMA that share its SIMD.  32-key tiles in four
// buffers were 4 % slower on the chunks and 7 % at head_dim 64, up to 10 %
// faster where runs are a few units; eight waves on 256 pairs were slower.
// --------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256, 2) void tree_many_kernel(TreeArgs a) {
  constexpr int R = 128, KB = 2, BK = 32 * KB, BLOCK = 256;
  constexpr int KS = D / 16, DB = D / 32;
  constexpr int TB = BK * D * 2;             // bytes of a tile
  constexpr int NL = TB / 4096;              // loads of a thread per tile
  constexpr int H = 8 * KB;                  // half the elements of a tile in a lane
  __shared__ __align__(1024) char sKb[2][TB];
  __shared__ __align__(1024) char sVb[2][TB];
  __shared__ __align__(16) int pg[4][128];
  __shared__ TreeShared sh;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int c = lane & 31, g = lane >> 5;
  Deal<R, BLOCK, true> deal(a, sh, run_of_block(a.groups));
  const int ps = 1 << a.psl;
  // A wave loads 16 rows of a tile, which lie in one page (its rows are a multiple
  // of 16): one look-up, one scalar address.
  uint32_t voff[NL];
  row_offsets<D>(lane, voff);
  const int wv = uniform(wave);
  const uint32_t ldsK = uniform(int(lds_addr(&sKb[0][0]) + wv * NL * 1024));
  const uint32_t ldsV = uniform(int(lds_addr(&sVb[0][0]) + wv * NL * 1024));

  for (; !deal.done(); deal.next()) {
    const Tile& t = deal.t;
    const int hk = deal.hk;

    auto my = [&]() {   // this lane's pair of the tile
      const int x = here(threadIdx.x);
      return (x >> 6) * 32 + (x & 31);
    };
    // a wave without pairs loads its share of the tiles and computes nothing
    const bool active = wv * 32 < t.rows;
    // this lane's pair, worked out again where it is needed rather than held
    auto pair = [&](const TreeArgs& b) {
      const int m = my();
      return Pair(b, t, hk, t.m0 + (m < t.rows ? m : 0));
    };
    f32x16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;

    const int key_base = deal.unit * kUnit;
    const int last = t.kmax - 1;
    // tiles of the segment
    const int n = (int(min(int64_t(t.kmax), int64_t(deal.unit + deal.n) * kUnit)) - key_base +
                   BK - 1) / BK;
    const uint32_t page_rows = uint32_t(a.Hkv) * ps;   // (a pool of 2^32 rows is past any memory)
    const char* kb = reinterpret_cast<const char*>(a.k) + int64_t(hk) * ps * D * 2;
    const char* vb = reinterpret_cast<const char*>(a.v) + int64_t(hk) * ps * D * 2;
    PageRing pages{nullptr, lds_addr(&pg[wv][0]), &pg[wv][0], 0, a.n_pages, a.psl};
    const bool keys = t.kmax > 0;   // block-uniform
    if (keys) {
      pages.row = deal.pages();
      pages.start(key_base, last);
    }
    // (lanes past the tile's pairs hold its first, and store nothing)
    bf16x8 qf[KS];
    {
      const TreeArgs& b = again();
      const Pair mine = pair(b);
      const u16* qp = b.q + (mine.row * b.Hq + mine.h) * D + here(g) * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[ks] = as_bf16x8(ld16(qp + ks * 16));
    }
    wait_loads<KS>();   // the page ids have landed, Q may be on its way
    // The first of this wave's rows of tile x.  (What rows past the last key hold
    // is masked.)
    auto locate = [&](int x) {
      return read_lane(pages.row_of(key_base + x * BK + wv * 16, last, page_rows), 0);
    };
    auto issue = [&](const char* base, uint32_t at, uint32_t lds) {
      load_rows16(base + uint64_t(at) * (D * 2), voff, lds);
    };
    uint32_t at_v, at_k;   // of the V tile and of the K tile to be asked for next
    auto kfrag = [&](int buf, int j) {
      return ld_row_swz<D>(&sKb[buf][0], (j % KB) * 32 + c, (j / KB) * 2 + g);
    };
    const int clear = a.tree ? t.c : t.c + by_heads(a, t.m0) + 1;   // keys every row of the tile sees
    auto masked = [&](int x) { return key_base + x * BK + BK > min(clear, t.kmax); };
    auto seen = [&](int x, int kb2) {   // of keys 32 kb2 .. + 32 of tile x
      const int key0 = key_base + x * BK + kb2 * 32, m = t.kmax - key0;
      const uint32_t in = m >= 32 ? ~0u : m <= 0 ? 0u : (1u << m) - 1u;
      const TreeArgs& b = again();
      const Pair mine = pair(b);
      return seen32(b, t, mine.row, mine.i, key0) & in;
    };
    f32x16 sc[2][KB];   // scores of tile x in sc[x & 1]
    auto mask_tile = [&](f32x16 (&s)[KB], int x) {
      if (!masked(x)) return;   // block-uniform
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        const uint32_t w = seen(x, b) >> (g * 4);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          s[b][r] = (w >> ((r >> 2) * 8 + (r & 3))) & 1u ? s[b][r] : -INFINITY;
      }
    };
    auto tile_max = [&](const f32x16 (&s)[KB]) {
      float mx = -INFINITY;
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[b][r]);
      return max_halves(mx) * a.scale_log2;
    };
    // As in the masked forward: probabilities are taken against the maximum of
    // a tile that the row has scored before; only where they would pass 2^16,
    // or a row has seen no key yet, is the tile's own maximum taken.  They are
    // rounded to bf16 for the product, as in the kernel for few pairs (outputs are
    // then 2.3e-3 from 64 bits in norm, where their own rounding gives 1.7e-3).
    auto m_off = [&]() { return m_run == -INFINITY ? 0.f : m_run; };
    auto pexp = [&](const f32x16 (&s)[KB], int i, float mu) {
      return fast_exp2(fmaf(s[i >> 4][i & 15], a.scale_log2, -mu));
    };
    auto pack8 = [](const float* q) {
      return as_bf16x8(make_uint4(pack2(q[0], q[1]), pack2(q[2], q[3]), pack2(q[4], q[5]),
                                  pack2(q[6], q[7])));
    };
    auto slow_tile = [&](const f32x16 (&s)[KB], bf16x8 (&pf)[2 * KB], float& psum)
                         __attribute__((always_inline)) {
      const float m_tile = tile_max(s);
      if (m_tile > m_run) {
        const float alpha = m_run == -INFINITY ? 0.f : fast_exp2(m_run - m_tile);
        m_run = m_tile;
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[db][r] *= alpha;
      }
      const float mu = m_off();
      psum = 0.f;
#pragma unroll
      for (int k = 0; k < 2 * KB; ++k) {
        float q[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          q[u] = pexp(s, 8 * k + u, mu);
          psum += q[u];
        }
        pf[k] = pack8(q);
      }
    };
    // Values that are not finite in a masked tile (see the kernel for few
    // pairs): added where they are seen, then made 0.
    auto odd_values = [&](const f32x16 (&s)[KB], int x, char* sV) __attribute__((always_inline)) {
      bool odd = false;
#pragma unroll
      for (int j = 0; j < NL; ++j)
        odd |= odd16(sV + (j * 4 + wv) * 1024 + (here(threadIdx.x) & 63) * 16);
      if (!__syncthreads_or(odd)) return;
      const float mu = m_off();
      const uint32_t see0 = seen(x, 0), see1 = seen(x, 1);
#pragma nounroll
      for (int key = 0; key < BK; ++key) {
        const int kk = key & 31, rr = (kk >> 3) * 4 + (kk & 3), hh = (kk >> 2) & 1;
        float sk = 0.f;
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) sk = b * 16 + r == (key >> 5) * 16 + rr ? s[b][r] : sk;
        sk = __shfl(sk, c + 32 * hh);
        add_odd_row<D>(sV, key, fast_exp2(fmaf(sk, a.scale_log2, -mu)),
                       ((key < 32 ? see0 : see1) >> kk) & 1u, oacc);
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < NL; ++j)
        clear_odd16(sV + (j * 4 + wv) * 1024 + (here(threadIdx.x) & 63) * 16);
      __syncthreads();
    };

    bf16x8 pf[2 * KB];
    float psum_a = 0.f;
    if (keys) {
      at_v = locate(0);
      issue(kb, at_v, ldsK);
      issue(vb, at_v, ldsV);
    }
    wait_loads<0>();
    settle(qf);
    if (keys) {
      at_v = locate(min(1, n - 1));
      if (n > 1) issue(kb, at_v, ldsK + TB);
      at_k = locate(min(2, n - 1));
      lds_barrier();
    }
    if (keys && active) {
#pragma unroll
      for (int j = 0; j < KB * KS; ++j)
        sc[0][j % KB] = mfma32(kfrag(0, j), qf[j / KB], j < KB ? f32x16{} : sc[0][j % KB]);
      mask_tile(sc[0], 0);
      m_run = tile_max(sc[0]);
      const float mu = m_off();
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        float q[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          q[u] = pexp(sc[0], 8 * k + u, mu);
          psum_a += q[u];
        }
        pf[k] = pack8(q);
      }
    }
    // One step: tile x (in buffer and score set S = x % 2, the operands of its
    // first half in pf) and the scores of tile x + 1.  On the last tile the score
    // MFMAs run on stale LDS and their results are dropped.
    auto step = [&](auto tag, int x) __attribute__((always_inline)) {
      constexpr int S = decltype(tag)::value;
      f32x16 (&cur)[KB] = sc[S];
      f32x16 (&nxt)[KB] = sc[S ^ 1];
      const bool next = x + 1 < n;   // block-uniform
      // K of tile x + 1 and V of tile x have landed, every wave is done with K of
      // tile x and V of tile x - 1
      wait_loads<0>();
      lds_barrier();
      if (x + 2 < n) issue(kb, at_k, ldsK + S * TB);
      if (next) issue(vb, at_v, ldsV + (S ^ 1) * TB);
      const float mu = m_off();
      if (active) {
        float psum = psum_a;
        bf16x8 kr[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) kr[j] = kfrag(S ^ 1, j);
        float q[H];
        __builtin_amdgcn_s_setprio(1);   // the matrix phases first (1 to 2 %)
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < KB * KS; ++j) {
          nxt[j % KB] = mfma32(kr[j & 3], qf[j / KB], j < KB ? f32x16{} : nxt[j % KB]);
          if (j + 4 < KB * KS) kr[j & 3] = kfrag(S ^ 1, j + 4);
          constexpr int NS = KB * KS;
          const int i0 = H * j / NS, i1 = H * (j + 1) / NS;
#pragma unroll
          for (int i = i0; i < i1; ++i) {
            q[i] = pexp(cur, H + i, mu);
            psum += q[i];
          }
          if (i1 / 8 != i0 / 8) {
            const int k = i1 / 8 - 1;
            pf[KB + k] = pack8(q + 8 * k);
            asm volatile("" : "+v"(pf[KB + k]));
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (__any(!(psum <= 65536.f) || m_run == -INFINITY)) slow_tile(cur, pf, psum);
        l_run += psum;
      }
      if (masked(x)) odd_values(cur, x, &sVb[S][0]);
      if (next && active) mask_tile(nxt, x + 1);
      // the tiles asked for after the next barrier: V follows K
      at_v = at_k;
      if (x + 3 < n) {
        pages.ahead((key_base + (x + 3) * BK) >> a.psl, last);
        at_k = locate(x + 3);
      }
      if (active) {
        const float mu1 = m_off();
        const char* sV = &sVb[S][0];
        auto vfrag = [&](int st) { return ld_tr_swz<D>(sV, (st / DB) * 16, (st % DB) * 32); };
        bf16x8 vr[4];
#pragma unroll
        for (int st = 0; st < 4; ++st) vr[st] = vfrag(st);
        float q[H];
        psum_a = 0.f;
        __builtin_amdgcn_s_setprio(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int st = 0; st < 2 * KB * DB; ++st) {
          oacc[st % DB] = mfma32(vr[st & 3], pf[st / DB], oacc[st % DB]);
          if (st + 4 < 2 * KB * DB) vr[st & 3] = vfrag(st + 4);
          constexpr int NS = 2 * KB * DB;
          const int i0 = H * st / NS, i1 = H * (st + 1) / NS;
#pragma unroll
          for (int i = i0; i < i1; ++i) {
            q[i] = pexp(nxt, i, mu1);
            psum_a += q[i];
          }
          if (i1 / 8 != i0 / 8) {
            const int k = i1 / 8 - 1;
            pf[k] = pack8(q + 8 * k);
            asm volatile("" : "+v"(pf[k]));
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        asm volatile("" : "+v"(psum_a));
        __builtin_amdgcn_s_setprio(0);
      }
    };
    if (keys) {
      for (int x = 0; x < n; x += 2) {
        step(std::integral_constant<int, 0>{}, x);
        if (x + 1 < n) step(std::integral_constant<int, 1>{}, x + 1);
      }
    }
    const float l = l_run + __shfl_xor(l_run, 32);
    if (const int m = my(); m < t.rows) {
      const TreeArgs& b = again();
      const Pair mine = pair(b);
      if (deal.whole()) {
        const float inv = l == 0.f ? 0.f : 1.f / l;   // l is 0 where no key was seen
        u16* op = b.o + (mine.row * b.Hq + mine.h) * D + here(g) * 4;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4)
            *reinterpret_cast<uint2*>(op + db * 32 + q4 * 8) =
                make_uint2(pack2(oacc[db][q4 * 4 + 0] * inv, oacc[db][q4 * 4 + 1] * inv),
                           pack2(oacc[db][q4 * 4 + 2] * inv, oacc[db][q4 * 4 + 3] * inv));
        if (g == 0)
          b.lse[int64_t(mine.h) * b.N + mine.row] = lse_of(m_run, l);
      } else {
        const int64_t s = deal.slot() * R + m;
        float* op = b.part_o + s * D + here(g) * 4;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4)
            *reinterpret_cast<float4*>(op + db * 32 + q4 * 8) =
                make_float4(oacc[db][q4 * 4 + 0], oacc[db][q4 * 4 + 1], oacc[db][q4 * 4 + 2],
                            oacc[db][q4 * 4 + 3]);
        if (g == 0) {
          b.part_ml[s * 2] = m_run;
          b.part_ml[s * 2 + 1] = l;
        }
      }
    }
    deal.note();
    lds_barrier();   // the tiles are read before the next segment's loads
  }
}

// Whether a record can be one (if row_ptr is not as it should be, some are not
// written): all it names lies inside the arrays.
template <int R>
__device__ __forceinline__ bool sound(const TreeArgs& a, const TreeJoin& j) {
  return j.rows <= R && j.run >= 0 && j.runs >= 0 && int64_t(j.run) + j.runs <= a.groups &&
         unsigned(j.slot) < 2u * unsigned(a.groups) && j.m0 >= 0 && j.m0 <= INT32_MAX - R &&
         j.r0 >= 0 && int64_t(j.r0) + by_heads(a, j.m0 + j.rows - 1) < a.N;
}

// --------------------------------------------------------------------------
// Joins the segments of a tile, in their order: block (tile place, KV head,
// RG pairs), JG groups of D / 8 threads to a pair, each for every JG-th segment.
// Bound by the read of the partial results (the chunks above: 65 MB read, 17 MB
// written in 13 us, 6 TB/s), or by its two dependent reads (one token: 3.2 us).
// --------------------------------------------------------------------------
template <int D, int R, int JG>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs a) {
  constexpr int TD = D / 8, RG = 256 / (TD * JG), NG = R / RG, U = 4;
  __shared__ float so[JG][RG][D], sml[JG][RG][2];
  const int rg = blockIdx.x % NG;
  const TreeJoin jn = a.join[blockIdx.x / NG];
  const int hk = blockIdx.x / NG % a.Hkv;
  if (rg * RG >= jn.rows || !sound<R>(a, jn)) return;   // block-uniform
  const int d0 = (threadIdx.x % TD) * 8, rr = threadIdx.x / TD % RG, jg = threadIdx.x / (TD * RG);
  const int r = rg * RG + rr;
  float M = -INFINITY, l = 0.f, y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (r < jn.rows) {
    for (int j0 = jg; j0 < jn.runs; j0 += JG * U) {
      float2 ml[U];
      float4 oj[U][2];
#pragma unroll
      for (int x = 0; x < U; ++x) {
        const int j = min(j0 + x * JG, jn.runs - 1);
        const int64_t s = int64_t(j == 0 ? jn.slot : 2 * (jn.run + j)) * R + r;
        ml[x] = *reinterpret_cast<const float2*>(a.part_ml + 2 * s);
        oj[x][0] = *reinterpret_cast<const float4*>(a.part_o + s * D + d0);
        oj[x][1] = *reinterpret_cast<const float4*>(a.part_o + s * D + d0 + 4);
      }
      float Mn = M;
#pragma unroll
      for (int x = 0; x < U; ++x) Mn = fmaxf(Mn, ml[x].x);   // (the last one again does not matter)
      float f = weight(M, Mn);
      l *= f;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] *= f;
#pragma unroll
      for (int x = 0; x < U; ++x) {
        if (j0 + x * JG >= jn.runs) break;
        f = weight(ml[x].x, Mn);
        l += ml[x].y * f;
        y[0] += oj[x][0].x * f, y[1] += oj[x][0].y * f;
        y[2] += oj[x][0].z * f, y[3] += oj[x][0].w * f;
        y[4] += oj[x][1].x * f, y[5] += oj[x][1].y * f;
        y[6] += oj[x][1].z * f, y[7] += oj[x][1].w * f;
      }
      M = Mn;
    }
  }
  if (JG > 1) {
    float* o = &so[jg][rr][d0];
    *reinterpret_cast<float4*>(o) = make_float4(y[0], y[1], y[2], y[3]);
    *reinterpret_cast<float4*>(o + 4) = make_float4(y[4], y[5], y[6], y[7]);
    if (d0 == 0) {
      sml[jg][rr][0] = M;
      sml[jg][rr][1] = l;
    }
    __syncthreads();
    if (jg != 0) return;
#pragma unroll
    for (int j = 1; j < JG; ++j) M = fmaxf(M, sml[j][rr][0]);
    l = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = 0.f;
#pragma unroll
    for (int j = 0; j < JG; ++j) {
      const float f = weight(sml[j][rr][0], M);
      l += sml[j][rr][1] * f;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] += so[j][rr][d0 + e] * f;
    }
  }
  if (r >= jn.rows) return;
  Tile t{};
  t.r0 = jn.r0;
  const Pair pr(a, t, hk, jn.m0 + r);
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] *= inv;
  store_v<8>(a.o + (pr.row * a.Hq + pr.h) * D + d0, y);
  if (d0 == 0)
    a.lse[int64_t(pr.h) * a.N + pr.row] = lse_of(M, l);
}

// A thread to a row: up the parents, its words from the highest down.  Latency:
// 24 trees of 8 to 61 tokens 4.6 us, 9 of 5 to 33 3.1.  (The parents held in LDS
// for the walk made no difference.)
__global__ __launch_bounds__(256) void tree_mask_kernel(int B, int N, const int32_t* __restrict__ ptr,
                                                        const int32_t* __restrict__ parent, int W,
                                                        uint32_t* __restrict__ tree,
                                                        int32_t* __restrict__ depth) {
  const int64_t place = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (place >= min(N, ptr[B])) return;
  const int t = int(place);
  int lo = 0, hi = B;   // the entry: the last with ptr <= t
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (ptr[mid] <= t) lo = mid; else hi = mid;
  }
  const int64_t r0 = min(max(ptr[lo], 0), t);
  uint32_t* out = tree + int64_t(t) * W;
  int w = W - 1, d = -1, x = int(t - r0);
  uint32_t bits = 0;
  while (x >= 0) {
    const int wx = x >> 5;
    for (; w > wx; --w) {
      out[w] = bits;
      bits = 0;
    }
    if (wx < W) bits |= 1u << (x & 31);
    ++d;
    const int p = parent[r0 + x];
    x = p < x ? p : -1;   // a row's ancestors come before it: the walk ends
  }
  for (; w >= 0; --w) {
    out[w] = bits;
    bits = 0;
  }
  if (depth) depth[t] = d;
}

// --------------------------------------------------------------------------
// launches
// --------------------------------------------------------------------------
constexpr int kFewWaves = 2, kWholeWaves = 8;
// Few pairs, sequences known not to be long and no more tiles than two to a CU:
// whole tiles by eight waves each, one launch in place of two and no deal.  A
// round of 256 keys takes 1.15 us, so where single tiles leave the chip idle the
// deal's splitting wins from some 1600 keys on, where they fill a good part of it
// later (us, whole / dealt and joined, 28/4 heads of 128: 1 sequence of 1024
// keys 14.5 / 16.2, of 2048 19.3 / 16.6; 16 of 1024 15.6 / 27.3, of 4096 32.9 /
// 37.0, of 512 to 4096 30.4 / 29.6; 32 of 512 to 4096 33.6 / 37.0; 64 of 1024
// 35.2 / 37.8, of 2048 60.7 / 56.0; 128 of 512 39.2 / 41.4, 256 of 64 39.9 / 35.0).
constexpr int kWholeLen = 1536, kWholeLenMid = 4096;
// Pairs per entry up to which the kernel for few pairs is used
constexpr int kFewPairs = 32;

struct TreePlan {
  bool many, whole;
  int R, tiles, groups;
  size_t o_bytes, ml_bytes, bytes;
};

// Two workgroups to a CU; no more than there are units, if the longest
// sequence is known.
static int tree_groups(const mv_cache_shape& c, const mv_tree_attn_shape& s, int64_t tiles) {
  const int64_t groups = 2 * kNumCu;
  if (s.max_len <= 0) return int(groups);
  return int(std::min(groups, tiles * c.n_heads_kv * ((int64_t(s.max_len) + kUnit - 1) / kUnit)));
}

static TreePlan tree_plan(const mv_cache_shape& c, const mv_tree_attn_shape& s) {
  TreePlan p;
  const int G = s.n_heads_q / c.n_heads_kv;
  const int64_t pairs = int64_t(s.n_rows) * G;
  p.many = pairs > int64_t(kFewPairs) * s.n_batch;
  p.R = p.many ? 128 : 32;
  p.tiles = int(pairs / p.R) + s.n_batch;
  const int64_t whole = int64_t(p.tiles) * c.n_heads_kv;   // workgroups, if so
  const bool mid = whole >= kNumCu / 4 && whole < kNumCu;
  p.whole = !p.many && s.max_len > 0 && s.max_len <= (mid ? kWholeLenMid : kWholeLen) &&
            whole <= 2 * kNumCu;
  p.groups = tree_groups(c, s, p.tiles);
  p.o_bytes = size_t(2 * p.groups) * p.R * c.head_dim * 4;
  p.ml_bytes = size_t(2 * p.groups) * p.R * 2 * 4;
  p.bytes = p.o_bytes + p.ml_bytes + sizeof(TreeJoin) * p.tiles * c.n_heads_kv;
  return p;
}

// What any call of at most this many rows and entries needs: which kernel it
// takes depends on both.
size_t tree_attn_ws_bytes(const mv_cache_shape& c, const mv_tree_attn_shape& s) {
  const int G = s.n_heads_q / c.n_heads_kv;
  const int64_t tiles = int64_t(s.n_rows) * G / 32 + s.n_batch;
  return size_t(2 * tree_groups(c, s, tiles)) * 128 * (c.head_dim + 2) * 4 +
         sizeof(TreeJoin) * size_t(tiles) * c.n_heads_kv;
}

// Whether the deal fits its LDS and the join a launch (2^32 threads)
bool tree_attn_fits(const mv_cache_shape& c, const mv_tree_attn_shape& s) {
  const TreePlan p = tree_plan(c, s);
  return p.tiles <= kChunks * (p.many ? 256 : 64 * kFewWaves) &&
         int64_t(p.tiles) * c.n_heads_kv * (p.R * c.head_dim / 2048) < (int64_t(1) << 24);
}

template <int D>
static hipError_t launch_tree(const TreePlan& p, TreeArgs a, hipStream_t stream) {
  {
    ProfScope prof("tree_attn", stream);
    if (p.many)
      hipLaunchKernelGGL((tree_many_kernel<D>), dim3(p.groups), dim3(256), 0, stream, a);
    else if (p.whole)
      hipLaunchKernelGGL((tree_few_kernel<D, kWholeWaves, true>), dim3(p.tiles * a.Hkv),
                         dim3(64 * kWholeWaves), 0, stream, a);
    else
      hipLaunchKernelGGL((tree_few_kernel<D, kFewWaves, false>), dim3(p.groups),
                         dim3(64 * kFewWaves), 0, stream, a);
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  // every tile was one workgroup's
  if (p.whole || p.groups == 1) return hipSuccess;
  ProfScope prof("tree_combine", stream);
  // The more segments a tile has on average, the more groups of threads share a
  // pair's, which otherwise wait for one after another (us by one, four and
  // sixteen groups: 9 trees, 17 segments a tile, - / 10.2 / 7.4; 16 trees, 5
  // segments, 10.4 / 7.5 / -); with fewer segments than threads to read them the
  // blocks are only smaller (8 trees, 8 segments, - / 8.5 / 10.8; 24 trees of 64
  // tokens, 3 segments, 12.6 / 16.7 / -).  Tiles of 32 pairs are single tokens',
  // whose long ones have many more than the average (64 tokens over 257 to 16384
  // rows, 2 segments, 8.4 / 7.1 / -).
  const int64_t segments = p.groups / (int64_t(p.tiles) * a.Hkv);
#define MV_JOIN(R, JG)                                                                         \
  hipLaunchKernelGGL((tree_join_kernel<D, R, JG>),                                             \
                     dim3(unsigned(p.tiles * a.Hkv * (R * JG * D / 2048))), dim3(256), 0, stream, \
                     a)
  if (p.many) {
    if (segments >= 16) MV_JOIN(128, 16);
    else if (segments >= 4) MV_JOIN(128, 4);
    else MV_JOIN(128, 1);
  } else {
    if (segments >= 16) MV_JOIN(32, 16);
    else if (segments >= 1) MV_JOIN(32, 4);
    else MV_JOIN(32, 1);
  }
#undef MV_JOIN
  return hipGetLastError();
}

hipError_t launch_tree_attn(const mv_cache_shape& cs, const CacheDev& cd, int layer,
                            const mv_tree_attn_shape& s, float scale, const int32_t* ids,
                            const int32_t* ptr, const uint32_t* tree, const void* q, void* o,
                            float* lse, void* ws, hipStream_t stream) {
  const TreePlan p = tree_plan(cs, s);
  const int64_t plane = int64_t(layer) * cs.n_pages * cs.n_heads_kv * cs.page_size * cs.head_dim;
  TreeArgs a;
  a.q = static_cast<const u16*>(q);
  a.k = cd.k + plane;
  a.v = cd.v + plane;
  a.o = static_cast<u16*>(o);
  a.lse = lse;
  char* w = static_cast<char*>(ws);
  a.part_o = reinterpret_cast<float*>(w);
  a.part_ml = reinterpret_cast<float*>(w + p.o_bytes);
  a.join = reinterpret_cast<TreeJoin*>(w + p.o_bytes + p.ml_bytes);
  a.table = cd.table;
  a.len = cd.len;
  a.ids = ids;
  a.ptr = ptr;
  a.tree = tree;
  a.words = s.tree_words;
  a.B = s.n_batch;
  a.N = s.n_rows;
  a.Hq = s.n_heads_q;
  a.Hkv = cs.n_heads_kv;
  a.G = s.n_heads_q / cs.n_heads_kv;
  a.g_shift = 31;
  while ((1 << (a.g_shift - 31)) < a.G) ++a.g_shift;
  a.g_mul = uint32_t(((uint64_t(1) << a.g_shift) + a.G - 1) / a.G);
  a.n_pages = cs.n_pages;
  a.n_seqs = cs.n_seqs;
  a.max_pages = cs.max_pages;
  a.psl = cd.psl;
  a.tiles = p.tiles;
  a.groups = p.groups;
  a.scale_log2 = scale * 1.4426950408889634f;
  return cs.head_dim == 128 ? launch_tree<128>(p, a, stream) : launch_tree<64>(p, a, stream);
}

hipError_t launch_tree_mask(int B, int N, const int32_t* ptr, const int32_t* parent, int words,
                            uint32_t* tree, int32_t* depth, hipStream_t stream) {
  ProfScope prof("tree_mask", stream);
  hipLaunchKernelGGL(tree_mask_kernel, dim3(unsigned((int64_t(N) + 255) / 256)), dim3(256), 0,
                     stream, B, N, ptr, parent, words, tree, depth);
  return hipGetLastError();
}

}  // namespace mv
