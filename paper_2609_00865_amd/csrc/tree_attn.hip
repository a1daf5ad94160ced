// Attention of a sequence's newest rows (one decoded token, a tree of drafted
// ones, a chunk of a prompt) over its rows in a paged cache, on gfx950.
//
// A tile is up to 32 (query row, query head) pairs of one KV head: they read
// the same keys.  A workgroup takes a tile's run of 64-key units; its waves
// take 32-key tiles of that run in turn, each with K and V of its own in LDS
// (two buffers, filled by direct loads a tile ahead, no barrier between
// waves), S^T = K Q^T and O^T += V^T P^T with bf16 MFMA (a query per lane, so
// the softmax statistics stay in a lane pair) and a running maximum and sum in
// fp32; the waves' results meet in LDS.
//
// With few tiles the work is the reading of long caches, so every tile's
// units are cut into runs of one common length, chosen on the device from
// the sequences' lengths: the workgroups then do equal work however uneven
// the batch is, and a second pass joins the runs of a tile in order.
#include "mv_cache_dev.h"

namespace mv {

struct TreeArgs {
  const u16* q;
  const u16* k;        // of the layer
  const u16* v;
  u16* o;
  float* lse;
  float* part_o;       // [slots][R][D] unnormalised
  float* part_ml;      // [slots][R][2] maximum (base 2, scaled), sum
  const int32_t* table;
  const int32_t* len;
  const int32_t* ids;
  const int32_t* ptr;
  const uint32_t* tree;
  int words;
  int B, N, Hq, Hkv, G, n_pages, n_seqs, max_pages, psl;
  int tiles;           // tile places: at least as many as there are tiles
  int target;          // runs aimed at, over all KV heads
  float scale_log2;
};

constexpr int kUnit = 64;      // keys of a unit of work
constexpr int kPlanB = 1024;   // entries whose sizes are held in LDS

struct TreeShared {
  int ptr[kPlanB + 1];
  int len[kPlanB];
  int tmp[17];
  int found[4];
};

// One tile: the entry, its first pair, and the keys any of its rows may see.
struct Tile {
  int b, n, c;      // entry, its rows, its context rows (negative: absent rows)
  int r0;           // its first row of q
  int m0, rows;     // first pair and pairs of the tile (0: no such tile)
  int kmax;         // keys [0, kmax)
};

// Entry b's first tile place: places of entries never overlap, because
// ceil(n G / R) <= floor((r + n) G / R) - floor(r G / R) + 1.
template <int R>
__device__ __forceinline__ int first_place(int64_t r, int b, int G) {
  return int(r * G / R) + b;
}

template <int R>
__device__ __forceinline__ Tile tile_of(const TreeArgs& a, const TreeShared& s, int u) {
  const bool lds = a.B <= kPlanB;
  auto at = [&](int b) { return lds ? s.ptr[b] : min(max(a.ptr[b], 0), a.N); };
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first_place<R>(at(mid), mid, a.G) <= u) lo = mid; else hi = mid;
  }
  Tile t;
  t.b = lo;
  t.r0 = at(lo);
  t.n = max(0, at(lo + 1) - t.r0);
  t.m0 = (u - first_place<R>(t.r0, lo, a.G)) * R;
  t.rows = t.m0 >= 0 ? min(R, t.n * a.G - t.m0) : 0;
  t.kmax = t.c = 0;
  if (t.rows <= 0) {
    t.rows = 0;
    return t;
  }
  int L;
  if (lds) {
    L = s.len[lo];
  } else {
    const int id = a.ids[lo];
    L = unsigned(id) < unsigned(a.n_seqs)
            ? int(min(int64_t(max(a.len[id], 0)), int64_t(a.max_pages) << a.psl)) : 0;
  }
  t.c = L - t.n;
  const int last = (t.m0 + t.rows - 1) / a.G;
  t.kmax = a.tree ? L : max(0, t.c + last + 1);
  return t;
}

__device__ __forceinline__ void load_sizes(const TreeArgs& a, TreeShared& s) {
  if (a.B <= kPlanB) {
    for (int b = threadIdx.x; b <= a.B; b += blockDim.x) {
      s.ptr[b] = min(max(a.ptr[b], 0), a.N);
      if (b < a.B) {
        const int id = a.ids[b];
        s.len[b] = unsigned(id) < unsigned(a.n_seqs)
                       ? int(min(int64_t(max(a.len[id], 0)), int64_t(a.max_pages) << a.psl)) : 0;
      }
    }
  }
  __syncthreads();
}

// The run length (in units) that cuts the tiles of all KV heads into about
// `target` runs.  A tile without keys is one unit: its rows are still written.
template <int R, int BLOCK>
__device__ __forceinline__ int run_length(const TreeArgs& a, TreeShared& s) {
  int64_t sum = 0;
  for (int u = threadIdx.x; u < a.tiles; u += BLOCK) {
    const Tile t = tile_of<R>(a, s, u);
    if (t.rows) sum += max(1, (t.kmax + kUnit - 1) / kUnit);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  __shared__ int64_t part[BLOCK / 64];
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  int64_t all = 0;
#pragma unroll
  for (int w = 0; w < BLOCK / 64; ++w) all += part[w];
  return int(max(int64_t(1), (all * a.Hkv + a.target - 1) / a.target));
}

// What a partial result with maximum m counts for beside maximum M.  Without
// a maximum it holds nothing (or only NaN, which has to stay).
__device__ __forceinline__ float weight(float m, float M) {
  return m == -INFINITY ? 1.f : fast_exp2(m - M);
}

// The tile and run of workgroup w of a KV head: found[0] = tile place,
// found[1] = run, found[2] = runs of the tile; found[0] = -1 past the last.
// With by_tile, w is a tile place and found[1] the tile's first run among all.
template <int R, int BLOCK>
__device__ __forceinline__ void find_run(const TreeArgs& a, TreeShared& s, int run, int w,
                                         bool by_tile) {
  if (threadIdx.x == 0) s.found[0] = -1;
  int before = 0;
  for (int u0 = 0; u0 < a.tiles; u0 += BLOCK) {
    const int u = u0 + threadIdx.x;
    int mine = 0, total;
    if (u < a.tiles) {
      const Tile t = tile_of<R>(a, s, u);
      if (t.rows) mine = (max(1, (t.kmax + kUnit - 1) / kUnit) + run - 1) / run;
    }
    const int first = before + block_scan<BLOCK>(mine, s.tmp, total);
    if (by_tile ? u == w && mine > 0 : w >= first && w < first + mine) {
      s.found[0] = u;
      s.found[1] = by_tile ? first : w - first;
      s.found[2] = mine;
    }
    before += total;
  }
  __syncthreads();
}

// The keys of [key0, key0 + 32) that new row i of a tile's entry sees, as bits.
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

// NW waves, each with two K and two V tiles of 32 keys.
template <int D, int NW>
__global__ __launch_bounds__(NW * 64) void tree_attn_kernel(TreeArgs a) {
  constexpr int R = 32, BLOCK = NW * 64;
  constexpr int KS = D / 16, DB = D / 32;
  constexpr int TB = 32 * D * 2;             // bytes of a tile
  constexpr int NI = TB / 1024;              // 1 KiB loads of a tile
  constexpr int LR = 512 / D;                // rows of a load
  constexpr int PG = 128;                    // page ids held per wave
  constexpr int OS = D + 4;                  // floats of a row of O where the waves meet
  static_assert(R * OS * 4 <= 4 * TB, "a wave's O fits its tiles");
  __shared__ __align__(1024) char buf[NW][4 * TB];   // K, K, V, V
  __shared__ TreeShared sh;
  __shared__ int pg[NW][PG];
  __shared__ float sm[NW][R], sl[NW][R];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int c = lane & 31, g = lane >> 5;
  const int hk = blockIdx.x % a.Hkv;

  load_sizes(a, sh);
  const int run = run_length<R, BLOCK>(a, sh);
  find_run<R, BLOCK>(a, sh, run, blockIdx.x / a.Hkv, false);
  const int place = sh.found[0];
  if (place < 0) return;
  const int ri = sh.found[1], runs = sh.found[2];
  const Tile t = tile_of<R>(a, sh, place);
  const int id = a.ids[t.b];
  const int64_t row0 = t.r0;

  // Q^T as the B operand: lane holds pair c, dims ks*16 + g*8 .. + 8
  const bool qok = c < t.rows;
  const int m = t.m0 + (qok ? c : 0);
  const int qi = m / a.G;
  const int64_t qrow = row0 + qi;
  const int64_t qat = (qrow * a.Hq + hk * a.G + (m - qi * a.G)) * D;
  bf16x8 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
    qf[ks] = as_bf16x8(qok ? ld16(a.q + qat + ks * 16 + g * 8) : make_uint4(0, 0, 0, 0));

  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;

  // this run's keys; wave w takes 32-key tiles w, w + NW, ...
  const int units = max(1, (t.kmax + kUnit - 1) / kUnit);
  const int k_begin = int(int64_t(ri) * run) * kUnit;
  const int k_end = int(min(int64_t(t.kmax), int64_t(min(units, (ri + 1) * run)) * kUnit));
  const int nt = max(0, (k_end - k_begin + 31) / 32);
  const int mine = nt > wave ? (nt - wave + NW - 1) / NW : 0;
  auto key_of = [&](int x) { return k_begin + (wave + x * NW) * 32; };

  // page ids of the keys ahead: entries [pg0, pg0 + PG) of the sequence's table
  const int last = t.kmax - 1;
  const int ps = 1 << a.psl;
  int pg0 = -PG;
  auto fill_pages = [&](int first) {
    pg0 = first;
    for (int j = lane; j < PG; j += 64) {
      int p = 0;
      if (first + j <= last >> a.psl) {
        p = a.table[int64_t(id) * a.max_pages + first + j];
        p = unsigned(p) < unsigned(a.n_pages) ? p : 0;
      }
      pg[wave][j] = p;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  const int64_t page_bytes = int64_t(a.Hkv) * ps * D * 2;
  const char* kb = reinterpret_cast<const char*>(a.k) + int64_t(hk) * ps * D * 2;
  const char* vb = reinterpret_cast<const char*>(a.v) + int64_t(hk) * ps * D * 2;
  const int lrow = lane / (D / 8), lpos = lane % (D / 8);
  const uint32_t lds0 = lds_addr(&buf[wave][0]);
  // Tile x of this wave into buffer x & 1.  Keys past the last read the last
  // (a load's rows lie in one page; what is past it is masked).
  auto issue = [&](int x) {
    const int key0 = key_of(x);
    const int p_lo = min(key0, last) >> a.psl, p_hi = min(key0 + 31, last) >> a.psl;
    if (p_lo < pg0 || p_hi >= pg0 + PG) fill_pages(p_lo);
    const uint32_t kl = lds0 + uint32_t(x & 1) * TB;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int key = min(key0 + j * LR, last);
      const int64_t page = __builtin_amdgcn_readfirstlane(pg[wave][(key >> a.psl) - pg0]);
      const int r = j * LR + lrow;
      const uint32_t off = uint32_t(min(key0 + r, last) & (ps - 1)) * (D * 2) +
                           uint32_t((lpos ^ kv_swz<D>(r)) << 4);
      lds_load16s(uniform_ptr(kb + page * page_bytes), off, kl + j * 1024);
      lds_load16s(uniform_ptr(vb + page * page_bytes), off, kl + 2 * TB + j * 1024);
    }
  };

  if (mine > 0) issue(0);
  if (mine > 1) issue(1);
  const int clear = a.tree ? t.c : t.c + t.m0 / a.G + 1;   // keys every row of the tile sees
  for (int x = 0; x < mine; ++x) {
    // the tile has landed (the next one's loads may be in flight)
    if (x + 1 < mine)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NI) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const char* sK = &buf[wave][(x & 1) * TB];
    const char* sV = sK + 2 * TB;
    f32x16 sc = {};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) sc = mfma32(ld_row_swz<D>(sK, c, ks * 2 + g), qf[ks], sc);
    const int key0 = key_of(x);
    uint32_t see = ~0u;
    const bool masked = key0 + 32 > min(clear, k_end);   // wave-uniform
    if (masked) {
      const int n = k_end - key0;
      see = seen32(a, t, qrow, qi, key0) & (n >= 32 ? ~0u : (1u << n) - 1u);
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
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sc[r] = fast_exp2(fmaf(sc[r], a.scale_log2, -mu));
      l_run += sc[r];
    }
    if (masked) {
      // A value that is not finite in a row that some query does not see
      // would reach it as 0 * inf: such elements are taken out of the tile
      // and added, query by query, where they are seen.
      bool odd = false;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const uint4 x4 = ld16(sV + j * 1024 + lane * 16);
        const uint32_t w[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          odd |= (w[e] & 0x7f80u) == 0x7f80u || (w[e] & 0x7f800000u) == 0x7f800000u;
      }
      if (__any(odd)) {
        for (int key = 0; key < 32; ++key) {
          const int rr = (key >> 3) * 4 + (key & 3), hh = (key >> 2) & 1;
          float p = 0.f;
#pragma unroll
          for (int r = 0; r < 16; ++r) p = r == rr ? sc[r] : p;
          p = __shfl(p, c + 32 * hh);
          if (!__any((see >> key) & 1u)) continue;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int dim = db * 32 + (r >> 2) * 8 + g * 4 + (r & 3);
              const u16 b = *reinterpret_cast<const u16*>(
                  sV + key * (D * 2) + (((dim >> 3) ^ kv_swz<D>(key)) << 4) + (dim & 7) * 2);
              if ((b & 0x7f80u) == 0x7f80u && ((see >> key) & 1u))
                oacc[db][r] += p * bf16_to_f32(b);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        char* wV = const_cast<char*>(sV);
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          uint4 x4 = ld16(wV + j * 1024 + lane * 16);
          uint32_t w[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if ((w[e] & 0x7f80u) == 0x7f80u) w[e] &= 0xffff0000u;
            if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] &= 0xffffu;
          }
          st16(wV + j * 1024 + lane * 16, make_uint4(w[0], w[1], w[2], w[3]));
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
    }
    const bf16x8 pf[2] = {to_operand(sc, 0), to_operand(sc, 8)};
#pragma unroll
    for (int st = 0; st < 2 * DB; ++st)
      oacc[st % DB] = mfma32(ld_tr_swz<D>(sV, (st / DB) * 16, (st % DB) * 32), pf[st / DB],
                             oacc[st % DB]);
    if (x + 2 < mine) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the buffer's reads are done
      issue(x + 2);
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
    for (int q4 = 0; q4 < 4; ++q4) {
      float4 x4;
      x4.x = oacc[db][q4 * 4 + 0] * f;
      x4.y = oacc[db][q4 * 4 + 1] * f;
      x4.z = oacc[db][q4 * 4 + 2] * f;
      x4.w = oacc[db][q4 * 4 + 3] * f;
      *reinterpret_cast<float4*>(so + c * OS + db * 32 + q4 * 8 + g * 4) = x4;
    }
  __syncthreads();
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
      const float* p = reinterpret_cast<const float*>(&buf[w][0]) + r * OS + d0;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] += p[e];
    }
    if (runs == 1) {
      const int mm = t.m0 + r, i = mm / a.G, h = hk * a.G + mm - i * a.G;
      const float inv = l == 0.f ? 0.f : 1.f / l;   // l is 0 where no key was seen
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] *= inv;
      store_v<8>(a.o + ((row0 + i) * a.Hq + h) * D + d0, y);
      if (d0 == 0)
        a.lse[int64_t(h) * a.N + row0 + i] =
            l == 0.f ? -INFINITY : (Mr + __log2f(l)) * 0.69314718055994531f;
    } else {
      float* p = a.part_o + (int64_t(blockIdx.x) * R + r) * D + d0;
      *reinterpret_cast<float4*>(p) = make_float4(y[0], y[1], y[2], y[3]);
      *reinterpret_cast<float4*>(p + 4) = make_float4(y[4], y[5], y[6], y[7]);
      if (d0 == 0) {
        a.part_ml[(int64_t(blockIdx.x) * R + r) * 2] = Mr;
        a.part_ml[(int64_t(blockIdx.x) * R + r) * 2 + 1] = l;
      }
    }
  }
}

// Joins the runs of a tile, in their order: block (tile place, KV head, rows
// rg * RG ..), a thread to 8 elements of a row.
template <int D, int R>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeArgs a) {
  constexpr int RG = 256 / (D / 8);   // rows of a block
  constexpr int NG = (R + RG - 1) / RG;
  __shared__ TreeShared sh;
  int x = blockIdx.x;
  const int rg = x % NG;
  x /= NG;
  const int hk = x % a.Hkv, place = x / a.Hkv;
  load_sizes(a, sh);
  const Tile t = tile_of<R>(a, sh, place);
  const int r = rg * RG + threadIdx.x / (D / 8), d0 = (threadIdx.x % (D / 8)) * 8;
  if (rg * RG >= t.rows) return;   // block-uniform
  const int run = run_length<R, 256>(a, sh);
  find_run<R, 256>(a, sh, run, place, true);
  const int first = sh.found[1], runs = sh.found[2];
  if (runs <= 1 || r >= t.rows) return;
  float M = -INFINITY;
  for (int j = 0; j < runs; ++j)
    M = fmaxf(M, a.part_ml[((int64_t(first + j) * a.Hkv + hk) * R + r) * 2]);
  float l = 0.f, y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int j = 0; j < runs; ++j) {
    const int64_t s = (int64_t(first + j) * a.Hkv + hk) * R + r;
    const float mj = a.part_ml[2 * s], lj = a.part_ml[2 * s + 1];
    const float f = weight(mj, M);
    l += lj * f;
    const float4 u = *reinterpret_cast<const float4*>(a.part_o + s * D + d0);
    const float4 v = *reinterpret_cast<const float4*>(a.part_o + s * D + d0 + 4);
    y[0] += u.x * f, y[1] += u.y * f, y[2] += u.z * f, y[3] += u.w * f;
    y[4] += v.x * f, y[5] += v.y * f, y[6] += v.z * f, y[7] += v.w * f;
  }
  const int mm = t.m0 + r, i = mm / a.G, h = hk * a.G + mm - i * a.G;
  const int64_t row = int64_t(t.r0) + i;
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] *= inv;
  store_v<8>(a.o + (row * a.Hq + h) * D + d0, y);
  if (d0 == 0)
    a.lse[int64_t(h) * a.N + row] =
        l == 0.f ? -INFINITY : (M + __log2f(l)) * 0.69314718055994531f;
}

// A thread to a row: up the parents, its words from the highest down.
__global__ __launch_bounds__(256) void tree_mask_kernel(int B, int N, const int32_t* __restrict__ ptr,
                                                        const int32_t* __restrict__ parent, int W,
                                                        uint32_t* __restrict__ tree,
                                                        int32_t* __restrict__ depth) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= min(N, ptr[B])) return;
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
struct TreePlan {
  int tiles, target;
  int64_t blocks;        // workgroups: runs there can be, over all KV heads
  size_t o_bytes, bytes;
};

static TreePlan tree_plan(const mv_cache_shape& c, const mv_tree_attn_shape& s) {
  constexpr int R = 32;
  TreePlan p;
  const int G = s.n_heads_q / c.n_heads_kv;
  p.tiles = int(int64_t(s.n_rows) * G / R) + s.n_batch;
  // Two workgroups to a CU, four of them in turn; not more than there are
  // units if the longest sequence is known.
  int64_t target = 4 * kNumCu;
  if (s.max_len > 0)
    target = std::min(target, int64_t(p.tiles) * c.n_heads_kv * ((s.max_len + kUnit - 1) / kUnit));
  p.target = int(std::max<int64_t>(1, target));
  p.blocks = int64_t(p.target) + int64_t(p.tiles) * c.n_heads_kv;
  p.o_bytes = size_t(p.blocks) * R * c.head_dim * 4;
  p.bytes = p.o_bytes + size_t(p.blocks) * R * 2 * 4;
  return p;
}

size_t tree_attn_ws_bytes(const mv_cache_shape& c, const mv_tree_attn_shape& s) {
  return tree_plan(c, s).bytes;
}

int64_t tree_attn_blocks(const mv_cache_shape& c, const mv_tree_attn_shape& s) {
  return tree_plan(c, s).blocks;
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
  a.part_o = static_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) + p.o_bytes);
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
  a.n_pages = cs.n_pages;
  a.n_seqs = cs.n_seqs;
  a.max_pages = cs.max_pages;
  a.psl = cd.psl;
  a.tiles = p.tiles;
  a.target = p.target;
  a.scale_log2 = scale * 1.4426950408889634f;
  const int combine = p.tiles * cs.n_heads_kv;
  if (cs.head_dim == 128) {
    {
      ProfScope prof("tree_attn", stream);
      hipLaunchKernelGGL((tree_attn_kernel<128, 2>), dim3(unsigned(p.blocks)), dim3(128), 0,
                         stream, a);
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    ProfScope prof("tree_combine", stream);
    hipLaunchKernelGGL((tree_combine_kernel<128, 32>), dim3(unsigned(combine * 2)), dim3(256), 0,
                       stream, a);
  } else {
    {
      ProfScope prof("tree_attn", stream);
      hipLaunchKernelGGL((tree_attn_kernel<64, 2>), dim3(unsigned(p.blocks)), dim3(128), 0, stream,
                         a);
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    ProfScope prof("tree_combine", stream);
    hipLaunchKernelGGL((tree_combine_kernel<64, 32>), dim3(unsigned(combine)), dim3(256), 0,
                       stream, a);
  }
  return hipGetLastError();
}

hipError_t launch_tree_mask(int B, int N, const int32_t* ptr, const int32_t* parent, int words,
                            uint32_t* tree, int32_t* depth, hipStream_t stream) {
  ProfScope prof("tree_mask", stream);
  hipLaunchKernelGGL(tree_mask_kernel, dim3((N + 255) / 256), dim3(256), 0, stream, B, N, ptr,
                     parent, words, tree, depth);
  return hipGetLastError();
}

}  // namespace mv
