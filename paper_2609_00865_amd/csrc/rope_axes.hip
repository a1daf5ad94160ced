// Rotary positions with several axes: rows rotated in place of a projection's
// output or its gradient, and keys rotated on their way into the pages of a
// cache.  Both are bandwidth-bound streams; the angles of a token are shared
// by its heads, so a block takes them once into LDS, and reads its first
// elements meanwhile.  32768 tokens of 32 heads of 128: 100 us, 537 MB, 5.4 TB/s;
// 64 tokens 3.4 us, a write of 16 sequences' 6 to 24 rows 3.9 us (an empty
// launch: 2.1), of a prompt's 32768 rows of 4 heads of 128 22 us as they are (134
// MB, 6 TB/s) and 42 rotated (a token to a block: its angles are waited for).
#include "mv_cache_dev.h"

namespace mv {

// What the kernels need of the ABI's spec.
struct RopeDev {
  uint8_t axis[MV_ROPE_MAX_PAIRS];
  double log_theta;
  int pairs, n_axes;
};

static RopeDev rope_dev(const mv_rope_axes_spec& s) {
  RopeDev r;
  r.pairs = s.rotary_dim / 2;
  r.n_axes = s.n_axes;
  r.log_theta = std::log(double(s.theta));
  for (int i = 0; i < MV_ROPE_MAX_PAIRS; ++i) r.axis[i] = i < r.pairs ? s.axis[i] : 0;
  return r;
}

// cos and sin of tokens [t0, t0 + nt) and every pair into LDS rows of P floats
__device__ __forceinline__ void fill_angles(const RopeDev& r, const int32_t* pos, int64_t n,
                                            int64_t t0, int nt, float sign, float* sc, float* ss) {
  const int P = r.pairs;
  for (int x = threadIdx.x; x < nt * P; x += blockDim.x) {
    const int t = x / P, i = x - t * P;
    const double f = exp(-(double(i) / P) * r.log_theta);
    float c, s;
    axes_cs(pos[int64_t(r.axis[i]) * n + t0 + t], f, c, s);
    sc[x] = c;
    ss[x] = sign * s;
  }
  __syncthreads();
}

constexpr int kRopeTokens = 4;   // tokens of a block, at most
constexpr int kSlice = 1 << 23;   // tokens of a launch, at most: a launch has 2^32 threads

// One block per nt tokens; a thread per (token, head, V pairs), then the
// elements that pass through.
template <int V>
__global__ __launch_bounds__(256) void rope_axes_kernel(RopeDev r, int n, int tokens, int H, int d,
                                                        int nt, const u16* x, int64_t xs,
                                                        const int32_t* __restrict__ pos,
                                                        float sign, u16* out, int64_t os) {
  __shared__ __align__(16) float sc[kRopeTokens * MV_ROPE_MAX_PAIRS];
  __shared__ __align__(16) float ss[kRopeTokens * MV_ROPE_MAX_PAIRS];
  const int64_t t0 = int64_t(blockIdx.x) * nt;
  nt = int(min(int64_t(nt), tokens - t0));
  const uint32_t P = r.pairs, C = P / V, total = nt * H * C;   // (a token has fewer than 2^30 elements)
  // where a thread's pairs are: its first are read while the angles are formed
  int t, i;
  int64_t at_x, at_out;
  auto place = [&](uint32_t w) {
    const uint32_t th = w / C;
    t = th / uint32_t(H);
    i = int(w - th * C) * V;
    const int64_t head = int64_t(th - t * uint32_t(H)) * d;
    at_x = (t0 + t) * xs + head;
    at_out = (t0 + t) * os + head;
  };
  Pairs<V> row;
  if (threadIdx.x < total) {
    place(threadIdx.x);
    row.read(x + at_x, i, P);
  }
  fill_angles(r, pos, n, t0, nt, sign, sc, ss);
  for (uint32_t w = threadIdx.x; w < total; w += 256) {
    if (w != threadIdx.x) {
      place(w);
      row.read(x + at_x, i, P);
    }
    row.turn(out + at_out, i, P, sc + t * P + i, ss + t * P + i);
  }
  if (x == out) return;
  const int rest = d - 2 * P;
  for (int64_t w = threadIdx.x; w < int64_t(nt) * H * rest; w += 256) {
    const int e = int(w % rest), h = int(w / rest % H), t = int(w / rest / H);
    const int64_t at = int64_t(h) * d + 2 * P + e;
    out[(t0 + t) * os + at] = x[(t0 + t) * xs + at];
  }
}

// K (rotated when ROPE) and V of one token per block row into their pages.
template <int V, bool ROPE>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheDev a, int layer, RopeDev r, int n,
                                                          const int32_t* __restrict__ slot,
                                                          const u16* __restrict__ k, int64_t ks,
                                                          const u16* __restrict__ v, int64_t vs,
                                                          const int32_t* __restrict__ pos) {
  __shared__ __align__(16) float sc[MV_ROPE_MAX_PAIRS];
  __shared__ __align__(16) float ss[MV_ROPE_MAX_PAIRS];
  const int64_t t = blockIdx.x;
  const int at = slot[t];
  const int D = a.D, place = at & ((1 << a.psl) - 1);
  const int CH = D / 8, P = r.pairs, C = ROPE ? P / V : CH;
  const int kw = a.Hkv * C, vw = a.Hkv * CH;
  // what a thread moves first is read while the slot and the angles are on their way
  Pairs<V> row;
  uint4 k0, v0;
  auto k_at = [&](int w, int& i) {   // of thread-sized piece w: element of the row, and of its head
    const int h = w / C;
    i = (w - h * C) * (ROPE ? V : 8);
    return h;
  };
  int ki, h = k_at(threadIdx.x, ki);
  if (int(threadIdx.x) < kw) {
    if (ROPE)
      row.read(k + t * ks + int64_t(h) * D, ki, P);
    else
      k0 = ld16(k + t * ks + int64_t(h) * D + ki);
  }
  if (int(threadIdx.x) < vw) v0 = ld16(v + t * vs + int64_t(threadIdx.x) * 8);
  if (ROPE) fill_angles(r, pos, n, t, 1, 1.f, sc, ss);
  if (at < 0 || (at >> a.psl) >= a.n_pages) return;   // block-uniform
  // element offset of head 0's row; heads lie page_size rows apart
  const int64_t base = (((int64_t(layer) * a.n_pages + (at >> a.psl)) * a.Hkv << a.psl) + place) * D;
  const int64_t hs = int64_t(D) << a.psl;
  for (int w = threadIdx.x; w < vw; w += 256) {
    const int h = w / CH;
    if (w != int(threadIdx.x)) v0 = ld16(v + t * vs + int64_t(w) * 8);
    st16(a.v + base + h * hs + (w - h * CH) * 8, v0);
  }
  for (int w = threadIdx.x; w < kw; w += 256) {
    if (w != int(threadIdx.x)) {
      h = k_at(w, ki);
      if (ROPE)
        row.read(k + t * ks + int64_t(h) * D, ki, P);
      else
        k0 = ld16(k + t * ks + int64_t(h) * D + ki);
    }
    if (ROPE)
      row.turn(a.k + base + h * hs, ki, P, sc + ki, ss + ki);
    else
      st16(a.k + base + h * hs + ki, k0);
  }
  if (!ROPE) return;
  const int rest = D - 2 * P;
  for (int w = threadIdx.x; w < a.Hkv * rest; w += 256) {
    const int h = w / rest, e = 2 * P + w - h * rest;
    a.k[base + h * hs + e] = k[t * ks + int64_t(h) * D + e];
  }
}

// The widest access that P pairs allow (rows start at multiples of 8
// elements, so the second element of a pair is aligned as P is).
static int pair_width(int P) { return P % 8 == 0 ? 8 : P % 4 == 0 ? 4 : P % 2 == 0 ? 2 : 1; }

hipError_t launch_rope_axes(const mv_rope_axes_spec& spec, int n, int H, int d, const void* x,
                            int64_t xs, const int32_t* pos, int direction, void* out, int64_t os,
                            hipStream_t stream) {
  const RopeDev r = rope_dev(spec);
  // Four tokens to a block where that still leaves several blocks per CU
  const int nt = n >= kRopeTokens * 4 * kNumCu ? kRopeTokens : 1;
  const float sign = direction > 0 ? 1.f : -1.f;
  const u16* xp = static_cast<const u16*>(x);
  u16* op = static_cast<u16*>(out);
  ProfScope prof("rope_axes", stream);
  for (int64_t first = 0; first < n; first += kSlice) {
    const int tokens = int(std::min(int64_t(kSlice), n - first));
    const dim3 grid(unsigned((tokens + nt - 1) / nt)), block(256);
#define MV_ROPE(V)                                                                           \
  hipLaunchKernelGGL((rope_axes_kernel<V>), grid, block, 0, stream, r, n, tokens, H, d, nt, \
                     xp + first * xs, xs, pos + first, sign, op + first * os, os)
    switch (pair_width(r.pairs)) {
      case 8: MV_ROPE(8); break;
      case 4: MV_ROPE(4); break;
      case 2: MV_ROPE(2); break;
      default: MV_ROPE(1); break;
    }
#undef MV_ROPE
  }
  return hipGetLastError();
}

hipError_t launch_cache_write(const CacheDev& a, int layer, int n, const int32_t* slot,
                              const void* k, int64_t ks, const void* v, int64_t vs,
                              const mv_rope_axes_spec* spec, const int32_t* pos,
                              hipStream_t stream) {
  RopeDev r{};
  if (spec) r = rope_dev(*spec);
  const u16* kp = static_cast<const u16*>(k);
  const u16* vp = static_cast<const u16*>(v);
  ProfScope prof("cache_write", stream);
  for (int64_t first = 0; first < n; first += kSlice) {
    const dim3 grid(unsigned(std::min(int64_t(kSlice), n - first))), block(256);
#define MV_WRITE(V, ROPE)                                                                      \
  hipLaunchKernelGGL((cache_write_kernel<V, ROPE>), grid, block, 0, stream, a, layer, r, n,    \
                     slot + first, kp + first * ks, ks, vp + first * vs, vs, ROPE ? pos + first : pos)
    if (!spec) {
      MV_WRITE(8, false);
    } else {
      switch (pair_width(r.pairs)) {
        case 8: MV_WRITE(8, true); break;
        case 4: MV_WRITE(4, true); break;
        case 2: MV_WRITE(2, true); break;
        default: MV_WRITE(1, true); break;
      }
    }
#undef MV_WRITE
  }
  return hipGetLastError();
}

}  // namespace mv
