// Shared by the cache's kernels: the state as the device sees it, a block-wide
// prefix sum, and the rotation of a row by several position axes.
#pragma once

#include "mv_device.h"

namespace mv {

// The cache as kernels take it: sizes in log2 where the ABI fixes a power of two.
struct CacheDev {
  u16* k;
  u16* v;
  int32_t* table;
  int32_t* len;
  int32_t* refs;
  int32_t* ctl;
  int n_layers, n_pages, n_seqs, max_pages, Hkv, D;
  int psl;   // log2(page_size)
  // rows of a sequence, kept inside what its table can hold
  __device__ __forceinline__ int length(int s) const {
    return int(min(int64_t(max(len[s], 0)), int64_t(max_pages) << psl));
  }
  __device__ __forceinline__ int pages_of(int rows) const {
    return int((int64_t(rows) + (1 << psl) - 1) >> psl);
  }
  // a table entry as a page that exists
  __device__ __forceinline__ int page(int s, int j) const {
    const int p = table[int64_t(s) * max_pages + j];
    return unsigned(p) < unsigned(n_pages) ? p : 0;
  }
};

// ctl words
enum { kCtlHint = 0, kCtlNoPages = 1, kCtlBad = 2, kCtlFree = 3 };

// A barrier that orders LDS alone.  __syncthreads also waits for every global
// store of the block to arrive, about a microsecond each time.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Inclusive prefix sum over the wave by data-parallel moves between lanes (six
// vector instructions; through LDS the same six steps take ten times as long).
// (Sums without a sign hold what passes 2^31.)
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  constexpr int kShr = 0x110, kBcast15 = 0x142, kBcast31 = 0x143;
  x += __builtin_amdgcn_update_dpp(0, x, kShr + 1, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, kShr + 2, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, kShr + 4, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, kShr + 8, 0xf, 0xf, false);   // rows of 16
  x += __builtin_amdgcn_update_dpp(0, x, kBcast15, 0xa, 0xf, false);   // rows 0 -> 1, 2 -> 3
  x += __builtin_amdgcn_update_dpp(0, x, kBcast31, 0xc, 0xf, false);   // rows 0, 1 -> 2, 3
  return x;
}

// Exclusive prefix sum of v over the block (BLOCK threads) and the total;
// tmp: BLOCK / 64 + 1 ints of LDS.
template <int BLOCK>
__device__ __forceinline__ int block_scan(int v, int* tmp, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int x = wave_scan(v);
  lds_barrier();   // tmp of an earlier call is read
  if (lane == 63) tmp[wave] = x;
  lds_barrier();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < BLOCK / 64; ++w) {
    const int t = tmp[w];
    before += w < wave ? t : 0;
    all += t;
  }
  total = all;
  return before + x - v;
}

// The angle of pair i at position p, and its cosine and sine.  The angle is
// formed and reduced to [-pi, pi] in fp64 (positions reach 2^31: an fp32
// product would be off by whole turns), its cosine and sine are fp32.
__device__ __forceinline__ void axes_cs(int p, double inv_freq, float& c, float& s) {
  const double a = double(p) * inv_freq;
  const double k = rint(a * 0.15915494309189535);   // 1 / (2 pi)
  sincosf(float(fma(-k, 6.283185307179586, a)), &s, &c);
}

// V consecutive bf16 elements as floats, and back with one rounding.
template <int V>
__device__ __forceinline__ void load_v(const u16* p, float (&x)[V]) {
  uint32_t w[(V + 1) / 2];
  if constexpr (V == 8) {
    const uint4 t = ld16(p);
    w[0] = t.x, w[1] = t.y, w[2] = t.z, w[3] = t.w;
  } else if constexpr (V == 4) {
    const uint2 t = *reinterpret_cast<const uint2*>(p);
    w[0] = t.x, w[1] = t.y;
  } else if constexpr (V == 2) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else {
    w[0] = *p;
  }
#pragma unroll
  for (int e = 0; e < V; ++e) x[e] = bf16_to_f32(uint16_t(w[e / 2] >> (16 * (e & 1))));
}

template <int V>
__device__ __forceinline__ void store_v(u16* p, const float (&x)[V]) {
  if constexpr (V == 8) {
    st16(p, make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]),
                       pack2(x[6], x[7])));
  } else if constexpr (V == 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2(x[0], x[1]), pack2(x[2], x[3]));
  } else if constexpr (V == 2) {
    *reinterpret_cast<uint32_t*>(p) = pack2(x[0], x[1]);
  } else {
    *p = uint16_t(bf16_bits(x[0]));
  }
}

// V consecutive pairs of one head row, from pair i of P on: (x[i], x[i + P]),
// read, and turned by the angles whose cosines and sines are c and s.
template <int V>
struct Pairs {
  float a[V], b[V];
  __device__ __forceinline__ void read(const u16* x, int i, int P) {
    load_v<V>(x + i, a);
    load_v<V>(x + i + P, b);
  }
  __device__ __forceinline__ void turn(u16* y, int i, int P, const float* c, const float* s) const {
    float u[V], w[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      u[e] = a[e] * c[e] - b[e] * s[e];
      w[e] = b[e] * c[e] + a[e] * s[e];
    }
    store_v<V>(y + i, u);
    store_v<V>(y + i + P, w);
  }
};

}  // namespace mv
