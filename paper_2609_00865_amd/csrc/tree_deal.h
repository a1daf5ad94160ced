// How the units of work of the cache attention's tiles are counted: host and
// device code, so that the largest counts can be checked without their keys.
#pragma once

#include <cstdint>

#include "mv_internal.h"

#if defined(__HIPCC__)
#define MV_DEAL_HD __host__ __device__ __forceinline__
#else
#define MV_DEAL_HD inline
#endif

namespace mv {

constexpr int kUnit = 64;       // keys of a unit of work

// Units of a tile that sees keys [0, kmax): at most 2^25, whatever the keys
// (kmax + 63 may pass 2^31).  Tiles of one entry, of forks, and of a sequence
// that several entries name see the same keys, so nothing bounds their sum by
// the memory that holds them.
MV_DEAL_HD int units_of(int kmax) { return int((uint32_t(kmax) + kUnit - 1) / kUnit); }

// The units of W waves' tiles from those of each wave: of the waves before
// `wave`, and of all.  A wave's 64 tiles have at most 2^31, which 32 bits hold
// without a sign; those of several waves are added in 64.
template <int W>
MV_DEAL_HD void add_waves(const uint32_t* units, int wave, int64_t& before, int64_t& all) {
  before = all = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const int64_t n = units[w];
    before += w < wave ? n : 0;
    all += n;
  }
}

}  // namespace mv
