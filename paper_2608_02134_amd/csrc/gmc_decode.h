// What the cache's decode kernels share: which tiles of keys a sequence's splits
// take, and the kernel that joins the splits.
#pragma once

#include "gmc_cache.h"

namespace gmc {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kDecodeWaves = 4, kDecodeShort = 8;   // waves of a block; where one block does a whole sequence

// Which tiles of TK slots a query in slot t looks at: all up to its own, or
// with a window over slots in order those of the first tokens and the window.
struct TileRange {
  int first, skip, count;   // tile i: i < first ? i : i + skip
};
__host__ __device__ inline TileRange tile_range(int len, int window, int sinks, bool ordered, int tk) {
  TileRange r;
  const int end = (len + tk - 1) / tk;
  if (window <= 0 || !ordered || window >= len) {
    r.first = end; r.skip = 0; r.count = end;
    return r;
  }
  const int lo = (len - window) / tk;
  const int sink = (sinks < len ? sinks + tk - 1 : len + tk - 1) / tk;
  r.first = sink < lo ? sink : lo;
  r.skip = lo - r.first;
  r.count = end - r.skip;
  return r;
}

struct DecodeScratch {
  float* part;     // [b][hq][nsplit][dh] unnormalised sums
  float* ml;       // [b][hq][nsplit][2] maximum (base 2) and sum
  float* logits;   // [b][hq][cap] or null
  int nsplit;
};

// Splits that a sequence's tiles are shared over, at most those of the grid:
// one tile a wave up to 32 splits, above that two, above 64 four, as the join
// reads every split (28 query heads on 4, bf16; one request of 32768 slots:
// 20.2 us with 64 splits, 22.1 with 128, 30 with 256; of 4096: 9.2 with 32,
// 10.5 with 16).
__host__ __device__ inline int used_splits(int tiles, int nsplit) {
  const int one = (tiles + kDecodeWaves - 1) / kDecodeWaves;
  const int two = (one + 1) / 2, four = (two + 1) / 2;
  const int want = one < 32 ? one : two < 32 ? 32 : two < 64 ? two : four < 64 ? 64 : four;
  return nsplit < want ? nsplit : want < 1 ? 1 : want;
}

// Joins the splits of a call's tiles of tk keys.
hipError_t launch_decode_join(const CacheView& c, const AttendArgs& a, const DecodeScratch& sc, bool accumulate, int tk,
                              hipStream_t st);

}  // namespace gmc
