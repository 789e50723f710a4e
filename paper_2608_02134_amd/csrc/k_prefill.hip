// Attention of the newest tokens of each sequence over the paged cache, with a
// window and first tokens that stay visible.
//
// The query heads of a kv head share its keys, so a block takes 128 rows of
// (token, head of the group), 32 a wave, against tiles of KT keys in shared
// memory, loaded from the pages straight into it (no registers between), one
// tile ahead of the products.  A wave keeps its queries in registers as the
// columns of
//   S^T = K Q^T (32x32x16 in bf16, 32x32x2 in fp32): every lane then holds 16
//         keys of one query for each 32 keys, so maxima and sums of a row need
//         one exchange between lane halves, and the keys a lane holds are the
//         k slots it has to supply as B of
//   O^T = V^T P^T, with A = V^T read in the same key order, in bf16 by
//         transposing reads.
// bf16 weights are rounded to bf16 for the second product (half a step, 2^-8
// of each weight; the sum that divides them is of unrounded ones): a second
// product for what the rounding drops would cost a quarter of the kernel's
// matrix work for an error that the output's own rounding matches.
//
// Rows in shared memory are swizzled in 16-byte chunks, so that the 16 rows
// that one read touches lie on different banks.
//
// 16448 tokens, window 4096, 28 heads on 4 of 128 in bf16: 0.94 to 1.01 ms, 840 to 900 TFLOP/s
// (a large matrix product of the library: 1217).  Of its time 0.69 ms are products
// and reads of shared memory alone, what the loads add is 0.13 and what the
// exponentials and maxima add 0.12.  (64 queries a wave, one wave a SIMD, halve the
// reads and took 1.36 ms; eight waves a block, loads spread over the products and
// weights interleaved with products by hand were no faster.)
#include <algorithm>

#include "gmc_prefill.h"

namespace gmc {

template <typename T, int DH>
__global__ void __launch_bounds__(64 * kPreWaves, sizeof(T) == 2 && DH <= 128 ? 2 : 1)
prefill_kernel(CacheView c, AttendArgs a, PreScratch sc, int row_blocks) {
  prefill_block<T, DH, false>(c, CacheScales{}, a, sc, row_blocks);
}

// Joins the splits: one wave per row and head, four elements a lane; lanes that a
// row leaves over take other splits (77 tokens of 3 requests, 8 heads of 64, 28
// splits: 5.2 us, 8.4 with 16 lanes at work).  Up to 8 splits every lane takes all
// statistics itself: 4 requests of 77 tokens, 6 splits, 49.5 us for both kernels,
// 51.3 with the exchange; 16 tokens, 64 splits, 37 with it.
template <typename T>
__global__ void __launch_bounds__(256)
prefill_join_kernel(CacheView c, AttendArgs a, PreScratch sc) {
  const int b = blockIdx.z, hq = blockIdx.y, i = blockIdx.x * 4 + wave_id(), lane = threadIdx.x & 63;
  long long first;
  int n;
  new_rows(a.starts, a.max_new, a.rows, b, &first, &n);
  if (i >= n) return;
  const long long row = (first + i) * c.hq + hq, part_row = (static_cast<long long>(b) * a.max_new + i) * c.hq + hq;
  const float2* ml = reinterpret_cast<const float2*>(sc.ml) + part_row * sc.nsplit;
  const int per = c.dh / 4, groups = 64 / per, g = lane / per;   // lanes of a row, rows at once
  const float* part = sc.part + part_row * sc.nsplit * c.dh + 4 * (lane - g * per);
  constexpr int kFlight = 8;
  floatx4 x[kFlight];
  float2 y[kFlight];
  auto load = [&](int s0) {
#pragma unroll
    for (int e = 0; e < kFlight; ++e) {
      const int s = min(s0 + e * groups, sc.nsplit - 1);
      y[e] = ml[s];
      x[e] = *reinterpret_cast<const floatx4*>(part + static_cast<long long>(s) * c.dh);
    }
  };
  load(g);                     // (on its way while the statistics are taken)
  float m = -INFINITY, l = 0.f;
  if (sc.nsplit <= kFlight) {  // every lane takes them all: no exchange between lanes
    float2 z[kFlight];
#pragma unroll
    for (int e = 0; e < kFlight; ++e) z[e] = e < sc.nsplit ? ml[e] : make_float2(-INFINITY, 0.f);
#pragma unroll
    for (int e = 0; e < kFlight; ++e) m = fmaxf(m, z[e].x);
#pragma unroll
    for (int e = 0; e < kFlight; ++e) l += z[e].y * __builtin_amdgcn_exp2f(z[e].x - (m == -INFINITY ? 0.f : m));
  } else {
    join_stats(reinterpret_cast<const float*>(ml), sc.nsplit, &m, &l);
  }
  const float base = m == -INFINITY ? 0.f : m;
  floatx4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = g; s0 < sc.nsplit; s0 += groups * kFlight) {
    if (s0 > g) load(s0);
#pragma unroll
    for (int e = 0; e < kFlight; ++e) {
      // (a split without a part has written its statistics only)
      if (s0 + e * groups >= sc.nsplit || (y[e].x == -INFINITY && y[e].y == 0.f)) continue;
      const float f = __builtin_amdgcn_exp2f(y[e].x - base);
#pragma unroll
      for (int u = 0; u < 4; ++u) o[u] += f * x[e][u];
    }
  }
  for (int k = 1; k < groups; ++k)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float other = __shfl(o[u], (lane + k * per) & 63);
      if (g == 0) o[u] += other;
    }
  if (g == 0) {
    T* to = static_cast<T*>(a.out) + row * c.dh + 4 * lane;
    const float inv = 1.f / l;
#pragma unroll
    for (int u = 0; u < 4; ++u) to[u] = from_f32<T>(l == 0.f ? 0.f : o[u] * inv);
  }
  if (a.lse && lane == 0)
    a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

static int pre_key_tile(const CacheView& c, bool four_bits) {
  return (c.dtype != 0 || four_bits) && c.dh <= 128 ? 64 : 32;
}

static int pre_row_blocks(const CacheView& c, int max_new) {
  return static_cast<int>((static_cast<long long>(max_new) * c.hg + kPreRows - 1) / kPreRows);
}

// Splits of a row block's keys, while the blocks find room on the chip together
// (512): a block's tiles, one after the other, against a second launch and the
// parts it reads.  512 is two to a CU, as kernels of up to 256 registers have it: bf16 with
// heads of up to 128, fp32 up to 64 over pages and 32 over 4 bits.  Of the others a CU holds
// one, and blocks from 257 on wait; another limit was not measured for them.  Estimates
// in us: a tile 1.7 for 64 keys of 128 dims (fp32: 1.9 for 32 of 64), the launch 4,
// parts 4 MB each.  Measured, us with the splits
// chosen and with others: 335 tokens (28 query heads on 4 of 128) 16.7 with 1,
// 20.7 with 2; 1000 tokens 32.5 with 1, 41 with 2; 77 tokens over 4100 slots 27.9
// with 16, 26.2 with 10, 29.8 with 25; 10 over 2000 14.1 with 15, 19.6 with 5;
// 200 over 500 (12 on 12 of 96, 2 sequences) 15.1 with 1, 16.7 with 4; fp32 (8 on
// 2 of 64) 300 tokens 17.0 with 5, 26.6 with 2.
// Over 4 bits also what a tile costs where two blocks share a CU (77 tokens over
// 4100 slots 29.8 us with 240 blocks, 32.4 with 280; three such requests 43.7 with 480, 57
// with 240; 16 over 32768 35.6 with 256, 38.6 with 348).
static int pre_splits(const CacheView& c, int max_new, bool four_bits, int slots) {
  const int kt = pre_key_tile(c, four_bits), tiles = (slots + kt - 1) / kt;
  const long long blocks = static_cast<long long>(pre_row_blocks(c, max_new)) * c.hkv * c.n_seq;
  const double tile = (c.dtype != 0 ? 1.7 / (64 * 128) : four_bits ? 3.0 / (64 * 128) : 1.9 / (32 * 64)) * kt * c.dh;
  const double part = 8e-6 / 4 * (c.dh + 2) * c.hq * max_new * c.n_seq;
  int best = 1;
  double least = tile * tiles;
  for (int s = 2; s <= tiles / 2 && blocks * s <= 512; ++s) {
    const double shared = four_bits && blocks * s > 256 ? 1.5 : 1;
    const double time = shared * tile * tiles / s + 4 + part * s;
    if (time < least) {
      least = time;
      best = s;
    }
  }
  return best;
}

long long prefill_scratch_bytes(const CacheView& c, int max_new, bool four_bits) {
  const int ns = pre_splits(c, max_new, four_bits, c.cap);
  return ns == 1 ? 0 : 4ll * c.n_seq * max_new * c.hq * ns * (c.dh + 2);
}

PreScratch pre_plan(const CacheView& c, const AttendArgs& a, bool four_bits, void* scratch, int* row_blocks) {
  const int max_new = a.max_new;
  PreScratch sc{};
  *row_blocks = pre_row_blocks(c, max_new);
  sc.nsplit = pre_splits(c, max_new, four_bits, c.cap);
  // Under a window a block looks at few of the slots: splits for those, of the scratch
  // memory that the capacity's splits need.  us so and with the capacity's: 43 tokens over
  // 5488 slots, window 700, 18.5 and 20.4; three requests of 77 over 4100, 512, 24.0 and
  // 27.6; 16 over 60000, 4096, 19.6 and 20.5; 300 over 32768, 1024, 33.0 and 32.4.  (Over
  // pages of the type it was not measured, and the capacity's stand.)
  if (four_bits && a.window > 0) {
    const long long slots = static_cast<long long>(a.window) + a.sinks + kPreRows / c.hg + 128;
    if (slots < c.cap) sc.nsplit = std::min(sc.nsplit, pre_splits(c, max_new, true, static_cast<int>(slots)));
  }
  if (sc.nsplit > 1) {
    sc.part = static_cast<float*>(scratch);
    sc.ml = sc.part + static_cast<long long>(c.n_seq) * max_new * c.hq * sc.nsplit * c.dh;
  }
  sc.grid = pre_grid(*row_blocks * sc.nsplit, static_cast<long long>(c.hkv) * c.n_seq);
  return sc;
}

hipError_t launch_prefill_join(const CacheView& c, const AttendArgs& a, const PreScratch& sc, hipStream_t st) {
  const dim3 grid((a.max_new + 3) / 4, c.hq, c.n_seq);
  if (c.dtype == 0)
    hipLaunchKernelGGL(prefill_join_kernel<float>, grid, dim3(256), 0, st, c, a, sc);
  else
    hipLaunchKernelGGL(prefill_join_kernel<bf16_t>, grid, dim3(256), 0, st, c, a, sc);
  return hipGetLastError();
}

hipError_t launch_cache_prefill(const CacheView& c, const AttendArgs& a, void* scratch, hipStream_t st) {
  int row_blocks;
  const PreScratch sc = pre_plan(c, a, false, scratch, &row_blocks);
#define GMC_PREFILL(T, DH)                                                                                       \
  case DH:                                                                                                       \
    hipLaunchKernelGGL((prefill_kernel<T, DH>), dim3(static_cast<unsigned>(sc.grid.blocks)), dim3(64 * kPreWaves), 0, st, c, a, sc, \
                       row_blocks); \
    break;
#define GMC_PREFILL_ALL(T)                                                                                       \
  switch (c.dh) {                                                                                                \
    GMC_PREFILL(T, 32) GMC_PREFILL(T, 64) GMC_PREFILL(T, 96) GMC_PREFILL(T, 128)                                 \
    GMC_PREFILL(T, 160) GMC_PREFILL(T, 192) GMC_PREFILL(T, 224) GMC_PREFILL(T, 256)                              \
    default: return hipErrorInvalidValue;                                                                        \
  }
  if (c.dtype == 0) { GMC_PREFILL_ALL(float) } else { GMC_PREFILL_ALL(bf16_t) }
#undef GMC_PREFILL_ALL
#undef GMC_PREFILL
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;   // (there is nothing to join)
  return sc.nsplit > 1 ? launch_prefill_join(c, a, sc, st) : hipSuccess;
}

}  // namespace gmc
