// The paged cache's data movement: appending rows and evicting them.
#include <algorithm>

#include "gmc_cache.h"
#include "gmc_device.h"

namespace gmc {

// New rows into slots lens[b] + i.  A thread moves one 16-byte chunk of K and
// V; slots past the capacity and on pages that are none are left out.
__global__ void __launch_bounds__(256)
cache_append_kernel(CacheView c, const uint4* __restrict__ k, const uint4* __restrict__ v, long long k_stride,
                    long long v_stride, long long rows, const int32_t* __restrict__ starts,
                    const int32_t* __restrict__ src, int max_new, int chunks) {
  const int b = blockIdx.y;
  long long first;
  int n;
  new_rows(starts, max_new, rows, b, &first, &n);
  const int len = cache_len(c, b);
  n = min(n, c.cap - len);
  const long long total = static_cast<long long>(n) * c.hkv * chunks;
  const long long per = rows / c.n_seq;   // with src: rows of one sequence
  uint4* ko = static_cast<uint4*>(c.k);
  uint4* vo = static_cast<uint4*>(c.v);
  for (long long x = blockIdx.x * 256ll + threadIdx.x; x < total; x += gridDim.x * 256ll) {
    const int ch = static_cast<int>(x % chunks);
    const int h = static_cast<int>(x / chunks % c.hkv);
    const int i = static_cast<int>(x / chunks / c.hkv);
    const int s = len + i;
    if (ch == 0) {
      const long long at = (static_cast<long long>(b) * c.hkv + h) * c.cap + s;
      if (c.slot_pos) c.slot_pos[at] = c.seen[b] + i;
      if (c.weights) c.weights[at] = 0.f;
    }
    const long long to = cache_row(c, b, h, s);
    if (to < 0) continue;
    long long from = first + i;
    if (src) from = b * per + min(max(static_cast<long long>(src[static_cast<long long>(b) * max_new + i]), 0ll), per - 1);
    ko[to * chunks + ch] = k[from * k_stride + h * chunks + ch];
    vo[to * chunks + ch] = v[from * v_stride + h * chunks + ch];
  }
}

__global__ void __launch_bounds__(256)
cache_advance_kernel(CacheView c, long long rows, const int32_t* __restrict__ starts, int max_new) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= c.n_seq) return;
  long long first;
  int n;
  new_rows(starts, max_new, rows, b, &first, &n);
  const int len = cache_len(c, b);
  n = min(n, c.cap - len);
  c.lens[b] = len + n;
  if (c.seen) c.seen[b] += n;
}

hipError_t launch_cache_append(const CacheView& c, const void* k, const void* v, long long k_stride,
                               long long v_stride, long long rows, const int32_t* starts, const int32_t* src,
                               int max_new, hipStream_t st) {
  const int esz = c.dtype == 0 ? 4 : 2, chunks = c.dh * esz / 16;
  const long long total = static_cast<long long>(max_new) * c.hkv * chunks;
  const int gx = static_cast<int>(std::max<long long>(1, std::min<long long>((total + 255) / 256, 4096)));
  hipLaunchKernelGGL(cache_append_kernel, dim3(gx, c.n_seq), dim3(256), 0, st, c, static_cast<const uint4*>(k),
                     static_cast<const uint4*>(v), k_stride * esz / 16, v_stride * esz / 16, rows, starts, src,
                     max_new, chunks);
  hipLaunchKernelGGL(cache_advance_kernel, dim3((c.n_seq + 255) / 256), dim3(256), 0, st, c, rows, starts, max_new);
  return hipGetLastError();
}

// --- eviction -------------------------------------------------------------------
// Order-preserving key of an accumulated weight: NaN lowest, -0 equal to +0;
// protected slots above all.
__device__ __forceinline__ uint32_t evict_key(float w, bool safe) {
  if (safe) return 0xFFFFFFFFu;
  if (!(w == w)) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u >> 31) ? ~u : (u | 0x80000000u);
}

// One block per (sequence, kv head): the budget-th largest key bit by bit,
// then the list of moves: the i-th free slot below the budget takes the i-th
// kept slot at or above it.
constexpr int kEvictThreads = 1024;
__global__ void __launch_bounds__(kEvictThreads)
evict_select_kernel(CacheView c, int budget, int sinks, int recent, int32_t* counts, int2* moves, int max_moves) {
  __shared__ int scan[16];
  const int g = blockIdx.x, b = g / c.hkv;
  const int len = cache_len(c, b);
  if (len <= budget) {
    if (threadIdx.x == 0) counts[g] = 0;
    return;
  }
  const float* w = c.weights + static_cast<long long>(g) * c.cap;
  const int32_t* pos = c.slot_pos + static_cast<long long>(g) * c.cap;
  const int from_pos = c.seen[b] - recent;
  auto key = [&](int s) { return evict_key(w[s], pos[s] < sinks || pos[s] >= from_pos); };
  // largest T with at least `budget` keys >= T
  uint32_t T = 0;
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t t = T | (1u << bit);
    int n = 0, all;
    for (int s = threadIdx.x; s < len; s += kEvictThreads) n += key(s) >= t;
    block_exclusive_scan(n, scan, &all);
    if (all >= budget) T = t;
  }
  int above = 0, all;
  for (int s = threadIdx.x; s < len; s += kEvictThreads) above += key(s) > T;
  block_exclusive_scan(above, scan, &all);
  const int ties = budget - all;   // of the keys equal to T, the first `ties` slots stay
  int tie0 = 0, hole0 = 0, stay0 = 0;
  int2* mv = moves + static_cast<long long>(g) * max_moves;
  for (int s0 = 0; s0 < len; s0 += kEvictThreads) {
    const int s = s0 + threadIdx.x;
    const uint32_t kk = s < len ? key(s) : 0u;
    const bool tie = s < len && kk == T;
    int n;
    const int rank = tie0 + block_exclusive_scan(tie, scan, &n);
    tie0 += n;
    const bool kept = s < len && (kk > T || (tie && rank < ties));
    const bool hole = s < budget && !kept, stay = kept && s >= budget;
    const int ih = hole0 + block_exclusive_scan(hole, scan, &n);
    hole0 += n;
    const int is = stay0 + block_exclusive_scan(stay, scan, &n);
    stay0 += n;
    if (hole && ih < max_moves) mv[ih].x = s;
    if (stay && is < max_moves) mv[is].y = s;
  }
  if (threadIdx.x == 0) counts[g] = min(hole0, max_moves);
}

__global__ void __launch_bounds__(256)
evict_move_kernel(CacheView c, int budget, const int32_t* __restrict__ counts, const int2* __restrict__ moves,
                  int max_moves, int chunks) {
  const int g = blockIdx.y, b = g / c.hkv, h = g % c.hkv;
  const int n = counts[g];
  uint4* k = static_cast<uint4*>(c.k);
  uint4* v = static_cast<uint4*>(c.v);
  const long long total = static_cast<long long>(n) * chunks;
  for (long long x = blockIdx.x * 256ll + threadIdx.x; x < total; x += gridDim.x * 256ll) {
    const int i = static_cast<int>(x / chunks), ch = static_cast<int>(x % chunks);
    const int2 m = moves[static_cast<long long>(g) * max_moves + i];
    if (ch == 0) {
      const long long base = static_cast<long long>(g) * c.cap;
      c.weights[base + m.x] = c.weights[base + m.y];
      c.slot_pos[base + m.x] = c.slot_pos[base + m.y];
    }
    const long long to = cache_row(c, b, h, m.x), from = cache_row(c, b, h, m.y);
    if (to < 0 || from < 0) continue;
    k[to * chunks + ch] = k[from * chunks + ch];
    v[to * chunks + ch] = v[from * chunks + ch];
  }
  if (h == 0 && blockIdx.x == 0 && threadIdx.x == 0) c.lens[b] = min(cache_len(c, b), budget);
}

hipError_t launch_cache_evict(const CacheView& c, int budget, int sinks, int recent, int32_t* scratch,
                              hipStream_t st) {
  const int esz = c.dtype == 0 ? 4 : 2, chunks = c.dh * esz / 16;
  const int groups = c.n_seq * c.hkv, max_moves = evict_moves(c.cap, budget);
  int32_t* counts = scratch;
  int2* moves = reinterpret_cast<int2*>(scratch + (groups + 3) / 4 * 4);
  hipLaunchKernelGGL(evict_select_kernel, dim3(groups), dim3(kEvictThreads), 0, st, c, budget, sinks, recent, counts,
                     moves, max_moves);
  const long long total = static_cast<long long>(max_moves) * chunks;
  const int gx = static_cast<int>(std::max<long long>(1, std::min<long long>((total + 255) / 256, 1024)));
  hipLaunchKernelGGL(evict_move_kernel, dim3(gx, groups), dim3(256), 0, st, c, budget, counts, moves, max_moves,
                     chunks);
  return hipGetLastError();
}

}  // namespace gmc
