// The paged cache's data movement: appending rows and evicting them.
#include <algorithm>

#include "gmc_cache.h"
#include "gmc_device.h"

namespace gmc {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// --- append ---------------------------------------------------------------------
// One wave per token: its K and V rows of all heads are runs of hkv * chunks
// 16-byte pieces, a lane moves every 64th.  Slots past the capacity and on
// pages that are none are left out.  (16 prompts of 335 rows picked from 1375, 4
// heads of 128 in bf16, 22 MB read and written: 13 us a call, two launches.)
__device__ __forceinline__ void append_token(const CacheView& c, const uint4* __restrict__ k,
                                             const uint4* __restrict__ v, long long k_stride, long long v_stride,
                                             int b, int s, int position, long long from, int chunks) {
  const int lane = threadIdx.x & 63;
  const long long at = static_cast<long long>(b) * c.hkv * c.cap + s;
  for (int h = lane; h < c.hkv; h += 64) {
    if (c.slot_pos) c.slot_pos[at + static_cast<long long>(h) * c.cap] = position;
    if (c.weights) c.weights[at + static_cast<long long>(h) * c.cap] = 0.f;
  }
  const long long row = cache_row(c, b, 0, s);   // of head 0; the others' lie a page's rows on
  if (row < 0) return;
  const int pieces = c.hkv * chunks;
  uint4* ko = static_cast<uint4*>(c.k);
  uint4* vo = static_cast<uint4*>(c.v);
  for (int p = lane; p < pieces; p += 64) {
    const int h = p / chunks, ch = p - h * chunks;
    const long long to = (row + (static_cast<long long>(h) << c.shift)) * chunks + ch;
    ko[to] = k[from * k_stride + p];
    vo[to] = v[from * v_stride + p];
  }
}

struct AppendArgs {
  const uint4 *k, *v;
  long long k_stride, v_stride, rows;   // strides in 16-byte pieces
  const int32_t *starts, *src;
  int max_new, chunks;
};

__device__ __forceinline__ long long append_source(const AppendArgs& a, int n_seq, int b, long long first, int i) {
  if (!a.src) return first + i;
  const long long per = a.rows / n_seq;   // rows of one sequence
  const long long x = a.src[static_cast<long long>(b) * a.max_new + i];
  return b * per + min(max(x, 0ll), per - 1);
}

// Few new tokens: one block per sequence, which also moves the length on.  16
// sequences, 4 heads of 128 in bf16: one token 3.3 us, 4.5 with the two launches
// below; 16 tokens 4.8 either way; 32 tokens 6.9 and 4.7.
constexpr int kAppendFew = 16;
__global__ void __launch_bounds__(256) cache_append_few_kernel(CacheView c, AppendArgs a) {
  const int b = blockIdx.x;
  long long first;
  int n;
  new_rows(a.starts, a.max_new, a.rows, b, &first, &n);
  const int len = cache_len(c, b), seen = c.seen ? c.seen[b] : 0;
  n = min(n, c.cap - len);
  for (int i = wave_id(); i < n; i += 4)
    append_token(c, a.k, a.v, a.k_stride, a.v_stride, b, len + i, seen + i, append_source(a, c.n_seq, b, first, i),
                 a.chunks);
  __syncthreads();   // (every wave has read the length)
  if (threadIdx.x == 0) {
    c.lens[b] = len + n;
    if (c.seen) c.seen[b] = seen + n;
  }
}

__global__ void __launch_bounds__(256) cache_append_kernel(CacheView c, AppendArgs a) {
  const int b = blockIdx.y;
  long long first;
  int n;
  new_rows(a.starts, a.max_new, a.rows, b, &first, &n);
  const int len = cache_len(c, b), seen = c.seen ? c.seen[b] : 0;
  n = min(n, c.cap - len);
  for (int i = blockIdx.x * 4 + wave_id(); i < n; i += gridDim.x * 4)
    append_token(c, a.k, a.v, a.k_stride, a.v_stride, b, len + i, seen + i, append_source(a, c.n_seq, b, first, i),
                 a.chunks);
}

// After every row has found its slot: the lengths.
__global__ void __launch_bounds__(256) cache_advance_kernel(CacheView c, AppendArgs a) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= c.n_seq) return;
  long long first;
  int n;
  new_rows(a.starts, a.max_new, a.rows, b, &first, &n);
  const int len = cache_len(c, b);
  n = min(n, c.cap - len);
  c.lens[b] = len + n;
  if (c.seen) c.seen[b] += n;
}

hipError_t launch_cache_append(const CacheView& c, const void* k, const void* v, long long k_stride,
                               long long v_stride, long long rows, const int32_t* starts, const int32_t* src,
                               int max_new, hipStream_t st) {
  const int esz = c.dtype == 0 ? 4 : 2;
  const AppendArgs a{static_cast<const uint4*>(k), static_cast<const uint4*>(v), k_stride * esz / 16,
                     v_stride * esz / 16, rows, starts, src, max_new, c.dh * esz / 16};
  if (max_new <= kAppendFew) {
    hipLaunchKernelGGL(cache_append_few_kernel, dim3(c.n_seq), dim3(256), 0, st, c, a);
  } else {
    hipLaunchKernelGGL(cache_append_kernel, dim3(std::min((max_new + 3) / 4, 4096), c.n_seq), dim3(256), 0, st, c, a);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;   // (rows that were not written are not counted)
    hipLaunchKernelGGL(cache_advance_kernel, dim3((c.n_seq + 255) / 256), dim3(256), 0, st, c, a);
  }
  return hipGetLastError();
}

// --- eviction -------------------------------------------------------------------
constexpr uint32_t kSafeKey = 0xFFFFFFFFu;
// Order-preserving key of an accumulated weight: NaN lowest, -0 equal to +0;
// protected slots above all.
__device__ __forceinline__ uint32_t evict_key(float w, bool safe) {
  if (safe) return kSafeKey;
  if (!(w == w)) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u >> 31) ? ~u : (u | 0x80000000u);
}

// One block per (sequence, kv head) finds the budget-th largest key T, then
// lists the slots below the budget that become free and the kept ones at or
// above it.
//
// The keys' upper halves (plus one; 0 past the length) are formed from weights and
// positions once: a cache of at most 8192 slots keeps them in shared memory, for
// longer ones a kernel of many blocks before this one leaves them in scratch
// memory, with histograms of their upper 11 bits (2 x 8 caches of 65536 slots:
// 5 and 28 us, 39 with all in the one block; at 8192 slots 512 caches take 40 us
// the short way and 55 the long one, 16 caches 27 either way).  Histograms of 2048 bins over the
// halves narrow T's half to a range [lo, hi] that few keys fall into; those are
// formed again from memory, and T is the one with the right number of larger
// ones.  (More than kEvictList keys with one half: histograms of their lower
// halves; comparing 1024 keys with each other would take 22 us.)
// One block has the work of a whole cache, so what counts is instructions per
// key, and that the loops over the keys stay loops (unrolled, the kernel waited
// for its own instructions: 21 us for 4160 slots).  A wave owns a run of
// consecutive slots, 256 per step, four a lane: slot order is (wave, step, lane,
// slot), and one scan per step counts free and moving slots together.  A wave's
// lists start at its own place, at the first slot of its run; the move kernel
// strings them together.
constexpr int kEvictBins = 2048, kEvictList = 256, kEvictRuns = 16, kEvictHead = 64;
constexpr int kEvictShort = 8192;                  // slots of a cache whose halves shared memory holds
constexpr int kEvictSlice = 4096;                  // slots a block of the first kernel takes
constexpr int kEvictThreads = 1024;                // threads of the selecting block of a long cache
constexpr uint32_t kSafeHalf = 0xFFFFu;            // protected; others are at most 0xFF81
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ uint32_t evict_half(float w, bool safe) {
  const uint32_t y = evict_key(w, safe);
  return y == kSafeKey ? kSafeHalf : (y >> 16) + 1u;
}

// Scratch memory: the lengths of the runs' lists, then the lists; for long caches
// the keys' halves and each slice's histogram.
struct EvictLists {
  int32_t* heads;    // [groups][kEvictHead]: free slots of each run, kept slots above
                     // the budget of each, slots of a run
  int32_t* to;       // [groups][cap]
  int32_t* from;     // [groups][cap]
  uint16_t* halves;  // [groups][cap]
  uint16_t* hist;    // [groups][slices][kEvictBins]
};

__host__ __device__ inline int evict_slices(int slots) { return (slots + kEvictSlice - 1) / kEvictSlice; }

// The halves and histogram of one slice of a long cache.
__global__ void __launch_bounds__(256)
evict_halves_kernel(CacheView c, int budget, int sinks, int recent, EvictLists out) {
  __shared__ int bins[kEvictBins];
  const int g = blockIdx.x, b = g / c.hkv, first = blockIdx.y * kEvictSlice;
  const int len = cache_len(c, b);
  if (len <= budget || first >= len) return;
  for (int x = threadIdx.x; x < kEvictBins; x += 256) bins[x] = 0;
  __syncthreads();
  const long long at = static_cast<long long>(g) * c.cap;
  const int from_pos = c.seen[b] - recent, end = min(first + kEvictSlice, c.cap);
  constexpr int kSteps = kEvictSlice / 1024;
  f32x4_any x[kSteps];
  i32x4_any p[kSteps];
#pragma unroll
  for (int e = 0; e < kSteps; ++e) {
    const int s = min(first + 1024 * e + 4 * static_cast<int>(threadIdx.x), c.cap - 4);
    x[e] = *reinterpret_cast<const f32x4_any*>(c.weights + at + s);
    p[e] = *reinterpret_cast<const i32x4_any*>(c.slot_pos + at + s);
  }
#pragma unroll
  for (int e = 0; e < kSteps; ++e) {
    const int s = first + 1024 * e + 4 * static_cast<int>(threadIdx.x);
    if (s >= end) break;
    uint32_t k[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      k[j] = s + j < len ? evict_half(x[e][j], p[e][j] < sinks || p[e][j] >= from_pos) : 0u;
      if (k[j]) atomicAdd(&bins[k[j] >> 5], 1);
    }
    *reinterpret_cast<uint2*>(out.halves + at + s) = make_uint2(k[0] | (k[1] << 16), k[2] | (k[3] << 16));
  }
  __syncthreads();
  uint32_t* to = reinterpret_cast<uint32_t*>(
      out.hist + (static_cast<long long>(g) * evict_slices(c.cap) + blockIdx.y) * kEvictBins);
  for (int x = threadIdx.x; x < kEvictBins / 2; x += 256)
    to[x] = static_cast<uint32_t>(bins[2 * x]) | (static_cast<uint32_t>(bins[2 * x + 1]) << 16);
}

template <int THREADS, int KEEP>
__global__ void __launch_bounds__(THREADS)
evict_select_kernel(CacheView c, int budget, int sinks, int recent, EvictLists out) {
  constexpr int WAVES = THREADS / 64, PER = kEvictBins / THREADS;
  __shared__ __align__(8) uint16_t upper[KEEP > 0 ? KEEP : 4];
  __shared__ int bins[kEvictBins];
  __shared__ uint32_t list[kEvictList];
  __shared__ int scan[16];
  __shared__ float range[2][WAVES];
  __shared__ int found[4];
  __shared__ int base[WAVES];
  const int g = blockIdx.x, b = g / c.hkv;
  const int len = cache_len(c, b);
  const int w = wave_id(), lane = threadIdx.x & 63;
  int32_t* head = out.heads + static_cast<long long>(g) * kEvictHead;
  if (len <= budget) {
    if (threadIdx.x < kEvictHead) head[threadIdx.x] = 0;
    return;
  }
  const float* wt = c.weights + static_cast<long long>(g) * c.cap;
  const int32_t* pos = c.slot_pos + static_cast<long long>(g) * c.cap;
  const int from_pos = c.seen[b] - recent;
  const uint16_t* halves = out.halves + static_cast<long long>(g) * c.cap;
  const int steps = (len + 4 * THREADS - 1) / (4 * THREADS);
  const int s_wave = w * steps * 256, s0 = s_wave + 4 * lane;
  auto again = [&](int s) { return evict_key(wt[s], pos[s] < sinks || pos[s] >= from_pos); };
  // f(the lane's first slot, its four halves) for the wave's steps
  auto from_memory = [&](auto f) {
    constexpr int kFlight = 4;   // steps whose loads are in flight together
    for (int i0 = 0; i0 < steps; i0 += kFlight) {
      f32x4_any x[kFlight];
      i32x4_any p[kFlight];
#pragma unroll
      for (int e = 0; e < kFlight; ++e) {
        const int s = min(s0 + 256 * (i0 + e), c.cap - 4);
        x[e] = *reinterpret_cast<const f32x4_any*>(wt + s);
        p[e] = *reinterpret_cast<const i32x4_any*>(pos + s);
      }
#pragma unroll
      for (int e = 0; e < kFlight; ++e) {
        if (i0 + e >= steps) break;
        const int s = s0 + 256 * (i0 + e);
        uint32_t k[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          k[j] = s + j >= len ? 0u : evict_half(x[e][j], p[e][j] < sinks || p[e][j] >= from_pos);
        }
        f(s, k);
      }
    }
  };
  auto each = [&](auto f) {
    constexpr int kFlight = KEEP > 0 ? 2 : 8;
    for (int i0 = 0; i0 < steps; i0 += kFlight) {
      uint2 y[kFlight];
#pragma unroll
      for (int e = 0; e < kFlight; ++e) {
        if constexpr (KEEP > 0) {
          y[e] = *reinterpret_cast<const uint2*>(&upper[s0 + 256 * min(i0 + e, steps - 1)]);
        } else {
          const int s = s0 + 256 * (i0 + e);
          y[e] = *reinterpret_cast<const uint2*>(halves + min(s, c.cap - 4));   // (no branch: all on their way together)
        }
      }
#pragma unroll
      for (int e = 0; e < kFlight; ++e) {
        if (i0 + e >= steps) break;
        if (KEEP == 0 && s0 + 256 * (i0 + e) >= len) y[e] = make_uint2(0u, 0u);
        const uint32_t k[4] = {y[e].x & 0xFFFFu, y[e].x >> 16, y[e].y & 0xFFFFu, y[e].y >> 16};
        f(s0 + 256 * (i0 + e), k);
      }
    }
  };
  // one histogram: the bin that the need-th largest of the counted values falls
  // into is left in found[0], the values above it in found[1], its own in found[2]
  auto clear_bins = [&] {
    for (int x = threadIdx.x; x < kEvictBins; x += THREADS) bins[x] = 0;
    __syncthreads();
  };
  auto find_bin = [&](int need) {
    __syncthreads();
    const int x = kEvictBins - PER * (threadIdx.x + 1);   // bins from the top, PER a thread
    int n[PER], sum = 0, all;
#pragma unroll
    for (int e = 0; e < PER; ++e) { n[e] = bins[x + e]; sum += n[e]; }
    int before = block_exclusive_scan(sum, scan, &all);
    if (before < need && before + sum >= need) {
#pragma unroll
      for (int e = PER - 1; e >= 0; --e) {
        if (before < need && before + n[e] >= need) {
          found[0] = x + e;
          found[1] = before;
          found[2] = n[e];
        }
        before += n[e];
      }
    }
    __syncthreads();
  };
  auto width = [](uint32_t span) {   // bins as wide as 2^ this cover span + 1 values
    const int bits = span ? 32 - __clz(span) : 0;
    return bits > 11 ? bits - 11 : 0;
  };

  // T is the need-th largest key of the `some` keys with halves in [lo, hi]
  uint32_t lo = kSafeHalf, hi = 1u;
  int need = budget, some = len;
  if constexpr (KEEP > 0) {
    // protected slots stay, first of all; the histograms need only span the others
    int safe = 0;
    from_memory([&](int s, const uint32_t* k) {
      // (read back by this lane only)
      *reinterpret_cast<uint2*>(&upper[s]) = make_uint2(k[0] | (k[1] << 16), k[2] | (k[3] << 16));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        safe += k[j] == kSafeHalf;
        lo = k[j] ? min(lo, k[j]) : lo;
        hi = k[j] != kSafeHalf ? max(hi, k[j]) : hi;
      }
    });
    const float l = wave_min(static_cast<float>(lo)), h = wave_max(static_cast<float>(hi));   // (exact)
    if (lane == 0) { range[0][w] = l; range[1][w] = h; }
    int all;
    block_exclusive_scan(safe, scan, &all);
    float fl = range[0][0], fh = range[1][0];
#pragma unroll
    for (int u = 1; u < WAVES; ++u) { fl = fminf(fl, range[0][u]); fh = fmaxf(fh, range[1][u]); }
    if (all >= budget) {     // (more protected slots than the budget: positions given twice)
      lo = hi = kSafeHalf;
      some = all;
    } else {
      lo = static_cast<uint32_t>(fl);
      hi = static_cast<uint32_t>(fh);
      need -= all;
      some -= all;
    }
  } else {
    int n[PER] = {};
    static_assert(PER == 2, "two bins a thread");
    const uint32_t* hist = reinterpret_cast<const uint32_t*>(
        out.hist + static_cast<long long>(g) * evict_slices(c.cap) * kEvictBins);
    const int slices = evict_slices(len);
#pragma unroll 8
    for (int u = 0; u < slices; ++u) {
      const uint32_t y = hist[static_cast<long long>(u) * (kEvictBins / 2) + threadIdx.x];
      n[0] += y & 0xFFFFu;
      n[1] += y >> 16;
    }
    bins[2 * threadIdx.x] = n[0];
    bins[2 * threadIdx.x + 1] = n[1];
    find_bin(need);
    if (found[0] == static_cast<int>(kSafeHalf >> 5)) {   // (more protected slots than the budget: positions given twice)
      hi = kSafeHalf;
    } else {
      lo = max(static_cast<uint32_t>(found[0]) << 5, 1u);
      hi = (static_cast<uint32_t>(found[0]) << 5) + 31u;
    }
    need -= found[1];
    some = found[2];
    __syncthreads();
  }
  while (lo < hi && need < some && some > kEvictList) {
    const int shift = width(hi - lo);
    clear_bins();
    each([&](int, const uint32_t* k) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (k[j] - lo <= hi - lo) atomicAdd(&bins[(k[j] - lo) >> shift], 1);
    });
    find_bin(need);
    lo += static_cast<uint32_t>(found[0]) << shift;
    hi = min(hi, lo + ((1u << shift) - 1u));
    need -= found[1];
    some = found[2];
    __syncthreads();
  }
  // Slots with a half above hi stay, those in [lo, hi] if their key is above T
  // or, for the first `need` of the `some` equal ones, T itself.
  uint32_t T = kSafeKey;
  const bool exact = lo == kSafeHalf || need < some;   // else every key in the range stays
  if (lo != kSafeHalf && exact) {
    if (some <= kEvictList) {
      if (threadIdx.x == 0) found[3] = 0;
      __syncthreads();
      each([&](int s, const uint32_t* k) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (k[j] - lo <= hi - lo) list[atomicAdd(&found[3], 1)] = s + j;
      });
      __syncthreads();
      for (int x = threadIdx.x; x < some; x += THREADS) list[x] = again(list[x]);
      __syncthreads();
      for (int x = threadIdx.x; x < some; x += THREADS) {
        const uint32_t k = list[x];
        int larger = 0, equal = 0;
#pragma unroll 8
        for (int j = 0; j < some; ++j) {
          const uint32_t y = list[j];
          larger += y > k;
          equal += y == k;
        }
        if (larger < need && larger + equal >= need) {   // (the same for every copy of T)
          found[0] = static_cast<int>(k);
          found[1] = need - larger;
          found[2] = equal;
        }
      }
      __syncthreads();
      T = static_cast<uint32_t>(found[0]);
      need = found[1];
      some = found[2];
    } else {                                  // one half, lo = hi
      uint32_t first = (lo - 1u) << 16, last = first | 0xFFFFu;
      while (first < last) {
        const int shift = width(last - first);
        clear_bins();
        each([&](int s, const uint32_t* h) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (h[j] == lo) {
              const uint32_t k = again(s + j);
              if (k - first <= last - first) atomicAdd(&bins[(k - first) >> shift], 1);
            }
        });
        find_bin(need);
        first += static_cast<uint32_t>(found[0]) << shift;
        last = min(last, first + ((1u << shift) - 1u));
        need -= found[1];
        some = found[2];
        __syncthreads();
      }
      T = first;
    }
  }
  const bool split = need < some;   // the cut falls between equal keys
  // keys of [lo, hi] above and equal to T, as bits of the lane's four slots
  auto compare = [&](int s, const uint32_t* h, int& above, int& equal) {
    above = equal = 0;
    bool any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      above |= h[j] > hi ? 1 << j : 0;
      any = any || h[j] - lo <= hi - lo;
    }
    if (any) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (h[j] - lo <= hi - lo) {
          const uint32_t k = exact ? again(s + j) : T;
          above |= k > T ? 1 << j : 0;
          equal |= k == T ? 1 << j : 0;
        }
    }
  };
  int ties = 0;   // equal keys in the waves before
  if (split) {
    int n = 0;
    each([&](int s, const uint32_t* h) {
      int above, equal;
      compare(s, h, above, equal);
      n += __popc(equal);
    });
    n = wave_sum_i(n);
    if (lane == 0) base[w] = n;
    __syncthreads();
    for (int u = 0; u < w; ++u) ties += base[u];
  }
  int32_t* to = out.to + static_cast<long long>(g) * c.cap + min(s_wave, c.cap);
  int32_t* from = out.from + static_cast<long long>(g) * c.cap + min(s_wave, c.cap);
  int holes = 0, movers = 0;
  each([&](int s, const uint32_t* h) {
    int kept, equal;
    compare(s, h, kept, equal);
    if (!split) {
      kept |= equal;
    } else {
      const int n = __popc(equal), upto = wave_scan_add(n);
      int rank = ties + upto - n;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if ((equal >> j) & 1) {
          kept |= rank < need ? 1 << j : 0;
          ++rank;
        }
      ties += __builtin_amdgcn_readlane(upto, 63);
    }
    const int left = budget - s;              // slots of the four below the budget
    const int low = left >= 4 ? 15 : left <= 0 ? 0 : (1 << left) - 1;
    const int hole = low & ~kept, move = kept & ~low;
    if (__ballot((hole | move) != 0)) {
      const int n = __popc(hole) | (__popc(move) << 16), upto = wave_scan_add(n);
      int ih = holes + ((upto - n) & 0xFFFF), im = movers + ((upto - n) >> 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if ((hole >> j) & 1) to[ih++] = s + j;
        if ((move >> j) & 1) from[im++] = s + j;
      }
      const int total = __builtin_amdgcn_readlane(upto, 63);
      holes += total & 0xFFFF;
      movers += total >> 16;
    }
  });
  if (lane == 0) {
    head[w] = holes;
    head[kEvictRuns + w] = movers;
  }
  if (WAVES < kEvictRuns && threadIdx.x >= WAVES && threadIdx.x < kEvictRuns)
    head[threadIdx.x] = head[kEvictRuns + threadIdx.x] = 0;
  if (threadIdx.x == 0) head[2 * kEvictRuns] = steps * 256;
}

// Rows from their slots to the free ones, kMoveDepth pieces of K and V in
// flight per thread: the i-th free slot takes the i-th kept slot above the
// budget, each counted through the runs of the lists.  (2 caches of 65536 slots on
// 8 heads of 128 in bf16 cut to 8192: 22 us, 5 TB/s.)
constexpr int kMoveDepth = 2;
__global__ void __launch_bounds__(256)
evict_move_kernel(CacheView c, int budget, EvictLists in, int chunks) {
  __shared__ int ends[2][kEvictRuns];   // of the runs' lists, counted from the first
  const int g = blockIdx.x, b = g / c.hkv, h = g - b * c.hkv;
  const int32_t* head = in.heads + static_cast<long long>(g) * kEvictHead;
  const int run = head[2 * kEvictRuns];
  if (threadIdx.x < 64) {
    const int x = threadIdx.x & 15, which = (threadIdx.x >> 4) & 1;
    int n = head[which * kEvictRuns + x];
#pragma unroll
    for (int o = 1; o < 16; o *= 2) {
      const int y = __shfl_up(n, o, 16);
      n += x >= o ? y : 0;
    }
    if (threadIdx.x < 32) ends[which][x] = n;
  }
  __syncthreads();
  const int n = ends[0][kEvictRuns - 1];
  const int32_t* lists[2] = {in.to + static_cast<long long>(g) * c.cap, in.from + static_cast<long long>(g) * c.cap};
  auto entry = [&](int which, int i) {
    int u = 0;
#pragma unroll
    for (int o = kEvictRuns / 2; o >= 1; o /= 2) u += ends[which][u + o - 1] <= i ? o : 0;
    return lists[which][u * run + i - (u ? ends[which][u - 1] : 0)];
  };
  u32x4* k = static_cast<u32x4*>(c.k);
  u32x4* v = static_cast<u32x4*>(c.v);
  const int stride = gridDim.y * 256, total = n * chunks;
  float* wt = c.weights + static_cast<long long>(g) * c.cap;
  int32_t* pos = c.slot_pos + static_cast<long long>(g) * c.cap;
  for (int x0 = blockIdx.y * 256 + threadIdx.x; x0 < total; x0 += kMoveDepth * stride) {
    int to[kMoveDepth], from[kMoveDepth], ch[kMoveDepth];
#pragma unroll
    for (int u = 0; u < kMoveDepth; ++u) {
      const int x = min(x0 + u * stride, total - 1), i = x / chunks;   // (past the end: the last piece again)
      ch[u] = x - i * chunks;
      to[u] = entry(0, i);
      from[u] = entry(1, i);
    }
    long long rt[kMoveDepth], rf[kMoveDepth];
#pragma unroll
    for (int u = 0; u < kMoveDepth; ++u) {
      rt[u] = cache_row(c, b, h, to[u]);
      rf[u] = cache_row(c, b, h, from[u]);
    }
    u32x4 kk[kMoveDepth], vv[kMoveDepth];
    float w[kMoveDepth];
    int p[kMoveDepth];
#pragma unroll
    for (int u = 0; u < kMoveDepth; ++u) {
      const long long f = rt[u] < 0 || rf[u] < 0 ? 0 : rf[u] * chunks + ch[u];   // (not moved: reads the first row)
      kk[u] = k[f];
      vv[u] = v[f];
      w[u] = wt[from[u]];
      p[u] = pos[from[u]];
    }
#pragma unroll
    for (int u = 0; u < kMoveDepth; ++u) {
      if (ch[u] == 0) {
        wt[to[u]] = w[u];
        pos[to[u]] = p[u];
      }
      if (rt[u] >= 0 && rf[u] >= 0) {
        k[rt[u] * chunks + ch[u]] = kk[u];
        v[rt[u] * chunks + ch[u]] = vv[u];
      }
    }
  }
  // (nothing else of this call reads the lengths any more)
  if (h == 0 && blockIdx.y == 0 && threadIdx.x == 0) c.lens[b] = min(cache_len(c, b), budget);
}

long long evict_max_groups(const CacheView& c) {
  return ((1ll << 32) - 1) / (c.cap <= kEvictShort ? 256 : kEvictThreads);
}

long long evict_scratch_bytes(const CacheView& c) {
  const long long groups = static_cast<long long>(c.n_seq) * c.hkv;
  const long long lists = 4 * groups * (kEvictHead + 2ll * c.cap);
  return c.cap <= kEvictShort ? lists : lists + 2 * groups * (c.cap + static_cast<long long>(evict_slices(c.cap)) * kEvictBins);
}

hipError_t launch_cache_evict(const CacheView& c, int budget, int sinks, int recent, void* scratch, hipStream_t st) {
  const int esz = c.dtype == 0 ? 4 : 2, chunks = c.dh * esz / 16;
  const long long groups = static_cast<long long>(c.n_seq) * c.hkv;
  EvictLists lists;   // (each part begins at a multiple of 16 bytes: cap is one of 16 slots)
  lists.heads = static_cast<int32_t*>(scratch);
  lists.to = lists.heads + groups * kEvictHead;
  lists.from = lists.to + groups * c.cap;
  lists.halves = reinterpret_cast<uint16_t*>(lists.from + groups * c.cap);
  lists.hist = lists.halves + groups * c.cap;
  if (c.cap <= kEvictShort) {
    hipLaunchKernelGGL((evict_select_kernel<256, kEvictShort>), dim3(groups), dim3(256), 0, st, c, budget, sinks, recent,
                       lists);
  } else {
    hipLaunchKernelGGL(evict_halves_kernel, dim3(groups, evict_slices(c.cap)), dim3(256), 0, st, c, budget, sinks, recent,
                       lists);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    hipLaunchKernelGGL((evict_select_kernel<kEvictThreads, 0>), dim3(groups), dim3(kEvictThreads), 0, st, c, budget, sinks, recent, lists);
  }
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;   // (the lists that the next kernel follows were not written)
  const long long total = static_cast<long long>(std::min(c.cap - budget, budget)) * chunks;   // pieces that can move
  const int gy =
      static_cast<int>(std::max<long long>(1, std::min<long long>((total + 256 * kMoveDepth - 1) / (256 * kMoveDepth), 1024)));
  hipLaunchKernelGGL(evict_move_kernel, dim3(groups, gy), dim3(256), 0, st, c, budget, lists, chunks);
  return hipGetLastError();
}

}  // namespace gmc
