// The paged K/V cache behind a compacted prompt: its view as the kernels take
// it, and the launchers of its operators.
//
// Slot s of sequence b lies in page table[b][s / page] at row s % page; a
// page holds one run of `page` rows of dh elements per kv head, so that the
// block that works on one head reads whole runs.  Lengths and page ids are
// device data: every kernel clamps a length to the table's capacity and takes
// a slot on a page id outside [0, n_pages) as not held.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#ifdef __HIPCC__
#include "gmc_device.h"
#endif

namespace gmc {

constexpr int kCacheMaxHeads = 256;   // GMC_CACHE_MAX_HEADS

struct CacheView {
  void* k;
  void* v;
  const int32_t* table;   // [n_seq][max_pages]
  int32_t* lens;          // [n_seq]
  int32_t* seen;          // [n_seq] or null: positions given out
  int32_t* slot_pos;      // [n_seq][hkv][cap] or null: position of a slot (null: its index)
  float* weights;         // [n_seq][hkv][cap] or null: accumulated attention weight
  long long n_pages;
  int n_seq, max_pages, shift, page, cap;   // page = 1 << shift rows; cap = max_pages * page
  int hq, hkv, hg, dh, dtype;
};

// One attention call: n query rows of sequence b at row first_b of q and out,
// the last n_b slots of the cache.
struct AttendArgs {
  const void* q;          // rows of hq * dh elements, q_stride elements apart
  long long q_stride, rows;
  const int32_t* starts;  // [n_seq + 1] or null: first_b = b * max_new, n_b = max_new
  int max_new;
  float scale;
  int window, sinks;      // window 0: none
  void* out;              // [rows][hq][dh]
  float* lse;             // [rows][hq] or null
};

// The scales of a cache of 4 bits, whose view holds its codes as k and v: a byte
// for each 32 elements of a row, `bytes` to a row (a power of two).
struct CacheScales {
  uint8_t* k;
  uint8_t* v;
  int bytes;
};
constexpr int scale_bytes(int dh) { return dh <= 32 ? 1 : dh <= 64 ? 2 : dh <= 128 ? 4 : 8; }

// A rotary table; pairs below t_end turn by the first of a token's `axes`
// positions, those below h_end by the second, the others by the third.
struct RotaryView {
  const float* cos;       // [n_pos][rot / 2]
  const float* sin;
  int n_pos, rot, interleaved;
  int axes, t_end, h_end;
};

// New rows of K and V, with the queries of their tokens.
struct RotaryArgs {
  const void *k, *v, *q;  // q may be null
  long long k_stride, v_stride, q_stride, rows, per_seq;   // strides in elements; rows of a sequence that src picks from
  const int32_t *starts, *src, *pos;
  int max_new;
  void* q_out;
};

#ifdef __HIPCC__
// Four integers of an array that is aligned as one is.
typedef int32_t i32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ int cache_len(const CacheView& c, int b) { return min(max(c.lens[b], 0), c.cap); }

// Row of slot s in the pages of head h, in rows of dh elements; -1: not held.
__device__ __forceinline__ long long cache_row(const CacheView& c, int b, int h, int s) {
  const int id = c.table[static_cast<long long>(b) * c.max_pages + (s >> c.shift)];
  if (id < 0 || id >= c.n_pages) return -1;
  return ((static_cast<long long>(id) * c.hkv + h) << c.shift) + (s & (c.page - 1));
}

// Takes a matrix product's result out of the accumulators here, in the same
// basic block.  (The compiler, clang 22 of ROCm 7.2, counts the wait between a
// matrix instruction and the first read of its result along the fall-through
// path only: with a taken branch in between the read came too early and gave
// stale last rows.)
template <typename V> __device__ __forceinline__ void settle(V& x) { asm volatile("" : "+v"(x)); }

// First row and number of rows of sequence b's new tokens, within [0, rows).
__device__ __forceinline__ void new_rows(const int32_t* starts, int max_new, long long rows, int b, long long* first,
                                         int* n) {
  if (!starts) {
    *first = static_cast<long long>(b) * max_new;
    *n = max_new;
  } else {
    const long long lo = min(max(static_cast<long long>(starts[b]), 0ll), rows);
    const long long hi = min(static_cast<long long>(starts[b + 1]), rows);
    *first = lo;
    *n = static_cast<int>(min(max(hi - lo, 0ll), static_cast<long long>(max_new)));
  }
}

// The maximum and sum (both base 2) of a row over its splits.
__device__ __forceinline__ void join_stats(const float* ml, int ns, float* m_out, float* l_out) {
  const int lane = threadIdx.x & 63;
  float m = -INFINITY, l = 0.f;
  for (int s = lane; s < ns; s += 64) {
    const float2 y = *reinterpret_cast<const float2*>(ml + 2 * s);
    const float mn = fmaxf(m, y.x), base = mn == -INFINITY ? 0.f : mn;
    l = l * __builtin_amdgcn_exp2f(m - base) + y.y * __builtin_amdgcn_exp2f(y.x - base);
    m = mn;
  }
  const float mw = wave_max(m), base = mw == -INFINITY ? 0.f : mw;
  *l_out = wave_sum(l * __builtin_amdgcn_exp2f(m - base));
  *m_out = mw;
}
#endif

hipError_t launch_cache_append(const CacheView& c, const void* k, const void* v, long long k_stride,
                               long long v_stride, long long rows, const int32_t* starts, const int32_t* src,
                               int max_new, hipStream_t st);

// Attention of every query row over its sequence's cache.  scratch:
// prefill_scratch_bytes of any content.
long long prefill_scratch_bytes(const CacheView& c, int max_new, bool four_bits = false);
hipError_t launch_cache_prefill(const CacheView& c, const AttendArgs& a, void* scratch, hipStream_t st);

// The same for one query row per sequence (a.starts null, a.max_new 1), with
// the attention weights added to c.weights if asked for.  scratch:
// decode_scratch_bytes of any content.
long long decode_scratch_bytes(const CacheView& c, bool accumulate);
hipError_t launch_cache_decode(const CacheView& c, const AttendArgs& a, bool accumulate, void* scratch,
                               hipStream_t st);

// scratch: evict_scratch_bytes of any content.  n_seq * hkv: at most
// evict_max_groups (a launch has fewer than 2^32 threads).
long long evict_max_groups(const CacheView& c);
long long evict_scratch_bytes(const CacheView& c);
hipError_t launch_cache_evict(const CacheView& c, int budget, int sinks, int recent, void* scratch, hipStream_t st);

// After every row has found its slot: the lengths (and positions given out).
hipError_t launch_cache_advance(const CacheView& c, const int32_t* starts, long long rows, int max_new,
                                hipStream_t st);

// Appending with rotation; into 4 bits with scales.  rotary: null for none, then
// into 4 bits only.
hipError_t launch_cache_append_rotary(const CacheView& c, const CacheScales* scales, const RotaryView* rotary,
                                      const RotaryArgs& a, hipStream_t st);

// Caches of 4 bits.
hipError_t launch_cache4_read(const CacheView& c, const CacheScales& s, long long rows, const int32_t* starts,
                              int max_new, void* k_out, void* v_out, hipStream_t st);
hipError_t launch_cache4_prefill(const CacheView& c, const CacheScales& s, const AttendArgs& a, void* scratch,
                                 hipStream_t st);
long long decode4_scratch_bytes(const CacheView& c);
hipError_t launch_cache4_decode(const CacheView& c, const CacheScales& s, const AttendArgs& a, void* scratch,
                                hipStream_t st);

}  // namespace gmc
