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
#include <limits.h>

#include <algorithm>

#include "gmc_cache.h"
#include "gmc_cache_grid.h"
#include "gmc_device.h"

namespace gmc {

// (the kernel's parts: out of line, what they share would live in memory)
#define GMC_INLINE __attribute__((always_inline))
constexpr int kPreWaves = 4, kPreRows = 32 * kPreWaves;
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Shared and global memory by their address spaces, as the loads into shared
// memory and the transposing reads take them.
typedef __attribute__((address_space(3))) unsigned char shared_u8;
typedef __attribute__((address_space(1))) uint32_t global_u32;
template <typename V> __device__ __forceinline__ V ld_shared(const shared_u8* p) {
  return *reinterpret_cast<const __attribute__((address_space(3))) V*>(p);
}

// A row of zeros: what a slot that is not held reads as.
__device__ const uint4 kZeroRow[64] = {};

template <typename T, int DH> struct KeyTile {
  static constexpr int CPR = DH * static_cast<int>(sizeof(T)) / 16;   // 16-byte chunks of a row
  static constexpr int KT = sizeof(T) == 2 && DH <= 128 ? 64 : 32;
  static constexpr bool kPow2 = (CPR & (CPR - 1)) == 0;
  // Where chunk c of a row stands, and which chunk stands at c.  Depends on
  // row % 16 (fp32: row % 8) only.
  static __device__ __forceinline__ int mix(int row) {
    if constexpr (!kPow2) return sizeof(T) == 4 ? row & 7 : (row >> 2) & 3;
    if constexpr (sizeof(T) == 4) return (row & 7) ^ (((row >> 2) & 1) << 3);
    if constexpr (CPR >= 16) return ((row & 3) << 2) | ((row >> 2) & 3);
    if constexpr (CPR == 8) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    return (row >> 2) & 3;
  }
  static __device__ __forceinline__ int place(int row, int c) {
    if constexpr (kPow2) return c ^ (mix(row) & (CPR - 1));
    return (c + mix(row)) % CPR;
  }
  static __device__ __forceinline__ int chunk_at(int row, int c) {
    if constexpr (kPow2) return c ^ (mix(row) & (CPR - 1));
    return (c + CPR - mix(row)) % CPR;
  }
};

// The rows and key tiles of one block.
struct PreWork {
  long long first;      // first row of the sequence's tokens
  int n, len;           // its tokens, its slots
  int row0, rows;       // the block's rows of (token, head)
  int t_min, t_max;     // slots of its first and last token
  int tiles, sink_tiles, skip;   // tile i: i < sink_tiles ? i : i + skip
};
__device__ __forceinline__ PreWork pre_work(const CacheView& c, const AttendArgs& a, int b, int block, int kt) {
  PreWork w;
  new_rows(a.starts, a.max_new, a.rows, b, &w.first, &w.n);
  w.len = cache_len(c, b);
  w.row0 = block * kPreRows;
  w.rows = min(kPreRows, w.n * c.hg - w.row0);
  if (w.rows <= 0) return w;
  w.t_min = w.len - w.n + w.row0 / c.hg;
  w.t_max = w.len - w.n + (w.row0 + w.rows - 1) / c.hg;
  const int end = w.t_max < 0 ? 0 : w.t_max / kt + 1;
  w.sink_tiles = end;
  w.skip = 0;
  if (a.window > 0 && !c.slot_pos && w.t_min >= a.window) {
    const int lo = (w.t_min - a.window + 1) / kt;
    const int sink = a.sinks / kt + (a.sinks % kt != 0);
    w.sink_tiles = min(sink, lo);
    w.skip = lo - w.sink_tiles;
  }
  w.tiles = end - w.skip;
  return w;
}

struct PreScratch {
  float* part;   // [n_seq * max_new][hq][nsplit][dh] unnormalised sums, or null
  float* ml;     // [n_seq * max_new][hq][nsplit][2] maximum (base 2) and sum
  int nsplit;
  PreGrid grid;
};
// Splits that a block's tiles are shared over: none with fewer than two tiles.
__device__ __forceinline__ int used_pre_splits(int tiles, int nsplit) { return min(nsplit, max(1, tiles / 2)); }

template <typename T, int DH>
__global__ void __launch_bounds__(64 * kPreWaves, sizeof(T) == 2 && DH <= 128 ? 2 : 1)
prefill_kernel(CacheView c, AttendArgs a, PreScratch sc, int row_blocks) {
  using KTile = KeyTile<T, DH>;
  constexpr int CPR = KTile::CPR, KT = KTile::KT, KB = KT / 32, NB = DH / 32, PITCH = CPR * 16;
  constexpr int NS = sizeof(T) == 2 ? DH / 16 : DH / 8;    // reads of 16 bytes a lane needs of its K row
  constexpr int GROUPS = KT / 16;                          // runs of 16 slots, each on one page
  constexpr int LOADS = CPR / 4;                           // 1 KB loads of one run
  __shared__ __align__(16) unsigned char k_even[KT * PITCH], v_even[KT * PITCH], k_odd[KT * PITCH], v_odd[KT * PITCH];
  __shared__ __align__(16) int pos_even[64], pos_odd[64];   // positions of the tiles' slots, if the window asks for them

  // (in a head, rows with the most keys come first)
  const int heads = c.hkv * c.n_seq;
  int bh, item;
  if (!pre_place(sc.grid, blockIdx.x, heads, &bh, &item)) return;
  const int split = item % sc.nsplit, block = row_blocks - 1 - item / sc.nsplit, h = bh % c.hkv, b = bh / c.hkv;
  const PreWork wk = pre_work(c, a, b, block, KT);
  if (wk.rows <= 0) return;
  const int ns = used_pre_splits(wk.tiles, sc.nsplit);
  if (split >= ns) {   // no part: the join leaves it out
    for (int x = threadIdx.x; x < wk.rows; x += 64 * kPreWaves) {
      const int r = wk.row0 + x;
      const long long part_row =
          ((static_cast<long long>(b) * a.max_new + r / c.hg) * c.hq + h * c.hg + r % c.hg) * sc.nsplit + split;
      sc.ml[2 * part_row] = -INFINITY;
      sc.ml[2 * part_row + 1] = 0.f;
    }
    return;
  }
  const int it0 = static_cast<int>(static_cast<long long>(wk.tiles) * split / ns);
  const int it1 = static_cast<int>(static_cast<long long>(wk.tiles) * (split + 1) / ns);

  const int lane = threadIdx.x & 63, w = wave_id(), half = lane >> 5, col = lane & 31;
  // the lane's query; rows past the block's last repeat it and are not written
  const int row = min(32 * w + col, wk.rows - 1) + wk.row0;
  const int tok = row / c.hg, hq = h * c.hg + row % c.hg;
  const int t = wk.len - wk.n + tok;
  const bool live = 32 * w + col < wk.rows;
  // slots of the wave's first and last query
  const int wt_min = wk.len - wk.n + (wk.row0 + min(32 * w, wk.rows - 1)) / c.hg;
  const int wt_max = wk.len - wk.n + (wk.row0 + min(32 * w + 31, wk.rows - 1)) / c.hg;
  const long long at = (static_cast<long long>(b) * c.hkv + h) * c.cap;
  const int32_t* pos = a.window ? c.slot_pos : nullptr;    // positions matter to the window only
  if (pos) pos += at;
  const int mine = pos && t >= 0 ? pos[t] : t;
  // exp2(scale log2(e) s): a negative scale goes to the queries' sign, and a
  // scale of zero to the least one that does not turn a hidden key's -inf into
  // NaN (the largest product then makes a logit of 5e-7)
  const float cs = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 0x1p-149f);

  const int32_t* table = c.table + static_cast<long long>(b) * c.max_pages;
  auto slot0 = [&](int it) GMC_INLINE { return (it < wk.sink_tiles ? it : it + wk.skip) * KT; };
  // The page ids of a tile's runs, one a lane (the first GROUPS lanes): fetched a
  // tile before its loads start, which would wait for them (3900 of 7100 cycles
  // a tile), and first looked at there: a look here would wait for all loads on
  // their way.
  auto fetch = [&](int it) GMC_INLINE { return table[min(slot0(it) + 16 * (lane & (GROUPS - 1)), c.cap - 1) >> c.shift]; };
  // Which runs of a tile are on a page.
  auto on_pages = [&](int it, int ids) GMC_INLINE {
    const bool on = slot0(it) + 16 * (lane & (GROUPS - 1)) < wk.len && ids >= 0 && ids < c.n_pages;
    return static_cast<unsigned>(__ballot(on)) & ((1u << GROUPS) - 1u);
  };
  const int ids0 = fetch(it0), ids1 = fetch(it0 + 1);

  uint4 q[NS];
  {
    const T* qp = static_cast<const T*>(a.q) + (wk.first + tok) * a.q_stride + static_cast<long long>(hq) * DH;
#pragma unroll
    for (int s = 0; s < NS; ++s) q[s] = ld16(reinterpret_cast<const char*>(qp) + 16 * (2 * s + half));
  }
  floatx16 o[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[n][i] = 0.f;
  float m = -INFINITY, l = 0.f;
  const float slack = fminf(8.f / cs, 0x1p126f);   // (not infinite: the first maximum is above -inf + slack)

  // Offsets of a lane's reads.  With a power of two of chunks to a row they are
  // exclusive ors of one offset each with constants, and are formed where they
  // are used: kept, they took the registers that hold the running sums.
  // Loads: piece u of a run of 16 slots, by position in shared memory; the source
  // chunk's byte offset in the run's rows.
  auto src_off = [&](int u) GMC_INLINE {
    const int p = 64 * u + lane, r = p / CPR;
    return r * PITCH + KTile::chunk_at(r, p % CPR) * 16;
  };
  constexpr bool kXor = KTile::kPow2;
  constexpr int VO = sizeof(T) == 2 ? 2 : 4;
  int k_base[kXor ? 1 : NS], v_base[kXor ? 1 : NB][VO];
#pragma unroll
  for (int s = 0; s < (kXor ? 1 : NS); ++s) k_base[s] = col * PITCH + KTile::place(col, 2 * s + half) * 16;
#pragma unroll
  for (int n = 0; n < (kXor ? 1 : NB); ++n)
#pragma unroll
    for (int e = 0; e < VO; ++e) {
      if constexpr (sizeof(T) == 2) {      // a transposing read of 4 keys x 16 dims
        const int i = lane & 15, r = 8 * e + 4 * half + (i >> 2);
        const int ch = 4 * n + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
        v_base[n][e] = r * PITCH + KTile::place(r, ch) * 16 + 8 * (i & 1);
      } else {                             // one value of a key
        const int r = 4 * half + e;        // of 8 keys; the next 8 lie 8 rows on
        v_base[n][e] = r * PITCH + KTile::place(r, 8 * n + (col >> 2)) * 16 + 4 * (col & 3);
      }
    }
  auto k_off = [&](int s) GMC_INLINE { return kXor ? k_base[0] ^ (32 * s) : k_base[kXor ? 0 : s]; };
  auto v_off = [&](int n, int e) GMC_INLINE {
    return kXor ? v_base[0][e] ^ ((sizeof(T) == 2 ? 64 : 128) * n) : v_base[kXor ? 0 : n][e];
  };

  const long long page_bytes = static_cast<long long>(c.page) * PITCH;
  // Starts the loads of a tile; returns which of its runs are on a page.  A wave
  // loads K and V of one run (64 keys a tile), or one of the two (32 keys).
  auto issue = [&](int it, int ids, shared_u8* ks, shared_u8* vs, shared_u8* ps) GMC_INLINE -> unsigned {
    const int s0 = slot0(it);
    if (pos && w == 0) __builtin_amdgcn_global_load_lds((const global_u32*)(pos + min(s0 + lane, c.cap - 1)), ps, 4, 0, 0);
    constexpr bool kBoth = GROUPS == kPreWaves;
    static_assert(kBoth || 2 * GROUPS == kPreWaves, "a wave loads K and V of a run, or one of them");
    const int mine = kBoth ? w : w >> 1;
    const unsigned ok = on_pages(it, ids);
    const int pid = (ok >> mine) & 1u ? __builtin_amdgcn_readlane(ids, mine) : -1;
    const int s = s0 + 16 * mine, held = pid < 0 ? 0 : wk.len - s;   // rows of the run that are held
    const long long base =
        (static_cast<long long>(pid) * c.hkv + h) * page_bytes + static_cast<long long>(s & (c.page - 1)) * PITCH;
    auto copy = [&](const void* pages, shared_u8* to) GMC_INLINE {
      const char* from = static_cast<const char*>(pages) + base;
      to += 16 * mine * PITCH;
      if (held >= 16) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u)
          __builtin_amdgcn_global_load_lds((const global_u32*)(from + src_off(u)), to + 1024 * u, 16, 0, 0);
      } else {
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
          const char* at = (64 * u + lane) / CPR < held ? from + src_off(u) : reinterpret_cast<const char*>(kZeroRow);
          __builtin_amdgcn_global_load_lds((const global_u32*)at, to + 1024 * u, 16, 0, 0);
        }
      }
    };
    if constexpr (kBoth) {
      copy(c.k, ks);
      copy(c.v, vs);
    } else {
      copy((w & 1) ? c.v : c.k, (w & 1) ? vs : ks);
    }
    return ok;
  };

  // Sets the infinities and NaN among a lane's 16 bytes of values to zero; returns
  // whether there were any.
  auto clean = [](u32x4& y) GMC_INLINE {
    constexpr uint32_t kExp = sizeof(T) == 2 ? 0x7F807F80u : 0x7F800000u, kOne = sizeof(T) == 2 ? 0x00800080u : 0x00800000u;
    constexpr uint32_t kTop = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
    const uint32_t hit = (((y.x & kExp) + kOne) | ((y.y & kExp) + kOne) | ((y.z & kExp) + kOne) | ((y.w & kExp) + kOne)) & kTop;
    if (!hit) return false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t top = ((y[e] & kExp) + kOne) & kTop;   // a bit for each value that goes
      y[e] = sizeof(T) == 2 ? y[e] & ~((top >> 15) * 0xFFFFu) : (top ? 0u : y[e]);
    }
    return true;
  };
  // whether some query of the block does not see some key of the tile
  auto edge_of_block = [&](int s0, unsigned ok) GMC_INLINE {
    return ok != (1u << GROUPS) - 1u || s0 + KT - 1 > wk.t_min || pos || (a.window && wk.t_max - s0 >= a.window);
  };
  // An infinity or NaN among the values must not reach a query that does not see
  // it, through a weight of zero.  That it did shows in the sums, so the block's
  // tiles are first taken as if there were none; if a sum is not finite, all over
  // again with care: the infinities and NaN of tiles where some query does not
  // see some key are taken out, and added at the end.
  bool care = false;
  auto compute = [&](int it, unsigned ok, shared_u8* ks, shared_u8* vs, shared_u8* ps) GMC_INLINE {
    const int s0 = slot0(it);
    if (care && edge_of_block(s0, ok)) {
      // (bf16 tiles of 160 and 224 dims have 640 and 896 chunks: the last round is
      // for half of the threads)
      constexpr int kChunks = KT * CPR, kThreads = 64 * kPreWaves;
#pragma unroll 1
      for (int x = 0; x < (kChunks + kThreads - 1) / kThreads; ++x) {
        if (kChunks % kThreads != 0 && kThreads * x + static_cast<int>(threadIdx.x) >= kChunks) break;
        shared_u8* at = vs + 16 * (kThreads * x + static_cast<int>(threadIdx.x));
        u32x4 y = ld_shared<u32x4>(at);
        if (clean(y)) *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(at) = y;
      }
      __syncthreads();
    }
    if (s0 > wt_max) return;
    const bool all = ok == (1u << GROUPS) - 1u;
    if constexpr (kXor) {
      asm volatile("" : "+v"(k_base[0]));   // (formed in each tile anew)
#pragma unroll
      for (int e = 0; e < VO; ++e) asm volatile("" : "+v"(v_base[0][e]));
    }
    floatx16 x[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[kb][i] = 0.f;
    typedef __attribute__((address_space(3))) shortx4 shared4;
    if constexpr (sizeof(T) == 2) {
      // kAhead steps of K's reads before the first product, then one step of
      // products for one of reads
      constexpr int kAhead = NS < 4 ? NS : 4;
      u32x4 kf[NS][KB];
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) kf[s][kb] = ld_shared<u32x4>(ks + k_off(s) + 32 * kb * PITCH);
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
          x[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[s][kb]),
                                                          __builtin_bit_cast(bf16x8, q[s]), x[kb], 0, 0, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, kAhead * KB, 0);
#pragma unroll
      for (int s = 0; s < NS - kAhead; ++s) {
        __builtin_amdgcn_sched_group_barrier(0x8, KB, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, KB, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x8, kAhead * KB, 0);
    } else {
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const u32x4 kf = ld_shared<u32x4>(ks + k_off(s));
        const uint32_t qe[4] = {q[s].x, q[s].y, q[s].z, q[s].w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          x[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e]), __uint_as_float(qe[e]), x[0], 0, 0, 0);
      }
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) settle(x[kb]);
    // (compared first: t may be negative and the window as large as an integer)
    const bool before = a.window && wt_min >= a.window && s0 + KT - 1 <= wt_min - a.window;   // the windows of all queries
    if (!all || pos || (a.window && s0 < a.sinks && !before)) {
      const int win = a.window ? a.window : INT_MAX;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int sl = 32 * kb + 8 * j + 4 * half, s = s0 + sl;   // four slots
          const bool on = (ok >> (2 * kb + (j >> 1))) & 1u;
          int p[4] = {s, s + 1, s + 2, s + 3};
          if (pos) {
            const u32x4 y = ld_shared<u32x4>(ps + 4 * sl);
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] = static_cast<int>(y[r]);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const bool see = on & (s + r <= t) & ((mine - p[r] < win) | (p[r] < a.sinks));
            x[kb][4 * j + r] = see ? x[kb][4 * j + r] : -INFINITY;
          }
        }
    } else if (s0 + KT - 1 > wt_min || (a.window && wt_max - s0 >= a.window)) {
      // the slots that a query sees are one run: of `span` + 1 from `lo` on (none:
      // lo is past the tile)
      int lo = a.window && t >= a.window ? t - a.window + 1 : 0, end = t;
      if (before) { lo = 0; end = a.sinks - 1; }
      if (end < 0) { lo = INT_MAX; end = INT_MAX; }
      const unsigned span = static_cast<unsigned>(end - lo);
      const unsigned at = static_cast<unsigned>(s0 + 4 * half) - static_cast<unsigned>(lo);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          x[kb][i] = at + (32 * kb + 8 * (i >> 2) + (i & 3)) <= span ? x[kb][i] : -INFINITY;
    }
    float mt = x[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mt = fmaxf(mt, x[kb][i]);
    mt = fmaxf(mt, xor_lane<32>(mt));
    // the running maximum follows in steps of at least 8 (base 2): weights stay
    // below 2^8 and most tiles rescale nothing.  Each query's own: its bits do
    // not depend on its neighbours'
    if (__any(mt > m + slack)) {
      const float mn = mt > m + slack ? mt : m;
      const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - mn) * cs);
      m = mn;
      l *= f;
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[n][i] *= f;
    }
    const float base = m == -INFINITY ? 0.f : m * cs;
    float sum = 0.f;
    // weight i of the lane's keys
    auto weight = [&](int kb, int i) GMC_INLINE {
      x[kb][i] = __builtin_amdgcn_exp2f(fmaf(x[kb][i], cs, -base));
      sum += x[kb][i];
    };
    if constexpr (sizeof(T) == 2) {
      // 16 keys at a time: their products are spread over the exponentials of
      // the next 16 keys, whose values are read meanwhile
      shortx4 v[2][NB][2];
      auto read_values = [&](int st) GMC_INLINE {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            v[st % 2][n][e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared4*)(vs + 16 * st * PITCH + v_off(n, e)));
      };
      bf16x8 p[2];
      auto weights = [&](int st) GMC_INLINE {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          weight(st / 2, 8 * (st % 2) + j);
          p[st % 2][j] = static_cast<__bf16>(x[st / 2][8 * (st % 2) + j]);
        }
      };
      read_values(0);
      weights(0);
#pragma unroll
      for (int st = 0; st < 2 * KB; ++st) {
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const auto both = __builtin_shufflevector(v[st % 2][n][0], v[st % 2][n][1], 0, 1, 2, 3, 4, 5, 6, 7);
          o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, both), p[st % 2], o[n], 0, 0, 0);
        }
        if (st + 1 < 2 * KB) {
          read_values(st + 1);
          weights(st + 1);
        }
      }
      l += sum;
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) weight(0, i);
      l += sum;
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int n = 0; n < NB; ++n)
          o[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(ld_shared<float>(vs + 8 * (i >> 2) * PITCH + v_off(n, i & 3)), x[0][i],
                                                      o[n], 0, 0, 0);
    }
  };
  // a tile is in shared memory for all waves once each has waited for its loads
  auto arrive = [&]() GMC_INLINE {
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __syncthreads();
  };

  shared_u8* const kb0 = (shared_u8*)k_even;
  shared_u8* const vb0 = (shared_u8*)v_even;
  shared_u8* const kb1 = (shared_u8*)k_odd;
  shared_u8* const vb1 = (shared_u8*)v_odd;
  shared_u8* const pb0 = (shared_u8*)pos_even;
  shared_u8* const pb1 = (shared_u8*)pos_odd;
  unsigned ok0 = 0, ok1 = 0;
  for (;;) {
    if (it0 < it1) ok0 = issue(it0, ids0, kb0, vb0, pb0);
    if (!care && a.scale < 0.f) {
      constexpr uint32_t kFlip = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
#pragma unroll
      for (int s = 0; s < NS; ++s) { q[s].x ^= kFlip; q[s].y ^= kFlip; q[s].z ^= kFlip; q[s].w ^= kFlip; }
    }
    int ids = ids1;
    for (int it = it0; it < it1; it += 2) {
      arrive();
      if (it + 1 < it1) ok1 = issue(it + 1, ids, kb1, vb1, pb1);
      ids = fetch(it + 2);
      compute(it, ok0, kb0, vb0, pb0);
      if (it + 1 >= it1) break;
      arrive();
      if (it + 2 < it1) ok0 = issue(it + 2, ids, kb0, vb0, pb0);
      ids = fetch(it + 3);
      compute(it + 1, ok1, kb1, vb1, pb1);
    }
    asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");   // (see settle)
    __builtin_amdgcn_sched_barrier(0);
    if (care) break;
    float odd = 0.f;   // not zero where a sum is not finite
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd = fmaf(o[n][i], 0.f, odd);
    if (!__syncthreads_or(odd != 0.f)) break;
    care = true;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[n][i] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }
  if (care) {
    // the infinities and NaN that were taken out, to the queries that see them
#pragma unroll 1
    for (int it = it0; it < it1; ++it) {
      if (!edge_of_block(slot0(it), on_pages(it, fetch(it)))) continue;
#pragma unroll 1
      for (int s = slot0(it); s < min(slot0(it) + KT, wk.len); ++s) {
        const long long row_at = cache_row(c, b, h, s);
        if (row_at < 0) continue;
        const int p = pos ? pos[s] : s;
        const bool see = s <= t && (!a.window || mine - p < a.window || p < a.sinks);
        const T* vp = static_cast<const T*>(c.v) + row_at * DH + 4 * half;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float v = to_f32<T>(vp[32 * n + 8 * (i >> 2) + (i & 3)]);
            o[n][i] += see && !(fabsf(v) < INFINITY) ? v : 0.f;
          }
      }
    }
  }
  l = add_xor32(l);
  if (!live) return;
  const long long out_row = (wk.first + tok) * c.hq + hq;
  const float mc = m * cs;
  if (sc.part) {
    const long long part_row = ((static_cast<long long>(b) * a.max_new + tok) * c.hq + hq) * sc.nsplit + split;
    float* to = sc.part + part_row * DH;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<floatx4*>(to + 32 * n + 2 * i + 4 * half) =
            floatx4{o[n][i], o[n][i + 1], o[n][i + 2], o[n][i + 3]};
    if (half == 0) {
      sc.ml[2 * part_row] = mc;
      sc.ml[2 * part_row + 1] = l;
    }
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* to = static_cast<T*>(a.out) + out_row * DH;
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = l == 0.f ? 0.f : o[n][i + e] * inv;
      T* p = to + 32 * n + 2 * i + 4 * half;
      if constexpr (sizeof(T) == 2) {
        uint2 u;
        u.x = f32_to_bf16(y[0]) | (static_cast<uint32_t>(f32_to_bf16(y[1])) << 16);
        u.y = f32_to_bf16(y[2]) | (static_cast<uint32_t>(f32_to_bf16(y[3])) << 16);
        *reinterpret_cast<uint2*>(p) = u;
      } else {
        *reinterpret_cast<floatx4*>(p) = floatx4{y[0], y[1], y[2], y[3]};
      }
    }
  if (a.lse && half == 0) a.lse[out_row] = l == 0.f ? -INFINITY : (mc + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
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

static int pre_key_tile(const CacheView& c) { return c.dtype != 0 && c.dh <= 128 ? 64 : 32; }

static int pre_row_blocks(const CacheView& c, int max_new) {
  return static_cast<int>((static_cast<long long>(max_new) * c.hg + kPreRows - 1) / kPreRows);
}

// Splits of a row block's keys, while the blocks find room on the chip together
// (512): a block's tiles, one after the other, against a second launch and the
// parts it reads.  Estimates in us: a tile 1.7 for 64 keys of 128 dims (fp32:
// 1.9 for 32 of 64), the launch 4, parts 4 MB each.  Measured, us with the splits
// chosen and with others: 335 tokens (28 query heads on 4 of 128) 16.7 with 1,
// 20.7 with 2; 1000 tokens 32.5 with 1, 41 with 2; 77 tokens over 4100 slots 27.9
// with 16, 26.2 with 10, 29.8 with 25; 10 over 2000 14.1 with 15, 19.6 with 5;
// 200 over 500 (12 on 12 of 96, 2 sequences) 15.1 with 1, 16.7 with 4; fp32 (8 on
// 2 of 64) 300 tokens 17.0 with 5, 26.6 with 2.
static int pre_splits(const CacheView& c, int max_new) {
  const int kt = pre_key_tile(c), tiles = (c.cap + kt - 1) / kt;
  const long long blocks = static_cast<long long>(pre_row_blocks(c, max_new)) * c.hkv * c.n_seq;
  const double tile = (c.dtype == 0 ? 1.9 / (32 * 64) : 1.7 / (64 * 128)) * kt * c.dh;
  const double part = 8e-6 / 4 * (c.dh + 2) * c.hq * max_new * c.n_seq;
  int best = 1;
  double least = tile * tiles;
  for (int s = 2; s <= tiles / 2 && blocks * s <= 512; ++s) {
    const double time = tile * tiles / s + 4 + part * s;
    if (time < least) {
      least = time;
      best = s;
    }
  }
  return best;
}

long long prefill_scratch_bytes(const CacheView& c, int max_new) {
  const int ns = pre_splits(c, max_new);
  return ns == 1 ? 0 : 4ll * c.n_seq * max_new * c.hq * ns * (c.dh + 2);
}

hipError_t launch_cache_prefill(const CacheView& c, const AttendArgs& a, void* scratch, hipStream_t st) {
  const int row_blocks = pre_row_blocks(c, a.max_new);
  PreScratch sc{};
  sc.nsplit = pre_splits(c, a.max_new);
  if (sc.nsplit > 1) {
    sc.part = static_cast<float*>(scratch);
    sc.ml = sc.part + static_cast<long long>(c.n_seq) * a.max_new * c.hq * sc.nsplit * c.dh;
  }
  sc.grid = pre_grid(row_blocks * sc.nsplit, static_cast<long long>(c.hkv) * c.n_seq);
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
  if (sc.nsplit > 1) {
    const dim3 grid((a.max_new + 3) / 4, c.hq, c.n_seq);
    if (c.dtype == 0)
      hipLaunchKernelGGL(prefill_join_kernel<float>, grid, dim3(256), 0, st, c, a, sc);
    else
      hipLaunchKernelGGL(prefill_join_kernel<bf16_t>, grid, dim3(256), 0, st, c, a, sc);
  }
  return hipGetLastError();
}

}  // namespace gmc
