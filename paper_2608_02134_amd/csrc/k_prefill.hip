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
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "gmc_cache.h"
#include "gmc_device.h"

namespace gmc {

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
};
// Splits that a block's tiles are shared over: none with fewer than two tiles.
__device__ __forceinline__ int used_pre_splits(int tiles, int nsplit) { return min(nsplit, max(1, tiles / 2)); }

template <typename T>
__device__ __forceinline__ bool not_finite(uint32_t u) {
  if constexpr (sizeof(T) == 4) return (u & 0x7F800000u) == 0x7F800000u;
  return (u & 0x7F80u) == 0x7F80u || (u & 0x7F800000u) == 0x7F800000u;
}

// A value's bits: of kind 0 with infinities and NaN set to zero, of kind 1, 2
// and 3 as 1 where it is +inf, -inf or NaN and 0 elsewhere.
template <typename T>
__device__ __forceinline__ uint32_t pick_special(uint32_t u, int kind) {
  constexpr int S = sizeof(T) == 2 ? 16 : 0;
  constexpr uint32_t kInf = 0x7F800000u >> S, kSign = 0x80000000u >> S, kOne = 0x3F800000u >> S;
  const uint32_t mag = u & ~kSign;
  if (kind == 0) return mag >= kInf ? 0u : u;
  const bool hit = kind == 3 ? mag > kInf : u == (kind == 1 ? kInf : (kInf | kSign));
  return hit ? kOne : 0u;
}

template <typename T, int DH>
__global__ void __launch_bounds__(64 * kPreWaves, sizeof(T) == 2 && DH <= 128 ? 2 : 1)
prefill_kernel(CacheView c, AttendArgs a, PreScratch sc, int row_blocks, int total) {
  using KTile = KeyTile<T, DH>;
  constexpr int CPR = KTile::CPR, KT = KTile::KT, KB = KT / 32, NB = DH / 32, PITCH = CPR * 16;
  constexpr int NS = sizeof(T) == 2 ? DH / 16 : DH / 8;    // reads of 16 bytes a lane needs of its K row
  constexpr int GROUPS = KT / 16;                          // runs of 16 slots, each on one page
  constexpr int LOADS = CPR / 4;                           // 1 KB loads of one run
  __shared__ __align__(16) unsigned char k0[KT * PITCH], v0[KT * PITCH], k1[KT * PITCH], v1[KT * PITCH];

  // blocks of one XCD (every eighth) work on neighbouring tiles of the same
  // heads, those with the most keys first
  int id = blockIdx.x;
  {
    const int per = total / 8, more = total % 8, x = id % 8;
    id = x * per + min(x, more) + id / 8;
  }
  const int split = id % sc.nsplit;
  id /= sc.nsplit;
  const int block = row_blocks - 1 - id % row_blocks, bh = id / row_blocks, h = bh % c.hkv, b = bh / c.hkv;
  const PreWork wk = pre_work(c, a, b, block, KT);
  if (wk.rows <= 0) return;
  const int ns = used_pre_splits(wk.tiles, sc.nsplit);
  if (split >= ns) return;
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
  // exp2(scale log2(e) s): a negative scale goes to the query's sign, and a
  // scale of zero to one that does not turn a hidden key's -inf into NaN
  const float cs = fmaxf(fabsf(a.scale) * 1.4426950408889634f, 1e-30f);

  uint4 q[NS];
  {
    const T* qp = static_cast<const T*>(a.q) + (wk.first + tok) * a.q_stride + static_cast<long long>(hq) * DH;
    const uint32_t flip = a.scale < 0.f ? (sizeof(T) == 2 ? 0x80008000u : 0x80000000u) : 0u;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      q[s] = ld16(reinterpret_cast<const char*>(qp) + 16 * (2 * s + half));
      q[s].x ^= flip; q[s].y ^= flip; q[s].z ^= flip; q[s].w ^= flip;
    }
  }
  floatx16 o[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[n][i] = 0.f;
  float m = -INFINITY, l = 0.f;
  const float slack = 8.f / cs;

  // loads of one run of 16 slots: piece u of 64 chunks, by position in shared
  // memory; the source chunk's byte offset in the run's rows
  int src_off[LOADS];
#pragma unroll
  for (int u = 0; u < LOADS; ++u) {
    const int p = 64 * u + lane, r = p / CPR;
    src_off[u] = r * PITCH + KTile::chunk_at(r, p % CPR) * 16;
  }
  int k_off[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) k_off[s] = col * PITCH + KTile::place(col, 2 * s + half) * 16;
  // bf16: two transposing reads of 4 keys x 16 dims; fp32: one value of a key
  constexpr int VO = sizeof(T) == 2 ? 2 : 4;
  int v_off[NB][VO];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int e = 0; e < VO; ++e) {
      if constexpr (sizeof(T) == 2) {
        const int i = lane & 15, r = 8 * e + 4 * half + (i >> 2);
        const int ch = 4 * n + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
        v_off[n][e] = r * PITCH + KTile::place(r, ch) * 16 + 8 * (i & 1);
      } else {
        const int r = 4 * half + e;      // of 8 keys; the next 8 lie 8 rows on
        v_off[n][e] = r * PITCH + KTile::place(r, 8 * n + (col >> 2)) * 16 + 4 * (col & 3);
      }
    }

  const int32_t* table = c.table + static_cast<long long>(b) * c.max_pages;
  const long long page_bytes = static_cast<long long>(c.page) * PITCH;
  // Starts the loads of a tile; returns which of its runs are on a page.  A wave
  // loads K and V of one run (64 keys a tile), or one of the two (32 keys).
  auto issue = [&](int it, shared_u8* ks, shared_u8* vs) -> unsigned {
    const int s0 = (it < wk.sink_tiles ? it : it + wk.skip) * KT;
    constexpr bool kBoth = GROUPS == kPreWaves;
    const int mine = kBoth ? w : w >> 1;
    unsigned ok = 0;
    int pid = -1;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int s = s0 + 16 * g;
      const int p = s < wk.len ? table[s >> c.shift] : -1;
      const bool on = p >= 0 && p < c.n_pages;
      ok |= on ? 1u << g : 0u;
      pid = g == mine ? (on ? p : -1) : pid;
    }
    const int s = s0 + 16 * mine, held = pid < 0 ? 0 : wk.len - s;   // rows of the run that are held
    const long long base =
        (static_cast<long long>(pid) * c.hkv + h) * page_bytes + static_cast<long long>(s & (c.page - 1)) * PITCH;
    auto copy = [&](const void* pages, shared_u8* to) {
      const char* from = static_cast<const char*>(pages) + base;
      to += 16 * mine * PITCH;
      if (held >= 16) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u)
          __builtin_amdgcn_global_load_lds((const global_u32*)(from + src_off[u]), to + 1024 * u, 16, 0, 0);
      } else {
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
          const char* at = (64 * u + lane) / CPR < held ? from + src_off[u] : reinterpret_cast<const char*>(kZeroRow);
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

  auto compute = [&](int it, unsigned ok, const shared_u8* ks, const shared_u8* vs) {
    const int s0 = (it < wk.sink_tiles ? it : it + wk.skip) * KT;
    // some query of the block does not see some key of the tile
    const bool block_edge = ok != (1u << GROUPS) - 1u || s0 + KT - 1 > wk.t_min || pos ||
                            (a.window && wk.t_max - s0 >= a.window);
    // then an infinity or NaN among the values must not reach that query
    bool careful = false;
    if (block_edge) {
      uint32_t bad = 0;
      for (int x = threadIdx.x; x < KT * CPR; x += 64 * kPreWaves) {
        const u32x4 y = ld_shared<u32x4>(vs + 16 * x);
        bad |= not_finite<T>(y.x) || not_finite<T>(y.y) || not_finite<T>(y.z) || not_finite<T>(y.w);
      }
      careful = __syncthreads_or(bad);
    }
    if (s0 > wt_max) return;
    const bool edge = ok != (1u << GROUPS) - 1u || s0 + KT - 1 > wt_min || pos || (a.window && wt_max - s0 >= a.window);

    floatx16 x[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[kb][i] = 0.f;
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const u32x4 kf = ld_shared<u32x4>(ks + k_off[s] + 32 * kb * PITCH);
        if constexpr (sizeof(T) == 2) {
          x[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf),
                                                          __builtin_bit_cast(bf16x8, q[s]), x[kb], 0, 0, 0);
        } else {
          const uint32_t qe[4] = {q[s].x, q[s].y, q[s].z, q[s].w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e]), __uint_as_float(qe[e]), x[kb], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) settle(x[kb]);
    if (edge) {
      const int win = a.window ? a.window : INT_MAX;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int sl = 32 * kb + 8 * j + 4 * half, s = s0 + sl;   // four slots
          const bool on = (ok >> (2 * kb + (j >> 1))) & 1u;
          int p[4] = {s, s + 1, s + 2, s + 3};
          if (pos) {
            const int4 y = on ? *reinterpret_cast<const int4*>(pos + s) : make_int4(0, 0, 0, 0);
            p[0] = y.x; p[1] = y.y; p[2] = y.z; p[3] = y.w;
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const bool see = on & (s + r <= t) & ((mine - p[r] < win) | (p[r] < a.sinks));
            x[kb][4 * j + r] = see ? x[kb][4 * j + r] : -INFINITY;
          }
        }
    }
    float mt = x[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mt = fmaxf(mt, x[kb][i]);
    mt = fmaxf(mt, xor_lane<32>(mt));
    // the running maximum follows in steps of at least 8 (base 2): weights stay
    // below 2^8 and most tiles rescale nothing
    if (__any(mt > m + slack)) {
      const float mn = fmaxf(m, mt);
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
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float y = x[kb][i];
        x[kb][i] = __builtin_amdgcn_exp2f(fmaf(y, cs, -base));
        sum += x[kb][i];
        // (a seen weight must not round to the zero of one that is not seen)
        if (careful && y != -INFINITY) x[kb][i] = fmaxf(x[kb][i], 0x1p-126f) + 0.f * x[kb][i];
      }
    l += sum;
    // kind 0: the product with the values (careful: those that are finite); 1 to
    // 3: which sums contain a seen +inf, -inf or NaN
    auto product = [&](auto clean, int kind, floatx16& acc, int n) {
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int st = 0; st < 2; ++st) {
            bf16x8 p;
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = static_cast<__bf16>(x[kb][8 * st + j]);
            typedef __attribute__((address_space(3))) shortx4 shared4;
            const shared_u8* vr = vs + (32 * kb + 16 * st) * PITCH;
            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared4*)(vr + v_off[n][0]));
            const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared4*)(vr + v_off[n][1]));
            auto both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            if constexpr (decltype(clean)::value) {
#pragma unroll
              for (int j = 0; j < 8; ++j) both[j] = static_cast<short>(pick_special<T>(static_cast<uint16_t>(both[j]), kind));
            }
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, both), p, acc, 0, 0, 0);
          }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          uint32_t v = ld_shared<uint32_t>(vs + 8 * (i >> 2) * PITCH + v_off[n][i & 3]);
          if constexpr (decltype(clean)::value) v = pick_special<T>(v, kind);
          acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(v), x[0][i], acc, 0, 0, 0);
        }
      }
    };
    if (careful) {
#pragma unroll
      for (int n = 0; n < NB; ++n) product(std::true_type{}, 0, o[n], n);
#pragma unroll 1
      for (int kind = 1; kind < 4; ++kind) {
        const float special = kind == 1 ? INFINITY : kind == 2 ? -INFINITY : NAN;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          floatx16 acc;
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[i] = 0.f;
          product(std::true_type{}, kind, acc, n);
          settle(acc);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[n][i] += acc[i] > 0.f ? special : 0.f;
        }
      }
      return;
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) product(std::false_type{}, 0, o[n], n);
  };
  // a tile is in shared memory for all waves once each has waited for its loads
  auto arrive = [&] {
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __syncthreads();
  };

  shared_u8* const kb0 = (shared_u8*)k0;
  shared_u8* const vb0 = (shared_u8*)v0;
  shared_u8* const kb1 = (shared_u8*)k1;
  shared_u8* const vb1 = (shared_u8*)v1;
  unsigned ok0 = 0, ok1 = 0;
  if (it0 < it1) ok0 = issue(it0, kb0, vb0);
  for (int it = it0; it < it1; it += 2) {
    arrive();
    if (it + 1 < it1) ok1 = issue(it + 1, kb1, vb1);
    compute(it, ok0, kb0, vb0);
    if (it + 1 >= it1) break;
    arrive();
    if (it + 2 < it1) ok0 = issue(it + 2, kb0, vb0);
    compute(it + 1, ok1, kb1, vb1);
  }

  asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");   // (see settle)
  __builtin_amdgcn_sched_barrier(0);
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

// Joins the splits: one wave per row and head.
template <typename T>
__global__ void __launch_bounds__(256)
prefill_join_kernel(CacheView c, AttendArgs a, PreScratch sc, int kt) {
  const int b = blockIdx.z, hq = blockIdx.y, i = blockIdx.x * 4 + wave_id(), lane = threadIdx.x & 63;
  long long first;
  int n;
  new_rows(a.starts, a.max_new, a.rows, b, &first, &n);
  if (i >= n) return;
  const PreWork wk = pre_work(c, a, b, (i * c.hg + hq % c.hg) / kPreRows, kt);
  const int ns = used_pre_splits(wk.tiles, sc.nsplit);
  const long long row = (first + i) * c.hq + hq, part_row = (static_cast<long long>(b) * a.max_new + i) * c.hq + hq;
  const float* ml = sc.ml + part_row * sc.nsplit * 2;
  float m = -INFINITY;
  for (int s = lane; s < ns; s += 64) m = fmaxf(m, ml[2 * s]);
  m = wave_max(m);
  const float base = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  for (int s = lane; s < ns; s += 64) l += ml[2 * s + 1] * __builtin_amdgcn_exp2f(ml[2 * s] - base);
  l = wave_sum(l);
  float o[4] = {0.f, 0.f, 0.f, 0.f};
  const float* part = sc.part + part_row * sc.nsplit * c.dh;
  for (int s = 0; s < ns; ++s) {
    const float f = __builtin_amdgcn_exp2f(ml[2 * s] - base);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (lane + 64 * e < c.dh) o[e] += f * part[static_cast<long long>(s) * c.dh + lane + 64 * e];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (lane + 64 * e < c.dh)
      static_cast<T*>(a.out)[row * c.dh + lane + 64 * e] = from_f32<T>(l == 0.f ? 0.f : o[e] / l);
  if (a.lse && lane == 0)
    a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

static int pre_key_tile(const CacheView& c) { return c.dtype != 0 && c.dh <= 128 ? 64 : 32; }

// Blocks of rows, and the splits of their keys: one while the rows alone fill
// the chip.
static int pre_row_blocks(const CacheView& c, int max_new) {
  return static_cast<int>((static_cast<long long>(max_new) * c.hg + kPreRows - 1) / kPreRows);
}
static int pre_splits(const CacheView& c, int max_new) {
  const long long blocks = static_cast<long long>(pre_row_blocks(c, max_new)) * c.hkv * c.n_seq;
  const long long most = std::max(1, c.cap / pre_key_tile(c) / 2);
  return static_cast<int>(std::max<long long>(1, std::min<long long>(most, 512 / blocks)));
}

long long prefill_scratch_bytes(const CacheView& c, int max_new) {
  const int ns = pre_splits(c, max_new);
  return ns == 1 ? 0 : 4ll * c.n_seq * max_new * c.hq * ns * (c.dh + 2);
}

hipError_t launch_cache_prefill(const CacheView& c, const AttendArgs& a, void* scratch, hipStream_t st) {
  const int row_blocks = pre_row_blocks(c, a.max_new), kt = pre_key_tile(c);
  PreScratch sc{};
  sc.nsplit = pre_splits(c, a.max_new);
  if (sc.nsplit > 1) {
    sc.part = static_cast<float*>(scratch);
    sc.ml = sc.part + static_cast<long long>(c.n_seq) * a.max_new * c.hq * sc.nsplit * c.dh;
  }
  const long long total = static_cast<long long>(row_blocks) * c.hkv * c.n_seq * sc.nsplit;
  if (total > (1ll << 31) - 1) return hipErrorInvalidValue;
#define GMC_PREFILL(T, DH)                                                                                    \
  case DH:                                                                                                    \
    hipLaunchKernelGGL((prefill_kernel<T, DH>), dim3(static_cast<unsigned>(total)), dim3(64 * kPreWaves), 0, st, c, a, sc, \
                       row_blocks, static_cast<int>(total));                                                  \
    break;
#define GMC_PREFILL_ALL(T)                                                                                    \
  switch (c.dh) {                                                                                             \
    GMC_PREFILL(T, 32) GMC_PREFILL(T, 64) GMC_PREFILL(T, 96) GMC_PREFILL(T, 128)                              \
    GMC_PREFILL(T, 160) GMC_PREFILL(T, 192) GMC_PREFILL(T, 224) GMC_PREFILL(T, 256)                           \
    default: return hipErrorInvalidValue;                                                                     \
  }
  if (c.dtype == 0) { GMC_PREFILL_ALL(float) } else { GMC_PREFILL_ALL(bf16_t) }
#undef GMC_PREFILL_ALL
#undef GMC_PREFILL
  if (sc.nsplit > 1) {
    const dim3 grid((a.max_new + 3) / 4, c.hq, c.n_seq);
    if (c.dtype == 0)
      hipLaunchKernelGGL(prefill_join_kernel<float>, grid, dim3(256), 0, st, c, a, sc, kt);
    else
      hipLaunchKernelGGL(prefill_join_kernel<bf16_t>, grid, dim3(256), 0, st, c, a, sc, kt);
  }
  return hipGetLastError();
}

}  // namespace gmc
