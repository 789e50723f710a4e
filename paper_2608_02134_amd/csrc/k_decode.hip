// Attention of one new token per sequence over the paged cache.
//
// The cache is read once and nothing else is large, so the kernel is bound by
// HBM: a block's waves each take tiles of 16 or 32 keys, loads of K and V go
// from the pages straight into the registers that the matrix instructions
// read, and no shared memory stands between.  With x = scale log2(e) q.k,
//   S^T = K Q^T:  A = K rows (lane: key l % 16, 8 dims of group l / 16),
//                 B = the group's query heads as columns (padded to 16);
//   the result has query l % 16 and keys 4 (l / 16) + 0..3 in each lane, which
//   is what B = P^T of the second product needs if its k slots are taken in
//   that order:
//   O^T = V^T P^T: A = V^T in the same slot order: lane (i = l % 16, g = l / 16)
//                 loads VEC consecutive dims VEC i.. of its group's keys 4 g +
//                 0..3, whole rows over 16 lanes, and turns them by byte
//                 permutations (bf16) or as they are (fp32).
// The running maximum and sum stay in fp32.  bf16 weights enter as a bf16 and
// the bf16 of what it leaves (16 bits together): the matrix cores idle, so
// the second product costs nothing and the weights lose nothing that the
// output's own rounding would not hide.
//
// The keys of a sequence are split over blocks; each writes its unnormalised
// sum with maximum and sum, and a second kernel joins them.  With weights to
// accumulate the logits go to scratch memory on the way (4 bytes per key and
// query head, beside 4 * dh per key and kv head of K and V), and the joining
// kernel adds exp2(x - lse) to each slot.
//
// 8 requests of 100000 to 131072 slots, 32 heads on 8 of 128 in bf16: 633 us, 6.0
// TB/s.  64 requests of 200 to 4096 slots, 28 heads on 4, weights accumulated: 58
// us (5.0 TB/s with the logits) and 9 for the joining kernel.
#include <algorithm>

#include "gmc_cache.h"
#include "gmc_device.h"

namespace gmc {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kDecodeWaves = 4, kDecodeShort = 8;   // waves of a block; where one block does a whole sequence

// Keys a wave takes at a time.
template <typename T> constexpr int kHalves = sizeof(T) == 2 ? 2 : 1;

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

template <int N> struct Raw;
template <> struct Raw<1> { uint32_t u[1]; };
template <> struct Raw<2> { uint32_t u[2]; };
template <> struct Raw<4> { uint32_t u[4]; };
template <int N> __device__ __forceinline__ Raw<N> load_raw(const void* p) {
  Raw<N> r;
  if constexpr (N == 4) {
    const uint4 v = *static_cast<const uint4*>(p);
    r.u[0] = v.x; r.u[1] = v.y; r.u[2] = v.z; r.u[3] = v.w;
  } else if constexpr (N == 2) {
    const uint2 v = *static_cast<const uint2*>(p);
    r.u[0] = v.x; r.u[1] = v.y;
  } else {
    r.u[0] = *static_cast<const uint32_t*>(p);
  }
  return r;
}

template <typename T, int DH, int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
decode_split_kernel(CacheView c, AttendArgs a, DecodeScratch sc, int qtiles) {
  constexpr int H = kHalves<T>, TK = 16 * H, NS = DH / 32;
  // dims a lane loads of a V row: up to 16 bytes, 16 lanes covering whole runs
  constexpr int VEC = sizeof(T) == 2 ? (DH % 128 == 0 ? 8 : DH % 64 == 0 ? 4 : 2) : (DH % 64 == 0 ? 4 : 2);
  constexpr int NB = DH / (16 * VEC), W = VEC * sizeof(T) / 4;
  __shared__ float red[WAVES / 2][16 * DH];
  __shared__ float stat[WAVES][2][16];
  const int split = blockIdx.x, h = blockIdx.y / qtiles, qt = blockIdx.y % qtiles, b = blockIdx.z;
  const int lane = threadIdx.x & 63, w = wave_id(), i16 = lane & 15, g = lane >> 4;
  const int len = cache_len(c, b);
  const TileRange tr = tile_range(len, a.window, a.sinks, c.slot_pos == nullptr, TK);
  const int ns = WAVES == kDecodeWaves ? used_splits(tr.count, sc.nsplit) : 1;
  if (split >= ns) return;
  const int t0 = static_cast<int>(static_cast<long long>(tr.count) * split / ns);
  const int t1 = static_cast<int>(static_cast<long long>(tr.count) * (split + 1) / ns);
  const int head = qt * 16 + i16;                 // of the group
  const bool live = head < c.hg;
  const int hq = h * c.hg + head;
  const long long at = (static_cast<long long>(b) * c.hkv + h) * c.cap;
  const int32_t* pos = c.slot_pos ? c.slot_pos + at : nullptr;
  const int mine = a.window && len > 0 ? (pos ? pos[len - 1] : len - 1) : 0;
  const float scale = a.scale * kLog2e;

  Frag<T> q[NS];
  {
    const T* qp = static_cast<const T*>(a.q) + b * a.q_stride + static_cast<long long>(hq) * DH + 8 * g;
#pragma unroll
    for (int s = 0; s < NS; ++s) q[s] = live ? frag_load<T>(qp + 32 * s) : frag_zero<T>();
  }
  floatx4 o[NB][VEC];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int j = 0; j < VEC; ++j) o[n][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  Frag<T> k[H][NS];
  Raw<W> v[H][4][NB];
  bool ok[H];             // the half tile is on a page
  int slot0 = 0;
  const long long page_elems = static_cast<long long>(c.page) * DH;
  const int32_t* table = c.table + static_cast<long long>(b) * c.max_pages;
  auto row0 = [&](int hh) -> long long {   // first element of a half tile's rows; 0 (read and dropped) where there is none
    const int s = slot0 + 16 * hh;
    ok[hh] = s < len;
    if (!ok[hh]) return 0;
    const int id = table[s >> c.shift];
    ok[hh] = id >= 0 && id < c.n_pages;
    return ok[hh] ? (static_cast<long long>(id) * c.hkv + h) * page_elems + static_cast<long long>(s & (c.page - 1)) * DH
                  : 0;
  };
  auto load = [&](int tile) {
    slot0 = (tile < tr.first ? tile : tile + tr.skip) * TK;
#pragma unroll
    for (int hh = 0; hh < H; ++hh) {
      const long long base = row0(hh);
      const T* kp = static_cast<const T*>(c.k) + base;
      const T* vp = static_cast<const T*>(c.v) + base;
#pragma unroll
      for (int s = 0; s < NS; ++s) k[hh][s] = frag_load<T>(kp + i16 * DH + 32 * s + 8 * g);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int n = 0; n < NB; ++n) v[hh][r][n] = load_raw<W>(vp + (4 * g + r) * DH + VEC * (16 * n + i16));
    }
  };

  int tile = t0 + w;
  if (tile < t1) load(tile);
  for (; tile < t1; tile += WAVES) {
    // keys that are not seen: only in the last tile, at the window's edges and
    // on pages that are none
    bool whole = slot0 + TK <= len && (!a.window || (!pos && len - 1 - slot0 < a.window));
#pragma unroll
    for (int hh = 0; hh < H; ++hh) whole = whole && ok[hh];
    floatx4 x[H];
#pragma unroll
    for (int hh = 0; hh < H; ++hh) {
      x[hh] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; ++s) x[hh] = mma(k[hh][s], q[s], x[hh]);
    }
#pragma unroll
    for (int hh = 0; hh < H; ++hh) settle(x[hh]);
#pragma unroll
    for (int hh = 0; hh < H; ++hh)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[hh][r] *= scale;
    if (!whole) {
#pragma unroll
      for (int hh = 0; hh < H; ++hh)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int s = slot0 + 16 * hh + 4 * g + r;
          bool see = ok[hh] && s < len;
          if (see && a.window) {
            const int p = pos ? pos[s] : s;
            see = mine - p < a.window || p < a.sinks;
          }
          if (!see) {
            x[hh][r] = -INFINITY;
            // a weight of zero does not silence an infinity or NaN
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
              for (int e = 0; e < W; ++e) v[hh][r][n].u[e] = 0u;
          }
        }
    }
    if (sc.logits && live) {
      float* to = sc.logits + (static_cast<long long>(b) * c.hq + hq) * c.cap + slot0 + 4 * g;
#pragma unroll
      for (int hh = 0; hh < H; ++hh)
        if (slot0 + 16 * hh < len) *reinterpret_cast<floatx4*>(to + 16 * hh) = x[hh];
    }
    float mt = x[0][0];
#pragma unroll
    for (int hh = 0; hh < H; ++hh)
#pragma unroll
      for (int r = 0; r < 4; ++r) mt = fmaxf(mt, x[hh][r]);
    mt = fmaxf(mt, xor_lane<16>(mt));
    mt = fmaxf(mt, xor_lane<32>(mt));
    const float mn = fmaxf(m, mt), base = mn == -INFINITY ? 0.f : mn;
    const float f = __builtin_amdgcn_exp2f(m - base);
    m = mn;
    float sum = 0.f;
#pragma unroll
    for (int hh = 0; hh < H; ++hh)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[hh][r] = __builtin_amdgcn_exp2f(x[hh][r] - base);
        sum += x[hh][r];
      }
    l = l * f + sum;   // this lane group's keys; joined at the end
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int j = 0; j < VEC; ++j) o[n][j] *= f;
    if constexpr (sizeof(T) == 2) {
      bf16x8 hi, lo;
#pragma unroll
      for (int hh = 0; hh < H; ++hh)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          // hi: the upper half of the fp32 (towards zero), so that lo is never
          // negative nor, for a weight above zero, zero: an infinite value
          // stays what it is
          const uint32_t u = __float_as_uint(x[hh][r]) & 0xFFFF0000u;
          hi[4 * hh + r] = __builtin_bit_cast(__bf16, static_cast<uint16_t>(u >> 16));
          lo[4 * hh + r] = static_cast<__bf16>(fmaxf(x[hh][r] - __uint_as_float(u), x[hh][r] * 0x1p-24f));
        }
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          // dim j of the lane's 8 keys
          uint32_t u[4];
          const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
#pragma unroll
          for (int hh = 0; hh < H; ++hh) {
            u[2 * hh] = __builtin_amdgcn_perm(v[hh][1][n].u[j / 2], v[hh][0][n].u[j / 2], sel);
            u[2 * hh + 1] = __builtin_amdgcn_perm(v[hh][3][n].u[j / 2], v[hh][2][n].u[j / 2], sel);
          }
          const bf16x8 av = __builtin_bit_cast(bf16x8, make_uint4(u[0], u[1], u[2], u[3]));
          o[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, hi, o[n][j], 0, 0, 0);
          o[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, lo, o[n][j], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            o[n][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[0][r][n].u[j]), x[0][r], o[n][j], 0, 0, 0);
    }
    if (tile + WAVES < t1) load(tile + WAVES);
  }

  // the waves' parts on their common maximum, added in a fixed order
  l = add_xor32(add_xor16(l));
  if (g == 0) { stat[w][0][i16] = m; stat[w][1][i16] = l; }
  __syncthreads();
  float mb = stat[0][0][i16];
#pragma unroll
  for (int u = 1; u < WAVES; ++u) mb = fmaxf(mb, stat[u][0][i16]);
  const float base = mb == -INFINITY ? 0.f : mb;
  float lb = 0.f;
#pragma unroll
  for (int u = 0; u < WAVES; ++u) lb += stat[u][1][i16] * __builtin_amdgcn_exp2f(stat[u][0][i16] - base);
  const float f = __builtin_amdgcn_exp2f(m - base);
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int j = 0; j < VEC; ++j) o[n][j] *= f;
#pragma unroll
  for (int step = WAVES / 2; step >= 1; step /= 2) {
    if (w >= step && w < 2 * step) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          *reinterpret_cast<floatx4*>(&red[w - step][((n * VEC + j) * 64 + lane) * 4]) = o[n][j];
    }
    __syncthreads();
    if (w < step) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          o[n][j] += *reinterpret_cast<const floatx4*>(&red[w][((n * VEC + j) * 64 + lane) * 4]);
    }
    __syncthreads();
  }
  if (w != 0 || !live) return;
  const long long row = static_cast<long long>(b) * c.hq + hq;
  if (sc.part) {
    float* to = sc.part + (row * sc.nsplit + split) * DH;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < VEC; ++j) to[VEC * (16 * n + 4 * g + r) + j] = o[n][j][r];
    if (g == 0) {
      sc.ml[(row * sc.nsplit + split) * 2] = mb;
      sc.ml[(row * sc.nsplit + split) * 2 + 1] = lb;
    }
    return;
  }
  const float inv = lb == 0.f ? 0.f : 1.f / lb;
  T* to = static_cast<T*>(a.out) + row * DH;
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        to[VEC * (16 * n + 4 * g + r) + j] = from_f32<T>(lb == 0.f ? 0.f : o[n][j][r] * inv);
  if (a.lse && g == 0) a.lse[row] = lb == 0.f ? -INFINITY : (mb + __builtin_amdgcn_logf(lb)) * kLn2;
}

// Joins a sequence's splits.  blockIdx.x < hg: output and lse of one query
// head of the kv head, its splits shared by the block's waves; above: the
// weights of one run of 1024 slots, for which each wave first takes the lse of
// some heads.
template <typename T>
__global__ void __launch_bounds__(256)
decode_join_kernel(CacheView c, AttendArgs a, DecodeScratch sc, int tk) {
  __shared__ __align__(16) float red[4][256];
  __shared__ float lse2[kCacheMaxHeads];
  const int h = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63, w = wave_id();
  const int len = cache_len(c, b);
  const TileRange tr = tile_range(len, a.window, a.sinks, c.slot_pos == nullptr, tk);
  const int ns = used_splits(tr.count, sc.nsplit);
  if (static_cast<int>(blockIdx.x) < c.hg) {
    const long long row = static_cast<long long>(b) * c.hq + h * c.hg + blockIdx.x;
    const float* ml = sc.ml + row * sc.nsplit * 2;
    const float* part = sc.part + row * sc.nsplit * c.dh + 4 * lane;
    const bool mine = 4 * lane < c.dh;
    constexpr int kFlight = 4;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    float m, l;
    // (the first parts are on their way while the statistics are taken)
    floatx4 x[kFlight];
    auto load = [&](int s0) {
#pragma unroll
      for (int e = 0; e < kFlight; ++e) {
        const int s = min(s0 + 4 * e, ns - 1);
        x[e] = mine ? *reinterpret_cast<const floatx4*>(part + static_cast<long long>(s) * c.dh) : floatx4{0.f, 0.f, 0.f, 0.f};
      }
    };
    load(w);
    join_stats(ml, ns, &m, &l);
    const float base = m == -INFINITY ? 0.f : m;
    for (int s0 = w; s0 < ns; s0 += 4 * kFlight) {
      if (s0 > w) load(s0);
#pragma unroll
      for (int e = 0; e < kFlight; ++e) {
        const int s = s0 + 4 * e;
        if (s >= ns) break;
        const float f = __builtin_amdgcn_exp2f(ml[2 * s] - base);
#pragma unroll
        for (int u = 0; u < 4; ++u) o[u] += f * x[e][u];
      }
    }
    *reinterpret_cast<floatx4*>(&red[w][4 * lane]) = o;
    __syncthreads();
    const int d = threadIdx.x;
    if (d < c.dh) {
      const float sum = red[0][d] + red[1][d] + red[2][d] + red[3][d];
      static_cast<T*>(a.out)[row * c.dh + d] = from_f32<T>(l == 0.f ? 0.f : sum / l);
    }
    if (a.lse && d == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    return;
  }
  const int s0 = (static_cast<int>(blockIdx.x) - c.hg) * 1024;
  if (s0 >= len) return;
  const int s = s0 + 4 * threadIdx.x;
  // tiles that no query looks at have no logits
  const int tile = s / tk;
  const bool mine = s < len && !(tile >= tr.first && tile < tr.first + tr.skip);
  const float* logits = sc.logits + (static_cast<long long>(b) * c.hq + h * c.hg) * c.cap + (mine ? s : 0);
  constexpr int kFlight = 8;
  floatx4 x[kFlight], add = {0.f, 0.f, 0.f, 0.f};
  auto load = [&](int head) {
#pragma unroll
    for (int e = 0; e < kFlight; ++e)
      x[e] = *reinterpret_cast<const floatx4*>(logits + static_cast<long long>(min(head + e, c.hg - 1)) * c.cap);
  };
  if (mine) load(0);
  for (int head = w; head < c.hg; head += 4) {
    float m, l;
    join_stats(sc.ml + (static_cast<long long>(b) * c.hq + h * c.hg + head) * sc.nsplit * 2, ns, &m, &l);
    // nothing seen: every logit is -inf, and any finite value gives 0
    if (lane == 0) lse2[head] = l == 0.f ? 0.f : m + __builtin_amdgcn_logf(l);
  }
  __syncthreads();
  if (!mine) return;
  for (int head = 0; head < c.hg; head += kFlight) {
    if (head > 0) load(head);
#pragma unroll
    for (int e = 0; e < kFlight; ++e) {
      if (head + e >= c.hg) break;
#pragma unroll
      for (int u = 0; u < 4; ++u) {   // (a slot that is not seen gains nothing, also where the lse is NaN)
        const float p = __builtin_amdgcn_exp2f(x[e][u] - lse2[head + e]);
        add[u] += x[e][u] == -INFINITY ? 0.f : p;
      }
    }
  }
  float* to = c.weights + (static_cast<long long>(b) * c.hkv + h) * c.cap + s;
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (s + u < len) to[u] += add[u];
}

// Splits of a call: enough blocks for the chip (64 requests of 4096 slots:
// 51.6 us with 1024 blocks, 57 with 2048, 70 with 4096).
static int decode_splits(const CacheView& c, int qtiles) {
  const int tk = c.dtype == 0 ? 16 : 32;
  const long long groups = static_cast<long long>(c.n_seq) * c.hkv * qtiles;
  return used_splits((c.cap + tk - 1) / tk, static_cast<int>((1024 + groups - 1) / groups));
}

static int decode_qtiles(const CacheView& c) { return (c.hg + 15) / 16; }

// Caches of at most two tiles for each of eight waves: one block a head and no
// second kernel (four tiles or fewer: four waves are that already).  GPU time, bf16,
// heads of 128, in us, with it and split: 28 heads on 4, 1 or 16 requests of 256
// slots 7.0 and 8.1, of 512 slots 9.6 and 8.2 to 9.2, where the launch saved makes
// up for it; 64 requests of 32 heads on 8, 512 slots 26 and 29, 768 slots 35 and 38;
// 100 slots 10.3 and 7.7.
static bool decode_short(const CacheView& c, bool accumulate) {
  const int tiles = (c.cap + (c.dtype == 0 ? 15 : 31)) / (c.dtype == 0 ? 16 : 32);
  return !accumulate && c.dh <= 128 && tiles > kDecodeWaves && tiles <= 2 * kDecodeShort;
}

long long decode_scratch_bytes(const CacheView& c, bool accumulate) {
  const int ns = decode_short(c, accumulate) ? 1 : decode_splits(c, decode_qtiles(c));
  if (ns == 1 && !accumulate) return 0;
  const long long rows = static_cast<long long>(c.n_seq) * c.hq;
  return 4 * rows * ns * (c.dh + 2) + (accumulate ? 4 * rows * c.cap : 0);
}

template <typename T>
static hipError_t start_decode(const CacheView& c, const AttendArgs& a, const DecodeScratch& sc, int qt, bool one_block,
                               hipStream_t st) {
  const dim3 grid(sc.nsplit, c.hkv * qt, c.n_seq);
#define GMC_DECODE(DH, WAVES)                                                                                        \
  case DH:                                                                                                           \
    hipLaunchKernelGGL((decode_split_kernel<T, DH, WAVES>), grid, dim3(64 * WAVES), 0, st, c, a, sc, qt);            \
    return hipGetLastError();
#define GMC_DECODE_NARROW(WAVES) GMC_DECODE(32, WAVES) GMC_DECODE(64, WAVES) GMC_DECODE(96, WAVES) GMC_DECODE(128, WAVES)
  if (one_block) {
    switch (c.dh) { GMC_DECODE_NARROW(kDecodeShort) default: return hipErrorInvalidValue; }
  }
  switch (c.dh) {
    GMC_DECODE_NARROW(kDecodeWaves)
    GMC_DECODE(160, kDecodeWaves) GMC_DECODE(192, kDecodeWaves) GMC_DECODE(224, kDecodeWaves) GMC_DECODE(256, kDecodeWaves)
    default: return hipErrorInvalidValue;
  }
#undef GMC_DECODE_NARROW
#undef GMC_DECODE
}

hipError_t launch_cache_decode(const CacheView& c, const AttendArgs& a, bool accumulate, void* scratch,
                               hipStream_t st) {
  const int qt = decode_qtiles(c), tk = c.dtype == 0 ? 16 : 32;
  const bool one_block = decode_short(c, accumulate);
  DecodeScratch sc{};
  sc.nsplit = one_block ? 1 : decode_splits(c, qt);
  const bool join = sc.nsplit > 1 || accumulate;
  if (join) {
    const long long rows = static_cast<long long>(c.n_seq) * c.hq;
    sc.logits = accumulate ? static_cast<float*>(scratch) : nullptr;   // first: rows of 16-byte pieces
    sc.part = static_cast<float*>(scratch) + (accumulate ? rows * c.cap : 0);
    sc.ml = sc.part + rows * sc.nsplit * c.dh;
  }
  const hipError_t err =
      c.dtype == 0 ? start_decode<float>(c, a, sc, qt, one_block, st) : start_decode<bf16_t>(c, a, sc, qt, one_block, st);
  if (err != hipSuccess || !join) return err;
  const dim3 jgrid(c.hg + (accumulate ? (c.cap + 1023) / 1024 : 0), c.hkv, c.n_seq);
  if (c.dtype == 0)
    hipLaunchKernelGGL(decode_join_kernel<float>, jgrid, dim3(256), 0, st, c, a, sc, tk);
  else
    hipLaunchKernelGGL(decode_join_kernel<bf16_t>, jgrid, dim3(256), 0, st, c, a, sc, tk);
  return hipGetLastError();
}

}  // namespace gmc
