// Attention of one new token per sequence over a paged cache of 4 bits.
//
// As over pages of bf16 (S^T = K Q^T, O^T = V^T P^T, keys split over blocks and
// joined by a second kernel), with codes and scales loaded from the pages and
// turned into bf16 operands by single instructions, exactly.  136 bytes a row of
// 128 elements for K and V instead of 512: bound by memory where the caches are long,
// and the instructions beside it have to stay few:
//   K: the order of the elements in a product is free, so lane (key l % 16, group g =
//      l / 16) takes a run of them: of each 128 the 32 from 32 g, one 16-byte load and
//      one scale; of what is left 16 from 16 g (64) and 8 from 8 g (32).
//   V: lane (i = l % 16, g) takes of each of its group's keys 4 g + 0..3 the 8
//      elements from 8 i of each 128 (4 of 64, 2 of 32), whole rows over 16 lanes,
//      and turns pairs of two keys into operands by byte permutations.
// Every value is a bf16, so fp32 queries and weights enter as three bf16 (24
// bits: exact but for the last, which is rounded) and the products are those of
// fp32; weights for bf16 outputs as two (16 bits).  The matrix cores idle, so this
// costs nothing.
#include <algorithm>

#include "gmc_cache.h"
#include "gmc_decode.h"
#include "gmc_device.h"
#include "gmc_fp4.h"

namespace gmc {

constexpr int kTile4 = 32;   // keys a wave takes at a time, in two halves

// A head as runs of 128 elements, then of 64 and 32.
template <int DH> struct Runs {
  static constexpr int n128 = DH / 128, n64 = DH % 128 / 64, n32 = DH % 64 / 32, count = n128 + n64 + n32;
  static constexpr int size(int n) { return n < n128 ? 128 : n < n128 + n64 ? 64 : 32; }
  static constexpr int base(int n) { return n <= n128 ? 128 * n : 128 * n128 + 64; }
};

template <int N> __device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* u) {
  static_assert(N == 1 || N == 2 || N == 4 || N == 8, "runs of 4 to 32 bytes");
  if constexpr (N == 1) {
    u[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    u[0] = v.x; u[1] = v.y;
  } else {
#pragma unroll
    for (int e = 0; e < N / 4; ++e) {
      const uint4 v = reinterpret_cast<const uint4*>(p)[e];
      u[4 * e] = v.x; u[4 * e + 1] = v.y; u[4 * e + 2] = v.z; u[4 * e + 3] = v.w;
    }
  }
}

// x as bf16 parts: the upper 8 significant bits, the next 8, and the rest rounded.
// Infinities and NaN are all in the first part.
__device__ __forceinline__ void split3(float x, __bf16* hi, __bf16* mid, __bf16* lo) {
  const uint32_t u = __float_as_uint(x);
  const bool finite = (u & 0x7F800000u) != 0x7F800000u;
  const float h = __uint_as_float(u & 0xFFFF0000u), rest = finite ? x - h : 0.f;
  const float m = __uint_as_float(__float_as_uint(rest) & 0xFFFF0000u);
  *hi = finite ? __builtin_bit_cast(__bf16, static_cast<uint16_t>(u >> 16)) : static_cast<__bf16>(x);
  *mid = __builtin_bit_cast(__bf16, static_cast<uint16_t>(__float_as_uint(m) >> 16));
  *lo = static_cast<__bf16>(rest - m);
}

template <typename T, int DH, int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
decode4_kernel(CacheView c, CacheScales sc4, AttendArgs a, DecodeScratch sc, int qtiles) {
  using R = Runs<DH>;
  constexpr int H = 2, TK = kTile4, NS = DH / 32, NO = DH / 16, ROW = DH / 2;
  constexpr int SB = scale_bytes(DH), SW = SB == 8 ? 2 : 1;
  constexpr int NQ = sizeof(T) == 2 ? 1 : 3, NP = sizeof(T) == 2 ? 2 : 3;   // bf16 parts of queries and weights
  __shared__ float red[WAVES / 2][16 * DH];
  __shared__ float stat[WAVES][2][16];
  const int split = blockIdx.x, h = blockIdx.y / qtiles, qt = blockIdx.y % qtiles, b = blockIdx.z;
  const int lane = threadIdx.x & 63, w = wave_id(), i16 = lane & 15, g = lane >> 4;
  const int len = cache_len(c, b);
  const TileRange tr = tile_range(len, a.window, a.sinks, true, TK);
  const int ns = WAVES == kDecodeWaves ? used_splits(tr.count, sc.nsplit) : 1;
  if (split >= ns) return;
  const int t0 = static_cast<int>(static_cast<long long>(tr.count) * split / ns);
  const int t1 = static_cast<int>(static_cast<long long>(tr.count) * (split + 1) / ns);
  const int head = qt * 16 + i16;                 // of the group
  const bool live = head < c.hg;
  const int hq = h * c.hg + head;
  const float scale = a.scale * kLog2e;

  struct Tile {
    uint32_t k[H][NS], v[H][4][R::count], sk[H][SW], sv[H][SB];
    bool ok[H];             // the half tile is on a page
    int slot0;
  };
  const int32_t* table = c.table + static_cast<long long>(b) * c.max_pages;
  auto load = [&](int tile, Tile& x) __attribute__((always_inline)) {
    x.slot0 = (tile < tr.first ? tile : tile + tr.skip) * TK;
#pragma unroll
    for (int hh = 0; hh < H; ++hh) {
      const int s = x.slot0 + 16 * hh;
      long long row = 0;    // read and dropped where there is none
      x.ok[hh] = s < len;
      if (x.ok[hh]) {
        const int id = table[s >> c.shift];
        x.ok[hh] = id >= 0 && id < c.n_pages;
        if (x.ok[hh]) row = ((static_cast<long long>(id) * c.hkv + h) << c.shift) + (s & (c.page - 1));
      }
      const uint8_t* kp = static_cast<const uint8_t*>(c.k) + row * ROW + i16 * ROW;
      const uint8_t* vp = static_cast<const uint8_t*>(c.v) + row * ROW + 4 * g * ROW;
#pragma unroll
      for (int n = 0; n < R::count; ++n) {
        constexpr int kWord = 32;   // elements of a group for each 128
        const int at = R::base(n) / 2, size = R::size(n);
        if (size == 128) load_words<4>(kp + at + 16 * g, &x.k[hh][R::base(n) / kWord]);
        if (size == 64) load_words<2>(kp + at + 8 * g, &x.k[hh][R::base(n) / kWord]);
        if (size == 32) load_words<1>(kp + at + 4 * g, &x.k[hh][R::base(n) / kWord]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint8_t* p = vp + r * ROW + at;
          x.v[hh][r][n] = size == 128  ? *reinterpret_cast<const uint32_t*>(p + 4 * i16)
                          : size == 64 ? *reinterpret_cast<const uint16_t*>(p + 2 * i16)
                                       : p[i16];
        }
      }
      const uint8_t* ks = sc4.k + row * SB + i16 * SB;
      if constexpr (SB == 1) x.sk[hh][0] = *ks;
      else if constexpr (SB == 2) x.sk[hh][0] = *reinterpret_cast<const uint16_t*>(ks);
      else load_words<SB / 4>(ks, x.sk[hh]);
      load_words<SB>(sc4.v + row * SB + 4 * g * SB, x.sv[hh]);
    }
  };

  bf16x8 q[NQ][NS];
  {
    const T* qp = static_cast<const T*>(a.q) + b * a.q_stride + static_cast<long long>(hq) * DH;
#pragma unroll
    for (int n = 0; n < R::count; ++n)
#pragma unroll
      for (int u = 0; u < R::size(n) / 32; ++u) {
        const int s = R::base(n) / 32 + u;
        const T* p = qp + R::base(n) + R::size(n) / 4 * g + 8 * u;
        if constexpr (sizeof(T) == 2) {
          q[0][s] = live ? __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(p)) : bf16x8{};
        } else {
          const Frag<float> f = live ? frag_load<float>(p) : frag_zero<float>();
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            __bf16 x0, x1, x2;
            split3(f.v[e], &x0, &x1, &x2);
            q[0][s][e] = x0; q[1][s][e] = x1; q[2][s][e] = x2;
          }
        }
      }
  }
  floatx4 o[NO];
#pragma unroll
  for (int n = 0; n < NO; ++n) o[n] = floatx4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  auto compute = [&](Tile& y) __attribute__((always_inline)) {
    // keys that are not seen: only in the last tile, at the window's edges and
    // on pages that are none
    const bool whole = y.slot0 + TK <= len && (!a.window || len - 1 - y.slot0 < a.window) && y.ok[0] && y.ok[1];
    floatx4 x[H];
#pragma unroll
    for (int hh = 0; hh < H; ++hh) {
      x[hh] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int n = 0; n < R::count; ++n)
#pragma unroll
        for (int u = 0; u < R::size(n) / 32; ++u) {
          const int s = R::base(n) / 32 + u;
          // block of the run's elements: of 128 one a group, of 64 one for two
          const int blk = R::base(n) / 32, sh = R::size(n) == 128 ? 8 * g : R::size(n) == 64 ? 8 * (g >> 1) : 0;
          const float f = scale_of((y.sk[hh][blk / 4] >> (8 * (blk % 4) + sh)) & 255u);
          const bf16x8 kf = __builtin_bit_cast(bf16x8, fp4_words(y.k[hh][s], f));
#pragma unroll
          for (int p = NQ - 1; p >= 0; --p) x[hh] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[p][s], x[hh], 0, 0, 0);
        }
    }
#pragma unroll
    for (int hh = 0; hh < H; ++hh) settle(x[hh]);
#pragma unroll
    for (int hh = 0; hh < H; ++hh)
#pragma unroll
      for (int r = 0; r < 4; ++r) x[hh][r] *= scale;
    uint32_t gone = 0;   // keys of this lane's eight that the query does not see
    if (!whole) {
#pragma unroll
      for (int hh = 0; hh < H; ++hh)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int s = y.slot0 + 16 * hh + 4 * g + r;
          const bool see = y.ok[hh] && s < len && (!a.window || len - 1 - s < a.window || s < a.sinks);
          if (!see) {
            x[hh][r] = -INFINITY;
            gone |= 1u << (4 * hh + r);
          }
        }
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
    bf16x8 p[NP];
#pragma unroll
    for (int hh = 0; hh < H; ++hh)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float e = __builtin_amdgcn_exp2f(x[hh][r] - base);
        sum += e;
        const int at = 4 * hh + r;
        if constexpr (NP == 2) {
          const uint32_t u = __float_as_uint(e) & 0xFFFF0000u;
          p[0][at] = __builtin_bit_cast(__bf16, static_cast<uint16_t>(u >> 16));
          // (no part of a weight above zero is zero: an infinite value, which
          // scales from 2^126 on have, stays what it is)
          p[1][at] = static_cast<__bf16>(fmaxf(e - __uint_as_float(u), e * 0x1p-24f));
        } else {
          const uint32_t u = __float_as_uint(e) & 0xFFFF0000u;
          const float rest = e - __uint_as_float(u);
          const uint32_t v = __float_as_uint(fmaxf(rest, e * 0x1p-25f)) & 0xFFFF0000u;
          p[0][at] = __builtin_bit_cast(__bf16, static_cast<uint16_t>(u >> 16));
          p[1][at] = __builtin_bit_cast(__bf16, static_cast<uint16_t>(v >> 16));
          p[2][at] = static_cast<__bf16>(fmaxf(rest - __uint_as_float(v), e * 0x1p-33f));
        }
      }
    l = l * f + sum;   // this lane group's keys; joined at the end
#pragma unroll
    for (int n = 0; n < NO; ++n) o[n] *= f;
#pragma unroll
    for (int n = 0; n < R::count; ++n) {
      const int pairs = R::size(n) / 32, blk = R::base(n) / 32;   // pairs of elements a lane has of each key
      uint32_t v[H][4][4];
#pragma unroll
      for (int hh = 0; hh < H; ++hh)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int sh = R::size(n) == 128 ? 8 * (i16 >> 2) : R::size(n) == 64 ? 8 * (i16 >> 3) : 0;
          const int at = r * SB + blk;
          uint32_t e = (y.sv[hh][at / 4] >> (8 * (at % 4) + sh)) & 255u, codes = y.v[hh][r][n];
          if (!whole && (gone >> (4 * hh + r)) & 1u) {   // a weight of zero does not silence a NaN
            e = 0u;
            codes = 0u;
          }
          const float fs = scale_of(e);
          v[hh][r][0] = fp4_pair<0>(codes, fs);
          if (pairs > 1) v[hh][r][1] = fp4_pair<1>(codes, fs);
          if (pairs > 2) { v[hh][r][2] = fp4_pair<2>(codes, fs); v[hh][r][3] = fp4_pair<3>(codes, fs); }
        }
#pragma unroll
      for (int j = 0; j < 2 * pairs; ++j) {
        // element j of the lane's 8 keys
        uint32_t u[4];
        const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
#pragma unroll
        for (int hh = 0; hh < H; ++hh) {
          u[2 * hh] = __builtin_amdgcn_perm(v[hh][1][j / 2], v[hh][0][j / 2], sel);
          u[2 * hh + 1] = __builtin_amdgcn_perm(v[hh][3][j / 2], v[hh][2][j / 2], sel);
        }
        const bf16x8 av = __builtin_bit_cast(bf16x8, make_uint4(u[0], u[1], u[2], u[3]));
        floatx4& to = o[R::base(n) / 16 + j];
#pragma unroll
        for (int e = NP - 1; e >= 0; --e) to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, p[e], to, 0, 0, 0);
      }
    }
  };

  Tile even, odd;
  int tile = t0 + w;
  if (tile < t1) load(tile, even);
  for (; tile < t1; tile += 2 * WAVES) {
    if (tile + WAVES < t1) load(tile + WAVES, odd);
    compute(even);
    if (tile + WAVES >= t1) break;
    if (tile + 2 * WAVES < t1) load(tile + 2 * WAVES, even);
    compute(odd);
  }
  asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");   // (see settle)
  __builtin_amdgcn_sched_barrier(0);

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
  for (int n = 0; n < NO; ++n) o[n] *= f;
#pragma unroll
  for (int step = WAVES / 2; step >= 1; step /= 2) {
    if (w >= step && w < 2 * step) {
#pragma unroll
      for (int n = 0; n < NO; ++n) *reinterpret_cast<floatx4*>(&red[w - step][(n * 64 + lane) * 4]) = o[n];
    }
    __syncthreads();
    if (w < step) {
#pragma unroll
      for (int n = 0; n < NO; ++n) o[n] += *reinterpret_cast<const floatx4*>(&red[w][(n * 64 + lane) * 4]);
    }
    __syncthreads();
  }
  if (w != 0 || !live) return;
  // accumulator j of a run of SIZE: element SIZE / 16 * (4 g + r) + j of it
  const long long row = static_cast<long long>(b) * c.hq + hq;
  if (sc.part) {
    float* to = sc.part + (row * sc.nsplit + split) * DH;
#pragma unroll
    for (int n = 0; n < R::count; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < R::size(n) / 16; ++j)
          to[R::base(n) + R::size(n) / 16 * (4 * g + r) + j] = o[R::base(n) / 16 + j][r];
    if (g == 0) {
      sc.ml[(row * sc.nsplit + split) * 2] = mb;
      sc.ml[(row * sc.nsplit + split) * 2 + 1] = lb;
    }
    return;
  }
  const float inv = lb == 0.f ? 0.f : 1.f / lb;
  T* to = static_cast<T*>(a.out) + row * DH;
#pragma unroll
  for (int n = 0; n < R::count; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < R::size(n) / 16; ++j)
        to[R::base(n) + R::size(n) / 16 * (4 * g + r) + j] =
            from_f32<T>(lb == 0.f ? 0.f : o[R::base(n) / 16 + j][r] * inv);
  if (a.lse && g == 0) a.lse[row] = lb == 0.f ? -INFINITY : (mb + __builtin_amdgcn_logf(lb)) * kLn2;
}

static int decode4_qtiles(const CacheView& c) { return (c.hg + 15) / 16; }

static int decode4_splits(const CacheView& c, int qtiles) {
  const long long groups = static_cast<long long>(c.n_seq) * c.hkv * qtiles;
  return used_splits((c.cap + kTile4 - 1) / kTile4, static_cast<int>((1024 + groups - 1) / groups));
}

// One block a head and no second kernel, as over pages of bf16.
static bool decode4_short(const CacheView& c) {
  const int tiles = (c.cap + kTile4 - 1) / kTile4;
  return c.dh <= 128 && tiles > kDecodeWaves && tiles <= 2 * kDecodeShort;
}

long long decode4_scratch_bytes(const CacheView& c) {
  const int ns = decode4_short(c) ? 1 : decode4_splits(c, decode4_qtiles(c));
  return ns == 1 ? 0 : 4ll * c.n_seq * c.hq * ns * (c.dh + 2);
}

template <typename T>
static hipError_t start_decode4(const CacheView& c, const CacheScales& s, const AttendArgs& a, const DecodeScratch& sc,
                                int qt, bool one_block, hipStream_t st) {
  const dim3 grid(sc.nsplit, c.hkv * qt, c.n_seq);
#define GMC_DECODE4(DH, WAVES)                                                                                   \
  case DH:                                                                                                       \
    hipLaunchKernelGGL((decode4_kernel<T, DH, WAVES>), grid, dim3(64 * WAVES), 0, st, c, s, a, sc, qt);          \
    return hipGetLastError();
#define GMC_DECODE4_NARROW(WAVES) \
  GMC_DECODE4(32, WAVES) GMC_DECODE4(64, WAVES) GMC_DECODE4(96, WAVES) GMC_DECODE4(128, WAVES)
  if (one_block) {
    switch (c.dh) { GMC_DECODE4_NARROW(kDecodeShort) default: return hipErrorInvalidValue; }
  }
  switch (c.dh) {
    GMC_DECODE4_NARROW(kDecodeWaves)
    GMC_DECODE4(160, kDecodeWaves) GMC_DECODE4(192, kDecodeWaves) GMC_DECODE4(224, kDecodeWaves)
    GMC_DECODE4(256, kDecodeWaves)
    default: return hipErrorInvalidValue;
  }
#undef GMC_DECODE4_NARROW
#undef GMC_DECODE4
}

hipError_t launch_cache4_decode(const CacheView& c, const CacheScales& s, const AttendArgs& a, void* scratch,
                                hipStream_t st) {
  const int qt = decode4_qtiles(c);
  const bool one_block = decode4_short(c);
  DecodeScratch sc{};
  sc.nsplit = one_block ? 1 : decode4_splits(c, qt);
  const bool join = sc.nsplit > 1;
  if (join) {
    sc.part = static_cast<float*>(scratch);
    sc.ml = sc.part + static_cast<long long>(c.n_seq) * c.hq * sc.nsplit * c.dh;
  }
  const hipError_t err = c.dtype == 0 ? start_decode4<float>(c, s, a, sc, qt, one_block, st)
                                      : start_decode4<bf16_t>(c, s, a, sc, qt, one_block, st);
  if (err != hipSuccess || !join) return err;
  return launch_decode_join(c, a, sc, false, kTile4, st);
}

}  // namespace gmc
