// Attention of one new token per sequence over a paged cache of 4 bits.
//
// As over pages of bf16 (S^T = K Q^T, O^T = V^T P^T, keys split over blocks and
// joined by a second kernel), with 136 bytes a row of 128 elements for K and V instead
// of 512: bound by memory where the caches are long, if enough loads are on their way
// and the instructions beside them are few.
//   Loads: tiles of 32 keys go from the pages into shared memory without registers
//      between, each wave its own, one tile ahead of the one it computes: five loads
//      a tile of 128 dims.  (Into registers, 14 loads a tile: 278 us where this takes 197;
//      loads alone take 179.  Two tiles ahead were 199, four waves a SIMD 233, with
//      spilt registers.)  What a lane loads is what it reads back, where K is
//      concerned; V is turned by the addresses of the reads.
//   K: the order of the elements in a product is free, so lane (key l % 16, group g =
//      l / 16) takes a run of them: of each 128 the 32 from 32 g, one block with one
//      scale; of what is left 16 from 16 g (64) and 8 from 8 g (32).
//   V: lane (i = l % 16, g) takes of each of its group's keys 4 g + 0..3 the 8
//      elements from 8 i of each 128 (4 of 64, 2 of 32), and turns pairs of two keys
//      into operands by byte permutations.
//   Codes become bf16 by single instructions, exactly; a scale's byte comes to its
//      place by one rotation.
// Every value is a bf16, so fp32 queries and weights enter as three bf16 (24
// bits: exact but for the last, which is rounded) and the products are those of
// fp32; weights for bf16 outputs as two (16 bits).  The matrix cores idle, so this
// costs nothing.
//
// 8 requests of 100000 to 131072 slots, 32 heads on 8 of 128 in bf16: 190 us, 5.3
// TB/s, and 5 for the joining kernel (over bf16 pages 633).  64 requests of 200 to 4096
// slots, 28 heads on 4: 20 us and 4.
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

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Byte n of four as a scale: the conversions look at the exponent's bits alone, so
// a rotation brings it there.
__device__ __forceinline__ uint32_t scale_at_bits(uint32_t bytes, int n) {
  return __builtin_amdgcn_alignbit(bytes, bytes, static_cast<uint32_t>(8 * n + 9) & 31u);
}
__device__ __forceinline__ float scale_at(uint32_t bytes, int n) { return __uint_as_float(scale_at_bits(bytes, n)); }

// Shared and global memory by their address spaces, as loads into shared memory
// take them.
typedef __attribute__((address_space(3))) uint8_t shared_u8;
typedef __attribute__((address_space(1))) uint32_t global_u32;
template <typename V> __device__ __forceinline__ V ld_shared(const shared_u8* p) {
  return *reinterpret_cast<const __attribute__((address_space(3))) V*>(p);
}

// A tile in shared memory: 16-byte blocks of K, of V (whole loads of 64 of
// them), then the rows' scales.  K's blocks stand block by block of the row, V's so
// that the blocks that one read touches lie on different banks.
template <int DH> struct Tile4 {
  static constexpr int kBlocks = DH / 32, kLoads = (kBlocks + 1) / 2, kScaleBytes = scale_bytes(DH);
  static constexpr int kScaleLoads = (kScaleBytes + 3) / 4;      // of 256 bytes
  static constexpr int kV = 1024 * kLoads, kScales = 2 * kV, kBytes = kScales + 256 * kScaleLoads;
  static constexpr int kInFlight = 2 * kLoads + kScaleLoads;     // loads of a tile
  static __device__ __forceinline__ int k_at(int half, int row, int blk) { return 16 * ((half * kBlocks + blk) * 16 + row); }
  static __device__ __forceinline__ int v_at(int half, int row, int blk) {
    return kV + 16 * (half * 16 * kBlocks + ((row & 3) * 4 + (row >> 2)) * kBlocks + blk);
  }
  static __device__ __forceinline__ int scales_at(bool values, int half, int row) {
    return kScales + (((values ? 2 : 0) + half) * 16 + row) * kScaleBytes;
  }
};

template <int N> __device__ __forceinline__ void arrive() {   // until at most N loads are on their way
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}

// As many blocks as find room on the chip together, three to a CU (with two tiles
// ahead, us with 512, 768, 1024 and 1536: 8 requests of 100000 to 131072 slots, 32 heads on
// 8 of 128, 205, 200, 197 and 194; 64 of 200 to 4096, 28 on 4, 28.2, 26.3, 27.5 and 28; 16 of
// them 13.0, 13.8, 15.4 and 17).  Splits of one length for all sequences, so that short ones
// have fewer, were slower: 210 and 28.1.  Wider heads, whose CUs hold two blocks or one
// (blocks_of_cu), have the same number; others were not measured for them.
constexpr int kDecode4Blocks = 768;

// Three blocks of four waves to a CU with heads of up to 128, two with wider ones and
// in fp32 with 96 to 160, one in fp32 from 192 on, whose registers are more.
constexpr int blocks_of_cu(int type_bytes, int dh, int waves) {
  return type_bytes == 4 && dh > 160 ? 1 : dh <= (type_bytes == 2 ? 128 : 64) && waves == kDecodeWaves ? 3 : 2;
}
template <typename T, int DH, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, (blocks_of_cu(sizeof(T), DH, WAVES)))
decode4_kernel(CacheView c, CacheScales sc4, AttendArgs a, DecodeScratch sc, int qtiles) {
  using R = Runs<DH>;
  using L = Tile4<DH>;
  constexpr int H = 2, TK = kTile4, NS = DH / 32, NO = DH / 16, ROW = DH / 2;
  constexpr int SB = scale_bytes(DH);
  constexpr int NQ = sizeof(T) == 2 ? 1 : 3, NP = sizeof(T) == 2 ? 2 : 3;   // bf16 parts of queries and weights
  __shared__ __align__(16) uint8_t even[WAVES * L::kBytes], odd[WAVES * L::kBytes];
  __shared__ float stat[WAVES][2][16];
  static_assert(sizeof(even) >= WAVES / 2 * 16 * DH * sizeof(float), "the waves' parts take the first tiles' place");
  const int split = blockIdx.x, h = blockIdx.y / qtiles, qt = blockIdx.y % qtiles, b = blockIdx.z;
  const int lane = threadIdx.x & 63, w = wave_id(), i16 = lane & 15, g = lane >> 4;
  const int len = cache_len(c, b);
  const TileRange tr = tile_range(len, a.window, a.sinks, true, TK);
  const int ns = WAVES == kDecodeWaves ? used_splits(tr.count, sc.nsplit) : 1;
  if (split >= ns) return;
  // (at most 2^19 tiles and kDecode4Blocks splits: their product is below 2^31)
  const int t0 = static_cast<int>(static_cast<unsigned>(tr.count * split) / static_cast<unsigned>(ns));
  const int t1 = static_cast<int>(static_cast<unsigned>(tr.count * (split + 1)) / static_cast<unsigned>(ns));
  const int head = qt * 16 + i16;                 // of the group
  const bool live = head < c.hg;
  const int hq = h * c.hg + head;
  // exp2(scale log2(e) s): a negative scale goes to the queries' sign, and a
  // scale of zero to the least one that does not turn a hidden key's -inf into NaN
  const float cs = fmaxf(fabsf(a.scale) * kLog2e, 0x1p-149f);
  const float slack = fminf(8.f / cs, 0x1p126f);   // (not infinite: the first maximum is above -inf + slack)

  // (as constant memory, which nothing here writes: page ids come by scalar loads, and
  // the vector loads on their way are those of tiles alone)
  typedef const __attribute__((address_space(4))) int32_t constant_i32;
  constant_i32* table = (constant_i32*)(c.table + static_cast<long long>(b) * c.max_pages);
  auto slot0 = [&](int tile) { return (tile < tr.first ? tile : tile + tr.skip) * TK; };
  // Page ids of a tile's halves; past the last tile as of it.
  auto ids_of = [&](int tile, int* id) {
    const int s = slot0(min(tile, t1 - 1));
#pragma unroll
    for (int hh = 0; hh < H; ++hh) id[hh] = table[min(s + 16 * hh, c.cap - 1) >> c.shift];
  };
  // Which halves of a tile are on a page: bits.
  auto on_pages = [&](int tile, const int* id) {
    unsigned ok = 0;
#pragma unroll
    for (int hh = 0; hh < H; ++hh)
      if (slot0(tile) + 16 * hh < len && id[hh] >= 0 && id[hh] < c.n_pages) ok |= 1u << hh;
    return ok;
  };
  // Where a lane's scale words come from (K, K, V, V of 4 SB words each): kept, as
  // the compiler would fetch the choice between the two anew, behind the loads on their way.
  const uint8_t* scales_from[L::kScaleLoads];
  bool second[L::kScaleLoads];
#pragma unroll
  for (int u = 0; u < L::kScaleLoads; ++u) {
    const int x = (64 * u + lane) % (16 * SB), part = x / (4 * SB);
    const uint8_t *k = sc4.k, *v = sc4.v;
    asm volatile("" : "+s"(k), "+s"(v));
    scales_from[u] = ((part & 2) ? v : k) + 4 * (x - part * 4 * SB);
    second[u] = part & 1;
  }
  // Loads a tile; rows that are none are those of the first page, and dropped.
  auto issue = [&](int tile, const int* id, unsigned ok, shared_u8* to) __attribute__((always_inline)) {
    // (pointers whose type depends on no template argument: clang drops the host's
    // side of a kernel in which this builtin is only checked with its arguments)
    shared_u8 *const values = to + L::kV, *const scales = to + L::kScales;
    long long row[H];
#pragma unroll
    for (int hh = 0; hh < H; ++hh)
      row[hh] = (ok >> hh) & 1u ? ((static_cast<long long>(id[hh]) * c.hkv + h) << c.shift) +
                                      ((slot0(tile) + 16 * hh) & (c.page - 1))
                                : 0;
#pragma unroll
    for (int u = 0; u < L::kLoads; ++u) {
      // (the last load of an odd number of blocks takes some of them twice)
      const int x = min(64 * u + lane, 32 * NS - 1), hh = x / (16 * NS), y = x - hh * 16 * NS;
      const long long r = hh ? row[1] : row[0];
      const int kr = y & 15, kblk = y >> 4;
      const int vx = y / NS, vblk = y - vx * NS, vr = (vx & 3) * 4 + (vx >> 2);
      const uint8_t* kp = static_cast<const uint8_t*>(c.k) + r * ROW + kr * ROW + 16 * kblk;
      const uint8_t* vp = static_cast<const uint8_t*>(c.v) + r * ROW + vr * ROW + 16 * vblk;
      __builtin_amdgcn_global_load_lds((const global_u32*)kp, to + 1024 * u, 16, 0, 0);
      __builtin_amdgcn_global_load_lds((const global_u32*)vp, values + 1024 * u, 16, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < L::kScaleLoads; ++u) {
      const uint8_t* p = scales_from[u] + (second[u] ? row[1] : row[0]) * SB;
      __builtin_amdgcn_global_load_lds((const global_u32*)p, scales + 256 * u, 4, 0, 0);
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
          uint4 y = live ? *reinterpret_cast<const uint4*>(p) : make_uint4(0u, 0u, 0u, 0u);
          if (a.scale < 0.f) { y.x ^= 0x80008000u; y.y ^= 0x80008000u; y.z ^= 0x80008000u; y.w ^= 0x80008000u; }
          q[0][s] = __builtin_bit_cast(bf16x8, y);
        } else {
          Frag<float> f = live ? frag_load<float>(p) : frag_zero<float>();
          if (a.scale < 0.f)
#pragma unroll
            for (int e = 0; e < 8; ++e) f.v[e] = -f.v[e];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            __bf16 part[3];
            split3(f.v[e], part);
            q[0][s][e] = part[0]; q[1][s][e] = part[1]; q[2][s][e] = part[2];
          }
        }
      }
  }
  floatx4 o[NO];
#pragma unroll
  for (int n = 0; n < NO; ++n) o[n] = floatx4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  auto compute = [&](int tile, unsigned ok, const shared_u8* in) __attribute__((always_inline)) {
    const int s0 = slot0(tile);
    // keys that are not seen: only in the last tile, at the window's edges and
    // on pages that are none
    const bool whole = s0 + TK <= len && (!a.window || len - 1 - s0 < a.window) && ok == 3u;
    floatx4 x[H];
#pragma unroll
    for (int hh = 0; hh < H; ++hh) {
      x[hh] = floatx4{0.f, 0.f, 0.f, 0.f};
      uint32_t sk[SB == 8 ? 2 : 1];
      {
        const shared_u8* p = in + L::scales_at(false, hh, i16);
        if constexpr (SB == 1) sk[0] = *p;
        else if constexpr (SB == 2) sk[0] = ld_shared<uint16_t>(p);
        else if constexpr (SB == 4) sk[0] = ld_shared<uint32_t>(p);
        else { const u32x2 y = ld_shared<u32x2>(p); sk[0] = y.x; sk[1] = y.y; }
      }
#pragma unroll
      for (int n = 0; n < R::count; ++n) {
        const int blk = R::base(n) / 32, size = R::size(n);
        // of 128 elements a group has a block, of 64 half of one, of 32 a quarter
        const int mine = size == 128 ? g : size == 64 ? g >> 1 : 0;
        const shared_u8* p = in + L::k_at(hh, i16, blk + mine);
        uint32_t u[4];
        if (size == 128) { const u32x4 y = ld_shared<u32x4>(p); u[0] = y.x; u[1] = y.y; u[2] = y.z; u[3] = y.w; }
        if (size == 64) { const u32x2 y = ld_shared<u32x2>(p + 8 * (g & 1)); u[0] = y.x; u[1] = y.y; }
        if (size == 32) u[0] = ld_shared<uint32_t>(p + 4 * g);
        const float f = scale_at(sk[blk / 4], blk % 4 + mine);
#pragma unroll
        for (int e = 0; e < size / 32; ++e) {
          const bf16x8 kf = __builtin_bit_cast(bf16x8, fp4_words(u[e], f));
#pragma unroll
          for (int y = NQ - 1; y >= 0; --y)
            x[hh] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[y][blk + e], x[hh], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int hh = 0; hh < H; ++hh) settle(x[hh]);
    uint32_t gone = 0;   // keys of this lane's eight that the query does not see
    if (!whole) {
#pragma unroll
      for (int hh = 0; hh < H; ++hh)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int s = s0 + 16 * hh + 4 * g + r;
          const bool see = ((ok >> hh) & 1u) && s < len && (!a.window || len - 1 - s < a.window || s < a.sinks);
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
    // the running maximum follows in steps of at least 8 (base 2): weights stay
    // below 2^8 and most tiles rescale nothing
    if (__any(mt > m + slack)) {
      const float mn = mt > m + slack ? mt : m;
      const float f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - mn) * cs);
      m = mn;
      l *= f;
#pragma unroll
      for (int n = 0; n < NO; ++n) o[n] *= f;
    }
    const float base = m == -INFINITY ? 0.f : m * cs;
    bf16x8 p[NP];
#pragma unroll
    for (int hh = 0; hh < H; ++hh)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float e = __builtin_amdgcn_exp2f(fmaf(x[hh][r], cs, -base));
        l += e;   // this lane group's keys; joined at the end
        const int at = 4 * hh + r;
        __bf16 part[3];
        if constexpr (NP == 2) split2_weight(e, part);
        else split3_weight(e, part);
#pragma unroll
        for (int y = 0; y < NP; ++y) p[y][at] = part[y];
      }
    uint32_t sv[H][SB];
#pragma unroll
    for (int hh = 0; hh < H; ++hh) {
      const shared_u8* ps = in + L::scales_at(true, hh, 4 * g);
      if constexpr (SB == 1) sv[hh][0] = ld_shared<uint32_t>(ps);
      if constexpr (SB == 2) { const u32x2 y = ld_shared<u32x2>(ps); sv[hh][0] = y.x; sv[hh][1] = y.y; }
      if constexpr (SB >= 4) {
#pragma unroll
        for (int e = 0; e < SB / 4; ++e) {
          const u32x4 y = ld_shared<u32x4>(ps + 16 * e);
#pragma unroll
          for (int k = 0; k < 4; ++k) sv[hh][4 * e + k] = y[k];
        }
      }
    }
#pragma unroll
    for (int n = 0; n < R::count; ++n) {
      const int size = R::size(n), pairs = size / 32, blk = R::base(n) / 32;   // pairs of elements a lane has of each key
      const int mine = size == 128 ? i16 >> 2 : size == 64 ? i16 >> 3 : 0;
      uint32_t codes[H][4], v[H][4][4];
#pragma unroll
      for (int hh = 0; hh < H; ++hh)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const shared_u8* p4 = in + L::v_at(hh, 4 * g + r, blk + mine);
          codes[hh][r] = size == 128  ? ld_shared<uint32_t>(p4 + 4 * (i16 & 3))
                         : size == 64 ? ld_shared<uint16_t>(p4 + 2 * (i16 & 7))
                                      : p4[i16];
        }
      uint32_t es[H][4];
#pragma unroll
      for (int hh = 0; hh < H; ++hh)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int at = r * SB + blk;
          es[hh][r] = scale_at_bits(sv[hh][at / 4], at % 4 + mine);
        }
      if (!whole) {   // a weight of zero does not silence a NaN
#pragma unroll
        for (int hh = 0; hh < H; ++hh)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if ((gone >> (4 * hh + r)) & 1u) codes[hh][r] = es[hh][r] = 0u;
      }
#pragma unroll
      for (int hh = 0; hh < H; ++hh)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float fs = __uint_as_float(es[hh][r]);
          v[hh][r][0] = fp4_pair<0>(codes[hh][r], fs);
          if (pairs > 1) v[hh][r][1] = fp4_pair<1>(codes[hh][r], fs);
          if (pairs > 2) { v[hh][r][2] = fp4_pair<2>(codes[hh][r], fs); v[hh][r][3] = fp4_pair<3>(codes[hh][r], fs); }
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

  // One tile is computed while the next one's loads are on their way; its page ids
  // come one tile before.
  shared_u8* const at0 = (shared_u8*)even + w * L::kBytes;
  shared_u8* const at1 = (shared_u8*)odd + w * L::kBytes;
  unsigned ok0 = 0, ok1 = 0;
  int tile = t0 + w, id[H];
  auto next = [&](int t, unsigned* ok, shared_u8* to) __attribute__((always_inline)) {
    if (t >= t1) return;
    *ok = on_pages(t, id);
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): what was read of the tile before is in registers
    issue(t, id, *ok, to);
    ids_of(t + WAVES, id);
  };
  auto step = [&](int t, unsigned ok, const shared_u8* in) __attribute__((always_inline)) {
    if (t + WAVES < t1) arrive<L::kInFlight>();   // those of the next tile may still be on their way
    else arrive<0>();
    compute(t, ok, in);
  };
  if (tile < t1) {
    ids_of(tile, id);
    next(tile, &ok0, at0);
  }
  for (; tile < t1; tile += 2 * WAVES) {
    next(tile + WAVES, &ok1, at1);
    step(tile, ok0, at0);
    if (tile + WAVES >= t1) break;
    next(tile + 2 * WAVES, &ok0, at0);
    step(tile + WAVES, ok1, at1);
  }
  asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");   // (see settle)
  __builtin_amdgcn_sched_barrier(0);
  m = m * cs;          // (as the parts' maxima are joined)
  float(*const red)[16 * DH] = reinterpret_cast<float(*)[16 * DH]>(even);

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
  return used_splits((c.cap + kTile4 - 1) / kTile4, static_cast<int>((kDecode4Blocks + groups - 1) / groups));
}

// One block of eight waves for a sequence's head and no second kernel, where a query
// looks at few tiles: up to 20 of them (caches of up to four are one block of four waves
// as it is), and more where the heads of all sequences are many, whose split parts cost
// more than they spread.  GPU time in us so and split, 28 heads on 4 of 128 in bf16: 1
// request of 640 slots 8.1 and 8.7, of 1024 10.3 and 8.7; 16 of 1024 10.5 and 10.6, of 2048
// 16 and 13; 64 of 1024 12.1 and 16.6, of 2048 18.6 and 23.1, of 200 to 4096 28.9 and 24.7.
// From kDecode4Blocks heads on nothing is split (256 of 640 22, so 32).
static bool decode4_short(const CacheView& c, int window, int sinks) {
  const long long heads = static_cast<long long>(c.n_seq) * c.hkv * decode4_qtiles(c);
  const int all = (c.cap + kTile4 - 1) / kTile4;
  long long seen = all;
  if (window > 0) seen = std::min(seen, (static_cast<long long>(window) + sinks) / kTile4 + 3);   // (two runs of slots)
  return c.dh <= 128 && all > kDecodeWaves && heads < kDecode4Blocks &&
         seen <= std::min(64ll, std::max(20ll, heads / 2));
}

long long decode4_scratch_bytes(const CacheView& c) {
  // (what is one block without a window is one with it)
  const int ns = decode4_short(c, 0, 0) ? 1 : decode4_splits(c, decode4_qtiles(c));
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
  const bool one_block = decode4_short(c, a.window, a.sinks);
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
