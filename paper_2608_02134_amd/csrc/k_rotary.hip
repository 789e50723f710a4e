// Appending to the paged cache with the position rotation on the way, into pages
// of the type or of 4 bits, with the tokens' queries rotated by the same call;
// and reading rows of 4 bits back.
//
// Nothing is used twice but the table, so the kernels are bound by memory.  A
// lane takes 8 neighbouring elements of a head ("piece"), and with pairs of
// halves loads the 8 that they turn with too (which a lane beside it has for its
// own: the second load is the cache's).  A lane keeps its piece over all heads of
// a token, so that it reads its cosines and sines once.  Four neighbouring lanes
// have a block of 32: its largest magnitude takes two exchanges.
//
// 16448 tokens, 28 query heads on 4 of 128 in bf16: 54 us, 5.6 TB/s.  16 prompts of
// 335 rows picked from 1375 into 4 bits, 4 heads of 128: 9.9 us, of which most are five
// trips to memory one after the other (pick, position, table, page, rows).  One token
// of 16 sequences with 28 query heads 5.0 us.
#include <algorithm>

#include "gmc_cache.h"
#include "gmc_device.h"
#include "gmc_fp4.h"

namespace gmc {

enum Pairs { kNoPairs, kHalves, kNeighbours };

template <typename T> struct Piece;   // eight elements as they are in memory
template <> struct Piece<bf16_t> { uint4 u; };
template <> struct Piece<float> { floatx4 u[2]; };

template <typename T> __device__ __forceinline__ Piece<T> load_piece(const T* p) {
  return *reinterpret_cast<const Piece<T>*>(p);
}
__device__ __forceinline__ void unpack(const Piece<float>& y, float* x) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = y.u[e / 4][e % 4];
}
__device__ __forceinline__ void unpack(const Piece<bf16_t>& y, float* x) {
  const uint32_t u[4] = {y.u.x, y.u.y, y.u.z, y.u.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e & 1 ? u[e / 2] & 0xFFFF0000u : u[e / 2] << 16);
}
__device__ __forceinline__ void store_piece(float* p, const float* x) {
  reinterpret_cast<floatx4*>(p)[0] = floatx4{x[0], x[1], x[2], x[3]};
  reinterpret_cast<floatx4*>(p)[1] = floatx4{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store_piece(bf16_t* p, const float* x) {
  bf16x8 y;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = static_cast<__bf16>(x[e]);
  *reinterpret_cast<bf16x8*>(p) = y;
}

// The cosines and sines of a lane's piece.
struct Turn {
  float c[8], s[8];   // neighbours: four pairs
};

template <int PAIRS>
__device__ __forceinline__ void load_turn(const RotaryView& r, const int32_t* pos, int position, int d0, Turn* t) {
  const int half = r.rot >> 1;
  const int f0 = PAIRS == kNeighbours ? d0 >> 1 : d0 < half ? d0 : d0 - half;
#pragma unroll
  for (int e = 0; e < (PAIRS == kNeighbours ? 1 : 2); ++e) {
    const int f = f0 + 4 * e;   // four pairs of one section
    int p = position;
    if (pos) p = pos[f < r.t_end ? 0 : f < r.h_end ? 1 : 2];
    const long long at = static_cast<long long>(min(max(p, 0), r.n_pos - 1)) * half + f;
    const floatx4 c = *reinterpret_cast<const floatx4*>(r.cos + at), s = *reinterpret_cast<const floatx4*>(r.sin + at);
#pragma unroll
    for (int u = 0; u < 4; ++u) { t->c[4 * e + u] = c[u]; t->s[4 * e + u] = s[u]; }
  }
}

// x turned in place; y: the elements of the other half.  Products are rounded
// before they are added, so that a result does not depend on which of the two a
// fused operation would take.
template <int PAIRS>
__device__ __forceinline__ void turn_piece(const Turn& t, bool second, const float* y, float* x) {
#pragma clang fp contract(off)
  if constexpr (PAIRS == kHalves) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float xc = x[e] * t.c[e], ys = y[e] * t.s[e];
      x[e] = second ? xc + ys : xc - ys;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float a = x[2 * e], b = x[2 * e + 1];
      const float ac = a * t.c[e], bs = b * t.s[e], bc = b * t.c[e], as = a * t.s[e];
      x[2 * e] = ac - bs;
      x[2 * e + 1] = bc + as;
    }
  }
}

// The largest magnitude's bits over a block's four lanes.
__device__ __forceinline__ uint32_t block_top(const float* x) {
  int top = 0;   // (as integers, infinities and NaN are largest)
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, static_cast<int>(__float_as_uint(x[e]) & 0x7FFFFFFFu));
  top = max(top, dpp_i<0xB1, 0xf>(top, top));
  return static_cast<uint32_t>(max(top, dpp_i<0x4E, 0xf>(top, top)));
}

// One token: heads of K, V and q, 64 / (dh / 8) at a time to a wave, by `parts`
// waves of which this is number `part`.  s: its slot (one past the capacity is not
// stored); from: its row in k, v, q and pos; to: in q_out.  (The first heads' loads
// before the position's and the page's, us with the launches around it: 66 where this
// takes 61 for 16448 tokens; 16 prompts of 335 picked rows into 4 bits and read back 19.7
// and 19.5; one token of 16 sequences 6.6 and 6.4.)
template <typename T, bool Q4, int PAIRS>
__device__ __forceinline__ void append_turned(const CacheView& c, const CacheScales& sc, const RotaryView& r,
                                              const RotaryArgs& a, int b, int s, int position, long long from,
                                              long long to, int part, int parts) {
  const int lane = threadIdx.x & 63, per = c.dh >> 3, heads = 64 / per;
  const int hl = lane / per, d0 = 8 * (lane - hl * per);
  if (hl >= heads) return;
  const int half = r.rot >> 1;
  const bool turns = PAIRS != kNoPairs && d0 < r.rot, second = d0 >= half;
  Turn t;
  if (turns) load_turn<PAIRS>(r, a.pos ? a.pos + from * r.axes : nullptr, position, d0, &t);
  const long long row = s < c.cap ? cache_row(c, b, 0, s) : -1;   // of head 0; the others' lie a page's rows on
  const int total = 2 * c.hkv + (a.q ? c.hq : 0);
  const T* const k = static_cast<const T*>(a.k) + from * a.k_stride + d0;
  const T* const v = static_cast<const T*>(a.v) + from * a.v_stride + d0;
  const T* const q = a.q ? static_cast<const T*>(a.q) + from * a.q_stride + d0 : nullptr;
  constexpr int kFlight = sizeof(T) == 2 ? 3 : 2;   // heads whose loads are on their way together
  for (int u0 = part * heads + hl; u0 < total; u0 += kFlight * parts * heads) {
    Piece<T> own[kFlight], other[kFlight];
#pragma unroll
    for (int f = 0; f < kFlight; ++f) {
      const int u = u0 + f * parts * heads;
      if (u >= total) break;
      const T* p = u < c.hkv ? k + u * c.dh : u < 2 * c.hkv ? v + (u - c.hkv) * c.dh : q + (u - 2 * c.hkv) * c.dh;
      own[f] = load_piece(p);
      if (PAIRS == kHalves && turns) other[f] = load_piece(p + (second ? -half : half));
    }
#pragma unroll
    for (int f = 0; f < kFlight; ++f) {
      const int u = u0 + f * parts * heads;
      if (u >= total) break;
      const bool values = u >= c.hkv && u < 2 * c.hkv, query = u >= 2 * c.hkv;
      float x[8];
      unpack(own[f], x);
      if (turns && !values) {
        float y[8];
        if constexpr (PAIRS == kHalves) unpack(other[f], y);
        turn_piece<PAIRS>(t, second, y, x);
      }
      if (query) {
        store_piece(static_cast<T*>(a.q_out) + (to * c.hq + (u - 2 * c.hkv)) * c.dh + d0, x);
        continue;
      }
      if (row < 0) continue;
      const long long at = row + (static_cast<long long>(values ? u - c.hkv : u) << c.shift);
      if constexpr (Q4) {
        const uint32_t e = fp4_scale(block_top(x));
        const long long word = at * (c.dh >> 3) + (d0 >> 3);
        static_cast<uint32_t*>(values ? c.v : c.k)[word] = fp4_codes(x, scale_of(e));
        if ((d0 & 31) == 0) (values ? sc.v : sc.k)[at * sc.bytes + (d0 >> 5)] = static_cast<uint8_t>(e);
      } else {
        store_piece(static_cast<T*>(values ? c.v : c.k) + at * c.dh + d0, x);
      }
    }
  }
}

__device__ __forceinline__ long long source_row(const RotaryArgs& a, int b, long long first, int i) {
  if (!a.src) return first + i;
  const long long x = a.src[static_cast<long long>(b) * a.max_new + i];
  return b * a.per_seq + min(max(x, 0ll), a.per_seq - 1);
}

// Token i of sequence b, by `parts` waves.
template <typename T, bool Q4, int PAIRS>
__device__ __forceinline__ void append_token_turned(const CacheView& c, const CacheScales& sc, const RotaryView& r,
                                                    const RotaryArgs& a, int b, long long first, int len, int seen,
                                                    int i, int part, int parts) {
  const int s = len + i, lane = threadIdx.x & 63;
  append_turned<T, Q4, PAIRS>(c, sc, r, a, b, s, c.seen ? seen + i : s, source_row(a, b, first, i), first + i,
                              part, parts);
  if (part != 0 || s >= c.cap) return;
  const long long at = static_cast<long long>(b) * c.hkv * c.cap + s;
  for (int h = lane; h < c.hkv; h += 64) {
    if (c.slot_pos) c.slot_pos[at + static_cast<long long>(h) * c.cap] = seen + i;
    if (c.weights) c.weights[at + static_cast<long long>(h) * c.cap] = 0.f;
  }
}

// Tokens whose heads four waves share (28 query heads on 4 of 128 in bf16, us with the
// length's kernel, shared and by one wave: 16 tokens 8.4 and 10.7, 335 8.9 and 11.0, 1375
// 14.4 and 13.0, 4096 25.9 and 20).
constexpr int kSplitTokens = 512;
constexpr int kGridBlocks = 1 << 22;   // of 256 threads, at most 65535 sequences: the others are loops

// Few new tokens: one block a sequence, four waves a token, which also moves the
// length on.  16 sequences, 28 query heads on 4 of 128, us so and with the two kernels
// below: 4 tokens 7.9, 8 tokens 10.6 and 8.5.
constexpr int kTurnedFew = 4;
template <typename T, bool Q4, int PAIRS>
__global__ void __launch_bounds__(1024)
rotary_append_few_kernel(CacheView c, CacheScales sc, RotaryView r, RotaryArgs a) {
  const int b = blockIdx.x, w = wave_id();
  long long first;
  int n;
  new_rows(a.starts, a.max_new, a.rows, b, &first, &n);
  const int len = cache_len(c, b), seen = c.seen ? c.seen[b] : 0;
  for (int i = w >> 2; i < n; i += blockDim.x >> 8)
    append_token_turned<T, Q4, PAIRS>(c, sc, r, a, b, first, len, seen, i, w & 3, 4);
  __syncthreads();   // (every wave has read the length)
  if (threadIdx.x == 0) {
    n = min(n, c.cap - len);
    c.lens[b] = len + n;
    if (c.seen) c.seen[b] = seen + n;
  }
}

template <typename T, bool Q4, int PAIRS>
__global__ void __launch_bounds__(256)
rotary_append_kernel(CacheView c, CacheScales sc, RotaryView r, RotaryArgs a, int parts) {
  const int b = blockIdx.y, w = wave_id(), part = w & (parts - 1), at_once = 4 / parts;   // tokens of a block
  long long first;
  int n;
  new_rows(a.starts, a.max_new, a.rows, b, &first, &n);
  const int len = cache_len(c, b), seen = c.seen ? c.seen[b] : 0;
  for (int i = blockIdx.x * at_once + w / parts; i < n; i += gridDim.x * at_once)
    append_token_turned<T, Q4, PAIRS>(c, sc, r, a, b, first, len, seen, i, part, parts);
}

template <typename T, bool Q4, int PAIRS>
static hipError_t start_append(const CacheView& c, const CacheScales& sc, const RotaryView& r, const RotaryArgs& a,
                               hipStream_t st) {
  if (a.max_new <= kTurnedFew) {
    hipLaunchKernelGGL((rotary_append_few_kernel<T, Q4, PAIRS>), dim3(c.n_seq), dim3(256 * a.max_new), 0, st,
                       c, sc, r, a);
    return hipGetLastError();
  }
  const int parts = static_cast<long long>(a.max_new) * c.n_seq <= kSplitTokens ? 4 : 1;
  const int blocks = (a.max_new + 4 / parts - 1) / (4 / parts);
  hipLaunchKernelGGL((rotary_append_kernel<T, Q4, PAIRS>), dim3(std::min(blocks, kGridBlocks / c.n_seq), c.n_seq), dim3(256),
                     0, st, c, sc, r, a, parts);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;   // (rows that were not written are not counted)
  return launch_cache_advance(c, a.starts, a.rows, a.max_new, st);
}

hipError_t launch_cache_append_rotary(const CacheView& c, const CacheScales* scales, const RotaryView* rotary,
                                      const RotaryArgs& a, hipStream_t st) {
  const CacheScales sc = scales ? *scales : CacheScales{};
  const RotaryView r = rotary ? *rotary : RotaryView{};
#define GMC_APPEND(T, Q4)                                                                       \
  (!rotary ? start_append<T, Q4, kNoPairs>(c, sc, r, a, st)                                     \
   : r.interleaved ? start_append<T, Q4, kNeighbours>(c, sc, r, a, st) : start_append<T, Q4, kHalves>(c, sc, r, a, st))
#define GMC_APPEND_TURNED(T) \
  (r.interleaved ? start_append<T, false, kNeighbours>(c, sc, r, a, st) : start_append<T, false, kHalves>(c, sc, r, a, st))
  if (scales) return c.dtype == 0 ? GMC_APPEND(float, true) : GMC_APPEND(bf16_t, true);
  return c.dtype == 0 ? GMC_APPEND_TURNED(float) : GMC_APPEND_TURNED(bf16_t);
#undef GMC_APPEND
#undef GMC_APPEND_TURNED
}

// --- rows of 4 bits back --------------------------------------------------------
// A wave a token; a lane turns a word of eight codes into eight values (16 x 335
// rows of 4 heads of 128 in bf16: 6.4 us).
template <typename T>
__global__ void __launch_bounds__(256)
cache4_read_kernel(CacheView c, CacheScales sc, long long rows, const int32_t* starts, int max_new, T* k_out, T* v_out) {
  const int b = blockIdx.y, lane = threadIdx.x & 63, per = c.dh >> 3;
  long long first;
  int n;
  new_rows(starts, max_new, rows, b, &first, &n);
  const int len = cache_len(c, b);
  for (int i = blockIdx.x * 4 + wave_id(); i < n; i += gridDim.x * 4) {
    const int s = len - n + i;
    const long long row = s < 0 ? -1 : cache_row(c, b, 0, s);
    constexpr int kFlight = 2;
    for (int p0 = lane; p0 < 2 * c.hkv * per; p0 += 64 * kFlight) {
      uint32_t codes[kFlight], e[kFlight];
#pragma unroll
      for (int f = 0; f < kFlight; ++f) {
        const int p = p0 + 64 * f, u = p / per, piece = p - u * per;
        const bool values = u >= c.hkv;
        const long long at = row + (static_cast<long long>(values ? u - c.hkv : u) << c.shift);
        codes[f] = e[f] = 0u;
        if (row < 0 || u >= 2 * c.hkv) continue;
        codes[f] = static_cast<const uint32_t*>(values ? c.v : c.k)[at * per + piece];
        e[f] = (values ? sc.v : sc.k)[at * sc.bytes + (piece >> 2)];
      }
#pragma unroll
      for (int f = 0; f < kFlight; ++f) {
        const int p = p0 + 64 * f, u = p / per, piece = p - u * per;
        if (u >= 2 * c.hkv) break;
        const uint4 y = fp4_words(codes[f], scale_of(e[f]));
        T* to = (u >= c.hkv ? v_out : k_out) + ((first + i) * c.hkv + (u >= c.hkv ? u - c.hkv : u)) * c.dh + 8 * piece;
        if constexpr (sizeof(T) == 2) {
          *reinterpret_cast<uint4*>(to) = y;
        } else {
          float x[8];
          unpack(Piece<bf16_t>{y}, x);
          store_piece(to, x);
        }
      }
    }
  }
}

hipError_t launch_cache4_read(const CacheView& c, const CacheScales& s, long long rows, const int32_t* starts,
                              int max_new, void* k_out, void* v_out, hipStream_t st) {
  const dim3 grid(std::min((max_new + 3) / 4, kGridBlocks / c.n_seq), c.n_seq);
  if (c.dtype == 0)
    hipLaunchKernelGGL(cache4_read_kernel<float>, grid, dim3(256), 0, st, c, s, rows, starts, max_new,
                       static_cast<float*>(k_out), static_cast<float*>(v_out));
  else
    hipLaunchKernelGGL(cache4_read_kernel<bf16_t>, grid, dim3(256), 0, st, c, s, rows, starts, max_new,
                       static_cast<bf16_t*>(k_out), static_cast<bf16_t*>(v_out));
  return hipGetLastError();
}

}  // namespace gmc
