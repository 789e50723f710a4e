// Values of 4 bits: blocks of 32 with a power of two, as caches of 4 bits hold
// them.  The conversions are single instructions and exact: a code times a scale
// has two significant bits, which bf16 and fp32 hold down to the least scale.
#pragma once

#include "gmc_device.h"

namespace gmc {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 2^(e - 127) as the conversions take it (255: infinity, which makes NaN of all
// codes; 0: their 2^-127).
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e << 23); }

// Codes 2 B and 2 B + 1 of the eight in a word, as two bf16.
template <int B> __device__ __forceinline__ uint32_t fp4_pair(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}

// Eight codes as eight bf16.
__device__ __forceinline__ uint4 fp4_words(uint32_t codes, float scale) {
  return make_uint4(fp4_pair<0>(codes, scale), fp4_pair<1>(codes, scale), fp4_pair<2>(codes, scale),
                    fp4_pair<3>(codes, scale));
}

// The scale byte of a block whose largest magnitude has the bits `top`: the
// least e >= 1 with top <= 7 * 2^(e - 127).  1.75 * 2^k is 7 * 2^(k - 2), so
// what is left after the leading bit decides between k - 2 and k - 1.  At most
// 252, whose 6 scales are the largest that does not overflow.
__device__ __forceinline__ uint32_t fp4_scale(uint32_t top) {
  const int e = static_cast<int>((top + 0x1FFFFFu) >> 23) - 2;
  return top >= 0x7F800000u ? 255u : static_cast<uint32_t>(min(max(e, 1), 252));
}

// Eight values as codes: nearest, ties to even; magnitudes above 6 scales become
// 6.
__device__ __forceinline__ uint32_t fp4_codes(const float* x, float scale) {
  uint32_t u = 0;
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[0], x[1], scale, 0);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[2], x[3], scale, 1);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[4], x[5], scale, 2);
  u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, x[6], x[7], scale, 3);
  return u;
}

// fp32 beside values of 4 bits, which are bf16: x as the upper 8 significant bits,
// the next 8, and the rest rounded; infinities and NaN in the first.
// An infinite value, which scales from 2^126 on have, times a part of zero would be NaN:
// the least bf16, 2^-133, with x's sign is added to the second and third part.
__device__ __forceinline__ __bf16 upper_half(uint32_t u) {
  return __builtin_bit_cast(__bf16, static_cast<uint16_t>(u >> 16));
}
__device__ __forceinline__ void split3(float x, __bf16* part) {
  const uint32_t u = __float_as_uint(x);
  const bool finite = (u & 0x7F800000u) != 0x7F800000u;
  const float least = __builtin_amdgcn_fmed3f(x, -0x1p-133f, 0x1p-133f);   // (0 for x = 0)
  const float rest = (finite ? x - __uint_as_float(u & 0xFFFF0000u) : 0.f) + least;
  const uint32_t v = __float_as_uint(rest) & 0xFFFF0000u;
  part[0] = finite ? upper_half(u) : static_cast<__bf16>(x);
  part[1] = upper_half(v);
  part[2] = static_cast<__bf16>(rest - __uint_as_float(v) + least);
}

// A weight (not negative) as two or three parts.  An infinite value, which scales from
// 2^126 on have, times a part of zero would be NaN: no part of a weight that is not zero
// is below the least bf16, 2^-133, which is under 2^-17 and 2^-25 of weights down to 2^-116
// and 2^-108.  (Weights below 2^-126 of the largest are zero as a whole in 32 bits.)
__device__ __forceinline__ void split2_weight(float e, __bf16* part) {
  const uint32_t u = __float_as_uint(e) & 0xFFFF0000u;
  part[0] = upper_half(u);
  part[1] = static_cast<__bf16>(fmaxf(e - __uint_as_float(u), fminf(e, 0x1p-133f)));
}
__device__ __forceinline__ void split3_weight(float e, __bf16* part) {
  const uint32_t u = __float_as_uint(e) & 0xFFFF0000u;
  const float rest = e - __uint_as_float(u), least = fminf(e, 0x1p-133f);
  const uint32_t v = __float_as_uint(fmaxf(rest, least)) & 0xFFFF0000u;
  part[0] = upper_half(u);
  part[1] = upper_half(v);
  part[2] = static_cast<__bf16>(fmaxf(rest - __uint_as_float(v), least));
}

}  // namespace gmc
