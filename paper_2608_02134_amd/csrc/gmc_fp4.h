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

}  // namespace gmc
