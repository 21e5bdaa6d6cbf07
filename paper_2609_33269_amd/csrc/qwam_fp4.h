// The 4-bit pages of the key-value cache (gfx950): e2m1 codes, two channels to a
// byte, and one power of two for 32 channels of a position (QWAM_CACHE_FP4).  The
// conversions are the hardware's, checked for every byte and exponent: reading is
// exact and takes the scale from a float's exponent bits alone, NaN where they are
// all ones; writing rounds to nearest, ties to the even code, and saturates at 6.
#pragma once
#include "qwam_device.h"
#include "qwam_internal.h"

namespace qwam {

typedef __bf16 v2bf16 __attribute__((ext_vector_type(2)));

// the two codes of byte `b` of a word (constant after unrolling) as a bf16 pair, times the power of two in
// the exponent bits of `scale`
__device__ __forceinline__ uint32_t fp4_pair(uint32_t w, uint32_t scale, int b) {
  const float s = __uint_as_float(scale);
  switch (b) {
    case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
    case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
    case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
    default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
  }
}

// The exponent byte E of a group whose largest |x| has these bf16 bits (sign cleared): the least power of two 2^(E - 127)
// with 7 of it at least that.  The largest is 1.m * 2^(e - 127), and 7 = 1.75 * 4, so E = e - 2 for m up to .75
// (0x60 in 7 bits) and one more above: a carry out of m + 0x1F.  E stays within [4, 252], where every stored value
// and every quotient that does not round to 0 is a normal bf16; infinities and NaN give 255.
__device__ __forceinline__ uint32_t fp4_exponent(uint32_t largest) {
  if (largest >= 0x7F80u) return 255u;
  const int e = static_cast<int>((largest + 0x1Fu) >> 7) - 2;
  return static_cast<uint32_t>(min(max(e, 4), 252));
}

// eight bf16 values in four words -> eight codes
__device__ __forceinline__ uint32_t fp4_codes(const uint4& x, uint32_t exponent) {
  const float s = __uint_as_float(exponent << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(v2bf16, x.x), s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(v2bf16, x.y), s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(v2bf16, x.z), s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(v2bf16, x.w), s, 3);
}

// bytes of scales in a page, and where a head's groups begin in it
__device__ __forceinline__ int64_t fp4_exp_page(const CacheParams& c) {
  return static_cast<int64_t>(c.heads * (c.dim / kFp4Group)) << c.page_bits;
}
__device__ __forceinline__ int64_t fp4_exp_group(const CacheParams& c, int head, int group) {
  return static_cast<int64_t>(head * (c.dim / kFp4Group) + group) << c.page_bits;
}

}  // namespace qwam
