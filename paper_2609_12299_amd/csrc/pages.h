// pages.h -- numbers on their way into a paged cache.
#pragma once

#include "decode.h"

namespace argus {
namespace decode {

// x / s rounded to nearest, limited to the range of e4m3.  y = 1 / s correctly
// rounded; then fma(x - q s, y, q) with q = x y is the correctly rounded
// quotient (Markstein), save where q overflows, which the limit settles.
ARGUS_DEV float quotient(float x, float s, float y) {
  const float q = x * y;
  float r = fmaf(fmaf(-q, s, x), y, q);
  r = fabsf(q) > 1000.0f ? q : r;  // beyond the range; infinities have no remainder
  r = r > 448.0f ? 448.0f : r;     // NaN stays
  return r < -448.0f ? -448.0f : r;
}

// Scales that quotient() takes.  Outside (0, infinities and NaN among them) the reciprocal, or the
// remainder of a quotient that is not rounded to zero, would leave the normal numbers of 32 bits.
ARGUS_DEV bool ordinary(float s) { return fabsf(s) >= 0x1p-80f && fabsf(s) <= 0x1p80f; }

typedef float f32_pair __attribute__((ext_vector_type(2)));

template <int T>  // 0: bf16, 1: fp16
ARGUS_DEV f32_pair pair(uint32_t w) {
  if constexpr (T == 0) {
    return (f32_pair){__builtin_bit_cast(float, w << 16), __builtin_bit_cast(float, w & 0xFFFF0000u)};
  } else {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_convertvector(__builtin_bit_cast(f16x2, w), f32_pair);
  }
}

}  // namespace decode
}  // namespace argus
