// rows.h -- rows of logits: their elements, the order of values and tokens, maxima and sums of a wave.
#pragma once

#include "decode.h"

namespace argus {
namespace decode {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// for elements read from LDS that was written as vectors
typedef float any_f32 __attribute__((may_alias));
typedef uint16_t any_u16 __attribute__((may_alias));

// Larger key: larger value, then lower token.  -0 and +0 are one value.
ARGUS_DEV uint32_t order_of(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
ARGUS_DEV float value_of(uint32_t o) { return __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7FFFFFFFu : ~o); }
ARGUS_DEV uint64_t key_of(float x, uint32_t token) { return join64(~token, order_of(x)); }

template <int TYPE>
ARGUS_DEV float of_word(uint32_t w, int half) {
  if constexpr (TYPE == ARGUS_FP32) return __builtin_bit_cast(float, w);
  if constexpr (TYPE == ARGUS_BF16) return __builtin_bit_cast(float, half ? w & 0xFFFF0000u : w << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(half ? w >> 16 : w));
}

// The largest value of the wave, without LDS.
ARGUS_DEV float wave_max(float v) {
  auto step = [&](auto ctrl, auto rows) {
    const int o = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, v), __builtin_bit_cast(int, v), ctrl(), rows(), 0xF, false);
    v = fmaxf(v, __builtin_bit_cast(float, o));
  };
#define ARGUS_K(x) []() constexpr { return x; }
  step(ARGUS_K(kDppRowShr + 1), ARGUS_K(0xF));
  step(ARGUS_K(kDppRowShr + 2), ARGUS_K(0xF));
  step(ARGUS_K(kDppRowShr + 4), ARGUS_K(0xF));
  step(ARGUS_K(kDppRowShr + 8), ARGUS_K(0xF));
  step(ARGUS_K(kDppBcast15), ARGUS_K(0xA));
  step(ARGUS_K(kDppBcast31), ARGUS_K(0xC));
#undef ARGUS_K
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
ARGUS_DEV uint32_t wave_max_u32(uint32_t v) {
  // (unsigned order as that of signed numbers, whose least the wave's helpers find)
  const int32_t x = (int32_t)(~v ^ 0x80000000u);
  return ~((uint32_t)rows_min32(row_min32(x)) ^ 0x80000000u);
}
ARGUS_DEV float wave_sum(float v) {
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}

}  // namespace decode
}  // namespace argus
