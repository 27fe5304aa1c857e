// Values into e4m3 codes with one power-of-two scale for each block of 128 columns: what
// lst_quantize, lst_scores and lst_norm_forward share.
#pragma once

#include "dtypes.h"

namespace lst {

constexpr int kBlock = 128;

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx2 __attribute__((ext_vector_type(2)));

// Biased exponent of the scale for the bits of a block's largest finite magnitude:
// 448 = 1.75 2^8, so 1.f 2^E needs 2^(E - 8) when 1.f <= 1.75, else 2^(E - 7).
__device__ inline int scale_of(uint32_t big) {
  const int e = (int)(big >> 23) - ((big & 0x7FFFFF) <= 0x600000 ? 8 : 7);
  return max(e, 0);
}

// Codes of values times 2^(127 - e), which is exact: e is at most 254 - 7.
template <int N>
__device__ inline void codes_of(const float (&v)[N], int e, uint32_t (&q)[N / 4]) {
  const float s = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * s, v[4 * i + 1] * s, 0, false);
    q[i] = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * s, v[4 * i + 3] * s, lo, true);
  }
}

// Largest finite magnitude of eight values, by its bits.  Values that are not finite become
// zero and set their bit of `bad`.
__device__ inline uint32_t largest_finite(float (&v)[8], uint32_t& bad) {
  uint32_t big = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) big = max(big, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  bad = 0;
  if (big >= 0x7F800000u) {
    big = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = __float_as_uint(v[i]) & 0x7FFFFFFFu;
      if (b >= 0x7F800000u) {
        bad |= 1u << i;
        v[i] = 0.f;
      } else {
        big = max(big, b);
      }
    }
  }
  return big;
}

// Codes of eight columns, a block being in 16 neighbouring lanes, and the block's biased
// exponent.  A value that is not finite gets the code that is no number.
__device__ inline void values_codes(float (&v)[8], uint32_t (&q)[2], int& e) {
  uint32_t bad, big = largest_finite(v, bad);
#pragma unroll
  for (int o = 8; o; o >>= 1) big = max(big, (uint32_t)__shfl_xor((int)big, o));
  e = scale_of(big);
  codes_of(v, e, q);
  if (bad) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (bad >> i & 1) q[i / 4] |= 0x7Fu << (8 * (i % 4));
  }
}

}  // namespace lst
