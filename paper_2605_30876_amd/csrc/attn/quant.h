// Values in 8 and 4 bits: 32 consecutive elements of a token's head share a
// scale 2^(b - 127), b a byte; an element is e4m3 or e2m1 times it.  b is the
// smallest at which no element of the group is off by more than half a step:
// its largest is at most 464 (7) times the scale, since 448 (6) is the largest
// code and the next one down is 32 (2) away.  Powers of two keep every product code * scale
// exact in bf16, so that what the cache holds enters the matrix products
// without another rounding.
#pragma once

#include "cache.h"

namespace dmoe {
namespace quant {

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kNan = 255;     // scale byte of a group with an element that is not finite: all of it reads as NaN
constexpr int kLowest = 17;   // 2^-110: the smallest code times it is a normal bf16
// the largest code times the largest scale fits bf16
template <int kBits>
constexpr int kHighest = kBits == 4 ? 252 : 246;

// The scale's byte, from the largest |element| as bits of a float32 (NaN and
// infinity are above all others).  Adding what is missing from the limit's fraction (7 =
// 1.75 * 4, 464 = 1.8125 * 256) to the next power of two carries into the exponent exactly
// for values above it.
template <int kBits>
__device__ __forceinline__ int scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return kNan;
  constexpr uint32_t kCarry = kBits == 4 ? 0x7fffffu - 0x600000u : 0x7fffffu - 0x680000u;
  const int b = static_cast<int>((top + kCarry) >> 23) - (kBits == 4 ? 2 : 8);
  return min(max(b, kLowest), kHighest<kBits>);
}

// Eight elements to codes at scale byte b, to nearest even, saturating: one dword of 4-bit
// codes, the first element lowest, or two of 8-bit ones.
template <int kBits>
struct alignas(kBits) Codes {
  uint32_t w[kBits / 4];
};
template <int kBits>
__device__ __forceinline__ Codes<kBits> encode(const float (&f)[8], int b) {
  const float inverse = __uint_as_float(static_cast<uint32_t>(254 - b) << 23);  // exact, and so is the product
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y[e] = b == kNan ? 0.f : f[e] * inverse;
    // e4m3 beyond the largest code would be NaN, e2m1 saturates
    if constexpr (kBits == 8) y[e] = __builtin_amdgcn_fmed3f(y[e], -448.f, 448.f);
  }
  Codes<kBits> c;
  if constexpr (kBits == 4) {
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.f, 2);
    c.w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.f, 3);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s16x2 w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s16x2{0, 0}, y[4 * i], y[4 * i + 1], 1.f, false);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, y[4 * i + 2], y[4 * i + 3], 1.f, true);
      c.w[i] = __builtin_bit_cast(uint32_t, w);
    }
  }
  return c;
}

__device__ __forceinline__ float scale_of(int b) { return __uint_as_float(static_cast<uint32_t>(b) << 23); }

// What eight codes stand for at a scale (NaN at scale_of(kNan), whatever the codes).
template <int kBits>
__device__ __forceinline__ bf16x8 decode(const uint32_t* w, float scale) {
  bf16x2 x[4];
  if constexpr (kBits == 4) {
    x[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 0);
    x[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 1);
    x[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 2);
    x[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale, 3);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false);
      x[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true);
    }
  }
  return bf16x8{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
}

}  // namespace quant
}  // namespace dmoe
