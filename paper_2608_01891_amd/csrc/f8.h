// Rows in 8 bits: e4m3 codes and a power of two.
#pragma once
#include <type_traits>

#include "common.h"

namespace aflex {

constexpr int kLeastRowExp = -100;

// Least e >= kLeastRowExp with m <= 448 2^e, from the fp32 bits of m >= 0 (finite):
// 448 = 1.75 2^8, and the added 2^21 - 1 carries into the exponent's bits where the
// mantissa is above 1.75.
__device__ __forceinline__ int row_exponent(uint32_t m) {
  return max((int)((m + 0x1fffffu) >> 23) - 135, kLeastRowExp);
}

__device__ __forceinline__ float exp2_whole(int n) { return __int_as_float((n + 127) << 23); }  // -126 <= n <= 127

// Codes of a and b in the low (HIGH: high) half of `old`. The conversion rounds to
// nearest, ties to even; what it gets is at most 448 where it is finite, and a NaN
// for anything else.
template <bool HIGH>
__device__ __forceinline__ uint32_t two_codes(float a, float b, uint32_t old) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, HIGH);
}

__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
  return two_codes<true>(c, d, two_codes<false>(a, b, 0));
}

// x 2^-e of a row whose finite values are at most 448 2^e; NaN for the others (inf
// would have no code of its own).
__device__ __forceinline__ float scaled(float x, float inv) {
  const float y = x * inv;
  return fabsf(y) <= 448.f ? y : __builtin_nanf("");
}

// Largest of the values of N neighbouring lanes (4, 8 or 16, from a multiple of N), in all of them.
template <int N>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
  const auto join = [&](auto dpp) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(dpp)::value, 0xf, 0xf, false));
  };
  join(std::integral_constant<int, 0xB1>{});                          // quad_perm [1, 0, 3, 2]
  join(std::integral_constant<int, 0x4E>{});                          // quad_perm [2, 3, 0, 1]
  if constexpr (N >= 8) join(std::integral_constant<int, 0x141>{});   // row_half_mirror
  if constexpr (N >= 16) join(std::integral_constant<int, 0x140>{});  // row_mirror
  return v;
}

// Magnitude bits of x where it is finite, else 0.
__device__ __forceinline__ uint32_t finite_mag(float x) {
  const uint32_t m = __float_as_uint(x) & 0x7fffffffu;
  return m < 0x7f800000u ? m : 0u;
}

}  // namespace aflex
