// One wave and one (cache block, kv head) tile of 16 keys: the lane layout and
// the tile's whole-number summary. Shared by the kernels that write keys and
// by the one that summarises blocks already written.
#pragma once
#include "common.h"

namespace aflex {

constexpr int kLeastExp = -100;  // exponents of summaries and queries are not below this
constexpr int kExpAlways = 127;  // block_exp of a block that holds a non-finite key

__device__ __forceinline__ int nblk16(int ctx) { return (ctx + 15) >> 4; }

// Lane layout: U = D / 16 lanes hold a row, 16 elements each in two 16-byte
// chunks (which channels: the caller's business), 64 / U rows at a time: lane
// (row r, unit u) = r U + u holds row r, for D = 128 rows r and r + 8.
template <int D>
struct TileLanes {
  static constexpr int U = D / 16;   // lanes per row
  static constexpr int NR = D / 64;  // rows per lane
  static constexpr int RS = 16 / NR; // row stride between a lane's rows
};

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// Largest magnitude bits of pairs of bf16 values, the two halves apart.
__device__ __forceinline__ u16x2 max_mag2(uint32_t w, u16x2 m) {
  return __builtin_elementwise_max(__builtin_bit_cast(u16x2, w & 0x7fff7fffu), m);
}

__device__ __forceinline__ int max_mag(const uint4& v, int m) {
  u16x2 p = {0, 0};
  p = max_mag2(v.x, max_mag2(v.y, max_mag2(v.z, max_mag2(v.w, p))));
  return max(m, (int)max(p[0], p[1]));
}

// Largest of the wave's values, none negative, in every lane (a scalar).
__device__ __forceinline__ int wave_max(int v) {
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));  // row_shr 1
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));  // row_shr 2
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));  // row_shr 4
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));  // row_shr 8
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));  // row_bcast 15
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));  // row_bcast 31
  return __builtin_amdgcn_readlane(v, 63);
}

// Halving sum over lanes that differ in bit M of their number: lanes without
// the bit get lo of both, lanes with it hi of both. (Unsigned, as all sums here:
// bits of two's complement, which may pass 2^31 on the way.)
template <int M>
__device__ __forceinline__ uint32_t halve(uint32_t lo, uint32_t hi, int lane) {
  if constexpr (M == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(lo, hi, false, false);
    return r[0] + r[1];
  } else if constexpr (M == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(lo, hi, false, false);
    return r[0] + r[1];
  } else {
    const bool up = lane & M;
    const uint32_t keep = up ? hi : lo, give = up ? lo : hi;
    if constexpr (M == 8)
      return keep + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)give, 0x128, 0xf, 0xf, false);  // row_ror 8
    return keep + __shfl_xor(give, M);
  }
}

// Least e >= kLeastExp with every magnitude below 2^e, from the largest
// magnitude's finite bf16 bits.
__device__ __forceinline__ int exponent_above(int mag_bits) { return max((mag_bits >> 7) - 126, kLeastExp); }

__device__ __forceinline__ float two_to(int n) { return __int_as_float((n + 127) << 23); }  // -126 <= n <= 127

// Summary of the tile whose rows the wave holds in `row` (chunk 0 and 1 of each
// of the lane's rows; their channels start at d0 and d1). Writes the codes to
// keys[0, D) and the exponent to *exp. Whole numbers throughout: a key value
// times 2^(14 - e) is below 2^14, and adding it to 1.5 2^23 in one fused step
// rounds it to a whole number (nearest, ties to even), which is then the
// difference of the bit patterns: one instruction to round, and sums of
// integers, the same in any order. The rows are added by halving: at each step
// a lane gives away half of its channels, 14 (D = 128) or 15 exchanges instead
// of 48 or 64, most of them without LDS. (With float sums and __shfl_xor 366 MB of
// keys took 165 us, so 78; about 200 vector instructions per 4 KiB tile.)
template <int D>
__device__ __forceinline__ void block_codes(const uint4 (&row)[D / 64][2], int d0, int d1, int lane, int8_t* keys,
                                            int8_t* exp) {
  constexpr int NR = TileLanes<D>::NR;
  constexpr uint32_t kOne = 0x4b400000;  // bits of 1.5 2^23
  u16x2 m2 = {0, 0};
#pragma unroll
  for (int i = 0; i < NR; ++i)
#pragma unroll
    for (int c = 0; c < 2; ++c)
      m2 = max_mag2(row[i][c].x, max_mag2(row[i][c].y, max_mag2(row[i][c].z, max_mag2(row[i][c].w, m2))));
  const int mag = wave_max(max(m2[0], m2[1]));
  const bool fine = mag < 0x7f80;
  const int e = exponent_above(mag);
  const float f = two_to(14 - e);
  uint32_t s[16];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t t = 0;
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const uint4& v = row[i][c];
        const uint32_t w = j < 2 ? v.x : j < 4 ? v.y : j < 6 ? v.z : v.w;
        const float k = __uint_as_float((j & 1) ? (w & 0xffff0000u) : (w << 16));
        t += __float_as_uint(fmaf(k, f, __uint_as_float(kOne)));
      }
      s[c * 8 + j] = t - NR * kOne;
    }
  }
  uint32_t a[8], b[4], h[2];
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = halve<32>(s[i], s[i + 8], lane);
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = halve<16>(a[i], a[i + 4], lane);
#pragma unroll
  for (int i = 0; i < 2; ++i) h[i] = halve<8>(b[i], b[i + 2], lane);
  int d = (lane & 32 ? d1 : d0) + (lane & 16 ? 4 : 0) + (lane & 8 ? 2 : 0);
  if constexpr (D == 64) {
    h[0] = halve<4>(h[0], h[1], lane);
    h[1] = 0;
    d += lane & 4 ? 1 : 0;
  }
  // (magnitudes below 2^18; of a tile that is not fine, any bits)
  const auto size = [](uint32_t x) { return (int)(x >> 31 ? 0u - x : x); };
  const int big = wave_max(max(size(h[0]), size(h[1])));
  const int r = max(32 - __clz(big) - 7, 0);  // (__clz(0) is 32)
  const float g = two_to(-r);
  int code[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) code[i] = fine ? (int)fminf(fmaxf(rintf((float)(int)h[i] * g), -127.f), 127.f) : 0;
  if constexpr (D == 128)
    *reinterpret_cast<uint16_t*>(keys + d) = (uint16_t)((code[0] & 0xff) | (code[1] << 8));
  else
    keys[d] = (int8_t)code[0];
  if (lane == 0) *exp = (int8_t)(fine ? e - 18 + r : kExpAlways);
}

}  // namespace aflex
