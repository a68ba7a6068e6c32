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
// chunks (which channels: the caller's business), 64 / U rows at a time;
// D = 128: lane = (row r, unit u) holds rows r and r + 8, D = 64: row r.
template <int D>
struct TileLanes {
  static constexpr int U = D / 16;   // lanes per row
  static constexpr int NR = D / 64;  // rows per lane
  static constexpr int RS = 16 / NR; // row stride between a lane's rows
};

__device__ __forceinline__ int max_mag(const uint4& v, int m) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m = max(m, (int)(w[i] & 0x7fffu));
    m = max(m, (int)((w[i] >> 16) & 0x7fffu));
  }
  return m;
}

// Least e >= kLeastExp with every magnitude below 2^e, from the largest
// magnitude's finite bf16 bits.
__device__ __forceinline__ int exponent_above(int mag_bits) { return max((mag_bits >> 7) - 126, kLeastExp); }

__device__ __forceinline__ float two_to(int n) { return __int_as_float((n + 127) << 23); }  // -126 <= n <= 127

// Summary of the tile whose rows the wave holds in `row` (chunk 0 and 1 of each
// of the lane's rows; their channels start at d0 and d1). Writes the codes to
// keys[0, D) and the exponent to *exp. Whole numbers throughout: each key value
// is rounded to a multiple of 2^(e - 14) below 2^14 in magnitude, 16 of them
// add up to less than 2^18, which fp32 holds exactly in any order. The rows are
// added by halving: at each step a lane gives away half of its channels, so
// that 14 (D = 128) or 15 exchanges replace 48 or 64.
template <int D>
__device__ __forceinline__ void block_codes(const uint4 (&row)[D / 64][2], int d0, int d1, int lane, int8_t* keys,
                                            int8_t* exp) {
  constexpr int NR = TileLanes<D>::NR, U = TileLanes<D>::U;
  int mag = 0;
#pragma unroll
  for (int i = 0; i < NR; ++i) mag = max_mag(row[i][1], max_mag(row[i][0], mag));
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) mag = max(mag, __shfl_xor(mag, o));
  const bool fine = mag < 0x7f80;
  const int e = exponent_above(mag);
  const float f = fine ? two_to(14 - e) : 0.f;
  float s[16];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const uint4& v = row[i][c];
        const uint32_t w = j < 2 ? v.x : j < 4 ? v.y : j < 6 ? v.z : v.w;
        t += rintf(__uint_as_float((j & 1) ? (w & 0xffff0000u) : (w << 16)) * f);
      }
      s[c * 8 + j] = t;
    }
  }
  int d = (lane & U) ? d1 : d0;
  constexpr int STEPS = D == 128 ? 3 : 4;
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const int half = 8 >> k;
    const bool up = lane & (U << k);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < half) {
        const float keep = up ? s[i + half] : s[i], give = up ? s[i] : s[i + half];
        s[i] = keep + __shfl_xor(give, U << k);
      }
    }
    if (k > 0 && up) d += half;
  }
  constexpr int NE = 16 >> STEPS;  // channels d .. d + NE of the finished sums
  float big = 0.f;
#pragma unroll
  for (int i = 0; i < NE; ++i) big = fmaxf(big, fabsf(s[i]));
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) big = fmaxf(big, __shfl_xor(big, o));
  const int r = max((__float_as_int(big) >> 23) - 126 - 7, 0);
  const float g = two_to(-r);
  int code[NE];
#pragma unroll
  for (int i = 0; i < NE; ++i) code[i] = fine ? (int)fminf(fmaxf(rintf(s[i] * g), -127.f), 127.f) : 0;
  if constexpr (NE == 2)
    *reinterpret_cast<uint16_t*>(keys + d) = (uint16_t)((code[0] & 0xff) | (code[1] << 8));
  else
    keys[d] = (int8_t)code[0];
  if (lane == 0) *exp = (int8_t)(fine ? e - 18 + r : kExpAlways);
}

}  // namespace aflex
