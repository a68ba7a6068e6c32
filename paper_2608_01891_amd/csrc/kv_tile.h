// Whole blocks into the token-fastest V tile: shared by the cache writes.
#pragma once
#include "common.h"

namespace aflex {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t chunk_word(const uint4& v, int i) {
  return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}

// A thread's 8 channels of the 16 tokens of a block (row) to its 8 rows of the V
// tile, 256 contiguous bytes at vc. exchange: the 16 threads of a group (4 KiB
// of contiguous V rows, lanes of one wave) exchange through LDS, so that a store
// of theirs covers 256 contiguous bytes instead of 16 in every 256, with 4 KiB
// of LDS per group at sm; or with HALVES 128 contiguous bytes, with 2 KiB.
template <bool HALVES = false>
__device__ __forceinline__ void store_v_rows(const uint4 (&row)[16], uint16_t* vc, bool exchange, uint8_t* sm) {
  uint4 out[16];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
    uint32_t r[8];
#pragma unroll
    for (int o = 0; o < 8; ++o)
      r[o] = __builtin_amdgcn_perm(chunk_word(row[2 * o + 1], e >> 1), chunk_word(row[2 * o], e >> 1), sel);
    out[2 * e] = make_uint4(r[0], r[1], r[2], r[3]);
    out[2 * e + 1] = make_uint4(r[4], r[5], r[6], r[7]);
  }
  const int t = threadIdx.x & 15;
  if (HALVES && exchange) {
    uint8_t* grp = sm + (threadIdx.x >> 4) * 2048;
    const int x = t & 7;
    uint16_t* vt = vc - t * 128 + x * 8;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      // Piece y of this half of thread t sits at y ^ (t & 7).
#pragma unroll
      for (int y = 0; y < 8; ++y) *reinterpret_cast<uint4*>(grp + t * 128 + ((y ^ x) << 4)) = out[p * 8 + y];
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the 16 threads are lanes of one wave
      __builtin_amdgcn_wave_barrier();
      u32x4 got[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int from = 2 * i + (t >> 3);
        got[i] = *reinterpret_cast<const u32x4*>(grp + from * 128 + ((x ^ (from & 7)) << 4));
      }
      __builtin_amdgcn_s_waitcnt(0xc07f);  // read before the second half is written
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < 8; ++i)
        *reinterpret_cast<u32x4*>(vt + (2 * i + (t >> 3)) * 128 + p * 64) = got[i];
    }
  } else if (exchange) {
    // Piece x of thread t sits at x ^ t.
    uint8_t* grp = sm + (threadIdx.x >> 4) * 4096;
#pragma unroll
    for (int x = 0; x < 16; ++x) *reinterpret_cast<uint4*>(grp + t * 256 + ((x ^ t) << 4)) = out[x];
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the 16 threads are lanes of one wave
    __builtin_amdgcn_wave_barrier();
    uint16_t* vt = vc - t * 128;  // the first thread's bytes
#pragma unroll
    for (int i = 0; i < 16; ++i)
      *reinterpret_cast<uint4*>(vt + i * 128 + t * 8) = *reinterpret_cast<const uint4*>(grp + i * 256 + ((t ^ i) << 4));
  } else {
#pragma unroll
    for (int x = 0; x < 16; ++x) *reinterpret_cast<uint4*>(vc + x * 8) = out[x];
  }
}

// The same for the tokens of `live` alone (bit o: token o, uniform): 8 of them in
// one 16-byte store where all are written, pairs in one of 4 bytes. (Token by
// token, the 128 two-byte stores of a thread, each of a wave to 64 lines, were
// 5 us of a 9 us launch.)
__device__ __forceinline__ void store_v_part(const uint4 (&row)[16], uint16_t* vc, uint32_t live) {
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const uint32_t here = live >> (8 * half) & 0xffu;
    if (here == 0) continue;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t sel = (e & 1) ? 0x07060302u : 0x05040100u;
      u32x4 r;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        r[i] = __builtin_amdgcn_perm(chunk_word(row[8 * half + 2 * i + 1], e >> 1),
                                     chunk_word(row[8 * half + 2 * i], e >> 1), sel);
      uint16_t* dst = vc + e * 16 + 8 * half;
      if (here == 0xffu) {
        *reinterpret_cast<u32x4*>(dst) = r;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t two = here >> (2 * i) & 3u;
          if (two == 3)
            *reinterpret_cast<uint32_t*>(dst + 2 * i) = r[i];
          else if (two == 1)
            dst[2 * i] = (uint16_t)r[i];
          else if (two == 2)
            dst[2 * i + 1] = (uint16_t)(r[i] >> 16);
        }
      }
    }
  }
}

}  // namespace aflex
