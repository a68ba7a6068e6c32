// What the writes of rotated tokens share: the 16 channels of a row that a lane
// turns, and the rows of a cache block that a packed prompt writes.
#pragma once
#include "common.h"

namespace aflex {

// Channels of unit u's two chunks: partners half a rotation apart, or 16
// neighbours (interleaved pairs, and the channels that are not rotated).
template <bool INTER>
__device__ __forceinline__ void unit_channels(int u, int rot, int& d0, int& d1) {
  const bool apart = !INTER && u * 16 < rot;
  d0 = apart ? u * 8 : u * 16;
  d1 = apart ? u * 8 + rot / 2 : u * 16 + 8;
}

struct Angles {
  float4 c[2], s[2];  // cosines and sines of the unit's 8 pairs
};

__device__ __forceinline__ Angles load_angles(const float* rope, int pos, int rot, int u) {
  const float* p = rope + (size_t)pos * rot + u * 8;
  const float* q = p + rot / 2;
  Angles a;
  a.c[0] = *reinterpret_cast<const float4*>(p);
  a.c[1] = *reinterpret_cast<const float4*>(p + 4);
  a.s[0] = *reinterpret_cast<const float4*>(q);
  a.s[1] = *reinterpret_cast<const float4*>(q + 4);
  return a;
}

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf(float lo, float hi) {
  return (uint32_t)f2bf(lo) | ((uint32_t)f2bf(hi) << 16);
}

__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
#pragma clang fp contract(off)
  const float x = a * c - b * s;
  const float y = b * c + a * s;
  a = x;
  b = y;
}

// Rotates a unit in place: x, y its two chunks.
template <bool INTER>
__device__ __forceinline__ void rotate_unit(uint4& x, uint4& y, const Angles& an) {
  const float c[8] = {an.c[0].x, an.c[0].y, an.c[0].z, an.c[0].w, an.c[1].x, an.c[1].y, an.c[1].z, an.c[1].w};
  const float s[8] = {an.s[0].x, an.s[0].y, an.s[0].z, an.s[0].w, an.s[1].x, an.s[1].y, an.s[1].z, an.s[1].w};
  uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
  if constexpr (INTER) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float a = lo_f(w[i]), b = hi_f(w[i]);
      turn(a, b, c[i], s[i]);
      w[i] = pack_bf(a, b);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a0 = lo_f(w[i]), a1 = hi_f(w[i]), b0 = lo_f(w[4 + i]), b1 = hi_f(w[4 + i]);
      turn(a0, b0, c[2 * i], s[2 * i]);
      turn(a1, b1, c[2 * i + 1], s[2 * i + 1]);
      w[i] = pack_bf(a0, a1);
      w[4 + i] = pack_bf(b0, b1);
    }
  }
  x = make_uint4(w[0], w[1], w[2], w[3]);
  y = make_uint4(w[4], w[5], w[6], w[7]);
}

// The same without the rounding to bf16: v holds the unit's 16 channels in order,
// chunk 0 and chunk 1.
template <bool INTER>
__device__ __forceinline__ void rotate_unit(float (&v)[16], const Angles& an) {
  const float c[8] = {an.c[0].x, an.c[0].y, an.c[0].z, an.c[0].w, an.c[1].x, an.c[1].y, an.c[1].z, an.c[1].w};
  const float s[8] = {an.s[0].x, an.s[0].y, an.s[0].z, an.s[0].w, an.s[1].x, an.s[1].y, an.s[1].z, an.s[1].w};
#pragma unroll
  for (int i = 0; i < 8; ++i) turn(v[INTER ? 2 * i : i], v[INTER ? 2 * i + 1 : 8 + i], c[i], s[i]);
}

__device__ __forceinline__ void unpack_unit(const uint4& x, const uint4& y, float (&v)[16]) {
  const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) v[2 * i] = lo_f(w[i]), v[2 * i + 1] = hi_f(w[i]);
}

__device__ __forceinline__ uint4 ld4(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void st4(uint16_t* p, const uint4& v) { *reinterpret_cast<uint4*>(p) = v; }

struct Slot {
  int blk;         // pool block, or -1
  int jb;          // logical block
  int o0, o1;      // its new rows [o0, o1)
  long long src;   // token row of the block's row 0 (rows outside [o0, o1) do not exist)
};

template <class Args>
__device__ __forceinline__ bool find_slot(const Args& a, int b, int jj, Slot& s) {
  int s1 = a.cu_seqlens[b + 1], s0 = a.cu_seqlens[b];
  s1 = min(max(s1, 0), a.T);
  s0 = min(max(s0, 0), s1);
  const int n = s1 - s0, ctx = a.context_lens[b];
  if (n <= 0 || ctx <= 0 || ctx > a.max_blocks_per_seq * 16) return false;
  const int start = ctx - n;
  s.jb = max(start, 0) / 16 + jj;
  const int lo = max(s.jb * 16, max(start, 0)), hi = min(s.jb * 16 + 16, ctx);
  if (lo >= hi) return false;
  s.o0 = lo - s.jb * 16;
  s.o1 = hi - s.jb * 16;
  s.src = (long long)s0 - start + s.jb * 16;
  s.blk = a.block_table[(size_t)b * a.max_blocks_per_seq + s.jb];
  if (s.blk < 0 || s.blk >= a.num_blocks) s.blk = -1;
  return true;
}

// Position of row o's token, or -1 where the token is left alone.
template <class Args>
__device__ __forceinline__ int slot_pos(const Args& a, const Slot& s, int o) {
  if (o < s.o0 || o >= s.o1) return -1;
  if (a.rotary_dim == 0) return 0;
  const int p = a.positions ? a.positions[s.src + o] : s.jb * 16 + o;
  return p >= 0 && p < a.rope_len ? p : -1;
}

// The strides that 0 stands for.
template <class Args>
inline Args with_strides(Args a) {
  if (a.q_stride == 0) a.q_stride = a.Hq * a.D;
  if (a.k_stride == 0) a.k_stride = a.Hkv * a.D;
  if (a.v_stride == 0) a.v_stride = a.Hkv * a.D;
  return a;
}

}  // namespace aflex
