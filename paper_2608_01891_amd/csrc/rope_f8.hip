// Rotation of new tokens' queries and keys on the way into an 8-bit paged KV
// cache, gfx950: e4m3 codes and one power of two per (token, kv head, K or V).
//
// The rotation is that of the bf16 writes (rope.hip); a rotated key stays in fp32
// until its one rounding to 8 bits. A row's exponent is the least that fits its
// largest magnitude, so the row's lanes exchange that maximum (3 steps inside a
// DPP row, no LDS), and scaling by the power of two is exact.
#include "block_codes.h"
#include "f8.h"
#include "kernels.h"
#include "profile.h"
#include "rope_unit.h"

namespace aflex {

// Exponent of the row whose lanes (N neighbours) hold 16 channels each.
template <int N>
__device__ __forceinline__ int unit_row_exponent(const float (&v)[16]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = max(m, finite_mag(v[i]));
  return row_exponent(lanes_max<N>(m));
}

__device__ __forceinline__ uint2 eight_codes(const float* v, float inv) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = scaled(v[i], inv);
  return make_uint2(four_codes(y[0], y[1], y[2], y[3]), four_codes(y[4], y[5], y[6], y[7]));
}

// ---------------------------------------------------------------------------
// One token per sequence: the first B Hkv waves take a (sequence, kv head) each,
// the key by the lanes of a row and the value by all 64, which spread its codes
// over a column of the V tile; the other waves rotate queries, a unit per lane.
// Bound by latency (sequence, block, row, store): 64 sequences of 64 / 8 heads x 128
// take 6.0 us; their 2.5 MB take 0.5 at the rate of a copy.
template <int D, bool INTER>
__global__ __launch_bounds__(256) void rope_append_f8_kernel(aflex_rope_f8_args a) {
  constexpr int U = TileLanes<D>::U, NR = TileLanes<D>::NR;
  const int lane = threadIdx.x & 63;
  const long long wave = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const long long nkv = (long long)a.B * a.Hkv;
  const int rot = a.rotary_dim;
  const int cap = a.max_blocks_per_seq * 16;
  if (wave >= nkv) {
    const long long idx = (wave - nkv) * 64 + lane;
    if (idx >= (long long)a.B * a.Hq * U) return;
    const int u = (int)(idx % U);
    const long long bh = idx / U;
    const int b = (int)(bh / a.Hq), h = (int)(bh - (long long)b * a.Hq);
    int d0, d1;
    unit_channels<INTER>(u, rot, d0, d1);
    const uint16_t* src = a.q + (size_t)b * a.q_stride + (size_t)h * D;
    uint4 x = ld4(src + d0), y = ld4(src + d1);
    const int ctx = a.context_lens[b];
    if (ctx <= 0 || ctx > cap) return;
    if (rot > 0) {
      const int pos = a.positions ? a.positions[b] : ctx - 1;
      if (pos < 0 || pos >= a.rope_len) return;
      if (u * 16 < rot) rotate_unit<INTER>(x, y, load_angles(a.rope, pos, rot, u));
    }
    uint16_t* dst = a.q_out + (size_t)bh * D;
    st4(dst + d0, x);
    st4(dst + d1, y);
    return;
  }
  const int b = (int)(wave / a.Hkv), g = (int)(wave - (long long)b * a.Hkv);
  const int u = lane % U;  // (every row of lanes holds the same key)
  int d0, d1;
  unit_channels<INTER>(u, rot, d0, d1);
  const uint16_t* ks = a.k_new + (size_t)b * a.k_stride + (size_t)g * D;
  const uint4 x = ld4(ks + d0), y = ld4(ks + d1);
  const uint16_t* vs = a.v_new + (size_t)b * a.v_stride + (size_t)g * D;
  float vv[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) vv[i] = bf2f(vs[i * 64 + lane]);
  const int ctx = a.context_lens[b];
  if (ctx <= 0 || ctx > cap) return;
  const int j = ctx - 1, o = j % 16;
  const int blk = a.block_table[(size_t)b * a.max_blocks_per_seq + j / 16];
  const int pos = rot > 0 && a.positions ? a.positions[b] : j;
  if (rot > 0 && (pos < 0 || pos >= a.rope_len)) return;
  if (blk < 0 || blk >= a.num_blocks) return;
  const size_t tile = (size_t)blk * a.Hkv + g;
  float k[16];
  unpack_unit(x, y, k);
  if (rot > 0 && u * 16 < rot) rotate_unit<INTER>(k, load_angles(a.rope, pos, rot, u));
  const int ke = unit_row_exponent<U>(k);
  const float kinv = exp2_whole(-ke);
  if (lane < U) {
    uint8_t* kt = a.k_cache + tile * 16 * D + o * D;
    *reinterpret_cast<uint2*>(kt + d0) = eight_codes(k, kinv);
    *reinterpret_cast<uint2*>(kt + d1) = eight_codes(k + 8, kinv);
  }
  uint32_t vm = 0;
#pragma unroll
  for (int i = 0; i < NR; ++i) vm = max(vm, finite_mag(vv[i]));
  const int ve = row_exponent((uint32_t)wave_max((int)vm));
  const float vinv = exp2_whole(-ve);
  uint8_t* vt = a.v_cache + tile * D * 16 + o;
#pragma unroll
  for (int i = 0; i < NR; ++i) vt[(i * 64 + lane) * 16] = (uint8_t)two_codes<false>(scaled(vv[i], vinv), 0.f, 0);
  if (lane < 2) a.kv_exp[tile * 32 + lane * 16 + o] = (int8_t)(lane ? ve : ke);
}

// ---------------------------------------------------------------------------
// Packed prompts, chunks and drafts: grid (block slot, part, sequence) as in the
// bf16 write. Bound by memory: prompts of 9518 tokens, 64 / 8 heads x 128, 371 MB in
// 78.0 us, 4.75 TB/s, as a large copy.
// A wave takes up to kHeadsPerWaveF8 heads with the angles it has loaded (the mixed
// prompts: 1 head 89.3 us, 2 81.6, 4 78.0, 8 89.2), one where that leaves few waves (61
// drafts: 6.7 us, 6.9 with 4). A handful of drafts is bound by its chain of loads: the
// sequence's numbers, block and rows, angles.
constexpr int kHeadsPerWaveF8 = 4;
constexpr long long kManyWavesF8 = 16384;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A wave's codes to the V tiles: its lanes hold 16 tokens x 8 channels each (`row`: a
// token's 8 bf16 values), which are 64 x 8 rows of 16 bytes, one behind the other in
// memory, `rows` of them in all at vt. The lanes exchange them through LDS (8 KiB at
// sm; row e of lane t sits at e ^ (t & 7)), so that a store covers 1 KiB without gaps. Where
// only some tokens are written (`live`), the rows' other bytes are read and written
// back: they belong to the block, which nobody else writes. (Byte by byte, the 20
// stores of a lane and channel, each of a wave to 64 lines, made 61 drafts 8.2 us.)
__device__ __forceinline__ void store_v_codes(const uint4 (&row)[16], const float (&inv)[16], uint8_t* vt, int rows,
                                              uint32_t live, uint8_t* sm) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float y[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint4& r = row[4 * i + t];
        const uint32_t c = e < 2 ? r.x : e < 4 ? r.y : e < 6 ? r.z : r.w;
        y[t] = scaled(e & 1 ? hi_f(c) : lo_f(c), inv[4 * i + t]);
      }
      w[i] = four_codes(y[0], y[1], y[2], y[3]);
    }
    *reinterpret_cast<u32x4*>(sm + lane * 128 + ((e ^ (lane & 7)) << 4)) = w;
  }
  u32x4 old[8];
  if (live != 0xffffu) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i * 64 + lane < rows) old[i] = *reinterpret_cast<const u32x4*>(vt + (i * 64 + lane) * 16);
  }
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the lanes are of one wave
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int at = i * 64 + lane, from = at >> 3;
    u32x4 w = *reinterpret_cast<const u32x4*>(sm + from * 128 + (((at & 7) ^ (from & 7)) << 4));
    if (live != 0xffffu) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t here = live >> (4 * k) & 0xfu;  // a byte of ones for each token that is written
        const uint32_t mask = ((here * 0x00204081u) & 0x01010101u) * 0xffu;
        w[k] = (w[k] & mask) | (old[i][k] & ~mask);
      }
    }
    if (at < rows) *reinterpret_cast<u32x4*>(vt + at * 16) = w;
  }
}

template <int D, bool INTER>
__global__ __launch_bounds__(256) void rope_write_f8_kernel(aflex_rope_f8_args a, int vparts, int kparts, int per_wave) {
  constexpr int U = TileLanes<D>::U, NR = TileLanes<D>::NR, RS = TileLanes<D>::RS;
  Slot s;
  if (!find_slot(a, blockIdx.z, blockIdx.x, s)) return;
  int part = blockIdx.y;
  const int rot = a.rotary_dim;
  if (part < vparts) {
    // V: a thread per (kv head, 8 channels) with the block's rows. (They and the positions
    // are loaded beside the block's id, which is looked at behind them.)
    constexpr int C = D / 8;
    const int t = part * 256 + threadIdx.x;
    const int g = t / C, c = t % C;
    // Rows that are written, the same for all threads: a lane looks at each (one after
    // the other, their positions took 16 rounds to memory).
    const int pos = slot_pos(a, s, threadIdx.x & 15);
    const uint16_t* src = a.v_new + (size_t)min(g, a.Hkv - 1) * D + c * 8;
    // (rows that do not exist repeat one that does)
    uint4 row[16];
#pragma unroll
    for (int o = 0; o < 16; ++o) row[o] = ld4(src + (size_t)(s.src + min(max(o, s.o0), s.o1 - 1)) * a.v_stride);
    const uint32_t live = (uint32_t)__ballot(pos >= 0) & 0xffffu;
    if (s.blk < 0 || live == 0) return;  // (all lanes stay: they store for each other)
    const size_t tile = (size_t)s.blk * a.Hkv + g;
    float inv[16];
    uint32_t ew[4] = {0, 0, 0, 0};
#pragma unroll
    for (int o = 0; o < 16; ++o) {
      const uint32_t w[4] = {row[o].x, row[o].y, row[o].z, row[o].w};
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) m = max(m, max(finite_mag(lo_f(w[i])), finite_mag(hi_f(w[i]))));
      const int e = row_exponent(lanes_max<C>(m));
      inv[o] = exp2_whole(-e);
      ew[o / 4] |= (uint32_t)(e & 0xff) << (8 * (o & 3));
    }
    const int wave0 = (int)((t & ~63) * 8);  // channel of the wave's first row, all heads'
    extern __shared__ __attribute__((aligned(16))) uint8_t sm[];
    store_v_codes(row, inv, a.v_cache + ((size_t)s.blk * a.Hkv * D + wave0) * 16, a.Hkv * D - wave0, live,
                  sm + (threadIdx.x >> 6) * 8192);
    if (c == 0 && g < a.Hkv) {
      int8_t* ex = a.kv_exp + tile * 32 + 16;
      if (live == 0xffffu) {
        *reinterpret_cast<uint4*>(ex) = make_uint4(ew[0], ew[1], ew[2], ew[3]);
      } else {
#pragma unroll
        for (int o = 0; o < 16; ++o)
          if (live >> o & 1u) ex[o] = (int8_t)(ew[o / 4] >> (8 * (o & 3)));
      }
    }
    return;
  }
  part -= vparts;
  const bool key = part < kparts;
  if (!key) part -= kparts;
  const int heads = key ? a.Hkv : a.Hq;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int h0 = (part * 4 + wave) * per_wave, h1 = min(h0 + per_wave, heads);
  if (h0 >= h1) return;
  const int u = lane % U, r = lane / U;
  int d0, d1;
  unit_channels<INTER>(u, rot, d0, d1);
  const size_t stride = key ? a.k_stride : a.q_stride;
  const uint16_t* base = key ? a.k_new : a.q;
  auto load = [&](int h, uint4(&row)[NR][2]) {
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int o = r + i * RS;  // (rows that exist, whether or not their position does)
      if (o < s.o0 || o >= s.o1) continue;
      const uint16_t* p = base + (size_t)(s.src + o) * stride + (size_t)h * D;
      row[i][0] = ld4(p + d0);
      row[i][1] = ld4(p + d1);
    }
  };
  uint4 next[NR][2] = {};
  load(h0, next);
  int pos[NR];
  Angles an[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    pos[i] = slot_pos(a, s, r + i * RS);
    if (pos[i] >= 0 && u * 16 < rot) an[i] = load_angles(a.rope, pos[i], rot, u);
  }
  if (key && s.blk < 0) return;
  for (int h = h0; h < h1; ++h) {
    uint4 row[NR][2];
#pragma unroll
    for (int i = 0; i < NR; ++i) row[i][0] = next[i][0], row[i][1] = next[i][1];
    if (h + 1 < h1) load(h + 1, next);
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int o = r + i * RS;
      if (!key) {
        if (pos[i] < 0) continue;
        if (u * 16 < rot) rotate_unit<INTER>(row[i][0], row[i][1], an[i]);
        uint16_t* dst = a.q_out + ((size_t)(s.src + o) * a.Hq + h) * D;
        st4(dst + d0, row[i][0]);
        st4(dst + d1, row[i][1]);
        continue;
      }
      // (a row's lanes share its position: all of them go on, or none)
      if (pos[i] < 0) continue;
      float k[16];
      unpack_unit(row[i][0], row[i][1], k);
      if (u * 16 < rot) rotate_unit<INTER>(k, an[i]);
      const int e = unit_row_exponent<U>(k);
      const float inv = exp2_whole(-e);
      const size_t tile = (size_t)s.blk * a.Hkv + h;
      uint8_t* kt = a.k_cache + (tile * 16 + o) * D;
      *reinterpret_cast<uint2*>(kt + d0) = eight_codes(k, inv);
      *reinterpret_cast<uint2*>(kt + d1) = eight_codes(k + 8, inv);
      if (u == 0) a.kv_exp[tile * 32 + o] = (int8_t)e;
    }
  }
}

// ---------------------------------------------------------------------------
// Host side.
hipError_t launch_rope_append_f8(const aflex_rope_f8_args& in, hipStream_t stream) {
  const aflex_rope_f8_args a = with_strides(in);
  const long long waves = (long long)a.B * a.Hkv + ((long long)a.B * a.Hq * (a.D / 16) + 63) / 64;
  const unsigned grid = (unsigned)((waves + 3) / 4);
  ProfScope ps("rope_append_f8", stream);
  if (a.D == 128 && a.interleaved)
    rope_append_f8_kernel<128, true><<<grid, 256, 0, stream>>>(a);
  else if (a.D == 128)
    rope_append_f8_kernel<128, false><<<grid, 256, 0, stream>>>(a);
  else if (a.interleaved)
    rope_append_f8_kernel<64, true><<<grid, 256, 0, stream>>>(a);
  else
    rope_append_f8_kernel<64, false><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_rope_write_f8(const aflex_rope_f8_args& in, hipStream_t stream) {
  if (in.T == 0 || in.max_seqlen == 0) return hipSuccess;
  const aflex_rope_f8_args a = with_strides(in);
  const int vparts = (a.Hkv * (a.D / 8) + 255) / 256;
  const int slots = (a.max_seqlen + 15) / 16 + 1;
  const int per_wave = (long long)slots * a.B * (a.Hq + a.Hkv) >= kManyWavesF8 * kHeadsPerWaveF8 ? kHeadsPerWaveF8 : 1;
  const int per = 4 * per_wave;
  const int kparts = (a.Hkv + per - 1) / per, qparts = (a.Hq + per - 1) / per;
  const dim3 grid(slots, vparts + kparts + qparts, a.B);
  const size_t lds = 4 * 8192;  // the exchange of V rows
  ProfScope ps("rope_write_f8", stream);
  if (a.D == 128 && a.interleaved)
    rope_write_f8_kernel<128, true><<<grid, 256, lds, stream>>>(a, vparts, kparts, per_wave);
  else if (a.D == 128)
    rope_write_f8_kernel<128, false><<<grid, 256, lds, stream>>>(a, vparts, kparts, per_wave);
  else if (a.interleaved)
    rope_write_f8_kernel<64, true><<<grid, 256, lds, stream>>>(a, vparts, kparts, per_wave);
  else
    rope_write_f8_kernel<64, false><<<grid, 256, lds, stream>>>(a, vparts, kparts, per_wave);
  return hipGetLastError();
}

}  // namespace aflex
