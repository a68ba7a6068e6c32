// Rotation of new tokens' queries and keys on the way into the paged KV cache,
// and the summaries of the blocks that get full, gfx950.
//
// Each pair of channels (a, b) at position p turns by the angle whose cosine c
// and sine s the caller's table holds for p: a' = a c - b s, b' = b c + a s in
// fp32 (products and sums rounded one by one, no fused multiply-add, so that
// the rotated bf16 bits are those of the formula read literally), rounded to
// bf16 once. Bound by HBM for prompts (every row is read and written once: 9518
// tokens of 64 + 2 x 8 heads x 128, 395 MB, 82 us, 93% of a copy's rate) and by
// the chain launch -> context length -> block id -> store for single tokens (64
// sequences 3.8 us).
//
// A lane handles a unit of 16 channels of a row: the 8 channels and their 8
// partners (or 16 neighbours), so that a rotation needs no other lane. A wave
// holds the 16 rows of a cache block for one head at a time and goes through a
// few heads with the same angles in registers; for the key heads it then has
// the tile that the summary is made of.
#include "block_codes.h"
#include "kernels.h"
#include "kv_tile.h"
#include "profile.h"

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

__device__ __forceinline__ uint4 ld4(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void st4(uint16_t* p, const uint4& v) { *reinterpret_cast<uint4*>(p) = v; }

// ---------------------------------------------------------------------------
// One token per sequence. The first B Hkv waves take a (sequence, kv head)
// each: the last row's lanes rotate the new key, the lanes spread the value
// over its column of the V tile, and where the token fills its block, the wave
// reads the 15 older keys and writes the summary. The other waves rotate
// queries, a unit per lane.
template <int D, bool INTER>
__global__ __launch_bounds__(256) void rope_append_kernel(aflex_rope_args a) {
  constexpr int U = TileLanes<D>::U, NR = TileLanes<D>::NR, RS = TileLanes<D>::RS;
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
  const int u = lane % U, r = lane / U;
  int d0, d1;
  unit_channels<INTER>(u, rot, d0, d1);
  const uint16_t* ks = a.k_new + (size_t)b * a.k_stride + (size_t)g * D;
  const uint4 nx = ld4(ks + d0), ny = ld4(ks + d1);
  const uint16_t* vs = a.v_new + (size_t)b * a.v_stride + (size_t)g * D;
  uint16_t vv[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) vv[i] = vs[i * 64 + lane];
  const int ctx = a.context_lens[b];
  if (ctx <= 0 || ctx > cap) return;
  const int j = ctx - 1, o = j % 16;
  const int blk = a.block_table[(size_t)b * a.max_blocks_per_seq + j / 16];
  const int pos = rot > 0 && a.positions ? a.positions[b] : j;
  if (rot > 0 && (pos < 0 || pos >= a.rope_len)) return;
  if (blk < 0 || blk >= a.num_blocks) return;
  const size_t tile = (size_t)blk * a.Hkv + g;
  uint16_t* kt = a.k_cache + tile * 16 * D;
  const bool full = o == 15 && a.block_keys;
  uint4 row[NR][2];
  if (full) {
#pragma unroll
    for (int i = 0; i < NR; ++i) {  // (row 15, the last one's lanes, is replaced below)
      row[i][0] = ld4(kt + (r + i * RS) * D + d0);
      row[i][1] = ld4(kt + (r + i * RS) * D + d1);
    }
  }
  uint4 x = nx, y = ny;
  if (rot > 0 && u * 16 < rot) rotate_unit<INTER>(x, y, load_angles(a.rope, pos, rot, u));
  if (r == 0) {
    st4(kt + o * D + d0, x);
    st4(kt + o * D + d1, y);
  }
  uint16_t* vt = a.v_cache + tile * D * 16 + o;
#pragma unroll
  for (int i = 0; i < NR; ++i) vt[(i * 64 + lane) * 16] = vv[i];
  if (full) {
    if (r == RS - 1) {
      row[NR - 1][0] = x;
      row[NR - 1][1] = y;
    }
    block_codes<D>(row, d0, d1, lane, a.block_keys + tile * D, a.block_exp + tile);
  }
}

// ---------------------------------------------------------------------------
// Packed prompts. Grid (block slot, part, sequence): slot jj of sequence b is
// logical block max(start, 0) / 16 + jj, start = ctx_b - n_b, as in the plain
// cache write. The parts share its 16 rows: V (transposed into the
// token-fastest tile), the key heads, the query heads.
// A wave takes up to kHeadsPerWave heads with the angles it has loaded, one where
// that leaves few waves (113 tokens, 32 + 8 heads: 5.3 us, with four heads in a
// row 7.5).
constexpr int kHeadsPerWave = 4;
constexpr long long kManyWaves = 16384;

struct Slot {
  int blk;         // pool block, or -1
  int jb;          // logical block
  int o0, o1;      // its new rows [o0, o1)
  long long src;   // token row of the block's row 0 (rows outside [o0, o1) do not exist)
};

__device__ __forceinline__ bool find_slot(const aflex_rope_args& a, int b, int jj, Slot& s) {
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
__device__ __forceinline__ int slot_pos(const aflex_rope_args& a, const Slot& s, int o) {
  if (o < s.o0 || o >= s.o1) return -1;
  if (a.rotary_dim == 0) return 0;
  const int p = a.positions ? a.positions[s.src + o] : s.jb * 16 + o;
  return p >= 0 && p < a.rope_len ? p : -1;
}

template <int D, bool INTER>
__global__ __launch_bounds__(256) void rope_write_kernel(aflex_rope_args a, int vparts, int kparts,
                                                            int per_wave) {
  constexpr int U = TileLanes<D>::U, NR = TileLanes<D>::NR, RS = TileLanes<D>::RS;
  Slot s;
  if (!find_slot(a, blockIdx.z, blockIdx.x, s)) return;
  int part = blockIdx.y;
  const int rot = a.rotary_dim;
  if (part < vparts) {
    // V: a thread per (kv head, 8 channels) with the block's rows, all loaded
    // before the first is stored
    if (s.blk < 0) return;
    constexpr int C = D / 8;
    extern __shared__ __attribute__((aligned(16))) uint8_t sm[];
    const int t = part * 256 + threadIdx.x;
    const int g = t / C, c = t % C;
    if (g >= a.Hkv) return;
    const uint16_t* src = a.v_new + (size_t)g * D + c * 8;
    uint16_t* vt = a.v_cache + (((size_t)s.blk * a.Hkv + g) * D + c * 8) * 16;
    uint4 row[16];
    uint32_t live = 0;  // rows that are written, the same for all threads
#pragma unroll
    for (int o = 0; o < 16; ++o) live |= slot_pos(a, s, o) >= 0 ? 1u << o : 0u;
    live = __builtin_amdgcn_readfirstlane(live);
    if (live == 0) return;
    // (rows that are not written repeat one that is)
    const int first = __builtin_ctz(live);
#pragma unroll
    for (int o = 0; o < 16; ++o) row[o] = ld4(src + (size_t)(s.src + (live >> o & 1 ? o : first)) * a.v_stride);
    if (live == 0xffffu)
      store_v_rows<true>(row, vt, (t | 15) < a.Hkv * C, sm);
    else
      store_v_part(row, vt, live);
    return;
  }
  part -= vparts;
  const bool key = part < kparts;
  if (!key) part -= kparts;
  const int heads = key ? a.Hkv : a.Hq;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int h0 = (part * 4 + wave) * per_wave;
  const int u = lane % U, r = lane / U;
  int d0, d1;
  unit_channels<INTER>(u, rot, d0, d1);
  int pos[NR];
  Angles an[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    pos[i] = slot_pos(a, s, r + i * RS);
    if (pos[i] >= 0 && u * 16 < rot) an[i] = load_angles(a.rope, pos[i], rot, u);
  }
  const bool full = key && s.blk >= 0 && a.block_keys && slot_pos(a, s, 15) >= 0;  // this write fills the block
  const size_t stride = key ? a.k_stride : a.q_stride;
  const uint16_t* base = key ? a.k_new : a.q;
  uint16_t* tiles = a.k_cache + (size_t)max(s.blk, 0) * a.Hkv * 16 * D;  // key: of the block's heads
  // Rows of head h: new ones, and the older keys of a block that this write fills.
  auto load = [&](int h, uint4(&row)[NR][2]) {
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int o = r + i * RS;
      const uint16_t* p = pos[i] >= 0 ? base + (size_t)(s.src + o) * stride + (size_t)h * D
                                      : tiles + ((size_t)h * 16 + o) * D;
      if (pos[i] >= 0 || full) {
        row[i][0] = ld4(p + d0);
        row[i][1] = ld4(p + d1);
      }
    }
  };
  const int h1 = min(h0 + per_wave, heads);
  if (h0 >= h1) return;
  uint4 next[NR][2];
  load(h0, next);
  for (int h = h0; h < h1; ++h) {
    uint4 row[NR][2];
#pragma unroll
    for (int i = 0; i < NR; ++i) row[i][0] = next[i][0], row[i][1] = next[i][1];
    if (h + 1 < h1) load(h + 1, next);
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int o = r + i * RS;
      if (pos[i] < 0) continue;
      if (u * 16 < rot) rotate_unit<INTER>(row[i][0], row[i][1], an[i]);
      if (key && s.blk < 0) continue;
      uint16_t* dst = key ? tiles + ((size_t)h * 16 + o) * D : a.q_out + ((size_t)(s.src + o) * a.Hq + h) * D;
      st4(dst + d0, row[i][0]);
      st4(dst + d1, row[i][1]);
    }
    if (full) {
      const size_t tile = (size_t)s.blk * a.Hkv + h;
      block_codes<D>(row, d0, d1, lane, a.block_keys + tile * D, a.block_exp + tile);
    }
  }
}

// ---------------------------------------------------------------------------
// Summaries of full blocks that are in the cache: a wave per tile.
// Tiles in a row per wave (375 MB of keys and summaries / 16 short contexts: one
// tile 77.3 / 5.5 us, two 76.3 / 6.3, four 78.7 / 7.6, eight 82.2 / 11.9).
constexpr int kTilesPerWave = 2;
// Work-groups in all, but 16 per sequence where that is more; they step on over a
// longer context. Enough for every tile of the bound / at most this many (lengths
// lognormal with sigma 0.5): 64 sequences of median 1500 tokens under a bound of
// 131072, 114.2 / 49.8 us, 256 of 400 under 32768, 116.6 / 56.6; 8 of 20000 under
// 65536, 77.1 / 77.0; 16 of 300 under 1024, 6.6 / 6.6.
constexpr int kSummaryWgs = 32768;

template <int D>
__global__ __launch_bounds__(256, 6) void block_summary_kernel(aflex_block_summary_args a) {
  constexpr int U = TileLanes<D>::U, NR = TileLanes<D>::NR, RS = TileLanes<D>::RS;
  const int lane = threadIdx.x & 63;
  const int b = blockIdx.y;
  const int ctx = min(max(a.context_lens[b], 0), a.max_context_len);
  const int tiles = ctx / 16 * a.Hkv;
  const int u = lane % U, r = lane / U;
  const int32_t* table = a.block_table + (size_t)b * a.max_blocks_per_seq;
  int j, g;
  // (tiles of a block one after the other in memory; the next one's loads go out first)
  auto tile_of = [&]() -> long long {
    const int blk = table[j];
    return blk < 0 || blk >= a.num_blocks ? -1 : (long long)blk * a.Hkv + g;
  };
  auto load = [&](long long tile, uint4(&row)[NR][2]) {
    const uint16_t* p = a.k_cache + (size_t)max(tile, 0ll) * 16 * D + r * D + u * 16;
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int c = 0; c < 2; ++c) row[i][c] = ld4(p + i * RS * D + c * 8);
  };
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (long long t0 = ((long long)blockIdx.x * 4 + wave) * kTilesPerWave; t0 < tiles;
       t0 += (long long)gridDim.x * 4 * kTilesPerWave) {
    j = (int)t0 / a.Hkv;
    g = (int)t0 - j * a.Hkv;
    const int count = min(kTilesPerWave, tiles - (int)t0);
    long long tile = tile_of();
    uint4 row[NR][2];
    load(tile, row);
    for (int k = 0; k < count; ++k) {
      uint4 next[NR][2];
      long long next_tile = -1;
      if (k + 1 < count) {
        if (++g == a.Hkv) g = 0, ++j;
        next_tile = tile_of();
        load(next_tile, next);
      }
      if (tile >= 0) block_codes<D>(row, u * 16, u * 16 + 8, lane, a.block_keys + tile * D, a.block_exp + tile);
      tile = next_tile;
#pragma unroll
      for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) row[i][c] = next[i][c];
    }
  }
}

// ---------------------------------------------------------------------------
// Host side.

// The strides that 0 stands for.
static aflex_rope_args with_strides(aflex_rope_args a) {
  if (a.q_stride == 0) a.q_stride = a.Hq * a.D;
  if (a.k_stride == 0) a.k_stride = a.Hkv * a.D;
  if (a.v_stride == 0) a.v_stride = a.Hkv * a.D;
  return a;
}

hipError_t launch_rope_append(const aflex_rope_args& in, hipStream_t stream) {
  const aflex_rope_args a = with_strides(in);
  const long long waves = (long long)a.B * a.Hkv + ((long long)a.B * a.Hq * (a.D / 16) + 63) / 64;
  const unsigned grid = (unsigned)((waves + 3) / 4);
  ProfScope ps("rope_append", stream);
  if (a.D == 128 && a.interleaved)
    rope_append_kernel<128, true><<<grid, 256, 0, stream>>>(a);
  else if (a.D == 128)
    rope_append_kernel<128, false><<<grid, 256, 0, stream>>>(a);
  else if (a.interleaved)
    rope_append_kernel<64, true><<<grid, 256, 0, stream>>>(a);
  else
    rope_append_kernel<64, false><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_rope_write(const aflex_rope_args& in, hipStream_t stream) {
  if (in.T == 0 || in.max_seqlen == 0) return hipSuccess;
  const aflex_rope_args a = with_strides(in);
  const int vparts = (a.Hkv * (a.D / 8) + 255) / 256;
  const int slots = (a.max_seqlen + 15) / 16 + 1;
  const int per_wave = (long long)slots * a.B * (a.Hq + a.Hkv) >= kManyWaves * kHeadsPerWave ? kHeadsPerWave : 1;
  const int per = 4 * per_wave;
  const int kparts = (a.Hkv + per - 1) / per, qparts = (a.Hq + per - 1) / per;
  const dim3 grid(slots, vparts + kparts + qparts, a.B);
  const size_t lds = 256 / 16 * 2048;  // the exchange of V rows
  ProfScope ps("rope_write", stream);
  if (a.D == 128 && a.interleaved)
    rope_write_kernel<128, true><<<grid, 256, lds, stream>>>(a, vparts, kparts, per_wave);
  else if (a.D == 128)
    rope_write_kernel<128, false><<<grid, 256, lds, stream>>>(a, vparts, kparts, per_wave);
  else if (a.interleaved)
    rope_write_kernel<64, true><<<grid, 256, lds, stream>>>(a, vparts, kparts, per_wave);
  else
    rope_write_kernel<64, false><<<grid, 256, lds, stream>>>(a, vparts, kparts, per_wave);
  return hipGetLastError();
}

hipError_t launch_block_summary(const aflex_block_summary_args& a, hipStream_t stream) {
  const long long tiles = (long long)(a.max_context_len / 16) * a.Hkv;
  if (tiles == 0) return hipSuccess;
  // Work-groups for the longest context, but no more than kSummaryWgs in all (or 16
  // per sequence): under a loose bound most would find nothing to do.
  const long long need = (tiles + 4 * kTilesPerWave - 1) / (4 * kTilesPerWave);
  const long long most = kSummaryWgs / a.B > 16 ? kSummaryWgs / a.B : 16;
  const dim3 grid((unsigned)(need < most ? need : most), a.B);
  ProfScope ps("block_summary", stream);
  if (a.D == 128)
    block_summary_kernel<128><<<grid, 256, 0, stream>>>(a);
  else
    block_summary_kernel<64><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace aflex
