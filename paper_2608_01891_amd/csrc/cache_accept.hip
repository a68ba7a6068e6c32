// The accepted drafts' cache entries to consecutive places, gfx950.
//
// Draft accepted[i] of a sequence moves to place i behind its context. The list
// ascends, so accepted[i] >= i, and what is read after the first k places are
// written lies at k or behind: a thread moves its own piece of the rows (16 bytes
// of the key, one channel of the value, one exponent) kAcceptBatch entries at a
// time, all of them read before the first is written, and needs no other thread.
// Bound by latency: numbers and list of the sequence, block ids, data, each a round
// of dependent loads: 5.5 us for 32 sequences with 8 drafts, 7.9 us for 64 drafts a
// sequence (batches of 8: 10.4 us, of 32, whose registers leave fewer waves: 8.9).
#include "common.h"
#include "kernels.h"
#include "profile.h"

namespace aflex {

constexpr int kAcceptBatch = 16;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Lane i's entry: where draft accepted[i] lies and where it goes; N entries.
struct Moves {
  int src, dst;    // slot in the block
  int sblk, dblk;  // pool blocks, -1 where the entry is not copied
  int n, ctx_out;
};

__device__ __forceinline__ Moves find_moves(const aflex_cache_accept_args& a, int b, int lane) {
  Moves m{0, 0, -1, -1, 0, 0};
  // (all of a sequence's numbers in one round of loads)
  const int ctx = a.context_lens[b];
  const long long n = (long long)a.cu_seqlens[b + 1] - a.cu_seqlens[b];
  const int most = min(a.accepted_counts[b], a.max_accepted);
  const int listed = a.accepted[(size_t)b * a.max_accepted + min(lane, a.max_accepted - 1)];
  m.ctx_out = ctx;
  if (ctx < 1 || ctx > a.max_blocks_per_seq * 16 || n < 0 || n > ctx) return m;
  const int start = ctx - (int)n;
  const int at = lane < most ? listed : -1;
  const int before = lane > 0 ? __shfl_up(at, 1) : -1;
  const unsigned long long bad = __ballot(!(lane < most && at > before && at < n));
  m.n = bad ? __builtin_ctzll(bad) : 64;
  m.ctx_out = start + m.n;
  if (lane < m.n && at != lane) {
    const int32_t* row = a.block_table + (size_t)b * a.max_blocks_per_seq;
    const int p = start + at, q = start + lane;
    m.src = p % 16;
    m.dst = q % 16;
    const int s = row[p / 16], d = row[q / 16];
    if (s >= 0 && s < a.num_blocks && d >= 0 && d < a.num_blocks) m.sblk = s, m.dblk = d;
  }
  return m;
}

// Moves one piece of every entry: `at(block, slot)` is its place in a pool. The
// entries sit in the lanes of the wave, so all of them stay; `mine`: the lane has a piece.
template <class T, class F>
__device__ __forceinline__ void move_pieces(const Moves& m, T* pool, bool mine, F at) {
  for (int i0 = 0; i0 < m.n; i0 += kAcceptBatch) {
    T got[kAcceptBatch] = {};
#pragma unroll
    for (int i = 0; i < kAcceptBatch; ++i) {
      const int blk = __builtin_amdgcn_readlane(m.sblk, i0 + i), o = __builtin_amdgcn_readlane(m.src, i0 + i);
      if (blk >= 0 && mine) got[i] = pool[at(blk, o)];
    }
#pragma unroll
    for (int i = 0; i < kAcceptBatch; ++i) {
      const int blk = __builtin_amdgcn_readlane(m.dblk, i0 + i), o = __builtin_amdgcn_readlane(m.dst, i0 + i);
      if (blk >= 0 && mine) pool[at(blk, o)] = got[i];
    }
  }
}

// Waves of each kind of piece: keys (16 bytes each), values (a channel each),
// exponents; a lane per piece.
struct AcceptWaves {
  int keys, values, exps;
};

static AcceptWaves accept_waves(const aflex_cache_accept_args& a) {
  const bool f8 = a.kv_exp != nullptr;
  const auto waves = [](long long pieces) { return (int)((pieces + 63) / 64); };
  return {waves((long long)a.Hkv * a.D * (f8 ? 1 : 2) / 16), waves((long long)a.Hkv * a.D),
          f8 ? waves(2ll * a.Hkv) : 0};
}

template <int D, class Elem>
__global__ __launch_bounds__(256) void cache_accept_kernel(aflex_cache_accept_args a, AcceptWaves w) {
  constexpr int KC = D * sizeof(Elem) / 16;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const int b = blockIdx.y;
  const Moves m = find_moves(a, b, lane);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.context_out[b] = m.ctx_out;
  const size_t Hkv = a.Hkv;
  if (wave < w.keys) {
    const size_t p = (size_t)wave * 64 + lane, g = p / KC, c = p % KC;
    move_pieces(m, static_cast<u32x4*>(a.k_cache), g < Hkv,
                [=](size_t blk, int o) { return ((blk * Hkv + g) * 16 + o) * KC + c; });
  } else if (wave < w.keys + w.values) {
    const size_t ch = (size_t)(wave - w.keys) * 64 + lane;  // g D + d
    move_pieces(m, static_cast<Elem*>(a.v_cache), ch < Hkv * D,
                [=](size_t blk, int o) { return (blk * Hkv * D + ch) * 16 + o; });
  } else if (wave < w.keys + w.values + w.exps) {
    const size_t ge = (size_t)(wave - w.keys - w.values) * 64 + lane;  // 2 g + (key or value)
    move_pieces(m, a.kv_exp, ge < Hkv * 2, [=](size_t blk, int o) { return (blk * Hkv * 2 + ge) * 16 + o; });
  }
}

hipError_t launch_cache_accept(const aflex_cache_accept_args& a, hipStream_t stream) {
  const bool f8 = a.kv_exp != nullptr;
  const AcceptWaves w = accept_waves(a);
  const dim3 grid((unsigned)((w.keys + w.values + w.exps + 3) / 4), a.B);
  ProfScope ps("cache_accept", stream);
  if (a.D == 128 && f8)
    cache_accept_kernel<128, uint8_t><<<grid, 256, 0, stream>>>(a, w);
  else if (a.D == 128)
    cache_accept_kernel<128, uint16_t><<<grid, 256, 0, stream>>>(a, w);
  else if (f8)
    cache_accept_kernel<64, uint8_t><<<grid, 256, 0, stream>>>(a, w);
  else
    cache_accept_kernel<64, uint16_t><<<grid, 256, 0, stream>>>(a, w);
  return hipGetLastError();
}

}  // namespace aflex
