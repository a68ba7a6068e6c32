// Choice of the cache blocks that each (sequence, kv head) attends, gfx950.
//
// score_j = max over the group's query heads of <q codes, block codes> times a
// power of two: a product of bytes on the matrix cores
// (v_mfma_i32_16x16x64_i8: 16 query heads x 16 blocks, D / 64 of them), summed
// in whole numbers, so every split gives the same bits. The summaries are read
// once (D + 1 bytes per block and head, a 64th of the block's K and V): bound
// by HBM for many long contexts, by latency for few.
//
// The scores become 32-bit keys whose unsigned order is theirs, forced blocks
// above all. The N-th largest key is found digit by digit (11, 11 and 10 bits,
// a histogram in LDS each), then the blocks above it and the first ones equal
// to it are written in order: the place of block j is the number of taken ones
// before it, from one scan of ballots.
#include "block_codes.h"
#include "kernels.h"
#include "profile.h"

namespace aflex {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kForced = 0xffffffffu;  // key of the blocks that are always taken
constexpr int kScoreThreads = 256;
constexpr int kScoreTiles = 4;             // tiles of 16 blocks a wave scores per round of loads
constexpr int kPickThreads = 1024;
constexpr int kBins = 2048;

// Unsigned order of the keys is the order of the floats.
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int clamp_len(const aflex_block_select_args& a, int b) {
  return min(max(a.context_lens[b], 0), a.max_context_len);
}

// The query heads of one group as whole numbers: lane (head r, slice qg) holds
// channels 64 c + 16 qg + [0, 16) of head r in code[c] (zero for r >= G), and
// eh[i] is the exponent of head 4 qg + i.
template <int D>
__device__ __forceinline__ void query_codes(const aflex_block_select_args& a, int b, int g, int lane,
                                            i32x4 (&code)[D / 64], int (&eh)[4]) {
  const int G = a.Hq / a.Hkv, r = lane & 15, qg = lane >> 4;
  uint4 w[D / 64][2];
  int mag = 0;
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    w[c][0] = w[c][1] = make_uint4(0, 0, 0, 0);
    if (r < G) {
      const uint16_t* p = a.q + ((size_t)b * a.Hq + g * G + r) * D + c * 64 + qg * 16;
      w[c][0] = *reinterpret_cast<const uint4*>(p);
      w[c][1] = *reinterpret_cast<const uint4*>(p + 8);
    }
  }
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t* x = reinterpret_cast<uint32_t*>(&w[c][k]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // non-finite channels count as zero
        if ((x[i] & 0x7f80u) == 0x7f80u) x[i] &= 0xffff0000u;
        if ((x[i] & 0x7f800000u) == 0x7f800000u) x[i] &= 0xffffu;
      }
      mag = max_mag(w[c][k], mag);
    }
  mag = max(mag, __shfl_xor(mag, 16));
  mag = max(mag, __shfl_xor(mag, 32));
  const int e = exponent_above(mag);
  const float f = two_to(7 - e);
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    const uint32_t* x = reinterpret_cast<const uint32_t*>(&w[c][0]);
    uint32_t out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t v = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t pair = x[i * 2 + k / 2];
        const float y = __uint_as_float((k & 1) ? (pair & 0xffff0000u) : (pair << 16)) * f;
        v |= ((uint32_t)(int)fminf(fmaxf(rintf(y), -127.f), 127.f) & 0xffu) << (8 * k);
      }
      out[i] = v;
    }
    code[c] = i32x4{(int)out[0], (int)out[1], (int)out[2], (int)out[3]};
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) eh[i] = __shfl(e, 4 * qg + i);
}

// Keys of blocks [j0, j1) of unit (b, g), n blocks in all, by the waves of a
// work-group (wave of nw), to out[j - j0].
template <int D>
__device__ __forceinline__ void score_blocks(const aflex_block_select_args& a, int b, int g, int n, int j0, int j1,
                                             int wave, int nw, int lane, uint32_t* out) {
  constexpr int NC = D / 64;
  const int G = a.Hq / a.Hkv, r = lane & 15, qg = lane >> 4;
  i32x4 qc[NC];
  int eh[4];
  query_codes<D>(a, b, g, lane, qc, eh);
  const int32_t* table = a.block_table + (size_t)b * a.max_blocks_per_seq;
  for (int t = j0 + wave * 16 * kScoreTiles; t < j1; t += nw * 16 * kScoreTiles) {
    int id[kScoreTiles];
#pragma unroll
    for (int k = 0; k < kScoreTiles; ++k) {
      const int j = t + k * 16 + r;
      id[k] = j < j1 ? table[j] : -1;
      if (id[k] >= a.num_blocks) id[k] = -1;
    }
    i32x4 kc[kScoreTiles][NC];
    int ex[kScoreTiles];
#pragma unroll
    for (int k = 0; k < kScoreTiles; ++k) {
      const size_t tile = id[k] >= 0 ? (size_t)id[k] * a.Hkv + g : 0;
#pragma unroll
      for (int c = 0; c < NC; ++c)
        kc[k][c] = *reinterpret_cast<const i32x4*>(a.block_keys + tile * D + c * 64 + qg * 16);
      ex[k] = a.block_exp[tile];
    }
#pragma unroll
    for (int k = 0; k < kScoreTiles; ++k) {
      i32x4 dot = {0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < NC; ++c) dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(qc[c], kc[k][c], dot, 0, 0, 0);
      float best = kNegInf;  // dot[i]: query head 4 qg + i, block r of the tile
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (4 * qg + i < G) best = fmaxf(best, ldexpf((float)dot[i], eh[i] - 7 + ex[k]));
      best = fmaxf(best, __shfl_xor(best, 16));
      best = fmaxf(best, __shfl_xor(best, 32));
      const int j = t + k * 16 + r;
      uint32_t key = order_key(ex[k] == kExpAlways ? -kNegInf : best);
      if (id[k] < 0) key = 0;
      if (j < a.sink_blocks || j >= n - a.recent_blocks) key = kForced;
      if (qg == 0 && j < j1) out[j - j0] = key;
    }
  }
}

// (sequence, kv head) or (group of them) of a linear work-group index: the kv
// heads of a sequence (or chunk) get indices equal modulo 8, which is how
// work-groups are dealt to the 8 XCDs, so that the line with a block's
// exponents for all heads is fetched into one L2 only.
__device__ __forceinline__ void unit_of(long long w, int groups, int Hkv, int& grp, int& g) {
  const long long span = 8LL * Hkv;
  const long long top = w / span, in = w - top * span;
  const int rest = min(8, groups - (int)(top * 8));  // sequences in this batch of up to 8
  g = (int)(in / rest);
  grp = (int)(top * 8 + in % rest);
}

// Scores of a chunk of one unit's blocks.
template <int D>
__global__ __launch_bounds__(kScoreThreads) void block_score_kernel(aflex_block_select_args a, int chunks,
                                                                    int chunk, int stride, uint32_t* keys) {
  int grp, g;
  unit_of(blockIdx.x, a.B * chunks, a.Hkv, grp, g);
  const int b = grp / chunks, j0 = (grp - b * chunks) * chunk;
  const int n = nblk16(clamp_len(a, b));
  if (n <= a.top_blocks || j0 >= n) return;
  score_blocks<D>(a, b, g, n, j0, min(j0 + chunk, n), threadIdx.x >> 6, kScoreThreads / 64, threadIdx.x & 63,
                  keys + ((size_t)b * a.Hkv + g) * stride + j0);
}

// Inclusive sum over a wave.
__device__ __forceinline__ int wave_scan(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(v, o);
    if (lane >= o) v += t;
  }
  return v;
}

struct PickShared {
  uint32_t hist[kBins];
  int wave_sum[kPickThreads / 64];
  int bin, above;
};

// Writes the N largest of keys[0, n) (N < n), ties to the lower index, to out
// in ascending order of index. All of a work-group of kPickThreads.
__device__ __forceinline__ void pick(const uint32_t* keys, int n, int N, int32_t* out, PickShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int NW = kPickThreads / 64;
  uint32_t prefix = 0;  // the digits found so far
  int need = N;         // how many keys with that prefix are taken
  constexpr int kShift[3] = {21, 10, 0}, kBits[3] = {11, 11, 10};
#pragma unroll
  for (int p = 0; p < 3; ++p) {
    for (int i = tid; i < kBins; i += kPickThreads) sh.hist[i] = 0;
    __syncthreads();
    const int shift = kShift[p], bits = kBits[p];
    for (int i = tid; i < n; i += kPickThreads) {
      const uint32_t k = keys[i];
      if (p == 0 || (k >> (shift + bits)) == prefix) atomicAdd(&sh.hist[(k >> shift) & ((1u << bits) - 1)], 1u);
    }
    __syncthreads();
    // thread t: bins 2t and 2t + 1 counted from the top
    const int top = kBins - 1 - 2 * tid;
    const int c0 = sh.hist[top], c1 = sh.hist[top - 1];
    const int incl = wave_scan(c0 + c1, lane);
    if (lane == 63) sh.wave_sum[wave] = incl;
    __syncthreads();
    int before = incl - c0 - c1;
    for (int w = 0; w < wave; ++w) before += sh.wave_sum[w];
    if (before < need && need <= before + c0) {
      sh.bin = top;
      sh.above = before;
    } else if (before + c0 < need && need <= before + c0 + c1) {
      sh.bin = top - 1;
      sh.above = before + c0;
    }
    __syncthreads();
    prefix = (prefix << bits) | (uint32_t)sh.bin;
    need -= sh.above;
  }
  // taken: keys above `prefix`, and the first `need` equal to it
  int base_gt = 0, base_eq = 0;
  for (int i0 = 0; i0 < n; i0 += kPickThreads) {
    const int i = i0 + tid;
    const uint32_t k = i < n ? keys[i] : 0;
    const bool gt = i < n && k > prefix, eq = i < n && k == prefix;
    const unsigned long long mg = __ballot(gt), me = __ballot(eq);
    __syncthreads();
    if (lane == 0) sh.wave_sum[wave] = __popcll(mg) << 16 | __popcll(me);
    __syncthreads();
    int gb = base_gt, eb = base_eq, gall = 0, eall = 0;
    for (int w = 0; w < NW; ++w) {
      const int s = sh.wave_sum[w];
      if (w < wave) gb += s >> 16, eb += s & 0xffff;
      gall += s >> 16;
      eall += s & 0xffff;
    }
    const unsigned long long below = (1ull << lane) - 1;
    gb += __popcll(mg & below);
    eb += __popcll(me & below);
    if (gt || (eq && eb < need)) out[gb + min(eb, need)] = i;
    base_gt += gall;
    base_eq += eall;
  }
}

__global__ __launch_bounds__(kPickThreads) void block_pick_kernel(aflex_block_select_args a, int stride,
                                                                  const uint32_t* keys) {
  __shared__ PickShared sh;
  const int unit = blockIdx.x, b = unit / a.Hkv;
  const int n = nblk16(clamp_len(a, b)), N = min(n, a.top_blocks);
  int32_t* out = a.selected + (size_t)unit * a.top_blocks;
  for (int i = N + threadIdx.x; i < a.top_blocks; i += kPickThreads) out[i] = -1;
  if (n == N) {
    for (int i = threadIdx.x; i < n; i += kPickThreads) out[i] = i;
    return;
  }
  pick(keys + (size_t)unit * stride, n, N, out, sh);
}

// ---------------------------------------------------------------------------
// Host side.
static int max_blocks_of(const aflex_block_select_args& a) { return (a.max_context_len + 15) / 16; }

size_t block_select_workspace_bytes(const aflex_block_select_args& a) {
  if (max_blocks_of(a) <= a.top_blocks) return 0;
  return align_up((size_t)a.B * a.Hkv * max_blocks_of(a) * sizeof(uint32_t), 256);
}

constexpr int kChunk = 512;  // blocks per work-group of the scores

hipError_t launch_block_select(const aflex_block_select_args& a, void* ws, hipStream_t stream) {
  uint32_t* keys = static_cast<uint32_t*>(ws);
  const int stride = max_blocks_of(a);
  if (stride > a.top_blocks) {
    ProfScope ps("block_score", stream);
    const int chunks = (stride + kChunk - 1) / kChunk;
    const unsigned grid = (unsigned)(a.B * chunks * a.Hkv);
    if (a.D == 128)
      block_score_kernel<128><<<grid, kScoreThreads, 0, stream>>>(a, chunks, kChunk, stride, keys);
    else
      block_score_kernel<64><<<grid, kScoreThreads, 0, stream>>>(a, chunks, kChunk, stride, keys);
  }
  {
    ProfScope ps("block_pick", stream);
    block_pick_kernel<<<a.B * a.Hkv, kPickThreads, 0, stream>>>(a, stride, keys);
  }
  return hipGetLastError();
}

}  // namespace aflex
