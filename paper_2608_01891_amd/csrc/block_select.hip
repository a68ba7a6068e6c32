// Choice of the cache blocks that each (sequence, kv head) attends, gfx950.
//
// score_j = max over the group's query heads of <q codes, block codes> times a
// power of two: a product of bytes on the matrix cores
// (v_mfma_i32_16x16x64_i8: 16 query heads x 16 blocks, D / 64 of them), summed
// in whole numbers, so every split gives the same bits. The summaries are read
// once (D + 1 bytes per block and head, a 64th of the block's K and V): bound
// by HBM for many long contexts, by latency for few.
//
// What the scores cost was, in turn: lanes that read 16 bytes of 16 rows each
// (four times the tag lookups of whole rows), chunks of sequences dealt to XCDs
// by their number (the first ones, which all sequences have, on two of 8), and
// grids over the longest context (idle work-groups; stretches of equal length
// instead): 64 sequences of median 20000 tokens, 95 MB, 63 -> 24 us. Rows of 1 KB
// (8 heads x 128) gathered at random reach 5.0-5.3 TB/s alone: 18.4 us.
//
// The scores become 32-bit keys whose unsigned order is theirs, forced blocks
// above all. The N-th largest is found digit by digit, a histogram in LDS each
// (bound by atomics that meet in one bin: absent keys are left out, and of long
// lists all but the keys that can be among the N), until the digits found leave
// exactly as many keys as are wanted. The blocks above the bound and the first
// ones inside it are written in order: the place of a block is the number of
// taken ones before it.
//
// Forms, by the bound on a sequence's blocks: up to 1024 one launch, a
// work-group per unit (128 sequences of median 2000 tokens 11.2 us, in two
// launches 16.9); else scores by all CUs and a work-group per unit that chooses
// from keys in memory, up to 4096 straight away, above from candidates.
#include <atomic>

#include "block_codes.h"
#include "kernels.h"
#include "profile.h"

namespace aflex {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kForced = 0xffffffffu;  // key of the blocks that are always taken
constexpr uint32_t kBad = 1;               // of those with a bad pool id; 0 stands for no block
constexpr int kScoreThreads = 512;
constexpr int kSelectThreads = 256;
constexpr int kChooseThreads = 512;
constexpr int kPickThreads = 1024;
constexpr int kBins = 2048;
constexpr int kListed = 4096;       // longest list of keys that a work-group holds
constexpr int kFusedBlocks = 1024;  // of those that it scores as well
constexpr int kSplitUnits = 1024;

// Unsigned order of the keys is the order of the floats (-0 and 0 are equal).
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(f == 0.f ? 0.f : f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int clamp_len(const aflex_block_select_args& a, int b) {
  return min(max(a.context_lens[b], 0), a.max_context_len);
}

// The query heads of one group as whole numbers: lane (row r, slice qg) holds
// channels 64 c + 16 qg + [0, 16) of head r mod G in code[c] (heads that repeat
// to fill the tile do not change a maximum) and the head's exponent. The lane
// gets the products of rows 4 qg + i; times scale[i] they are the heads' scores
// over 2^(top - 7), exactly, unless a head with whole codes is smaller than the
// largest by more than fp32's range (wide): there the exponents are applied one
// by one.
template <int D>
struct Query {
  i32x4 code[D / 64];
  int e;
  float scale[4];
  int top;
  bool wide;
};

template <int D>
struct QueryRows {
  uint4 w[D / 64][2];
};

template <int D>
__device__ __forceinline__ QueryRows<D> load_query(const aflex_block_select_args& a, int b, int g, int lane) {
  const int G = a.Hq / a.Hkv, r = (lane & 15) % G, qg = lane >> 4;
  QueryRows<D> q;
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    const uint16_t* p = a.q + ((size_t)b * a.Hq + g * G + r) * D + c * 64 + qg * 16;
    q.w[c][0] = *reinterpret_cast<const uint4*>(p);
    q.w[c][1] = *reinterpret_cast<const uint4*>(p + 8);
  }
  return q;
}

template <int D>
__device__ __forceinline__ void query_codes(QueryRows<D> rows, int lane, Query<D>& q) {
  const int qg = lane >> 4;
  auto& w = rows.w;
  int mag = 0;
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
  uint32_t any = 0;
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
    q.code[c] = i32x4{(int)out[0], (int)out[1], (int)out[2], (int)out[3]};
    any |= out[0] | out[1] | out[2] | out[3];
  }
  int top = e;
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) top = max(top, __shfl_xor(top, o));
  q.e = e;
  q.top = __builtin_amdgcn_readfirstlane(top);
  q.wide = __any(any != 0 && e < top - 120);
#pragma unroll
  for (int i = 0; i < 4; ++i) q.scale[i] = two_to(max(__shfl(e, 4 * qg + i) - top, -120));
}

// The summaries of 64 blocks on their way to a wave: a load instruction takes
// whole rows, D / 16 lanes each, so that a row's line is asked for once, and
// leaves them in registers; id and ex are block `lane`'s (-1: none).
template <int D>
struct Round {
  static constexpr int U = D / 16;   // lanes per row
  static constexpr int RPI = 64 / U; // rows per instruction
  i32x4 part[U];
  int ex, id;
};

template <int D>
__device__ __forceinline__ void load_round(const aflex_block_select_args& a, int g, int id, int lane, Round<D>& s) {
  constexpr int U = Round<D>::U, RPI = Round<D>::RPI;
  s.id = id >= 0 && id < a.num_blocks ? id : -1;
  const uint32_t tile = (uint32_t)max(s.id, 0) * a.Hkv + g;
  s.ex = a.block_exp[tile];
  // slice (lane % U) ^ (row % U) of the row: see stage_round
  const int8_t* base = a.block_keys + (((lane % U) ^ (lane / U % U)) << 4);
#pragma unroll
  for (int i = 0; i < U; ++i)
    s.part[i] = *reinterpret_cast<const i32x4*>(base + (size_t)(uint32_t)__shfl((int)tile, i * RPI + lane / U) * D);
}

// Turns the round's rows into matrix operands through the wave's LDS (64 D
// bytes): slice x of row r is kept at x ^ (r % U), which spreads the reads of
// one slice of 16 rows over the banks.
template <int D>
__device__ __forceinline__ void stage_round(const Round<D>& s, int lane, uint8_t* lds) {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < Round<D>::U; ++i) *reinterpret_cast<i32x4*>(lds + i * 1024 + lane * 16) = s.part[i];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Key of block t + lane, whose pool id and exponent are given, from the staged
// rows. The 16 x 16 products of 4 tiles leave lane (r, qg) with 4 heads of
// block r of each tile; the maximum over the heads is taken by halving, so that
// lane group qg ends with tile qg (3 exchanges instead of 8).
template <int D>
__device__ __forceinline__ uint32_t finish_round(const aflex_block_select_args& a, int n, int t, const Query<D>& q,
                                                 const uint8_t* lds, int id, int ex, int lane) {
  constexpr int U = Round<D>::U;
  const int r = lane & 15, qg = lane >> 4;
  float best[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    i32x4 dot = {0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      const i32x4 codes = *reinterpret_cast<const i32x4*>(lds + (k * 16 + r) * D + (((c * 4 + qg) ^ (r % U)) << 4));
      dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(q.code[c], codes, dot, 0, 0, 0);
    }
    float s[4];
    if (q.wide) {
      const int ek = __shfl(ex, k * 16 + r) - 7;
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = ldexpf((float)dot[i], __shfl(q.e, 4 * qg + i) + ek);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = (float)dot[i] * q.scale[i];
    }
    best[k] = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
  }
  const bool hi = qg & 2, up = qg & 1;
  const float b0 = fmaxf(hi ? best[2] : best[0], __shfl_xor(hi ? best[0] : best[2], 32));
  const float b1 = fmaxf(hi ? best[3] : best[1], __shfl_xor(hi ? best[1] : best[3], 32));
  float s = fmaxf(up ? b1 : b0, __shfl_xor(up ? b0 : b1, 16));
  if (!q.wide) s = ldexpf(s, q.top - 7 + ex);
  const int j = t + lane;
  uint32_t key = order_key(ex == kExpAlways ? -kNegInf : s);
  if (id < 0) key = kBad;
  if (j < a.sink_blocks || j >= n - a.recent_blocks) key = kForced;
  return key;
}

// Keys of blocks t, .. of unit (b, g), n blocks in all, below j1, to
// out[number], by a wave with 64 D bytes of LDS: 64 of them, then those `step`
// further on. It loads its next round while it finishes one.
template <int D>
__device__ __forceinline__ void score_blocks(const aflex_block_select_args& a, int b, int g, int n, int t, int step,
                                             int j1, uint8_t* lds, uint32_t* out) {
  if (t >= j1) return;
  const int lane = threadIdx.x & 63;
  const int32_t* table = a.block_table + (size_t)b * a.max_blocks_per_seq;
  auto id_of = [&](int j) { return j < j1 ? table[j] : -1; };
  const int first = id_of(t + lane);
  int next = id_of(t + step + lane);
  const QueryRows<D> rows = load_query<D>(a, b, g, lane);
  Round<D> s;
  load_round<D>(a, g, first, lane, s);
  Query<D> q;
  query_codes<D>(rows, lane, q);
  for (; t < j1; t += step) {
    stage_round<D>(s, lane, lds);
    const int now = s.id, ex = s.ex;
    if (t + step < j1) load_round<D>(a, g, next, lane, s);
    next = id_of(t + 2 * step + lane);
    const uint32_t key = finish_round<D>(a, n, t, q, lds, now, ex, lane);
    if (t + lane < j1) out[t + lane] = key;
  }
}

// (sequence, kv head) or (group of them) of a linear work-group index: the kv
// heads of a sequence (or chunk) get indices equal modulo 8, which is how
// work-groups are dealt to the 8 XCDs, so that the line with a block's
// exponents for all heads is fetched into one L2 only.
__device__ __forceinline__ void unit_of(int w, int groups, int Hkv, int& grp, int& g) {
  const int top = w / (8 * Hkv), in = w - top * (8 * Hkv);
  const int rest = min(8, groups - top * 8);  // groups in this batch of up to 8
  g = in / rest;
  grp = top * 8 + in - g * rest;
}

// Inclusive sum over a wave, by data movement between lanes of the vector unit.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr 1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);  // row_shr 2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);  // row_shr 4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);  // row_shr 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast 15 to rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast 31 to rows 2 and 3
  return v;
}

// Wave slots along the kv heads in a work-group of the scores (the others take
// further rounds of blocks): the next power of two, though with 3, 5, 6 or 7
// heads some of the waves then have nothing to do. With the power below, so that
// waves take two heads one after the other, or with one slot and every wave its
// own rounds (us of the scores, D = 128, this / below / one slot): 3 heads, 64
// sequences of median 20000 tokens 15.7 / 15.5 / 16.3, one of 400000 8.6 / 11.3 /
// 14.8; 5 heads 18.1 / 21.4 / 21.9 and 10.9 / 11.8 / 20.9; 7 heads 21.2 / 24.7 /
// 28.1 and 11.5 / 12.3 / 26.5.
__host__ __device__ constexpr int head_slots(int Hkv) { return Hkv > 4 ? 8 : Hkv > 2 ? 4 : Hkv; }

// Scores of all units whose blocks are not all taken, as rounds of 64 blocks of
// a sequence laid end to end. Each of the grid's workers (the waves of a
// work-group that share a slot) takes an equal stretch of them, whatever the
// lengths of the sequences, for all kv heads, a wave per head (more heads than
// waves: one after the other), so that the rows of a block (Hkv D bytes in a
// row) are asked for together.
template <int D>
__global__ __launch_bounds__(kScoreThreads, 4) void block_score_kernel(aflex_block_select_args a, int stride,
                                                                       uint32_t* keys) {
  constexpr int NW = kScoreThreads / 64;
  __shared__ __attribute__((aligned(16))) uint8_t rows[NW][64 * D];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int heads = head_slots(a.Hkv), slots = NW / heads;
  const int workers = gridDim.x * slots, worker = blockIdx.x * slots + wave / heads;
  auto rounds_of = [&](int b) {
    const int n = nblk16(clamp_len(a, min(b, a.B - 1)));
    return b < a.B && n > a.top_blocks ? (n + 63) >> 6 : 0;
  };
  int total = 0;
  for (int b = lane; b < a.B; b += 64) total += rounds_of(b);
  total = __builtin_amdgcn_readlane(wave_scan(total), 63);
  const int per = (total + workers - 1) / workers;
  int x = worker * per;
  const int end = min(x + per, total);
  if (x >= end) return;
  int b = 0, base = 0;  // rounds before sequence b
  while (x < end) {
    // on to the sequence that holds round x, 64 of them at a time
    while (true) {
      const int mine = rounds_of(b + lane), incl = wave_scan(mine);
      const unsigned long long past = __ballot(base + incl > x);
      const int l = past ? __builtin_ctzll(past) : 63;
      base += __builtin_amdgcn_readlane(past ? incl - mine : incl, l);
      b = __builtin_amdgcn_readfirstlane(b + (past ? l : 64));
      if (past) break;
    }
    const int n = nblk16(clamp_len(a, b)), here = (n + 63) >> 6;
    const int stop = min(end, base + here);
    for (int g = wave % heads; g < a.Hkv; g += heads)
      score_blocks<D>(a, b, g, n, (x - base) * 64, 64, min((stop - base) * 64, n), rows[wave],
                      keys + ((size_t)b * a.Hkv + g) * stride);
    x = stop;
    base += here;
    ++b;
  }
}

// (below, NT: threads of the work-group)
struct PickShared {
  uint32_t hist[2][kBins];  // the pass's bins, and the next one's being cleared
  int wave_sum[2][16];
  int bin, above, inside;
};

// Sum over the work-group of what the threads before this one hold; `all`: of
// all. The two halves of a value may be two sums below 2^16. Uses half w of
// wave_sum, alternately.
template <int NT>
__device__ __forceinline__ int before_me(int v, int w, int& all, PickShared& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int incl = wave_scan(v);
  if (lane == 63) sh.wave_sum[w][wave] = incl;
  __syncthreads();
  int before = incl - v;
  all = 0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) {
    const int s = sh.wave_sum[w][i];
    before += i < wave ? s : 0;
    all += s;
  }
  return before;
}

// Where bin x is kept: the 32 bins of a lane of find_bounds, 8 times 16 bytes,
// in an order of its own, so that the lanes' reads meet all banks.
__device__ __forceinline__ int bin_at(int x) { return x ^ ((x >> 3) & 28); }

// Clears the bins of the first pass; a barrier has to follow.
template <int NT>
__device__ __forceinline__ void clear_bins(PickShared& sh) {
  for (int i = threadIdx.x; i < kBins; i += NT) sh.hist[0][i] = 0;
}

// Bounds [lo, hi] of the `need`-th largest key, digit by digit (11, 11 and 10
// bits, a histogram each), at most `passes` of them: keys above hi are fewer
// than need, by which need is lowered; of those in [lo, hi], `need` are wanted.
// Ends early where the bounds hold exactly that many. each(f) calls f(key) for
// every key of the thread, 0 for none; the bins are clear before, not after.
template <int NT, class Each>
__device__ __forceinline__ void find_bounds(const Each& each, int& need, int passes, uint32_t& lo, uint32_t& hi,
                                            PickShared& sh) {
  const int lane = threadIdx.x & 63;
  uint32_t prefix = 0;
  for (int p = 0; p < passes; ++p) {
    const int shift = p == 0 ? 21 : p == 1 ? 10 : 0, bits = p == 2 ? 10 : 11;
    uint32_t* hist = sh.hist[p & 1];
    each([&](uint32_t k) {
      if (p == 0 ? k != 0 : (k >> (shift + bits)) == prefix) atomicAdd(&hist[bin_at((k >> shift) & ((1u << bits) - 1))], 1u);
    });
    __syncthreads();
    if (threadIdx.x < 64) {  // one wave: lane l has 32 bins, from the top
      const int row = kBins / 32 - 1 - lane;
      const uint4* mine = reinterpret_cast<const uint4*>(hist + row * 32);
      int four[8], sum = 0;  // of 4 bins each, from the top
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint4 v = mine[(7 - i) ^ (row & 7)];
        four[i] = v.x + v.y + v.z + v.w;
        sum += four[i];
      }
      int before = wave_scan(sum) - sum;
      if (before < need && need <= before + sum) {
        int group = 0, start = before;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool here = before < need && need <= before + four[i];
          group = here ? i : group;
          start = here ? before : start;
          before += four[i];
        }
        const uint4 v = mine[(7 - group) ^ (row & 7)];
        const int c[4] = {(int)v.w, (int)v.z, (int)v.y, (int)v.x};
        int at = 0, above = start, inside = 0;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const bool here = start < need && need <= start + c[m];
          at = here ? 4 * group + m : at;
          above = here ? start : above;
          inside = here ? c[m] : inside;
          start += c[m];
        }
        sh.bin = kBins - 1 - 32 * lane - at;
        sh.above = above;
        sh.inside = inside;
      }
    } else if (p + 1 < passes) {
      for (int i = threadIdx.x - 64; i < kBins; i += NT - 64) sh.hist[(p + 1) & 1][i] = 0;
    }
    __syncthreads();
    prefix = (prefix << bits) | (uint32_t)sh.bin;
    need -= sh.above;
    lo = prefix << shift;
    hi = lo + ((1u << shift) - 1);
    if (sh.inside == need) return;
  }
}

// Stretch of a list of up to kListed keys that a thread holds in registers.
template <int NT, int MOST = kListed>
struct Held {
  static constexpr int kEach = MOST / NT;
  uint32_t k[kEach];
  // (the list may end at n, rounded up to 4)
  __device__ __forceinline__ explicit Held(const uint32_t* list, int n = MOST) {
#pragma unroll
    for (int i = 0; i < kEach; i += 4) {
      const int at = threadIdx.x * kEach + i;
      const uint4 v = at < n ? *reinterpret_cast<const uint4*>(list + at) : make_uint4(0, 0, 0, 0);
      k[i] = v.x;
      k[i + 1] = at + 1 < n ? v.y : 0;
      k[i + 2] = at + 2 < n ? v.z : 0;
      k[i + 3] = at + 3 < n ? v.w : 0;
    }
  }
  template <class F>
  __device__ __forceinline__ void operator()(F f) const {
#pragma unroll
    for (int i = 0; i < kEach; ++i) f(k[i]);
  }
};

// Writes the block numbers of the list's N largest keys (N of them at least;
// ties to the lower place) to out, in the list's order: number(place). Absent
// keys are 0 and stand behind the others.
template <int NT, class Held, class Number>
__device__ __forceinline__ void choose(const Held& held, int N, const Number& number, int32_t* out,
                                       PickShared& sh) {
  int need = N;
  uint32_t lo, hi;
  find_bounds<NT>(held, need, 3, lo, hi, sh);
  int v = 0, all;
  held([&](uint32_t k) { v += (k > hi ? 1 << 16 : 0) + (k >= lo && k <= hi ? 1 : 0); });
  v = before_me<NT>(v, 0, all, sh);
  int gt = v >> 16, eq = v & 0xffff;
#pragma unroll
  for (int i = 0; i < held.kEach; ++i) {
    const uint32_t k = held.k[i];
    const bool above = k > hi, in = k >= lo && k <= hi;
    if (above || (in && eq < need)) out[gt + min(eq, need)] = number(threadIdx.x * held.kEach + i);
    gt += above;
    eq += in;
  }
}

// The part of a row that needs no choice: -1 behind the list, and all blocks
// where they are no more than the list's places (true then).
template <int NT>
__device__ __forceinline__ bool trivial_row(int n, int top, int32_t* out) {
  const int N = min(n, top);
  for (int i = N + threadIdx.x; i < top; i += NT) out[i] = -1;
  if (n > N) return false;
  for (int i = threadIdx.x; i < n; i += NT) out[i] = i;
  return true;
}

// Choice from a unit's scores in memory, at most kListed (longer units are
// another launch's).
__global__ __launch_bounds__(kChooseThreads, 6) void block_choose_kernel(aflex_block_select_args a, int stride,
                                                                         const uint32_t* keys) {
  constexpr int NT = kChooseThreads;
  __shared__ PickShared sh;
  const int unit = blockIdx.x, n = nblk16(clamp_len(a, unit / a.Hkv));
  int32_t* out = a.selected + (size_t)unit * a.top_blocks;
  if (n > kListed || trivial_row<NT>(n, a.top_blocks, out)) return;
  const Held<NT> held(keys + (size_t)unit * stride, n);  // (rows are padded to a multiple of 4)
  clear_bins<NT>(sh);
  __syncthreads();
  choose<NT>(held, a.top_blocks, [](int place) { return place; }, out, sh);
}

// Choice from a unit's scores in memory, any number of them. A wave takes a
// stretch of the keys, 256 at a time, four per lane. The N-th largest of the
// lanes' own maxima, cut to 22 bits, is a bound that at least N keys reach and
// few others do; those go to a list in LDS and the choice is made there. Where
// they are more than the list holds (equal scores, or N above the lanes that have
// keys: all 1024 from 8192 blocks on, little more than half of them just above
// 4096), the bounds are found digit by digit over all keys. R: rounds of keys that
// a lane keeps in registers, or 0: they are read again for every pass (us, kept /
// read again, 8 units of 5000 blocks 11.4 / 11.4, 16400 12.0 / 13.9, 25000 13.6 /
// 16.8, 32500 14.0 / 18.1; 512 of median 6250 21.4 / 24.8).
template <int R>
__global__ __launch_bounds__(kPickThreads) void block_pick_kernel(aflex_block_select_args a, int stride,
                                                                  const uint32_t* keys, bool long_only) {
  constexpr int NT = kPickThreads;
  __shared__ PickShared sh;
  __shared__ __attribute__((aligned(16))) uint32_t list_key[kListed];
  __shared__ int list_at[kListed];
  const int unit = blockIdx.x, b = unit / a.Hkv, tid = threadIdx.x, lane = tid & 63;
  const int n = nblk16(clamp_len(a, b)), N = a.top_blocks;
  int32_t* out = a.selected + (size_t)unit * N;
  if ((long_only && n <= kListed) || trivial_row<NT>(n, N, out)) return;
  const uint32_t* src = keys + (size_t)unit * stride;  // (rows are padded to a multiple of 4)
  clear_bins<NT>(sh);
  // a short sequence among long ones, or under a loose bound (131072 tokens: 64
  // sequences of median 20000 40.6 -> 32.7 us, of 3000 25.7 -> 15.3)
  if (n <= kListed) {
    const Held<NT> held(src, n);
    __syncthreads();
    choose<NT>(held, N, [](int place) { return place; }, out, sh);
    return;
  }
  const int rounds = (n + 4 * NT - 1) / (4 * NT);
  const long long base = (long long)(tid >> 6) * rounds * 256 + lane * 4;
  auto load = [&](int i) {
    const long long j = base + (long long)i * 256;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (i < rounds && j < n) v = *reinterpret_cast<const uint4*>(src + j);
    return make_uint4(v.x, j + 1 < n ? v.y : 0, j + 2 < n ? v.z : 0, j + 3 < n ? v.w : 0);
  };
  uint4 kept[R > 0 ? R : 1];
  if constexpr (R > 0) {
#pragma unroll
    for (int i = 0; i < R; ++i) kept[i] = load(i);
  }
  // f(the lane's four keys of a round, 0 for none; the first one's number)
  auto each4 = [&](auto f) {
    auto one = [&](int i, const uint4& v) {
      const uint32_t k[4] = {v.x, v.y, v.z, v.w};
      f(k, (int)(base + (long long)i * 256));
    };
    if constexpr (R > 0) {
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (i < rounds) one(i, kept[i]);
    } else {
      for (int i = 0; i < rounds; ++i) one(i, load(i));
    }
  };
  auto each = [&](auto f) {
    each4([&](const uint32_t(&k)[4], int) {
#pragma unroll
      for (int m = 0; m < 4; ++m) f(k[m]);
    });
  };
  uint32_t lo = 1, hi;
  if (N <= NT) {
    uint32_t most = 1;
    each([&](uint32_t k) { most = max(most, k); });
    __syncthreads();
    int need = N;
    find_bounds<NT>([&](auto f) { f(most); }, need, 2, lo, hi, sh);
    lo = max(lo, 1u);
    clear_bins<NT>(sh);
  }
  int c = 0, all;
  each([&](uint32_t k) { c += k >= lo; });
  const int before = before_me<NT>(c, 0, all, sh);
  if (all <= kListed) {
    for (int i = tid; i < kListed; i += NT) list_key[i] = 0;
    __syncthreads();
    int w = __builtin_amdgcn_readfirstlane(before);  // of the wave's first lane: place of its stretch
    each4([&](const uint32_t(&k)[4], int j) {
      const int mine = (k[0] >= lo) + (k[1] >= lo) + (k[2] >= lo) + (k[3] >= lo);
      const int incl = wave_scan(mine);
      int at = w + incl - mine;
#pragma unroll
      for (int m = 0; m < 4; ++m)
        if (k[m] >= lo) {
          list_key[at] = k[m];
          list_at[at++] = j + m;
        }
      w += __builtin_amdgcn_readlane(incl, 63);
    });
    __syncthreads();
    choose<NT>(Held<NT>(list_key), N, [&](int place) { return list_at[place]; }, out, sh);
    return;
  }
  __syncthreads();
  int need = N;
  find_bounds<NT>(each, need, 3, lo, hi, sh);
  int gt = 0, eq = 0, total;
  each([&](uint32_t k) {
    gt += k > hi;
    eq += k >= lo && k <= hi;
  });
  int g = __builtin_amdgcn_readfirstlane(before_me<NT>(gt, 1, total, sh));
  int e = __builtin_amdgcn_readfirstlane(before_me<NT>(eq, 0, total, sh));
  each4([&](const uint32_t(&k)[4], int j) {
    int mg = 0, me = 0;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      mg += k[m] > hi;
      me += k[m] >= lo && k[m] <= hi;
    }
    const int ig = wave_scan(mg), ie = wave_scan(me);
    int ag = g + ig - mg, ae = e + ie - me;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const bool above = k[m] > hi, in = k[m] >= lo && k[m] <= hi;
      if (above || (in && ae < need)) out[ag + min(ae, need)] = j + m;
      ag += above;
      ae += in;
    }
    g += __builtin_amdgcn_readlane(ig, 63);
    e += __builtin_amdgcn_readlane(ie, 63);
  });
}

// Scores and choice of a unit in one work-group, the keys in LDS (the bins of
// the choice where the rows of the scores were: 36 KiB, four work-groups per CU).
template <int D>
__global__ __launch_bounds__(kSelectThreads, 4) void block_select_kernel(aflex_block_select_args a) {
  constexpr int NT = kSelectThreads, NW = NT / 64;
  constexpr int kBytes = NW * 64 * D > (int)sizeof(PickShared) ? NW * 64 * D : (int)sizeof(PickShared);
  __shared__ __attribute__((aligned(16))) uint32_t keys[kFusedBlocks];
  __shared__ __attribute__((aligned(16))) uint8_t shared[kBytes];
  int b, g;
  unit_of(blockIdx.x, a.B, a.Hkv, b, g);
  const int n = nblk16(clamp_len(a, b)), wave = threadIdx.x >> 6;
  int32_t* out = a.selected + ((size_t)b * a.Hkv + g) * a.top_blocks;
  if (trivial_row<NT>(n, a.top_blocks, out)) return;
  score_blocks<D>(a, b, g, n, wave * 64, NT, n, shared + wave * 64 * D, keys);
  __syncthreads();
  PickShared& sh = *reinterpret_cast<PickShared*>(shared);
  clear_bins<NT>(sh);
  __syncthreads();
  choose<NT>(Held<NT, kFusedBlocks>(keys, n), a.top_blocks, [](int place) { return place; }, out, sh);
}

// ---------------------------------------------------------------------------
// Host side.
static int max_blocks_of(const aflex_block_select_args& a) { return (a.max_context_len + 15) / 16; }

static int cu_count() {
  static std::atomic<int> cached{0};
  int v = cached.load(std::memory_order_relaxed);
  if (v > 0) return v;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || v <= 0)
    v = 256;
  cached.store(v, std::memory_order_relaxed);
  return v;
}

// One launch, a work-group per unit, where a unit's keys fit the list in LDS.
static bool fused(const aflex_block_select_args& a) { return max_blocks_of(a) <= kFusedBlocks; }

// Rows of keys start at multiples of 16 bytes.
static int key_stride(const aflex_block_select_args& a) { return (max_blocks_of(a) + 3) / 4 * 4; }

size_t block_select_workspace_bytes(const aflex_block_select_args& a) {
  if (fused(a)) return 0;
  return align_up((size_t)a.B * a.Hkv * key_stride(a) * sizeof(uint32_t), 256);
}

hipError_t launch_block_select(const aflex_block_select_args& a, void* ws, hipStream_t stream) {
  const int units = a.B * a.Hkv;
  if (fused(a)) {
    ProfScope ps("block_select", stream);
    if (a.D == 128)
      block_select_kernel<128><<<units, kSelectThreads, 0, stream>>>(a);
    else
      block_select_kernel<64><<<units, kSelectThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  uint32_t* keys = static_cast<uint32_t*>(ws);
  const int stride = key_stride(a);
  {
    ProfScope ps("block_score", stream);
    // no more work-groups than the GPU holds at once (two of 8 waves per CU)
    const int slots = kScoreThreads / 64 / head_slots(a.Hkv);
    const long long most = ((long long)a.B * ((stride + 63) / 64) + slots - 1) / slots;
    const unsigned grid = (unsigned)(most < 2 * cu_count() ? most : 2 * cu_count());
    if (a.D == 128)
      block_score_kernel<128><<<grid, kScoreThreads, 0, stream>>>(a, stride, keys);
    else
      block_score_kernel<64><<<grid, kScoreThreads, 0, stream>>>(a, stride, keys);
  }
  {
    ProfScope ps("block_pick", stream);
    // rounds of keys in registers, 32 per lane: bounds of up to 32768 blocks (524288
    // tokens); a kernel for longer ones cannot know that a unit is shorter
    constexpr int kRounds = 8;
    // Where units may be long but are many, the short ones are chosen by the
    // smaller kernel, three work-groups of which a CU holds, and a launch of its
    // own (under a bound of 131072 tokens, lengths lognormal with sigma 0.5, the whole
    // choice in one launch / two: 2048 units of median 3000 tokens 42.7 / 32.2 us, 1024
    // of 5000 30.3 / 25.6, 512 of 20000 34.8 / 38.6, 256 of 20000 20.7 / 22.2).
    const bool split = stride > kListed && units >= kSplitUnits;
    if (stride <= kListed || split) block_choose_kernel<<<units, kChooseThreads, 0, stream>>>(a, stride, keys);
    if (stride > kRounds * 4 * kPickThreads)
      block_pick_kernel<0><<<units, kPickThreads, 0, stream>>>(a, stride, keys, split);
    else if (stride > kListed)
      block_pick_kernel<kRounds><<<units, kPickThreads, 0, stream>>>(a, stride, keys, split);
  }
  return hipGetLastError();
}

}  // namespace aflex
