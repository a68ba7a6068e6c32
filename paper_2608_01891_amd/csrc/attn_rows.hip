// Attention of a few query rows per (sequence, kv head) over a paged KV cache,
// gfx950: one new token per sequence over an 8-bit cache, and trees of drafted
// tokens over an 8-bit or a bf16 cache.
//
// The rows of a (sequence, kv head) are its n tokens times the G query heads of
// the group, row i G + h. They share every cached key and value:
//
//   S^T[tok][row] = K[tok][:] . q[row][:]      (v_mfma_f32_16x16x32_bf16: 16 tokens
//                                               x 16 rows, a row tile)
//   O^T[d][row] += V^T[d][tok] . P^T[tok][row]
//
// with the running maximum and sum of a softmax per row, in log2 units. The order
// of the tokens in the first product is chosen so that its output registers are
// the second product's operand.
//
// 8-bit rows are c 2^e. A key's codes become bf16 with its 2^e on the way, exactly.
// A value's exponent joins the weight: P' = p 2^e enters the product with the codes
// as fp16, exactly, and the row's sum is that of p. p = 2^(s - M') with M' the
// largest s + e, to within 2^kSlack: the largest contribution has a P' of 2^7 to 2^15,
// and P' is rounded to fp16 (11 bits; below 2^-14 steps of 2^-24), with up to 16 rows to
// two fp16 values. Over a bf16 cache a weight enters as two bf16 values, the rounded
// weight and what its rounding left: 16 bits. (One bf16 value, 8 bits, would show beside
// the output's own rounding: 2.1e-3 of the norm instead of 1.65e-3.)
//
// Two kernels. Up to 16 rows (decode attention; 8-bit cache: 32, with D = 64 also 64):
// the waves of a work-group take the tokens in turns, keys and values go from memory
// straight into the matrix operands' registers, a step ahead. More rows: the waves share
// the tokens, 64 a step, which the work-group turns into 16-bit operands in LDS once, and
// each has row tiles of its own.
//
// The blocks of all units (sequence, kv head, pass over the rows) are laid end to
// end, and each work-group takes a consecutive range of them, so that long and
// short contexts fill the GPU alike; a unit cut between work-groups leaves fp32
// partials that a second launch merges in order.
//
// Bounds, and what was measured (caches that no call has read just before; 8-bit and
// 64 / 8 heads x 128 but where it says otherwise). Decode attention: the cache's bytes.
// 64 sequences of median 4096 tokens, 740 MB: 133.0 us, 5.6 TB/s; one of 400000, 826
// MB: 140.4 us, 5.9 TB/s, where loads alone reach 6.4. Trees: the chain of a step
// (barrier, widening into LDS, barrier, operands, products, softmax, products) with two
// waves on a SIMD. 32 sequences of median 4096 tokens, up to 8 drafts each, 328 MB: 94
// us, 3.5 TB/s, the vector units busy for 43% of it, the matrix units 19%, LDS 34%; one
// context of 65536 with 64 drafts: 190 us, 0.72 PFLOP/s (a large matrix product reaches
// 1.41), 55%, 32% and 33%; 8 sequences of median 8192, up to 32 drafts, 32 / 8 heads,
// bf16, 301 MB: 82 us, 3.7 TB/s.
#include <math.h>

#include <atomic>
#include <type_traits>

#include "common.h"
#include "f8.h"
#include "kernels.h"
#include "profile.h"

namespace aflex {

namespace {

constexpr int kRowWaves = 4;
// Row tiles (16 rows each) of a wave, where there is more than one tile. (Three leave no
// registers for the loads ahead: one context of 65536 with 64 drafts took 282 us
// instead of 231; one, with all four waves on the same tokens, 99.9 instead of 93.3 us
// for 32 sequences with 8 drafts.)
constexpr int kTiles = 2;

struct RowsParams {
  const uint16_t* q;
  const uint8_t* kc;
  const uint8_t* vc;
  const int8_t* ke;
  const int32_t* bt;
  const int32_t* cl;
  const int32_t* cu;        // NULL: one row token per sequence
  const uint64_t* masks;    // NULL: a chain
  uint16_t* out;
  float* part_o;            // [slots][D]
  float* part_ml;           // [slots][2]  (running maximum, sum)
  int2* span;               // [B Hkv passes]  first and last work-group of each unit's pieces
  int B, T, Hq, Hkv, G;
  int max_n, max_passes, pass_rows;  // bounds: tokens, passes, rows of a pass
  int pass_tiles;           // row tiles that one pass takes
  int max_blocks, num_blocks, max_ctx;
  int unit_cost;
  int whole;                // a work-group per unit: a position each
  float scale_log2;
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// A sequence as its lanes see it.
struct Seq {
  int row0;   // first token row
  int n;      // its tokens
  int take;   // those that are computed (n, or the caller's bound)
  int ctx;    // cached tokens
  int tiles;  // row tiles of a pass (0: nothing to compute)
  int passes;
};

__device__ __forceinline__ Seq seq_of(const RowsParams& p, int b) {
  Seq s;
  s.ctx = min(max(p.cl[b], 0), p.max_ctx);
  if (p.cu) {
    const int s1 = min(max(p.cu[b + 1], 0), p.T);
    s.row0 = min(max(p.cu[b], 0), s1);
    s.n = s1 - s.row0;
  } else {
    s.row0 = b;
    s.n = 1;
  }
  s.take = min(s.n, p.max_n);
  const int all = s.ctx > 0 ? (s.take * p.G + 15) >> 4 : 0;
  s.passes = (all + p.pass_tiles - 1) / p.pass_tiles;
  s.tiles = s.passes > 1 ? (all + s.passes - 1) / s.passes : all;
  return s;
}

// Positions of a unit in the flattened range: its blocks, and a charge for the
// piece it adds; or one.
__device__ __forceinline__ int unit_len(const RowsParams& p, const Seq& s) {
  return p.whole ? 1 : ((s.ctx + 15) >> 4) + p.unit_cost;
}

__device__ __forceinline__ int seq_len(const RowsParams& p, int b) {
  if (b >= p.B) return 0;
  const Seq s = seq_of(p, b);
  return p.Hkv * s.passes * unit_len(p, s);
}

__device__ __forceinline__ int sum64(int v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o);
  return __builtin_amdgcn_readfirstlane(v);
}

__device__ __forceinline__ int scan64(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(v, o);
    if (lane >= o) v += t;
  }
  return v;
}

// A work-group's range [x0, x1) of the flattened positions, `per` each; b: the
// sequence of x0, base: its first position. False: nothing is left for it.
__device__ __forceinline__ bool find_range(const RowsParams& p, int least, int lane, int& per, int& x0, int& x1, int& b,
                                           int& base) {
  const int P = gridDim.x, wg = blockIdx.x;
  int total = 0;
  for (int c = 0; c < p.B; c += 64) total += sum64(seq_len(p, c + lane));
  per = p.whole ? 1 : max((total + P - 1) / P, least);
  const long long xs = (long long)wg * per;
  if (xs >= total) return false;
  x0 = (int)xs;
  x1 = min(x0 + per, total);
  b = base = 0;
  for (int c = 0; c < p.B; c += 64) {
    const int len = seq_len(p, c + lane);
    const int incl = scan64(len, lane);
    const unsigned long long past = __ballot(base + incl > x0);
    if (past) {
      const int l = __builtin_ctzll(past);
      b = c + l;
      base += __builtin_amdgcn_readlane(incl - len, l);
      break;
    }
    base += __builtin_amdgcn_readlane(incl, 63);
  }
  b = __builtin_amdgcn_readfirstlane(b);
  base = __builtin_amdgcn_readfirstlane(base);
  return true;
}

// Blocks [j0, j1) of a unit.
struct Piece {
  int kvh, pass, j0, j1;
  int first, last;  // work-groups that hold pieces of the unit
  int row0, rows;   // its rows in the sequence's
  int tiles;
};

__device__ __forceinline__ Piece piece_at(const RowsParams& p, const Seq& s, int base, int x, int x1, int per, int& xn) {
  Piece c;
  const int len = unit_len(p, s), unit = (x - base) / len;
  c.kvh = unit / s.passes;
  c.pass = unit - c.kvh * s.passes;
  if (p.whole) {
    c.j0 = 0;
    c.j1 = (s.ctx + 15) >> 4;
    c.first = c.last = blockIdx.x;
    xn = x1;
  } else {
    const int ustart = base + unit * len + p.unit_cost, nb = len - p.unit_cost;
    c.j0 = max(x - ustart, 0);
    c.j1 = min(nb, x1 - ustart);  // (j0 or less where the range ends inside the unit's charge)
    c.first = ustart / per;
    c.last = (ustart + nb - 1) / per;
    xn = min(ustart + nb, x1);
  }
  c.row0 = c.pass * s.tiles * 16;
  c.rows = min(s.take * p.G - c.row0, s.tiles * 16);
  c.tiles = (c.rows + 15) >> 4;
  return c;
}

// Row of a sequence's (kv head's) rows: its place in q and out.
__device__ __forceinline__ size_t row_of(const RowsParams& p, const Seq& s, int kvh, int row) {
  const int tok = row / p.G;
  return (size_t)(s.row0 + tok) * p.Hq + (size_t)kvh * p.G + (row - tok * p.G);
}

__device__ __forceinline__ uint64_t mask_of_row(const RowsParams& p, const Seq& s, int row) {
  const int tok = row / p.G;
  return p.masks ? p.masks[s.row0 + tok] : (2ull << tok) - 1ull;
}

// Partial row of a row of a unit's piece in work-group wg. Pieces are numbered along
// the range, and from one to the next either the unit advances by its rows or the
// work-group by one, or both: no two pieces share a row.
__device__ __forceinline__ size_t part_row(const RowsParams& p, const Seq& s, int kvh, int row, int wg) {
  return (size_t)s.row0 * p.Hq + (size_t)kvh * s.take * p.G + (size_t)row + (size_t)wg * p.pass_rows;
}

// Rows of sequences without cached tokens are zeros.
template <int D>
__device__ __forceinline__ void clear_empty(const RowsParams& p) {
  for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
    const Seq s = seq_of(p, b);
    if (s.ctx == 0) {
      uint4* o = reinterpret_cast<uint4*>(p.out + (size_t)s.row0 * p.Hq * D);
      for (size_t i = threadIdx.x; i < (size_t)s.take * p.Hq * (D / 8); i += 64 * kRowWaves) o[i] = make_uint4(0, 0, 0, 0);
    }
  }
}

// What a work-group has to do behind its pieces (add_odd): values that are not finite were
// taken out of products, or a result over a bf16 cache is not finite.
constexpr int kOddTaken = 1, kOddResult = 2;
constexpr uint16_t kNoSum = 0x7fff;  // the NaN of rows whose weights' sum is none (others are made as 0x7fc0)

// A row tile's result (lane: row `row`, channels 16 mt + 4 qg ..) to out, or to the piece's partial.
template <int D, bool F8>
__device__ __forceinline__ void store_rows(const RowsParams& p, const Seq& s, const Piece& c, int row, int qg, float m,
                                           float l, const f32x4 (&acc)[D / 16], int* odd) {
  if (row >= c.row0 + c.rows) return;
  if constexpr (!F8) {
    float zero = 0.f;
#pragma unroll
    for (int mt = 0; mt < D / 16; ++mt)
#pragma unroll
      for (int i = 0; i < 4; ++i) zero = fmaf(acc[mt][i], 0.f, zero);
    if (zero != 0.f) *odd |= kOddResult;
  }
  if (c.first == c.last) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
    uint16_t* o = p.out + row_of(p, s, c.kvh, row) * D + 4 * qg;
#pragma unroll
    for (int mt = 0; mt < D / 16; ++mt) {
      ushort4 v;
      v.x = f2bf(acc[mt][0] * inv);
      v.y = f2bf(acc[mt][1] * inv);
      v.z = f2bf(acc[mt][2] * inv);
      v.w = f2bf(acc[mt][3] * inv);
      if (!F8 && l != l) v.x = v.y = v.z = v.w = kNoSum;
      *reinterpret_cast<ushort4*>(o + mt * 16) = v;
    }
  } else {
    const size_t at = part_row(p, s, c.kvh, row, blockIdx.x);
    float* o = p.part_o + at * D + 4 * qg;
#pragma unroll
    for (int mt = 0; mt < D / 16; ++mt) *reinterpret_cast<f32x4*>(o + mt * 16) = acc[mt];
    if (qg == 0) *reinterpret_cast<float2*>(p.part_ml + at * 2) = make_float2(m, l);
  }
}

template <class V>
__device__ __forceinline__ V stream(const uint8_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
}

// Eight codes (two words) as bf16 times 2^scale's exponent, and as fp16.
__device__ __forceinline__ bf16x8 widen_bf16(uint32_t a, uint32_t b, float scale) {
  const bf16x2 w[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true)};
  return bf16x8{w[0][0], w[0][1], w[1][0], w[1][1], w[2][0], w[2][1], w[3][0], w[3][1]};
}

__device__ __forceinline__ f16x8 widen_f16(uint32_t a, uint32_t b) {
  const f16x2 w[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false),
                      __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true),
                      __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false),
                      __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true)};
  return f16x8{w[0][0], w[0][1], w[1][0], w[1][1], w[2][0], w[2][1], w[3][0], w[3][1]};
}

// The first n of the bytes, zeros behind them (n may be <= 0).
template <class V>
__device__ __forceinline__ V keep_bytes(V v, int n) {
#pragma unroll
  for (int i = 0; i < (int)(sizeof(V) / 4); ++i) {
    const int k = n - 4 * i;
    v[i] = k >= 4 ? v[i] : k <= 0 ? 0u : v[i] & ((1u << (8 * k)) - 1u);
  }
  return v;
}

// Exponents (bytes) as they can be, -100 to 120. Those of tokens that no row sees may hold
// anything, and a weight of 0 does not take away a 2^e that is not finite.
constexpr int kLeastExp = -100, kMostExp = 120;

__device__ __forceinline__ u32x2 legal_exponents(u32x2 v) {
  typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
  const auto limit = [](uint32_t x) {  // the high byte of each half
    const i16x2 least = {kLeastExp * 256, kLeastExp * 256}, most = {kMostExp * 256, kMostExp * 256};
    return __builtin_bit_cast(
        uint32_t, __builtin_elementwise_min(__builtin_elementwise_max(__builtin_bit_cast(i16x2, x), least), most));
  };
#pragma unroll
  for (int i = 0; i < 2; ++i) v[i] = limit(v[i] & 0xff00ff00u) | limit(v[i] << 8 & 0xff00ff00u) >> 8;
  return v;
}

// Which of the 8 tokens from place `tb` on a draft with these mask bits sees, as
// bits; the first nv of them are cached, and the sequence's drafts start at `start`.
__device__ __forceinline__ uint32_t seen_bits(uint64_t mask, int tb, int start, int nv) {
  const uint32_t cached = nv >= 8 ? 0xffu : nv <= 0 ? 0u : (1u << nv) - 1u;
  const int off = tb - start;
  if (off >= 64) return 0;
  if (off >= 0) return cached & (uint32_t)(mask >> off);
  if (off <= -8) return cached;
  return cached & (((uint32_t)mask << -off) | ((1u << -off) - 1u));
}

// Largest over the four lanes that hold a row (lane % 16).
__device__ __forceinline__ float row_max(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// The weights of 8 tokens as operands of the second product. 8-bit cache: fp16, which
// loses up to 2^-11 of a weight, or fp16 and what it leaves as fp16, 2^-22. With one row tile
// the second part costs little, as the call waits for memory: 64 sequences of decode
// attention 132.9 us with one part, 133.5 with two, one of 400000 tokens 139.7 and 140.4. The
// output's difference from one of 32-bit weights falls from 8.5e-4 of its norm to 6e-5. With
// more rows there is one part: two take 102.3 us instead of 94.3 for 32 sequences with 8
// drafts, 223 instead of 190 for 64 drafts over 65536 tokens, 84.5 instead of 83.5 for 64
// sequences with 4, 43.8 instead of 40.9 for 32 with 8 of D = 64, and the output, whose own
// rounding is 1.66e-3 of its norm, is 1.67e-3 off with either. bf16 cache: the rounded bf16
// and what the rounding left, 2^-17. (Its leading 8 bits and what those leave: 2^-16.)
struct HalfWeights {
  f16x8 w;
  __device__ __forceinline__ void set(int i, float a, float b) {
    w[i] = static_cast<_Float16>(a);
    w[i + 1] = static_cast<_Float16>(b);
  }
  static constexpr int kParts = 1;
  __device__ __forceinline__ f32x4 mul(int, f16x8 v, f32x4 acc) const {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w, acc, 0, 0, 0);
  }
};

struct TwoHalfWeights {
  f16x8 hi, lo;
  __device__ __forceinline__ void set(int i, float a, float b) {
    hi[i] = static_cast<_Float16>(a);
    hi[i + 1] = static_cast<_Float16>(b);
    lo[i] = static_cast<_Float16>(a - static_cast<float>(hi[i]));
    lo[i + 1] = static_cast<_Float16>(b - static_cast<float>(hi[i + 1]));
  }
  static constexpr int kParts = 2;
  __device__ __forceinline__ f32x4 mul(int part, f16x8 v, f32x4 acc) const {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(v, part ? lo : hi, acc, 0, 0, 0);
  }
};

struct TwoWeights {
  u32x4 hi, lo;
  __device__ __forceinline__ void set(int i, float a, float b) {
    uint32_t h = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
    asm("" : "+v"(h));  // (the rounded values are taken from the pair, not made again one by one)
    hi[i / 2] = h;
    lo[i / 2] = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a - __uint_as_float(h << 16)),
                                                    static_cast<__bf16>(b - __uint_as_float(h & 0xffff0000u))});
  }
  static constexpr int kParts = 2;
  __device__ __forceinline__ f32x4 mul(int part, bf16x8 v, f32x4 acc) const {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, part ? lo : hi), acc, 0, 0, 0);
  }
};

// Values that are not finite, in steps where not every row sees every token. A weight
// of 0 does not take one out of a product, so a row would get those of drafts that it
// does not see. The products have zeros in their place (m: one bit for each), and the
// rows that see them get them afterwards.
template <bool F8, class V>
__device__ __forceinline__ V without_odd(V v, bool& odd) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(V) / 4); ++i) {
    const uint32_t m = F8 ? ((v[i] & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u
                          : ((v[i] & 0x7f807f80u) + 0x00800080u) >> 15 & 0x00010001u;
    v[i] &= ~(m * (F8 ? 0xffu : 0xffffu));
    any |= m;
  }
  odd = odd || any != 0;
  return v;
}

// A work-group's pieces once more, if s_odd says so for one of its waves. First, where a
// result over a bf16 cache is not finite: it is the sum of the values that are not, if there
// are such values in the steps (of BLOCKS blocks) whose products took them. (The second
// part of a weight is 0 or negative at times, and times an infinity a NaN or one of the other sign.)
// Then the values that without_odd took out of the other steps' products, added to what is
// stored of the rows that see them. A pass of its own that reads the kernel's
// arguments (a RowsParams alone) again, so that the loop of the products need not keep
// anything for it.
template <int D, bool F8, int BLOCKS>
__device__ __forceinline__ void add_odd(int least, const int* s_odd) {
  __shared__ float s_sum[F8 ? 1 : 64 * kRowWaves];
  const int tid = threadIdx.x, lane = tid & 63;
  __syncthreads();  // (and what was stored is there for the others)
  const int odd = s_odd[0] | s_odd[1] | s_odd[2] | s_odd[3];
  if (!odd) return;
  auto* args = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(args));
  RowsParams p;
  __builtin_memcpy(&p, (const void*)args, sizeof(p));
  int per, x, x1, b, base;
  if (!find_range(p, least, lane, per, x, x1, b, base)) return;
  while (x < x1) {
    const Seq s = seq_of(p, b);
    const int all = p.Hkv * s.passes * unit_len(p, s);
    if (x >= base + all) {
      base += all;
      ++b;
      continue;
    }
    int xn;
    const Piece c = piece_at(p, s, base, x, x1, per, xn);
    x = xn;
    if (c.j1 <= c.j0) break;
    const int start = s.ctx - s.n;
    const int32_t* table = p.bt + (size_t)b * p.max_blocks;
    const auto whole_step = [&](int step) {
      bool whole = (step + BLOCKS) * 16 <= start && step + BLOCKS <= c.j1;
      for (int j = step; j < min(step + BLOCKS, c.j1); ++j) whole = whole && (uint32_t)table[j] < (uint32_t)p.num_blocks;
      return whole;
    };
    // the sum of the values of channel d in block j that are not finite, of tokens of the set bits
    const auto odd_sum = [&](int j, int d, uint32_t seen) {
      const uint8_t* at = p.vc + (((size_t)table[j] * p.Hkv + c.kvh) * D + d) * (F8 ? 16 : 32);
      bool any = false;
#pragma unroll
      for (int i = 0; i < (F8 ? 1 : 2); ++i) without_odd<F8>(reinterpret_cast<const u32x4*>(at)[i], any);
      float sum = 0.f;
      for (int k = 0; any && k < 16; ++k) {
        float v;
        if constexpr (F8)
          v = (at[k] & 0x7f) == 0x7f ? __builtin_nanf("") : 0.f;
        else
          v = bf2f(reinterpret_cast<const uint16_t*>(at)[k]);
        sum += (seen >> k & 1u) && !(fabsf(v) < __builtin_inff()) ? v : 0.f;
      }
      return sum;
    };
    if (!F8 && (odd & kOddResult)) {
      // (A channel's sum is that of all rows: each is found once, a thread a share of the steps.
      // 8 sequences of 8192 tokens with 32 drafts take 168 us with a NaN in one token, 88 without; a
      // thread a row and channel 1137.)
      constexpr int kShares = 64 * kRowWaves / D;
      const int d = tid % D;
      float sum = 0.f;
      for (int step = c.j0 + tid / D * BLOCKS; step < c.j1; step += kShares * BLOCKS) {
        if (!whole_step(step)) continue;
        for (int j = step; j < step + BLOCKS; ++j) sum += odd_sum(j, d, 0xffffu);
      }
      __syncthreads();  // (the sums of the piece before are read)
      s_sum[tid] = sum;
      __syncthreads();
      sum = 0.f;
      for (int i = 0; i < kShares; ++i) sum += s_sum[i * D + d];
      for (int r = sum != 0.f ? tid / D : c.rows; r < c.rows; r += kShares) {
        uint16_t* o = p.out + row_of(p, s, c.kvh, c.row0 + r) * D + d;
        const size_t part = part_row(p, s, c.kvh, c.row0 + r, blockIdx.x);
        if (c.first == c.last) {
          if (!(fabsf(bf2f(*o)) < __builtin_inff()) && *o != kNoSum) *o = f2bf(sum);
        } else {
          const float l = p.part_ml[part * 2 + 1];
          if (!(fabsf(p.part_o[part * D + d]) < __builtin_inff()) && l == l) p.part_o[part * D + d] = sum;
        }
      }
    }
    for (int step = c.j0; step < c.j1; step += BLOCKS) {
      if (whole_step(step)) continue;
      for (int j = step; j < min(step + BLOCKS, c.j1); ++j) {
        const int cached = s.ctx - j * 16;
        if ((uint32_t)table[j] >= (uint32_t)p.num_blocks) continue;
        for (int it = tid; it < c.rows * D; it += 64 * kRowWaves) {
          const int row = c.row0 + it / D, d = it % D;
          const uint64_t mask = mask_of_row(p, s, row);
          const float sum = odd_sum(
              j, d, seen_bits(mask, j * 16, start, cached) | seen_bits(mask, j * 16 + 8, start, cached - 8) << 8);
          if (sum == 0.f) continue;
          if (c.first == c.last) {
            uint16_t* o = p.out + row_of(p, s, c.kvh, row) * D + d;
            *o = f2bf(bf2f(*o) + sum);
          } else {
            p.part_o[part_row(p, s, c.kvh, row, blockIdx.x) * D + d] += sum;
          }
        }
      }
    }
  }
}

// x 2^d for d <= 0, where 2^d alone may be too small for a float.
__device__ __forceinline__ float times_exp2(float x, float d) {
  const float h = fast_exp2(0.5f * d);
  return x * h * h;
}

constexpr float kSlack = 8.f;

// Over a bf16 cache weights are 2^-24 where they are largest, up to 2^-16 with the slack: the
// sum of 2^16 values of any magnitude is a float, as their mean is. (Values below 2^-113 lose
// bits for that, as the least float is 2^-149.)
constexpr float kBf16Shift = -24.f;

// Of a value's exponent where it is a byte (15 to 235); what the weights' sum counts u in, and
// what that takes of the product at the end: 2^(kExpBias - 127) in all.
constexpr int kExpBias = 115;
constexpr float kSumUnit = 0x1p-20f, kProductUnit = 0x1p-8f;

// The softmax of N row tiles over 8 tokens per lane: scores x (masked: -inf) to
// weights, the references m and sums l, and the accumulators' rescaling.
// F8: ve holds the tokens' value exponents, a byte each with kExpBias added, in the
// references too. u = 2^(s - m + 134) is 2^(19 - e) where P' is largest; one shift makes
// 2^(e - 12) of the byte, and P' = u 2^(e - 12), at least 2^7 there: fp16 holds 11 bits of
// weights down to 2^-21 of the largest, and what it drops is below 2^-32 of that. The sum is
// that of u 2^-20, product and sum in one instruction. No u overflows for an e of -100; exp2
// gives nothing below 2^-126, so that what the sum loses is below 2^-25 of the largest p where
// that token's e is 120, and a bit less for each below. (The sum itself is 2^-121 or more, and
// floats below 2^-126 count. At e = -100 it holds 2^20 tokens.)
template <bool F8, int N, int NMT, class Weights>
__device__ __forceinline__ void softmax_step(f32x4 (&x)[N][2], u32x2 ve, float scale_log2, float (&m)[N], float (&l)[N],
                                             f32x4 (&acc)[N][NMT], Weights (&w)[N]) {
  const auto byte = [&](int e) { return ve[e / 4] >> (8 * (e & 3)) & 0xffu; };
  // A row's reference m is its maximum when it was set last, and stays while no score
  // is more than kSlack above it: weights are up to 2^kSlack then. So the hot path
  // compares a lane's own scores alone, and the four lanes of a row exchange theirs
  // where one is above.
  bool above = false;
  float mx[N];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float v = F8 ? (float)byte(e) : 0.f;
#pragma unroll
    for (int t = 0; t < N; ++t) {
      const float s = F8 ? fmaf(x[t][e / 4][e & 3], scale_log2, v) : x[t][e / 4][e & 3];
      mx[t] = e == 0 ? s : fmaxf(mx[t], s);
    }
  }
#pragma unroll
  for (int t = 0; t < N; ++t) {
    if constexpr (!F8) mx[t] *= scale_log2;
    above = above || mx[t] > m[t] + kSlack;
  }
  if (__any(above)) {
#pragma unroll
    for (int t = 0; t < N; ++t) {
      const float m_new = fmaxf(m[t], row_max(mx[t]));
      const float d = m_new == kNegInf ? 0.f : m[t] - m_new, alpha = fast_exp2(d);
      l[t] = F8 ? times_exp2(l[t], d) : l[t] * alpha;
#pragma unroll
      for (int mt = 0; mt < NMT; ++mt) acc[t][mt] *= alpha;
      m[t] = m_new;
    }
  }
  float m_use[N];
#pragma unroll
  for (int t = 0; t < N; ++t) m_use[t] = m[t] == kNegInf ? 0.f : m[t] - (F8 ? 134.f : kBf16Shift);
  float ps[N][2];
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float f[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) f[i] = F8 ? __uint_as_float(byte(e + i) << 23) : 1.f;  // 2^(exponent - 12)
#pragma unroll
    for (int t = 0; t < N; ++t) {
      float u[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        u[i] = fast_exp2(fmaf(x[t][(e + i) / 4][(e + i) & 3], scale_log2, -m_use[t]));
        if constexpr (F8)
          ps[t][i] = e == 0 ? u[i] * kSumUnit : fmaf(u[i], kSumUnit, ps[t][i]);
        else
          ps[t][i] = e == 0 ? u[i] : ps[t][i] + u[i];
        if constexpr (F8) u[i] *= f[i];
      }
      w[t].set(e, u[0], u[1]);
    }
  }
#pragma unroll
  for (int t = 0; t < N; ++t) l[t] += ps[t][0] + ps[t][1];
}

// A row's sum over the lanes that hold it, and its product in the same unit.
template <bool F8, int NMT>
__device__ __forceinline__ void finish_row(float& l, f32x4 (&acc)[NMT]) {
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
#pragma unroll
  for (int mt = 0; mt < NMT; ++mt)
    if constexpr (F8) acc[mt] *= kProductUnit;
}

// A lane's share of a row's partial to LDS and from there to another wave's: O, then (m, l).
template <int D>
__device__ __forceinline__ void put_partial(float* o, int qg, float m, float l, const f32x4 (&acc)[D / 16]) {
#pragma unroll
  for (int mt = 0; mt < D / 16; ++mt) *reinterpret_cast<f32x4*>(o + mt * 16 + 4 * qg) = acc[mt];
  if (qg == 0) *reinterpret_cast<float2*>(o + D) = make_float2(m, l);
}

template <int D>
__device__ __forceinline__ void add_partial(const float* o, int qg, float& m, float& l, f32x4 (&acc)[D / 16]) {
  const float2 ml = *reinterpret_cast<const float2*>(o + D);
  const float mn = fmaxf(m, ml.x);
  const float mu = (mn == kNegInf) ? 0.f : mn;
  const float wa = fast_exp2(m - mu), wb = fast_exp2(ml.x - mu);
  l = times_exp2(l, m - mu) + times_exp2(ml.y, ml.x - mu);
  m = mn;
#pragma unroll
  for (int mt = 0; mt < D / 16; ++mt) acc[mt] = acc[mt] * wa + *reinterpret_cast<const f32x4*>(o + mt * 16 + 4 * qg) * wb;
}

// Block ids of a piece's steps of two blocks by scalar loads: raw ones are fetched a
// step ahead, and become ids (-1: no such block) when their step's loads are made.
struct BlockIds {
  typedef const int32_t __attribute__((address_space(4))) * Table;
  Table table;
  int j0, j1, num_blocks;
  int raw0, raw1;
  int id0, id1;

  __device__ __forceinline__ BlockIds(const RowsParams& p, int b, int j0, int j1)
      : table((Table)(reinterpret_cast<uintptr_t>(p.bt + (size_t)b * p.max_blocks))), j0(j0), j1(j1),
        num_blocks(p.num_blocks), raw0(-1), raw1(-1), id0(-1), id1(-1) {}
  __device__ __forceinline__ void fetch(int st) {
    const int j = j0 + st * 2, e = j1 - 1;
    raw0 = table[min(j, e)];
    raw1 = table[min(j + 1, e)];
  }
  __device__ __forceinline__ int fine(int id, int j) const { return j < j1 && id >= 0 && id < num_blocks ? id : -1; }
  __device__ __forceinline__ void take(int st) {
    const int j = j0 + st * 2;
    id0 = fine(raw0, j);
    id1 = fine(raw1, j + 1);
  }
  __device__ __forceinline__ int pick(int i) const { return i ? id1 : id0; }
};

// Waits for the global loads so far. In front of a loop whose loads run a step ahead:
// what the loop only reads (the queries) would else be waited for inside it, each time
// with the loads of the next step.
__device__ __forceinline__ void wait_for_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }  // vmcnt(0)

// Work-groups that a CU holds at once. Few rows: two, one tile of D = 64 three (at D = 128 a third
// costs the registers of the step ahead: 139.9 us instead of 136.8 for 64 sequences,
// 153.7 instead of 145.8 for one of 400000).
constexpr int few_per_cu(int D, int RT) { return D == 64 && RT == 1 ? 3 : 2; }

// Least positions of a work-group: a step for each wave, two steps.
constexpr int kFewLeast = 2 * kRowWaves, kManyLeast = 8;

// More rows, or tiles: by registers.
constexpr int kManyPerCu = 2;

}  // namespace

// ---------------------------------------------------------------------------
// Up to 16 rows, or RT tiles of 16: a step is 32 tokens (two blocks) of one wave. (64:
// 146 us instead of 138 for 64 sequences, as fewer loads are on their way.) DRAFTS: rows
// may differ in the tokens that they see. Two tiles for an 8-bit cache alone: 4 drafts
// of 64 / 8 heads x 128 over 400000 tokens 149.6 us instead of the other kernel's 166, of
// 32 / 4 x 64 in 32 sequences 30.1 instead of 35.4; over bf16, whose step ahead takes
// twice the registers, 145.6 instead of 135.4 (200000 tokens). Four tiles where D = 64:
// 8 drafts of 32 / 4 heads over 400000 tokens 63.7 us instead of 77.5, in 32 sequences
// 40.8 instead of 42.5; where D = 128 they would take the registers of a second
// work-group a CU (118 us for 32 sequences with 8 drafts instead of 96).
template <int D, bool F8, bool DRAFTS, int RT>
__global__ __launch_bounds__(64 * kRowWaves, few_per_cu(D, RT)) void attn_few_kernel(RowsParams p) {
  constexpr int NC = D / 32;       // k-chunks of the first product
  constexpr int NMT = D / 16;      // d-tiles of the second
  constexpr int NK = F8 ? NC : 2 * NC;  // 16-byte loads of a step's keys
  constexpr int LDO = D + 4;       // row of a partial in LDS: O, then (m, l)
  typedef std::conditional_t<F8, u32x2, u32x4> VLoad;  // a lane's 8 tokens of a channel
  typedef std::conditional_t<!F8, TwoWeights, std::conditional_t<RT == 1, TwoHalfWeights, HalfWeights>> Weights;
  typedef std::conditional_t<F8, f16x8, bf16x8> VFrag;
  __shared__ __attribute__((aligned(16))) float so[2 * RT * 16 * LDO];  // partials of two waves
  __shared__ int s_odd[kRowWaves];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int r = lane & 15, qg = lane >> 4;
  // The lane's places in a step: block and token of its key row (token + 4 t in tile
  // t), block and first token of its values.
  const int kblk = r >> 3, ktok = ((r >> 2) & 1) * 8 + (r & 3);
  const int vblk = qg >> 1, vtok = (qg & 1) * 8;

  clear_empty<D>(p);
  int per, x, x1, b, base;
  if (!find_range(p, kFewLeast, lane, per, x, x1, b, base)) return;
  if (lane == 0) s_odd[wave] = 0;
  while (x < x1) {
    const Seq s = seq_of(p, b);
    const int all = p.Hkv * s.passes * unit_len(p, s);
    if (x >= base + all) {
      base += all;
      ++b;
      continue;
    }
    int xn;
    const Piece c = piece_at(p, s, base, x, x1, per, xn);
    x = xn;
    if (c.j1 <= c.j0) break;
    const int start = s.ctx - s.n;  // place of the first draft
    const int steps = (c.j1 - c.j0 + 1) / 2;
    BlockIds ids(p, b, c.j0, c.j1);

    u32x4 kraw[NK];  // (8-bit codes come 16 channels a load, and the k-chunks take the channels in that order)
    VLoad vraw[NMT];
    u32x2 kx = {0, 0}, vx = {0, 0};  // exponents of the 8 tokens around the lane's key rows, and of its values
    int tb = 0, nv = 0, jb = 0;  // place of the lane's first token, how many of them are cached; first block
    // (blocks that do not exist are read at block 0 and masked)
    auto load_keys = [&]() __attribute__((always_inline)) {
      const size_t tile = (size_t)max(ids.pick(kblk), 0) * p.Hkv + c.kvh;
      if constexpr (F8) {
        kx = *reinterpret_cast<const u32x2*>(p.ke + tile * 32 + (ktok & 8));
        const uint8_t* kb = p.kc + (tile * 16 + ktok) * D + qg * 16;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < NC / 2; ++i) kraw[t * (NC / 2) + i] = stream<u32x4>(kb + 4 * t * D + i * 64);
      } else {
        const uint8_t* kb = p.kc + ((tile * 16 + ktok) * D + qg * 8) * 2;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < NC; ++i) kraw[t * NC + i] = stream<u32x4>(kb + (4 * t * D + i * 32) * 2);
      }
    };
    auto load_values = [&](int st) __attribute__((always_inline)) {
      const int vid = ids.pick(vblk);
      const size_t tile = (size_t)max(vid, 0) * p.Hkv + c.kvh;
      jb = c.j0 + st * 2;
      tb = (jb + vblk) * 16 + vtok;
      nv = vid >= 0 ? s.ctx - tb : 0;
      if constexpr (F8) vx = *reinterpret_cast<const u32x2*>(p.ke + tile * 32 + 16 + vtok);
      const uint8_t* vb = p.vc + ((tile * D + r) * 16 + vtok) * (F8 ? 1 : 2);
#pragma unroll
      for (int mt = 0; mt < NMT; ++mt) vraw[mt] = stream<VLoad>(vb + mt * (F8 ? 256 : 512));
    };

    int st = wave;
    if (st < steps) {
      ids.fetch(st);
      ids.take(st);
      load_keys();
      load_values(st);
      ids.fetch(min(st + kRowWaves, steps - 1));
    }

    uint64_t mask[RT];
    bf16x8 qf[RT][NC];
    float m_run[RT], l_run[RT];
    f32x4 acc[RT][NMT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int row = t * 16 + r, at = c.row0 + min(row, c.rows - 1);
      const uint16_t* qrow = p.q + row_of(p, s, c.kvh, at) * D;
      mask[t] = DRAFTS ? mask_of_row(p, s, at) : 0;
#pragma unroll
      for (int i = 0; i < NC; ++i)
        qf[t][i] =
            row < c.rows ? ld_bf16x8(qrow + (F8 ? (i >> 1) * 64 + qg * 16 + (i & 1) * 8 : i * 32 + qg * 8)) : zero_bf16x8();
      m_run[t] = kNegInf;
      l_run[t] = 0.f;
#pragma unroll
      for (int mt = 0; mt < NMT; ++mt) acc[t][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    wait_for_loads();
    for (; st < steps; st += kRowWaves) {
      const int next = st + kRowWaves;  // (behind the last step: block 0, which all waves read there)
      f32x4 sc[RT][2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        bf16x8 kf[NC];
        if constexpr (F8) {
          const float f = exp2_whole((int8_t)(kx[k] >> (8 * (r & 3))));
#pragma unroll
          for (int i = 0; i < NC / 2; ++i) {
            const u32x4 w = kraw[k * (NC / 2) + i];
            kf[2 * i] = widen_bf16(w[0], w[1], f);
            kf[2 * i + 1] = widen_bf16(w[2], w[3], f);
          }
        } else {
#pragma unroll
          for (int i = 0; i < NC; ++i) kf[i] = __builtin_bit_cast(bf16x8, kraw[k * NC + i]);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) sc[t][k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
          for (int t = 0; t < RT; ++t)
            sc[t][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[i], qf[t][i], sc[t][k], 0, 0, 0);
      }
      // (nothing moves across: the loads take the registers that the keys leave)
      __builtin_amdgcn_sched_barrier(0);
      const int tb_now = tb, nv_now = nv, jb_now = jb;
      ids.take(next);
      load_keys();
      ids.fetch(min(next + kRowWaves, steps - 1));
      __builtin_amdgcn_sched_barrier(0);

      if (!((!DRAFTS || (jb_now + 2) * 16 <= start) && __all(nv_now >= 8))) {  // drafts, or places that hold nothing
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const uint32_t seen =
              DRAFTS ? seen_bits(mask[t], tb_now, start, nv_now) : seen_bits(0, tb_now, tb_now + 8, nv_now);
#pragma unroll
          for (int e = 0; e < 8; ++e) sc[t][e / 4][e & 3] = (seen >> e & 1u) ? sc[t][e / 4][e & 3] : kNegInf;
        }
        // zeros behind the context, so that 0 times what lies there is 0
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt) vraw[mt] = keep_bytes(vraw[mt], F8 ? nv_now : 2 * nv_now);
        if constexpr (DRAFTS) {
          bool odd = false;
#pragma unroll
          for (int mt = 0; mt < NMT; ++mt) vraw[mt] = without_odd<F8>(vraw[mt], odd);
          if (odd) s_odd[wave] |= kOddTaken;
        }
        if constexpr (F8) vx = keep_bytes(vx, nv_now);
        if constexpr (F8 && DRAFTS) vx = legal_exponents(vx);
      }
      const u32x2 ve = F8 ? (vx ^ 0x80808080u) - (128 - kExpBias) * 0x01010101u : vx;  // (no byte borrows)
      Weights w[RT];
      softmax_step<F8>(sc, ve, p.scale_log2, m_run, l_run, acc, w);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int part = 0; part < Weights::kParts; ++part)
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt) {
          VFrag v;
          if constexpr (F8)
            v = widen_f16(vraw[mt][0], vraw[mt][1]);
          else
            v = __builtin_bit_cast(bf16x8, vraw[mt]);
#pragma unroll
          for (int t = 0; t < RT; ++t) acc[t][mt] = w[t].mul(part, v, acc[t][mt]);
        }
      __builtin_amdgcn_sched_barrier(0);
      load_values(next);
    }

    // ---- merge the waves, in a fixed order: the upper half deposits, the lower adds ----
#pragma unroll
    for (int t = 0; t < RT; ++t) finish_row<F8>(l_run[t], acc[t]);
#pragma unroll
    for (int half = kRowWaves / 2; half >= 1; half /= 2) {
      __syncthreads();
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
          put_partial<D>(so + (((wave % half) * RT + t) * 16 + r) * LDO, qg, m_run[t], l_run[t], acc[t]);
      }
      __syncthreads();
      if (wave < half) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
          add_partial<D>(so + ((wave * RT + t) * 16 + r) * LDO, qg, m_run[t], l_run[t], acc[t]);
      }
    }
    if (wave == 0) {
      if (lane == 0 && (int)blockIdx.x == c.first)
        p.span[((size_t)b * p.Hkv + c.kvh) * p.max_passes + c.pass] = make_int2(c.first, c.last);
#pragma unroll
      for (int t = 0; t < RT; ++t) store_rows<D, F8>(p, s, c, c.row0 + t * 16 + r, qg, m_run[t], l_run[t], acc[t], s_odd);
    }
  }
  if constexpr (DRAFTS) add_odd<D, F8, 2>(kFewLeast, s_odd);
}

// ---------------------------------------------------------------------------
// More rows, WR waves on row tiles of their own, and 4 / WR on
// halves of a step's tokens: up to 64 rows WR = 2 (two tiles a wave share what it reads from LDS), else 4.
// A step is 64 tokens (four blocks) of the work-group. Its threads load
// the tiles as they lie (16 bytes each, whole 128-byte lines), a step ahead, and put
// them into LDS as 16-bit operands: K [token][D] with the tokens in the order of the
// first product's tiles, V^T [D][token], padded rows.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int D, bool F8, int WR>
__global__ __launch_bounds__(64 * kRowWaves, kManyPerCu) void attn_many_kernel(RowsParams p) {
  constexpr int NC = D / 32, NMT = D / 16;
  constexpr int ES = F8 ? 1 : 2;
  constexpr int CPB = D * ES;                     // 16-byte chunks of a block's K (and V) tile
  constexpr int NL = 4 * CPB / (64 * kRowWaves);  // those of a thread, 4 blocks
  constexpr int LDK = D + 16, LDV = 64 + 16;      // padded rows in LDS (16-bit elements; 8: 0.7% slower)
  constexpr int LDO = D + 4;                      // row of a partial in LDS: O, then (m, l)
  constexpr int TS = kRowWaves / WR;              // waves that share a step's tokens
  typedef std::conditional_t<F8, HalfWeights, TwoWeights> Weights;
  typedef std::conditional_t<F8, f16x8, bf16x8> VFrag;
  constexpr int kTileBytes = (64 * LDK + D * LDV) * 2, kPartBytes = TS == 2 ? WR * kTiles * 16 * LDO * 4 : 0;
  __shared__ __attribute__((aligned(16))) uint8_t sm[kTileBytes > kPartBytes ? kTileBytes : kPartBytes];
  __shared__ __attribute__((aligned(16))) uint8_t sx[F8 ? 64 : 8];  // the values' exponents, kExpBias added
  __shared__ int s_odd[kRowWaves];
  uint16_t* sk = reinterpret_cast<uint16_t*>(sm);
  uint16_t* sv = sk + 64 * LDK;
  float* so = reinterpret_cast<float*>(sm);

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int r = lane & 15, qg = lane >> 4;

  clear_empty<D>(p);
  int per, x, x1, b, base;
  if (!find_range(p, kManyLeast, lane, per, x, x1, b, base)) return;
  if (lane == 0) s_odd[wave] = 0;
  while (x < x1) {
    const Seq s = seq_of(p, b);
    const int all = p.Hkv * s.passes * unit_len(p, s);
    if (x >= base + all) {
      base += all;
      ++b;
      continue;
    }
    int xn;
    const Piece c = piece_at(p, s, base, x, x1, per, xn);
    x = xn;
    if (c.j1 <= c.j0) break;
    const int start = s.ctx - s.n;  // place of the first draft
    const int steps = (c.j1 - c.j0 + 3) / 4;
    // the wave's row tiles
    const int per_wave = (c.tiles + WR - 1) / WR;
    const int group = wave % WR, half = wave / WR;
    const int t0 = group * per_wave, mine = max(min(c.tiles - t0, per_wave), 0);
    // Block ids by vector loads, 64 a register and the next 64 ahead. -1: no such block.
    // (Plain variables: a struct of them stayed in memory.)
    const int32_t* table = p.bt + (size_t)b * p.max_blocks;
    auto load_id = [&](int j) __attribute__((always_inline)) { return table[min(j, c.j1 - 1)]; };
    int ids_now = load_id(c.j0 + lane), ids_next = load_id(c.j0 + 64 + lane), chunk = 0;
    int id0 = -1, id1 = -1, id2 = -1, id3 = -1;
    auto take_ids = [&](int st) __attribute__((always_inline)) {
      const int at = st * 4;
      if (at >> 6 != chunk) {  // (steps come one by one)
        chunk = at >> 6;
        ids_now = ids_next;
        ids_next = load_id(c.j0 + (chunk + 1) * 64 + lane);
      }
      const auto id_at = [&](int i) {
        const int id = __builtin_amdgcn_readlane(ids_now, (at & 63) + i);
        return (uint32_t)id < (uint32_t)p.num_blocks && c.j0 + at + i < c.j1 ? id : -1;
      };
      id0 = id_at(0);
      id1 = id_at(1);
      id2 = id_at(2);
      id3 = id_at(3);
    };
    auto pick = [&](int i) __attribute__((always_inline)) {
      const int low = (i & 1) ? id1 : id0, high = (i & 1) ? id3 : id2;
      return (i & 2) ? high : low;
    };

    // ---- a step's chunks: chunk i of the thread lies in block blk(i), the wave's ----
    u32x4 kraw[NL], vraw[NL];
    uint32_t kx[NL];
    int vx[NL];
    auto blk = [&](int i) __attribute__((always_inline)) { return (i * kRowWaves + wave) * 64 / CPB; };
    auto within = [&](int i) __attribute__((always_inline)) { return (i * 64 * kRowWaves + tid) % CPB; };
    auto heads_block = [&](int i) __attribute__((always_inline)) { return (i * kRowWaves + wave) * 64 % CPB == 0; };
    auto load = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const size_t tile = (size_t)max(pick(blk(i)), 0) * p.Hkv + c.kvh;
        // (a scalar base and an offset of 32 bits per lane)
        const uint8_t *kb = p.kc + tile * (16 * D * ES), *vb = p.vc + tile * (16 * D * ES);
        const uint32_t off = within(i) * 16;
        kraw[i] = stream<u32x4>(kb + off);
        vraw[i] = stream<u32x4>(vb + off);
        if constexpr (F8) {
          const int8_t* eb = p.ke + tile * 32;
          kx[i] = *reinterpret_cast<const uint32_t*>(eb + (uint32_t)(within(i) / (D / 16) & 12));
          if (heads_block(i)) vx[i] = eb[(uint32_t)(16 + (lane & 15))];
        }
      }
    };
    // (n0 .. n3: cached tokens of the blocks; zeros behind them, so that 0 times what lies there is 0)
    auto store = [&](bool whole, int n0, int n1, int n2, int n3) __attribute__((always_inline)) {
      if (!whole) {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const int k = blk(i), nv = k == 0 ? n0 : k == 1 ? n1 : k == 2 ? n2 : n3;
          vraw[i] = without_odd<F8>(keep_bytes(vraw[i], F8 ? nv : 2 * (nv - (within(i) & 1) * 8)), odd);
          if constexpr (F8) vx[i] = (lane & 15) < nv ? vx[i] : 0;
        }
        if (odd) s_odd[wave] |= kOddTaken;
      }
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int k = blk(i), w = within(i);
        const int o = w / (D * ES / 16), u = (k & 1) * 16 + o;
        uint16_t* kd = sk + ((k >> 1) * 32 + ((u >> 2) & 1) * 16 + (u >> 3) * 4 + (u & 3)) * LDK +
                       (w % (D * ES / 16)) * (16 / ES);
        const u32x4 v = vraw[i];
        if constexpr (F8) {
          const float f = exp2_whole((int8_t)(kx[i] >> (8 * (o & 3))));
          *reinterpret_cast<bf16x8*>(kd) = widen_bf16(kraw[i][0], kraw[i][1], f);
          *reinterpret_cast<bf16x8*>(kd + 8) = widen_bf16(kraw[i][2], kraw[i][3], f);
          uint16_t* vd = sv + w * LDV + k * 16;
          *reinterpret_cast<f16x8*>(vd) = widen_f16(v[0], v[1]);
          *reinterpret_cast<f16x8*>(vd + 8) = widen_f16(v[2], v[3]);
          // (0 to 242, whatever a draft that nobody sees holds: its 2^e is finite)
          if (heads_block(i) && lane < 16) sx[k * 16 + lane] = (uint8_t)max(vx[i] + kExpBias, 0);
        } else {
          *reinterpret_cast<u32x4*>(kd) = kraw[i];
          *reinterpret_cast<u32x4*>(sv + (w >> 1) * LDV + k * 16 + (w & 1) * 8) = v;
        }
      }
    };

    take_ids(0);
    load();

    auto run_steps = [&](auto count) __attribute__((always_inline)) {
      constexpr int N = decltype(count)::value;
      constexpr int N1 = N > 0 ? N : 1;
      bf16x8 qf[N1][NC];
      uint64_t mask[N1];
      float m_run[N1], l_run[N1];
      f32x4 acc[N1][NMT];
#pragma unroll
      for (int t = 0; t < N; ++t) {
        const int row = (t0 + t) * 16 + r;
        const int at = c.row0 + min(row, c.rows - 1);
        const uint16_t* src = p.q + row_of(p, s, c.kvh, at) * D + qg * 8;
        mask[t] = mask_of_row(p, s, at);
#pragma unroll
        for (int i = 0; i < NC; ++i) qf[t][i] = row < c.rows ? ld_bf16x8(src + i * 32) : zero_bf16x8();
        m_run[t] = kNegInf;
        l_run[t] = 0.f;
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt) acc[t][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      wait_for_loads();
      for (int st = 0; st < steps; ++st) {
        const int jb = c.j0 + st * 4;
        const bool whole = (jb + 4) * 16 <= start && (id0 | id1 | id2 | id3) >= 0;  // every row sees every token
        int n0 = 16, n1 = 16, n2 = 16, n3 = 16;
        if (!whole) {
          const auto cached = [&](int id, int i) { return id >= 0 ? min(max(s.ctx - (jb + i) * 16, 0), 16) : 0; };
          n0 = cached(id0, 0), n1 = cached(id1, 1), n2 = cached(id2, 2), n3 = cached(id3, 3);
        }
        lds_barrier();  // every wave is done with the step before
        store(whole, n0, n1, n2, n3);
        if (st + 1 < steps) {
          take_ids(st + 1);
          load();
        }
        lds_barrier();
        if constexpr (N > 0) {
#pragma unroll
          for (int part = 0; part < 2 / TS; ++part) {
            const int h = TS == 2 ? half : part;  // the slice of 32 tokens
            const u32x2 ve = F8 ? *reinterpret_cast<const u32x2*>(sx + h * 32 + qg * 8) : u32x2{0, 0};
            f32x4 sc[N][2];
#pragma unroll
            for (int t = 0; t < N; ++t) sc[t][0] = sc[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
            auto key = [&](int k, int i) __attribute__((always_inline)) {
              return ld_bf16x8(sk + ((h * 2 + k) * 16 + r) * LDK + i * 32 + qg * 8);
            };
            auto value = [&](int mt) __attribute__((always_inline)) {
              return *reinterpret_cast<const VFrag*>(sv + (mt * 16 + r) * LDV + h * 32 + qg * 8);
            };
            // (8-bit cache: all of a product's operands are read before it starts, the values'
            // before the softmax. A bf16 step ahead takes twice the registers and leaves none
            // for that.)
            bf16x8 kf[2][NC];
            VFrag vf[NMT];
            if constexpr (F8) {
#pragma unroll
              for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < NC; ++i) kf[k][i] = key(k, i);
              __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < NC; ++i) {
              if constexpr (!F8) kf[0][i] = key(0, i), kf[1][i] = key(1, i);
#pragma unroll
              for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int t = 0; t < N; ++t)
                  sc[t][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[k][i], qf[t][i], sc[t][k], 0, 0, 0);
            }
            if constexpr (F8) {
#pragma unroll
              for (int mt = 0; mt < NMT; ++mt) vf[mt] = value(mt);
              __builtin_amdgcn_sched_barrier(0);
            }
            if (!whole) {
              // the lane's 8 tokens lie in block 2 h + (qg >> 1)
              const int tb = jb * 16 + h * 32 + qg * 8;
              const int nv = (h == 0 ? ((qg & 2) ? n1 : n0) : ((qg & 2) ? n3 : n2)) - (qg & 1) * 8;
#pragma unroll
              for (int t = 0; t < N; ++t) {
                const uint32_t seen = seen_bits(mask[t], tb, start, nv);
#pragma unroll
                for (int e = 0; e < 8; ++e) sc[t][e / 4][e & 3] = (seen >> e & 1u) ? sc[t][e / 4][e & 3] : kNegInf;
              }
            }
            Weights w[N];
            softmax_step<F8>(sc, ve, p.scale_log2, m_run, l_run, acc, w);
            // (two channel tiles at a time: no product waits for the one before it)
#pragma unroll
            for (int mt = 0; mt < NMT; mt += 2) {
              if constexpr (!F8) vf[mt] = value(mt), vf[mt + 1] = value(mt + 1);
#pragma unroll
              for (int part = 0; part < Weights::kParts; ++part)
#pragma unroll
                for (int i = mt; i < mt + 2; ++i)
#pragma unroll
                  for (int t = 0; t < N; ++t) acc[t][i] = w[t].mul(part, vf[i], acc[t][i]);
            }
          }
        }
      }
#pragma unroll
      for (int t = 0; t < N; ++t) finish_row<F8>(l_run[t], acc[t]);
      if constexpr (TS == 2) {  // the second half's waves deposit, the first half's add
        lds_barrier();
        if (half == 1) {
#pragma unroll
          for (int t = 0; t < N; ++t)
            put_partial<D>(so + ((group * kTiles + t) * 16 + r) * LDO, qg, m_run[t], l_run[t], acc[t]);
        }
        lds_barrier();
        if (half == 0) {
#pragma unroll
          for (int t = 0; t < N; ++t)
            add_partial<D>(so + ((group * kTiles + t) * 16 + r) * LDO, qg, m_run[t], l_run[t], acc[t]);
        }
      }
      if (half == 0) {
#pragma unroll
        for (int t = 0; t < N; ++t)
          store_rows<D, F8>(p, s, c, c.row0 + (t0 + t) * 16 + r, qg, m_run[t], l_run[t], acc[t], s_odd + wave);
      }
    };
    if (mine == 0) run_steps(std::integral_constant<int, 0>{});
    if (mine == 1) run_steps(std::integral_constant<int, 1>{});
    if (mine == 2) run_steps(std::integral_constant<int, 2>{});
    if (tid == 0 && (int)blockIdx.x == c.first)
      p.span[((size_t)b * p.Hkv + c.kvh) * p.max_passes + c.pass] = make_int2(c.first, c.last);
  }
  add_odd<D, F8, 4>(kManyLeast, s_odd);
}

// ---------------------------------------------------------------------------
// Four channels of a row, merged from its unit's partials.
struct Merged {
  float M = kNegInf, L = 0.f;
  f32x4 O = {0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ void join(float2 ml, f32x4 o) {
    const float mn = fmaxf(M, ml.x);
    const float mu = (mn == kNegInf) ? 0.f : mn;
    const float wa = fast_exp2(M - mu), wb = fast_exp2(ml.x - mu);
    L = times_exp2(L, M - mu) + times_exp2(ml.y, ml.x - mu);
    O = O * wa + o * wb;
    M = mn;
  }
  __device__ __forceinline__ void store(uint16_t* out) const {
    const float inv = L > 0.f ? 1.f / L : 0.f;
    ushort4 v;
    v.x = f2bf(O[0] * inv);
    v.y = f2bf(O[1] * inv);
    v.z = f2bf(O[2] * inv);
    v.w = f2bf(O[3] * inv);
    *reinterpret_cast<ushort4*>(out) = v;
  }
};

// Sequence of a token row: the last one that starts at it or before it.
__device__ __forceinline__ int seq_of_row(const RowsParams& p, int trow) {
  if (!p.cu) return trow;
  int lo = 0, hi = p.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (p.cu[mid] <= trow)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// Merge launch: work-group (token row, kv head) merges the token's G rows over the
// pieces of its unit in work-group order, a thread 4 channels of a row.
template <int D>
__global__ __launch_bounds__(256) void attn_rows_merge_kernel(RowsParams p) {
  constexpr int D4 = D / 4;
  const int trow = blockIdx.x, kvh = blockIdx.y;
  const int b = seq_of_row(p, trow);
  const Seq s = seq_of(p, b);
  const int tok = trow - s.row0;
  if (s.ctx == 0 || tok < 0 || tok >= s.take) return;
  const int G = p.G;
  for (int it = threadIdx.x; it < G * D4; it += 256) {
    const int h = it / D4, d4 = it - h * D4;
    const int row = tok * G + h, pass = row / (s.tiles * 16);
    const int2 sp = p.span[((size_t)b * p.Hkv + kvh) * p.max_passes + pass];
    if (sp.x == sp.y) continue;  // written by the first launch
    Merged a;
#pragma unroll 4
    for (int w = sp.x; w <= sp.y; ++w) {
      const size_t at = part_row(p, s, kvh, row, w);
      a.join(*reinterpret_cast<const float2*>(p.part_ml + at * 2), *reinterpret_cast<const f32x4*>(p.part_o + at * D + d4 * 4));
    }
    a.store(p.out + ((size_t)trow * p.Hq + kvh * G + h) * D + d4 * 4);
  }
}

// The same for units cut into many pieces (a few long contexts): a work-group per
// (token row, query head), whose 256 / (D / 4) groups of lanes each take a share of
// the pieces, then the shares in order through LDS.
template <int D>
__global__ __launch_bounds__(256) void attn_rows_merge_many_kernel(RowsParams p) {
  constexpr int D4 = D / 4, NG = 256 / D4;
  __shared__ float sm_m[NG], sm_l[NG];
  __shared__ __attribute__((aligned(16))) float sm_o[NG][D];
  const int trow = blockIdx.x, head = blockIdx.y;
  const int kvh = head / p.G;
  const int b = seq_of_row(p, trow);
  const Seq s = seq_of(p, b);
  const int tok = trow - s.row0;
  if (s.ctx == 0 || tok < 0 || tok >= s.take) return;
  const int row = tok * p.G + (head - kvh * p.G), pass = row / (s.tiles * 16);
  const int2 sp = p.span[((size_t)b * p.Hkv + kvh) * p.max_passes + pass];
  if (sp.x == sp.y) return;
  const int grp = threadIdx.x / D4, d4 = threadIdx.x - grp * D4;
  const int per = (sp.y - sp.x + NG) / NG;
  const int w0 = sp.x + grp * per, w1 = min(w0 + per, sp.y + 1);
  Merged a;
#pragma unroll 4
  for (int w = w0; w < w1; ++w) {
    const size_t at = part_row(p, s, kvh, row, w);
    a.join(*reinterpret_cast<const float2*>(p.part_ml + at * 2), *reinterpret_cast<const f32x4*>(p.part_o + at * D + d4 * 4));
  }
  if (d4 == 0) {
    sm_m[grp] = a.M;
    sm_l[grp] = a.L;
  }
  *reinterpret_cast<f32x4*>(&sm_o[grp][d4 * 4]) = a.O;
  __syncthreads();
  if (grp != 0) return;
#pragma unroll
  for (int i = 1; i < NG; ++i)
    a.join(make_float2(sm_m[i], sm_l[i]), *reinterpret_cast<const f32x4*>(&sm_o[i][d4 * 4]));
  a.store(p.out + ((size_t)trow * p.Hq + head) * D + d4 * 4);
}

// ---------------------------------------------------------------------------
// Host side.
namespace {

// What a launch takes: the kernel for few rows with one, two or four row tiles, or the
// one for more rows with two or four waves on them.
enum RowsKind { kFewOne, kFewTwo, kFewFour, kManyTwo, kManyFour };
struct RowsPlan {
  RowsKind kind;
  int pass_tiles, passes, pass_rows, grid;
  bool whole;  // a work-group per unit, no merge
};

// Blocks that a unit's piece is charged for (its queries, merge of waves, partials). 8
// and 24 instead: 64 sequences of decode attention 134.3 and 133.1 us, with 16 132.4; 32 with 8
// drafts 96.4 and 94.1, with 16 93.5.
constexpr int kRowsUnitCost = 16;

// Units take a work-group each, without partials and the merge's launch, where
// contexts are at most kWholeCtx and one round of work-groups holds all units (4
// sequences of about 80 tokens, 8 / 2 heads x 64: 6.3 us a call, 9.5 with the even
// split), and where contexts are at most kWholeManyCtx and the units fill 3/4 to one
// round of what the GPU holds at once, or 3/2 rounds and more: dealt out as
// work-groups end, they balance themselves (256 sequences of median 500 tokens, 64 / 8
// heads x 128: 79.6 us, 86.8 with the even split; 128 of median 1000: 64.4 and 66.7; 128 of
// median 400 with up to 8 drafts: 61.7 and 71.4). Between one round and 3/2 the last units run
// alone. Numbers of rounds, 64 / 8 heads x 128, us with a work-group per unit and with
// the even split:
//                             0.75       1          1.02       1.25       1.5        2
//   one token, 2048 each    44.6 44.2  48.1 50.1  64.1 59.3  66.9 69.0  70.9 79.4  93.3 106
//   one token, median 1000  33.4 29.2  40.0 36.7  40.7 38.1  44.1 42.6  46.6 49.5  64.7 64.5
//   8 drafts, 2048 each     68.4 70.6  69.4 76.8   108 93.2   109 107    111 125    139 158
//   8 drafts, median 1000   59.1 50.8  66.0 64.6  67.0 65.2  83.6 72.7  86.3 83.4   105 107
constexpr int kWholeCtx = 512;
constexpr int kWholeManyCtx = 2048;
constexpr long long kWholeUnits = 1ll << 23;  // (a launch has less than 2^32 threads)

// Pieces per unit from which the merge shares a unit's pieces among lanes, if there are
// few rows: at most kFewRows a CU (one row of 64 heads in 64 pieces: 139.6 us in all, 148.5
// in one chain of loads; 8 rows: 200 and 204; 64 rows in 16 pieces: 199.8 and 197.8; 200
// of 32 heads in 8 pieces: 87.6 and 83.7).
constexpr int kManyPieces = 8;
constexpr int kFewRows = 8;

int compute_units() {
  static std::atomic<int> cached{0};
  int cus = cached.load(std::memory_order_relaxed);
  if (cus == 0) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess ||
        hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
      cus = 256;
    cached.store(cus, std::memory_order_relaxed);
  }
  return cus;
}

long long positions_bound(const RowsShape& s, int passes) {
  return (long long)s.B * s.Hkv * passes * ((s.max_ctx + 15) / 16 + kRowsUnitCost);
}

RowsPlan rows_plan(const RowsShape& s) {
  RowsPlan r;
  const int rows = s.max_n * (s.Hq / s.Hkv), all = (rows + 15) / 16;
  r.kind = kManyFour;
  if (all <= 1)
    r.kind = kFewOne;
  else if (all <= 2 && s.f8)
    r.kind = kFewTwo;
  else if (all <= 2 * kTiles)
    r.kind = s.f8 && s.D == 64 ? kFewFour : kManyTwo;
  r.pass_tiles = r.kind == kFewOne ? 1 : r.kind == kFewTwo ? 2 : r.kind == kManyFour ? 4 * kTiles : 4;
  r.passes = all > r.pass_tiles ? (all + r.pass_tiles - 1) / r.pass_tiles : 1;
  r.pass_rows = rows < r.pass_tiles * 16 ? rows : r.pass_tiles * 16;
  const long long most = (long long)compute_units() * (r.kind == kFewOne ? few_per_cu(s.D, 1) : kManyPerCu);
  const long long units = (long long)s.B * s.Hkv * r.passes;
  r.whole = (s.max_ctx <= kWholeCtx && units <= most) ||
            (s.max_ctx <= kWholeManyCtx && 4 * units >= 3 * most && (units <= most || 2 * units >= 3 * most) &&
             units <= kWholeUnits);
  const long long P = r.whole ? units : (positions_bound(s, r.passes) + 7) / 8;
  r.grid = (int)(P < 1 ? 1 : P < most || r.whole ? P : most);
  return r;
}

size_t part_rows(const RowsShape& s, const RowsPlan& r) {
  return r.whole ? 1 : (size_t)s.T * s.Hq + (size_t)r.grid * r.pass_rows;
}

template <int D, bool F8>
void launch_tiles(const RowsParams& p, const RowsPlan& r, hipStream_t stream) {
  const dim3 grid(r.grid), block(64 * kRowWaves);
  if (!p.cu)
    attn_few_kernel<D, true, false, 1><<<grid, block, 0, stream>>>(p);
  else if (r.kind == kFewOne)
    attn_few_kernel<D, F8, true, 1><<<grid, block, 0, stream>>>(p);
  else if (r.kind == kFewTwo)
    attn_few_kernel<D, true, true, 2><<<grid, block, 0, stream>>>(p);
  else if (r.kind == kFewFour)
    attn_few_kernel<64, true, true, 4><<<grid, block, 0, stream>>>(p);
  else if (r.kind == kManyFour)
    attn_many_kernel<D, F8, 4><<<grid, block, 0, stream>>>(p);
  else if constexpr (!(F8 && D == 64))  // (that takes kFewFour in its place)
    attn_many_kernel<D, F8, 2><<<grid, block, 0, stream>>>(p);
}

}  // namespace

bool rows_shape_fits(const RowsShape& s) {
  static_assert(kRowsUnitCost == 16, "the bound as the header states it");
  const int rows = s.max_n * (s.Hq / s.Hkv), most = kTiles * kRowWaves * 16;
  const int passes = rows > most ? (rows + most - 1) / most : 1;
  return positions_bound(s, passes) < (1ll << 30) && (long long)s.T * s.Hq < (1ll << 30);
}

size_t rows_workspace_bytes(const RowsShape& s) {
  const RowsPlan r = rows_plan(s);
  return align_up(part_rows(s, r) * s.D * sizeof(float), 256) + align_up(part_rows(s, r) * 2 * sizeof(float), 256) +
         align_up((size_t)s.B * s.Hkv * r.passes * sizeof(int2), 256);
}

hipError_t launch_attn_rows(const RowsShape& s, const RowsTensors& t, void* ws, hipStream_t stream) {
  if (s.T == 0 || s.max_n == 0) return hipSuccess;
  const RowsPlan r = rows_plan(s);
  RowsParams p;
  p.q = t.q;
  p.kc = static_cast<const uint8_t*>(t.k_cache);
  p.vc = static_cast<const uint8_t*>(t.v_cache);
  p.ke = t.kv_exp;
  p.bt = t.block_table;
  p.cl = t.context_lens;
  p.cu = t.cu_seqlens;
  p.masks = t.masks;
  p.out = t.out;
  char* w = static_cast<char*>(ws);
  p.part_o = reinterpret_cast<float*>(w);
  w += align_up(part_rows(s, r) * s.D * sizeof(float), 256);
  p.part_ml = reinterpret_cast<float*>(w);
  w += align_up(part_rows(s, r) * 2 * sizeof(float), 256);
  p.span = reinterpret_cast<int2*>(w);
  p.B = s.B;
  p.T = s.T;
  p.Hq = s.Hq;
  p.Hkv = s.Hkv;
  p.G = s.Hq / s.Hkv;
  p.max_n = s.max_n;
  p.max_passes = r.passes;
  p.pass_rows = r.pass_rows;
  p.pass_tiles = r.pass_tiles;
  p.max_blocks = s.max_blocks;
  p.num_blocks = s.num_blocks;
  p.max_ctx = s.max_ctx;
  p.unit_cost = kRowsUnitCost;
  p.whole = r.whole;
  p.scale_log2 = (s.scale != 0.f ? s.scale : 1.0f / sqrtf((float)s.D)) * kLog2e;
  {
    ProfScope ps("attn_rows", stream);
    if (s.D == 128 && s.f8)
      launch_tiles<128, true>(p, r, stream);
    else if (s.D == 128)
      launch_tiles<128, false>(p, r, stream);
    else if (s.f8)
      launch_tiles<64, true>(p, r, stream);
    else
      launch_tiles<64, false>(p, r, stream);
  }
  if (r.grid > 1 && !r.whole) {  // (else no unit is cut)
    ProfScope ps("attn_rows_merge", stream);
    const bool many = r.grid >= kManyPieces * (long long)s.B * s.Hkv * r.passes &&
                      (long long)s.T * s.Hq <= kFewRows * compute_units();
    const dim3 grid(s.T, many ? s.Hq : s.Hkv);
    if (many && s.D == 128)
      attn_rows_merge_many_kernel<128><<<grid, 256, 0, stream>>>(p);
    else if (many)
      attn_rows_merge_many_kernel<64><<<grid, 256, 0, stream>>>(p);
    else if (s.D == 128)
      attn_rows_merge_kernel<128><<<grid, 256, 0, stream>>>(p);
    else
      attn_rows_merge_kernel<64><<<grid, 256, 0, stream>>>(p);
  }
  return hipGetLastError();
}

}  // namespace aflex
