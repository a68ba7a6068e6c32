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
// A value's exponent joins the score: with s' = s + e the weight of the codes is
// P' = 2^(s' - M'), M' the running maximum of s', and the row's sum is that of
// P' 2^-e. So the largest contribution has weight 1, and P' enters the product as
// fp16 (11 bits; below 2^-14 steps of 2^-24 of the largest) with the codes as fp16,
// exactly. Over a bf16 cache a weight enters as two bf16 values, the rounded
// weight and what its rounding left: 16 bits. (One bf16 value, 8 bits, would show
// beside the output's own rounding: 2.1e-3 of the norm instead of 1.65e-3.)
//
// Two kernels. Up to 16 rows (decode attention): the waves of a work-group take the
// tokens in turns, keys and values go from memory straight into the matrix
// operands' registers, a step ahead. More rows: the waves share the tokens, 64 a
// step, which the work-group turns into 16-bit operands in LDS once, and each has
// row tiles of its own.
//
// The blocks of all units (sequence, kv head, pass over the rows) are laid end to
// end, and each work-group takes a consecutive range of them, so that long and
// short contexts fill the GPU alike; a unit cut between work-groups leaves fp32
// partials that a second launch merges in order.
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
constexpr int kMostTiles = 3;  // row tiles of a wave (16 rows each)

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
// piece it adds.
__device__ __forceinline__ int unit_len(const RowsParams& p, const Seq& s) { return ((s.ctx + 15) >> 4) + p.unit_cost; }

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
  per = max((total + P - 1) / P, least);
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
  const int ustart = base + unit * len + p.unit_cost, nb = len - p.unit_cost;
  c.j0 = max(x - ustart, 0);
  c.j1 = min(nb, x1 - ustart);  // (j0 or less where the range ends inside the unit's charge)
  c.first = ustart / per;
  c.last = (ustart + nb - 1) / per;
  c.row0 = c.pass * s.tiles * 16;
  c.rows = min(s.take * p.G - c.row0, s.tiles * 16);
  c.tiles = (c.rows + 15) >> 4;
  xn = min(ustart + nb, x1);
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

// A row tile's result (lane: row `row`, channels 16 mt + 4 qg ..) to out, or to the piece's partial.
template <int D>
__device__ __forceinline__ void store_rows(const RowsParams& p, const Seq& s, const Piece& c, int row, int qg, float m,
                                           float l, const f32x4 (&acc)[D / 16]) {
  if (row >= c.row0 + c.rows) return;
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

// The weights of 8 tokens as operands of the second product: fp16 (8-bit cache), or
// the rounded bf16 and what the rounding left.
struct HalfWeights {
  f16x8 w;
  __device__ __forceinline__ void set(int i, float a, float b) {
    w[i] = static_cast<_Float16>(a);
    w[i + 1] = static_cast<_Float16>(b);
  }
  __device__ __forceinline__ f32x4 mul(f16x8 v, f32x4 acc) const {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(v, w, acc, 0, 0, 0);
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
  __device__ __forceinline__ f32x4 mul(bf16x8 v, f32x4 acc) const {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, hi), acc, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, lo), acc, 0, 0, 0);
  }
};

// One row tile's softmax over NS slices of 8 tokens per lane: scores x (masked: -inf)
// to weights, the running maximum m and sum l, and the accumulators' rescaling. F8:
// ve and vinv are the tokens' value exponents and 2^-exponent.
template <bool F8, int NS, int NMT, class Weights>
__device__ __forceinline__ void softmax_step(f32x4 (&x)[2 * NS], const float (*ve)[8], const float (*vinv)[8],
                                             float scale_log2, float& m, float& l, f32x4 (&acc)[NMT], Weights (&w)[NS]) {
  if constexpr (F8) {
#pragma unroll
    for (int e = 0; e < 8 * NS; ++e) x[e / 4][e & 3] = fmaf(x[e / 4][e & 3], scale_log2, ve[e / 8][e & 7]);
  }
  float mx = x[0][0];
#pragma unroll
  for (int e = 1; e < 8 * NS; ++e) mx = fmaxf(mx, x[e / 4][e & 3]);
  const float m_new = fmaxf(m, F8 ? row_max(mx) : row_max(mx) * scale_log2);
  const float m_use = (m_new == kNegInf) ? 0.f : m_new;
  if (!__all(m_new == m)) {
    const float alpha = fast_exp2(m - m_use);
    l *= alpha;
#pragma unroll
    for (int mt = 0; mt < NMT; ++mt) acc[mt] *= alpha;
    m = m_new;
  }
#pragma unroll
  for (int e = 0; e < 8 * NS; e += 2) {
    float u[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float s = x[(e + i) / 4][(e + i) & 3];
      u[i] = fast_exp2(F8 ? s - m_use : fmaf(s, scale_log2, -m_use));
      l = F8 ? fmaf(u[i], vinv[e / 8][(e + i) & 7], l) : l + u[i];
    }
    w[e / 8].set(e & 7, u[0], u[1]);
  }
}

// Block ids of a piece by scalar loads: raw ones are fetched a step ahead, and become
// ids (-1: no such block) when their step's loads are made.
template <int NB>
struct BlockIds {
  typedef const int32_t __attribute__((address_space(4))) * Table;
  Table table;
  int j0, j1, num_blocks;
  int raw0, raw1, raw2, raw3;
  int id0, id1, id2, id3;

  __device__ __forceinline__ BlockIds(const RowsParams& p, int b, int j0, int j1)
      : table((Table)(reinterpret_cast<uintptr_t>(p.bt + (size_t)b * p.max_blocks))), j0(j0), j1(j1),
        num_blocks(p.num_blocks), raw0(-1), raw1(-1), raw2(-1), raw3(-1), id0(-1), id1(-1), id2(-1), id3(-1) {}
  __device__ __forceinline__ void fetch(int st) {
    const int j = j0 + st * NB, e = j1 - 1;
    raw0 = table[min(j, e)];
    raw1 = table[min(j + 1, e)];
    if constexpr (NB == 4) {
      raw2 = table[min(j + 2, e)];
      raw3 = table[min(j + 3, e)];
    }
  }
  __device__ __forceinline__ int fine(int id, int j) const { return j < j1 && id >= 0 && id < num_blocks ? id : -1; }
  __device__ __forceinline__ void take(int st) {
    const int j = j0 + st * NB;
    id0 = fine(raw0, j);
    id1 = fine(raw1, j + 1);
    if constexpr (NB == 4) {
      id2 = fine(raw2, j + 2);
      id3 = fine(raw3, j + 3);
    }
  }
  __device__ __forceinline__ int pick(int i) const {
    const int low = (i & 1) ? id1 : id0;
    if constexpr (NB == 4) return (i & 2) ? ((i & 1) ? id3 : id2) : low;
    return low;
  }
};

constexpr int few_per_cu(int D) { return D == 64 ? 3 : 2; }

// Work-groups that a CU holds at once (by registers and LDS).
constexpr int many_per_cu(int tiles) { return tiles == 1 ? 3 : 2; }

}  // namespace

// ---------------------------------------------------------------------------
// Up to 16 rows: a step is 32 tokens (two blocks) of one wave.
template <int D, bool F8>
__global__ __launch_bounds__(64 * kRowWaves, few_per_cu(D)) void attn_few_kernel(RowsParams p) {
  constexpr int NC = D / 32;       // k-chunks of the first product
  constexpr int NMT = D / 16;      // d-tiles of the second
  constexpr int NK = F8 ? NC : 2 * NC;  // 16-byte loads of a step's keys
  constexpr int LDO = D + 4;       // row of a partial in LDS: O, then (m, l)
  typedef std::conditional_t<F8, u32x2, u32x4> VLoad;  // a lane's 8 tokens of a channel
  typedef std::conditional_t<F8, HalfWeights, TwoWeights> Weights;
  __shared__ __attribute__((aligned(16))) float so[2 * 16 * LDO];  // partials of two waves

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int r = lane & 15, qg = lane >> 4;
  // The lane's places in a step: block and token of its key row (token + 4 t in tile
  // t), block and first token of its values.
  const int kblk = r >> 3, ktok = ((r >> 2) & 1) * 8 + (r & 3);
  const int vblk = qg >> 1, vtok = (qg & 1) * 8;

  clear_empty<D>(p);
  int per, x, x1, b, base;
  if (!find_range(p, 2 * kRowWaves, lane, per, x, x1, b, base)) return;
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
    BlockIds<2> ids(p, b, c.j0, c.j1);

    u32x4 kraw[NK];  // (8-bit codes come 16 channels a load, and the k-chunks take the channels in that order)
    VLoad vraw[NMT];
    u32x2 kx, vx;    // exponents of the 8 tokens around the lane's key rows, and of its values
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

    const int row = min(r, c.rows - 1);
    const uint16_t* qrow = p.q + row_of(p, s, c.kvh, row) * D;
    const uint64_t mask = mask_of_row(p, s, row);
    bf16x8 qf[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i)
      qf[i] = r < c.rows ? ld_bf16x8(qrow + (F8 ? (i >> 1) * 64 + qg * 16 + (i & 1) * 8 : i * 32 + qg * 8)) : zero_bf16x8();

    float m_run = kNegInf, l_run = 0.f;
    f32x4 acc[NMT];
#pragma unroll
    for (int mt = 0; mt < NMT; ++mt) acc[mt] = f32x4{0.f, 0.f, 0.f, 0.f};

    for (; st < steps; st += kRowWaves) {
      const int next = st + kRowWaves < steps ? st + kRowWaves : st;  // (the last step's loads are repeated)
      f32x4 sc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        bf16x8 kf[NC];
        if constexpr (F8) {
          const float f = exp2_whole((int8_t)(kx[t] >> (8 * (r & 3))));
#pragma unroll
          for (int i = 0; i < NC / 2; ++i) {
            const u32x4 w = kraw[t * (NC / 2) + i];
            kf[2 * i] = widen_bf16(w[0], w[1], f);
            kf[2 * i + 1] = widen_bf16(w[2], w[3], f);
          }
        } else {
#pragma unroll
          for (int i = 0; i < NC; ++i) kf[i] = __builtin_bit_cast(bf16x8, kraw[t * NC + i]);
        }
#pragma unroll
        for (int i = 0; i < NC; ++i) sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[i], qf[i], sc[t], 0, 0, 0);
      }
      // (nothing moves across: the loads take the registers that the keys leave)
      __builtin_amdgcn_sched_barrier(0);
      const int tb_now = tb, nv_now = nv, jb_now = jb;
      ids.take(next);
      load_keys();
      ids.fetch(min(next + kRowWaves, steps - 1));
      __builtin_amdgcn_sched_barrier(0);

      if (!((jb_now + 2) * 16 <= start && __all(nv_now >= 8))) {  // drafts, or places that hold nothing
        const uint32_t seen = seen_bits(mask, tb_now, start, nv_now);
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[e / 4][e & 3] = (seen >> e & 1u) ? sc[e / 4][e & 3] : kNegInf;
        // zeros behind the context, so that 0 times what lies there is 0
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt) vraw[mt] = keep_bytes(vraw[mt], F8 ? nv_now : 2 * nv_now);
        if constexpr (F8) vx = keep_bytes(vx, nv_now);
      }
      float ve[1][8], vinv[1][8];
      if constexpr (F8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int v = (int8_t)(vx[e / 4] >> (8 * (e & 3)));
          ve[0][e] = (float)v;
          vinv[0][e] = exp2_whole(-v);
        }
      }
      Weights w[1];
      softmax_step<F8, 1>(sc, ve, vinv, p.scale_log2, m_run, l_run, acc, w);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int mt = 0; mt < NMT; ++mt) {
        if constexpr (F8)
          acc[mt] = w[0].mul(widen_f16(vraw[mt][0], vraw[mt][1]), acc[mt]);
        else
          acc[mt] = w[0].mul(__builtin_bit_cast(bf16x8, vraw[mt]), acc[mt]);
      }
      __builtin_amdgcn_sched_barrier(0);
      load_values(next);
    }

    // ---- merge the waves, in a fixed order: the upper half deposits, the lower adds ----
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);
#pragma unroll
    for (int half = kRowWaves / 2; half >= 1; half /= 2) {
      float* o = so + ((wave % half) * 16 + r) * LDO;
      __syncthreads();
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt) *reinterpret_cast<f32x4*>(o + mt * 16 + 4 * qg) = acc[mt];
        if (qg == 0) *reinterpret_cast<float2*>(o + D) = make_float2(m_run, l_run);
      }
      __syncthreads();
      if (wave < half) {
        const float2 ml = *reinterpret_cast<const float2*>(o + D);
        const float mn = fmaxf(m_run, ml.x);
        const float mu = (mn == kNegInf) ? 0.f : mn;
        const float wa = fast_exp2(m_run - mu), wb = fast_exp2(ml.x - mu);
        l_run = l_run * wa + ml.y * wb;
        m_run = mn;
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt)
          acc[mt] = acc[mt] * wa + *reinterpret_cast<const f32x4*>(o + mt * 16 + 4 * qg) * wb;
      }
    }
    if (wave == 0) {
      if (lane == 0 && (int)blockIdx.x == c.first)
        p.span[((size_t)b * p.Hkv + c.kvh) * p.max_passes + c.pass] = make_int2(c.first, c.last);
      store_rows<D>(p, s, c, c.row0 + r, qg, m_run, l_run, acc);
    }
  }
}

// ---------------------------------------------------------------------------
// More rows: a step is 64 tokens (four blocks) of the work-group. Its threads load
// the tiles as they lie (16 bytes each, whole 128-byte lines), a step ahead, and put
// them into LDS as 16-bit operands: K [token][D] with the tokens in the order of the
// first product's tiles, V^T [D][token], padded rows.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int D, bool F8, int RT>
__global__ __launch_bounds__(64 * kRowWaves, many_per_cu(RT)) void attn_many_kernel(RowsParams p) {
  constexpr int NC = D / 32, NMT = D / 16;
  constexpr int ES = F8 ? 1 : 2;
  constexpr int CPB = D * ES;                     // 16-byte chunks of a block's K (and V) tile
  constexpr int NL = 4 * CPB / (64 * kRowWaves);  // those of a thread, 4 blocks
  constexpr int LDK = D + 8, LDV = 64 + 8;        // padded rows in LDS (16-bit elements)
  constexpr int NS = RT == 3 ? 1 : 2;             // 32-token slices per softmax step
  typedef std::conditional_t<F8, HalfWeights, TwoWeights> Weights;
  typedef std::conditional_t<F8, f16x8, bf16x8> VFrag;
  __shared__ __attribute__((aligned(16))) uint16_t sk[64 * LDK];
  __shared__ __attribute__((aligned(16))) uint16_t sv[D * LDV];
  __shared__ __attribute__((aligned(16))) float sx[2][F8 ? 64 : 1];  // the values' exponents, and 2^-exponent

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int r = lane & 15, qg = lane >> 4;

  clear_empty<D>(p);
  int per, x, x1, b, base;
  if (!find_range(p, 8, lane, per, x, x1, b, base)) return;
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
    const int per_wave = (c.tiles + kRowWaves - 1) / kRowWaves;
    const int t0 = wave * per_wave, mine = max(min(c.tiles - t0, per_wave), 0);
    BlockIds<4> ids(p, b, c.j0, c.j1);

    // ---- a step's chunks: chunk i of the thread lies in block blk(i), the wave's ----
    u32x4 kraw[NL], vraw[NL];
    uint32_t kx[NL];
    int vx = 0;
    auto blk = [&](int i) __attribute__((always_inline)) { return (i * kRowWaves + wave) * 64 / CPB; };
    auto within = [&](int i) __attribute__((always_inline)) { return (i * 64 * kRowWaves + tid) % CPB; };
    auto load = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const size_t tile = (size_t)max(ids.pick(blk(i)), 0) * p.Hkv + c.kvh;
        const size_t at = tile * (16 * D * ES) + within(i) * 16;
        kraw[i] = stream<u32x4>(p.kc + at);
        vraw[i] = stream<u32x4>(p.vc + at);
        if constexpr (F8) kx[i] = *reinterpret_cast<const uint32_t*>(p.ke + tile * 32 + (within(i) / (D / 16) & 12));
      }
      if constexpr (F8) {
        if (wave == 0) {
          const size_t tile = (size_t)max(ids.pick(lane >> 4), 0) * p.Hkv + c.kvh;
          vx = p.ke[tile * 32 + 16 + (lane & 15)];
        }
      }
    };
    // (n0 .. n3: cached tokens of the blocks; zeros behind them, so that 0 times what lies there is 0)
    auto store = [&](int n0, int n1, int n2, int n3) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int k = blk(i), w = within(i);
        const int nv = k == 0 ? n0 : k == 1 ? n1 : k == 2 ? n2 : n3;  // cached tokens of the block
        const int o = w / (D * ES / 16), u = (k & 1) * 16 + o;
        uint16_t* kd = sk + ((k >> 1) * 32 + ((u >> 2) & 1) * 16 + (u >> 3) * 4 + (u & 3)) * LDK +
                       (w % (D * ES / 16)) * (16 / ES);
        u32x4 v = vraw[i];
        if constexpr (F8) {
          if (nv < 16) v = keep_bytes(v, nv);
          const float f = exp2_whole((int8_t)(kx[i] >> (8 * (o & 3))));
          *reinterpret_cast<bf16x8*>(kd) = widen_bf16(kraw[i][0], kraw[i][1], f);
          *reinterpret_cast<bf16x8*>(kd + 8) = widen_bf16(kraw[i][2], kraw[i][3], f);
          uint16_t* vd = sv + w * LDV + k * 16;
          *reinterpret_cast<f16x8*>(vd) = widen_f16(v[0], v[1]);
          *reinterpret_cast<f16x8*>(vd + 8) = widen_f16(v[2], v[3]);
        } else {
          if (nv < 16) v = keep_bytes(v, 2 * (nv - (w & 1) * 8));
          *reinterpret_cast<u32x4*>(kd) = kraw[i];
          *reinterpret_cast<u32x4*>(sv + (w >> 1) * LDV + k * 16 + (w & 1) * 8) = v;
        }
      }
      if constexpr (F8) {
        if (wave == 0) {
          const int i = lane >> 4, nv = i == 0 ? n0 : i == 1 ? n1 : i == 2 ? n2 : n3;
          const int v = (lane & 15) < nv ? vx : 0;
          sx[0][lane] = (float)v;
          sx[1][lane] = exp2_whole(-v);
        }
      }
    };

    ids.fetch(0);
    ids.take(0);
    load();
    ids.fetch(min(1, steps - 1));

    auto run_steps = [&](auto count) __attribute__((always_inline)) {
      constexpr int N = decltype(count)::value;
      bf16x8 qf[N > 0 ? N : 1][NC];
      uint64_t mask[N > 0 ? N : 1];
      float m_run[N > 0 ? N : 1], l_run[N > 0 ? N : 1];
      f32x4 acc[N > 0 ? N : 1][NMT];
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
      for (int st = 0; st < steps; ++st) {
        const int jb = c.j0 + st * 4;
        const auto cached = [&](int id, int i) { return id >= 0 ? min(max(s.ctx - (jb + i) * 16, 0), 16) : 0; };
        const int n0 = cached(ids.id0, 0), n1 = cached(ids.id1, 1), n2 = cached(ids.id2, 2), n3 = cached(ids.id3, 3);
        lds_barrier();  // every wave is done with the step before
        store(n0, n1, n2, n3);
        if (st + 1 < steps) {
          ids.take(st + 1);
          load();
          ids.fetch(min(st + 2, steps - 1));
        }
        lds_barrier();
        if constexpr (N > 0) {
          const bool whole = (jb + 4) * 16 <= start && n0 + n1 + n2 + n3 == 64;
#pragma unroll
          for (int h = 0; h < 2 / NS; ++h) {
            f32x4 sc[N][2 * NS];
#pragma unroll
            for (int t = 0; t < N; ++t)
#pragma unroll
              for (int k = 0; k < 2 * NS; ++k) sc[t][k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 2 * NS; ++k)
#pragma unroll
              for (int i = 0; i < NC; ++i) {
                const bf16x8 kf = ld_bf16x8(sk + ((h * 2 * NS + k) * 16 + r) * LDK + i * 32 + qg * 8);
#pragma unroll
                for (int t = 0; t < N; ++t)
                  sc[t][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][i], sc[t][k], 0, 0, 0);
              }
            if (!whole) {
#pragma unroll
              for (int k = 0; k < NS; ++k) {
                const int sl = h * NS + k;  // 32-token slice: the lane's 8 tokens lie in its block 2 sl + (qg >> 1)
                const int in = sl == 0 ? ((qg & 2) ? n1 : n0) : ((qg & 2) ? n3 : n2);
                const int tb = jb * 16 + sl * 32 + qg * 8;
#pragma unroll
                for (int t = 0; t < N; ++t) {
                  const uint32_t seen = seen_bits(mask[t], tb, start, in - (qg & 1) * 8);
#pragma unroll
                  for (int e = 0; e < 8; ++e)
                    sc[t][2 * k + e / 4][e & 3] = (seen >> e & 1u) ? sc[t][2 * k + e / 4][e & 3] : kNegInf;
                }
              }
            }
            float ve[NS][8], vinv[NS][8];
            if constexpr (F8) {
#pragma unroll
              for (int k = 0; k < NS; ++k)
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                  const int at = (h * NS + k) * 32 + qg * 8 + e;
                  const f32x4 a = *reinterpret_cast<const f32x4*>(&sx[0][at]);
                  const f32x4 d = *reinterpret_cast<const f32x4*>(&sx[1][at]);
#pragma unroll
                  for (int i = 0; i < 4; ++i) ve[k][e + i] = a[i], vinv[k][e + i] = d[i];
                }
            }
            Weights w[N][NS];
#pragma unroll
            for (int t = 0; t < N; ++t)
              softmax_step<F8, NS>(sc[t], ve, vinv, p.scale_log2, m_run[t], l_run[t], acc[t], w[t]);
#pragma unroll
            for (int mt = 0; mt < NMT; ++mt)
#pragma unroll
              for (int k = 0; k < NS; ++k) {
                const VFrag vf = *reinterpret_cast<const VFrag*>(sv + (mt * 16 + r) * LDV + (h * NS + k) * 32 + qg * 8);
#pragma unroll
                for (int t = 0; t < N; ++t) acc[t][mt] = w[t][k].mul(vf, acc[t][mt]);
              }
          }
        }
      }
#pragma unroll
      for (int t = 0; t < N; ++t) {
        l_run[t] += __shfl_xor(l_run[t], 16);
        l_run[t] += __shfl_xor(l_run[t], 32);
        store_rows<D>(p, s, c, c.row0 + (t0 + t) * 16 + r, qg, m_run[t], l_run[t], acc[t]);
      }
    };
    if (mine == 0) run_steps(std::integral_constant<int, 0>{});
    if (mine == 1) run_steps(std::integral_constant<int, 1>{});
    if constexpr (RT >= 2) {
      if (mine == 2) run_steps(std::integral_constant<int, 2>{});
    }
    if constexpr (RT >= 3) {
      if (mine == 3) run_steps(std::integral_constant<int, 3>{});
    }
    if (tid == 0 && (int)blockIdx.x == c.first)
      p.span[((size_t)b * p.Hkv + c.kvh) * p.max_passes + c.pass] = make_int2(c.first, c.last);
  }
}

// ---------------------------------------------------------------------------
// Merge launch: work-group (token row, kv head) merges the token's G rows over the
// pieces of its unit in work-group order, a thread 4 channels of a row.
template <int D>
__global__ __launch_bounds__(256) void attn_rows_merge_kernel(RowsParams p) {
  constexpr int D4 = D / 4;
  const int trow = blockIdx.x, kvh = blockIdx.y;
  int b = trow;
  if (p.cu) {  // the last sequence that starts at trow or before it
    int lo = 0, hi = p.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (p.cu[mid] <= trow)
        lo = mid;
      else
        hi = mid - 1;
    }
    b = lo;
  }
  const Seq s = seq_of(p, b);
  const int tok = trow - s.row0;
  if (s.ctx == 0 || tok < 0 || tok >= s.take) return;
  const int G = p.G;
  for (int it = threadIdx.x; it < G * D4; it += 256) {
    const int h = it / D4, d4 = it - h * D4;
    const int row = tok * G + h, pass = row / (s.tiles * 16);
    const int2 sp = p.span[((size_t)b * p.Hkv + kvh) * p.max_passes + pass];
    if (sp.x == sp.y) continue;  // written by the first launch
    float M = kNegInf, L = 0.f;
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int w = sp.x; w <= sp.y; ++w) {
      const size_t at = part_row(p, s, kvh, row, w);
      const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + at * 2);
      const f32x4 o = *reinterpret_cast<const f32x4*>(p.part_o + at * D + d4 * 4);
      const float mn = fmaxf(M, ml.x);
      const float mu = (mn == kNegInf) ? 0.f : mn;
      const float wa = fast_exp2(M - mu), wb = fast_exp2(ml.x - mu);
      L = L * wa + ml.y * wb;
      O = O * wa + o * wb;
      M = mn;
    }
    const float inv = L > 0.f ? 1.f / L : 0.f;
    ushort4 v;
    v.x = f2bf(O[0] * inv);
    v.y = f2bf(O[1] * inv);
    v.z = f2bf(O[2] * inv);
    v.w = f2bf(O[3] * inv);
    *reinterpret_cast<ushort4*>(p.out + ((size_t)trow * p.Hq + kvh * G + h) * D + d4 * 4) = v;
  }
}

// ---------------------------------------------------------------------------
// Host side.
namespace {

// What a launch takes: row tiles of a wave (0: the kernel for up to 16 rows).
struct RowsPlan {
  int tiles, pass_tiles, passes, pass_rows, grid;
};

constexpr int kRowsUnitCost = 8;

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
  r.tiles = all <= 1 ? 0 : all <= kRowWaves ? 1 : all <= 2 * kRowWaves ? 2 : kMostTiles;
  r.pass_tiles = r.tiles == 0 ? 1 : r.tiles * kRowWaves;
  r.passes = all > r.pass_tiles ? (all + r.pass_tiles - 1) / r.pass_tiles : 1;
  r.pass_rows = rows < r.pass_tiles * 16 ? rows : r.pass_tiles * 16;
  const long long most = (long long)compute_units() * (r.tiles == 0 ? few_per_cu(s.D) : many_per_cu(r.tiles));
  const long long P = (positions_bound(s, r.passes) + 7) / 8;
  r.grid = (int)(P < 1 ? 1 : P < most ? P : most);
  return r;
}

size_t part_rows(const RowsShape& s, const RowsPlan& r) { return (size_t)s.T * s.Hq + (size_t)r.grid * r.pass_rows; }

template <int D, bool F8>
void launch_tiles(const RowsParams& p, const RowsPlan& r, hipStream_t stream) {
  const dim3 grid(r.grid), block(64 * kRowWaves);
  if (r.tiles == 0)
    attn_few_kernel<D, F8><<<grid, block, 0, stream>>>(p);
  else if (r.tiles == 1)
    attn_many_kernel<D, F8, 1><<<grid, block, 0, stream>>>(p);
  else if (r.tiles == 2)
    attn_many_kernel<D, F8, 2><<<grid, block, 0, stream>>>(p);
  else
    attn_many_kernel<D, F8, 3><<<grid, block, 0, stream>>>(p);
}

}  // namespace

bool rows_shape_fits(const RowsShape& s) {
  const int rows = s.max_n * (s.Hq / s.Hkv), most = kMostTiles * kRowWaves * 16;
  const long long passes = rows > most ? (rows + most - 1) / most : 1;
  return (long long)s.B * s.Hkv * passes * ((s.max_ctx + 15) / 16 + 16) < (1ll << 30) &&
         (long long)s.T * s.Hq < (1ll << 30);
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
  if (r.grid > 1) {  // one work-group cuts no unit
    ProfScope ps("attn_rows_merge", stream);
    const dim3 grid(s.T, s.Hkv);
    if (s.D == 128)
      attn_rows_merge_kernel<128><<<grid, 256, 0, stream>>>(p);
    else
      attn_rows_merge_kernel<64><<<grid, 256, 0, stream>>>(p);
  }
  return hipGetLastError();
}

}  // namespace aflex
