// Attention of a few query rows per (sequence, kv head) over a paged KV cache,
// gfx950: one new token per sequence over an 8-bit cache, and trees of drafted
// tokens over an 8-bit or a bf16 cache.
//
// The rows of a (sequence, kv head) are its n tokens times the G query heads of
// the group, row i G + h; they share every cached key and value, so a unit reads
// its cache once for up to 256 rows (a pass; more rows take more passes).
//
//   S^T[tok][row] = K[tok][:] . q[row][:]      (v_mfma_f32_16x16x32_bf16: 16 tokens
//                                               x 16 rows, a row tile)
//   O^T[d][row] += V^T[d][tok] . P^T[tok][row]
//
// with the running maximum and sum of a softmax per row. K and V go from memory
// straight into the matrix operands' registers, K and V of a step (32 bf16 or 64
// 8-bit tokens: 16 loads of 16 bytes per lane for D = 128) feed RT row tiles. The
// order of the tokens in the first product is chosen so that its output
// registers are the second product's operand. An 8-bit row is c 2^e: codes are
// turned into bf16 exactly, the key's 2^e on the way, the value's goes into the
// softmax weight. A weight enters the second product as two bf16 values, the
// rounded weight and what its rounding left: 16 bits.
//
// Work-groups of 4 waves. The blocks of all units are laid end to end, and each
// work-group takes a consecutive range of them, so that long and short contexts
// fill the GPU alike; a unit cut between work-groups leaves fp32 partials that a
// second launch merges in order. Inside a work-group up to 64 rows take their
// tokens in turns, a step per wave (the partials are merged through LDS in a fixed
// order); with up to 128 rows two waves share a step's rows, and above that four.
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
constexpr int kPassRows = 256;  // rows of a unit in one pass

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
  float* part_ml;           // [slots][2]  (running maximum in log2 units, sum)
  int2* span;               // [B Hkv passes]  first and last work-group of each unit's pieces
  int B, T, Hq, Hkv, G;
  int max_n, max_passes, pass_rows;  // bounds: tokens, passes, rows of a pass
  int max_blocks, num_blocks, max_ctx;
  int unit_cost;
  float scale_log2;
};

// A sequence as its lanes see it.
struct Seq {
  int row0;  // first token row
  int n;     // its tokens
  int take;  // those that are computed (n, or the caller's bound)
  int ctx;   // cached tokens
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
  return s;
}

// Units of a sequence (0 without rows or cached tokens) and positions of each in
// the flattened range.
__device__ __forceinline__ int units_of(const RowsParams& p, const Seq& s) {
  return s.ctx > 0 && s.take > 0 ? p.Hkv * ((s.take * p.G + kPassRows - 1) / kPassRows) : 0;
}

__device__ __forceinline__ int unit_len(const RowsParams& p, const Seq& s) { return ((s.ctx + 15) >> 4) + p.unit_cost; }

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

// First partial row of a unit's piece in work-group wg. Pieces are numbered along
// the range, and from one to the next either the unit advances by its rows or the
// work-group by one, or both: no two pieces share a row.
__device__ __forceinline__ size_t part_row(const RowsParams& p, const Seq& s, int kvh, int pass, int wg) {
  return (size_t)s.row0 * p.Hq + (size_t)kvh * s.take * p.G + (size_t)pass * kPassRows + (size_t)wg * p.pass_rows;
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ u32x4 stream16(const uint8_t* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
}

// Eight codes (two words) as bf16 times 2^scale's exponent.
__device__ __forceinline__ bf16x8 widen(uint32_t a, uint32_t b, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 w[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true)};
  return bf16x8{w[0][0], w[0][1], w[1][0], w[1][1], w[2][0], w[2][1], w[3][0], w[3][1]};
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

// How many of the TOK tokens from place `tb` on a draft with these mask bits sees,
// as bits; the sequence's drafts start at place `start`.
__device__ __forceinline__ uint32_t seen_bits(uint64_t mask, int tb, int start) {
  const int off = tb - start;
  if (off >= 64) return 0;
  if (off >= 0) return (uint32_t)(mask >> off);
  if (off <= -32) return ~0u;
  return ((uint32_t)mask << -off) | ((1u << -off) - 1u);
}

// Largest over the four lanes that hold a row (lane % 16).
__device__ __forceinline__ float row_max(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// Two weights as bf16 pairs: the rounded weights, and what the rounding left.
__device__ __forceinline__ void split_weights(float a, float b, uint32_t& hi, uint32_t& lo) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  hi = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
  lo = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a - __uint_as_float(hi << 16)),
                                           static_cast<__bf16>(b - __uint_as_float(hi & 0xffff0000u))});
}

}  // namespace

// D, 8-bit cache or bf16, row tiles of a wave, tokens of a lane in a step.
template <int D, bool F8, int RT, int TOK>
__global__ __launch_bounds__(64 * kRowWaves, 2) void attn_rows_kernel(RowsParams p) {
  constexpr int NC = D / 32;       // k-chunks of the first product
  constexpr int NMT = D / 16;      // d-tiles of the second
  constexpr int SB = TOK / 4;      // blocks of a step (4 TOK tokens), and its tiles in the first product
  constexpr int NK = SB * D / (F8 ? 64 : 32);  // loads of 16 bytes of its keys
  typedef std::conditional_t<F8 && TOK == 8, u32x2, u32x4> VLoad;  // a lane's values of a channel
  constexpr int PS = TOK / 8;      // 32-token slices of a step
  // Few rows: q in registers, values loaded a step ahead like the keys. Many: q in
  // LDS, and the values take the keys' registers behind the first product.
  constexpr bool EARLY = RT <= 2;
  constexpr int LDQ = D + 8;       // padded row of q in LDS
  constexpr int LDO = D + 4;       // row of a partial in LDS: O, then (m, l)
  constexpr int kQBytes = EARLY ? 0 : kPassRows * LDQ * 2;
  constexpr int kPartBytes = 2 * 16 * RT * LDO * 4;  // partials of two waves
  __shared__ __attribute__((aligned(16))) uint8_t sm[kQBytes > kPartBytes ? kQBytes : kPartBytes];
  __shared__ uint64_t sm_mask[EARLY ? 1 : kPassRows];
  uint16_t* sq = reinterpret_cast<uint16_t*>(sm);
  float* so = reinterpret_cast<float*>(sm);

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int r = lane & 15, qg = lane >> 4;
  const int G = p.G, wg = blockIdx.x, P = gridDim.x;
  // places of the lane in a step: block and token of its key row (token + 4 t in tile
  // t), block and first token of its values
  const int kblk = TOK == 16 ? r >> 2 : r >> 3, ktok = TOK == 16 ? r & 3 : ((r >> 2) & 1) * 8 + (r & 3);
  const int vblk = TOK == 16 ? qg : qg >> 1, vtok = TOK == 16 ? 0 : (qg & 1) * 8;

  // Rows of sequences without cached tokens are zeros.
  for (int b = wg; b < p.B; b += P) {
    const Seq s = seq_of(p, b);
    if (s.ctx == 0) {
      uint4* o = reinterpret_cast<uint4*>(p.out + (size_t)s.row0 * p.Hq * D);
      for (size_t i = tid; i < (size_t)s.take * p.Hq * (D / 8); i += 64 * kRowWaves) o[i] = make_uint4(0, 0, 0, 0);
    }
  }

  // ---- this work-group's range [x0, x1) of the flattened positions ----
  int total = 0;
  for (int c = 0; c < p.B; c += 64) {
    int len = 0;
    if (c + lane < p.B) {
      const Seq s = seq_of(p, c + lane);
      len = units_of(p, s) * unit_len(p, s);
    }
    total += sum64(len);
  }
  const int per = max((total + P - 1) / P, SB * kRowWaves);
  const long long xs = (long long)wg * per;
  if (xs >= total) return;
  const int x0 = (int)xs, x1 = min(x0 + per, total);
  int b = 0, base = 0;  // sequence of x0, and its first position
  for (int c = 0; c < p.B; c += 64) {
    int len = 0;
    if (c + lane < p.B) {
      const Seq s = seq_of(p, c + lane);
      len = units_of(p, s) * unit_len(p, s);
    }
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

  int x = x0;
  while (x < x1) {
    // ---- the piece: blocks [j0, j1) of unit (b, kvh, pass) ----
    const Seq s = seq_of(p, b);
    const int units = units_of(p, s), len = unit_len(p, s);
    if (units == 0 || x >= base + units * len) {
      base += units * len;
      ++b;
      continue;
    }
    const int unit = (x - base) / len;
    const int passes = units / p.Hkv;
    const int kvh = unit / passes, pass = unit - kvh * passes;
    const int ustart = base + unit * len + p.unit_cost;  // position of the unit's first block
    const int nb = len - p.unit_cost;
    const int j0 = max(x - ustart, 0), j1 = min(nb, x1 - ustart);
    x = min(ustart + nb, x1);
    if (j1 <= j0) break;  // the range ends inside the unit's leading charge
    const int start = s.ctx - s.n;  // place of the first draft
    const int rows = min(s.take * G - pass * kPassRows, kPassRows);
    const int tiles = (rows + 15) >> 4;
    // waves that share a step's rows, and the row tiles of each
    const int share = tiles <= RT ? 1 : tiles <= 2 * RT ? 2 : 4;
    const int per_wave = (tiles + share - 1) / share;
    const int t0 = (wave % share) * per_wave;
    const int mine = max(min(tiles - t0, per_wave), 0);
    const int turns = kRowWaves / share, turn = wave / share;
    const int row_base = pass * kPassRows;

    // ---- block ids: scalar loads, a step ahead of the keys' ----
    typedef const int32_t __attribute__((address_space(4))) * ScalarTable;
    const ScalarTable table = (ScalarTable)(reinterpret_cast<uintptr_t>(p.bt + (size_t)b * p.max_blocks));
    const int steps = mine > 0 ? (j1 - j0 + SB - 1) / SB : 0;
    int raw0 = -1, raw1 = -1, raw2 = -1, raw3 = -1;  // as the table has them
    int id0 = -1, id1 = -1, id2 = -1, id3 = -1;      // of the step at hand; -1: no such block
    auto fetch_ids = [&](int st) __attribute__((always_inline)) {
      const int j = j0 + st * SB;
      raw0 = table[min(j, j1 - 1)];
      raw1 = table[min(j + 1, j1 - 1)];
      if constexpr (SB == 4) {
        raw2 = table[min(j + 2, j1 - 1)];
        raw3 = table[min(j + 3, j1 - 1)];
      }
    };
    auto take_ids = [&](int st) __attribute__((always_inline)) {
      const int j = j0 + st * SB;
      const auto fine = [&](int id, int at) { return at < j1 && id >= 0 && id < p.num_blocks ? id : -1; };
      id0 = fine(raw0, j);
      id1 = fine(raw1, j + 1);
      if constexpr (SB == 4) {
        id2 = fine(raw2, j + 2);
        id3 = fine(raw3, j + 3);
      }
    };
    // (blocks that do not exist are read at block 0 and masked)
    auto pick = [&](int blk) __attribute__((always_inline)) {
      const int low = (blk & 1) ? id1 : id0;
      if constexpr (SB == 4) return (blk & 2) ? ((blk & 1) ? id3 : id2) : low;
      return low;
    };
    u32x4 kraw[NK];   // (8-bit codes come 16 channels a load, and the k-chunks take the channels in that order)
    VLoad vraw[NMT];
    u32x4 kx, vx;     // exponents of the lane's key block, and of its value block
    int tb = 0, nv = 0, jb = 0;  // place of the lane's first token, how many of them are cached; first block
    auto load_keys = [&]() __attribute__((always_inline)) {
      const size_t tile = (size_t)max(pick(kblk), 0) * p.Hkv + kvh;
      if constexpr (F8) {
        kx = *reinterpret_cast<const u32x4*>(p.ke + tile * 32);
        const uint8_t* kb = p.kc + (tile * 16 + ktok) * D + qg * 16;
#pragma unroll
        for (int t = 0; t < SB; ++t)
#pragma unroll
          for (int c = 0; c < NC / 2; ++c) kraw[t * (NC / 2) + c] = stream16(kb + 4 * t * D + c * 64);
      } else {
        const uint8_t* kb = p.kc + ((tile * 16 + ktok) * D + qg * 8) * 2;
#pragma unroll
        for (int t = 0; t < SB; ++t)
#pragma unroll
          for (int c = 0; c < NC; ++c) kraw[t * NC + c] = stream16(kb + (4 * t * D + c * 32) * 2);
      }
    };
    auto load_values = [&](int st) __attribute__((always_inline)) {
      const int vid = pick(vblk);
      const size_t tile = (size_t)max(vid, 0) * p.Hkv + kvh;
      jb = j0 + st * SB;
      tb = (jb + vblk) * 16 + vtok;
      nv = vid >= 0 ? s.ctx - tb : 0;
      if constexpr (F8) {
        vx = *reinterpret_cast<const u32x4*>(p.ke + tile * 32 + 16);
        const uint8_t* vb = p.vc + (tile * D + r) * 16 + vtok;
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt)
          vraw[mt] = __builtin_nontemporal_load(reinterpret_cast<const VLoad*>(vb + mt * 256));
      } else {
        const uint8_t* vb = p.vc + ((tile * D + r) * 16 + vtok) * 2;
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt) vraw[mt] = stream16(vb + mt * 512);
      }
    };

    int st = turn;
    if (st < steps) {
      fetch_ids(st);
      take_ids(st);
      load_keys();
      if constexpr (EARLY) load_values(st);
      fetch_ids(min(st + turns, steps - 1));
    }

    // ---- q: row i G + h of the pass is token i, head kvh G + h ----
    auto q_row = [&](int row) {
      const int tok = (row_base + row) / G, h = row_base + row - tok * G;
      return p.q + ((size_t)(s.row0 + tok) * p.Hq + kvh * G + h) * D;
    };
    auto q_channel = [&](int c) { return F8 ? (c >> 1) * 64 + qg * 16 + (c & 1) * 8 : c * 32 + qg * 8; };
    auto mask_row = [&](int row) {
      const int tok = (row_base + row) / G;
      return p.masks ? p.masks[s.row0 + tok] : (2ull << tok) - 1ull;
    };
    bf16x8 qreg[EARLY ? RT : 1][NC];
    uint64_t mask_of[EARLY ? RT : 1];
    if constexpr (EARLY) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const int row = t * 16 + r;
        mask_of[t] = mask_row(min(row, rows - 1));
        const uint16_t* src = q_row(min(row, rows - 1));
#pragma unroll
        for (int c = 0; c < NC; ++c) qreg[t][c] = row < rows ? ld_bf16x8(src + q_channel(c)) : zero_bf16x8();
      }
    } else {
      __syncthreads();
      for (int i = tid; i < tiles * 16 * (D / 8); i += 64 * kRowWaves) {
        const int row = i / (D / 8), c = i % (D / 8);
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row < rows) v = *reinterpret_cast<const uint4*>(q_row(row) + c * 8);
        *reinterpret_cast<uint4*>(sq + row * LDQ + c * 8) = v;
      }
      for (int row = tid; row < tiles * 16; row += 64 * kRowWaves) sm_mask[row] = mask_row(min(row, rows - 1));
      __syncthreads();
    }

    float m_run[RT], l_run[RT];
    f32x4 acc[RT][NMT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      m_run[t] = kNegInf;
      l_run[t] = 0.f;
#pragma unroll
      for (int mt = 0; mt < NMT; ++mt) acc[t][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // The steps of this wave with N row tiles.
    auto run_steps = [&](auto count) __attribute__((always_inline)) {
      constexpr int N = decltype(count)::value;
      for (; st < steps; st += turns) {
        const int next = st + turns < steps ? st + turns : st;  // (the last step's loads are repeated, of data at hand)
        // ---- S^T: the tiles of the step, each against all row tiles ----
        f32x4 sc[N][SB];
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
          for (int k = 0; k < SB; ++k) sc[t][k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < SB; ++k) {
          bf16x8 kf[NC];
          if constexpr (F8) {
            const uint32_t ex = TOK == 16 ? kx[k] : (r & 4) ? kx[(2 + k) & 3] : kx[k & 1];
            const float f = exp2_whole((int8_t)(ex >> (8 * (r & 3))));
#pragma unroll
            for (int c = 0; c < NC / 2; ++c) {
              const u32x4 w = kraw[k * (NC / 2) + c];
              kf[2 * c] = widen(w[0], w[1], f);
              kf[2 * c + 1] = widen(w[2], w[3], f);
            }
          } else {
#pragma unroll
            for (int c = 0; c < NC; ++c) kf[c] = __builtin_bit_cast(bf16x8, kraw[k * NC + c]);
          }
#pragma unroll
          for (int t = 0; t < N; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c) {
              bf16x8 qf;
              if constexpr (EARLY)
                qf = qreg[t][c];
              else
                qf = ld_bf16x8(sq + ((t0 + t) * 16 + r) * LDQ + q_channel(c));
              sc[t][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[c], qf, sc[t][k], 0, 0, 0);
            }
        }
        // (nothing moves across: the loads take the registers that the keys leave)
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!EARLY) load_values(st);
        const int tb_now = tb, nv_now = nv, jb_now = jb;
        if constexpr (EARLY) {
          take_ids(next);
          load_keys();
          fetch_ids(min(next + turns, steps - 1));
        }
        __builtin_amdgcn_sched_barrier(0);

        // ---- weights ----
        if (!((jb_now + SB) * 16 <= start && __all(nv_now >= TOK))) {  // drafts, or places that hold nothing
          const uint32_t cached = nv_now >= TOK ? (1u << TOK) - 1u : nv_now <= 0 ? 0u : (1u << nv_now) - 1u;
#pragma unroll
          for (int t = 0; t < N; ++t) {
            const uint64_t mask = EARLY ? mask_of[t] : sm_mask[(t0 + t) * 16 + r];
            const uint32_t seen = cached & seen_bits(mask, tb_now, start);
#pragma unroll
            for (int e = 0; e < TOK; ++e) sc[t][e / 4][e & 3] = (seen >> e & 1u) ? sc[t][e / 4][e & 3] : kNegInf;
          }
          if (!__all(nv_now >= TOK)) {  // zeros behind the context, so that 0 times what lies there is 0
#pragma unroll
            for (int mt = 0; mt < NMT; ++mt) vraw[mt] = keep_bytes(vraw[mt], F8 ? nv_now : 2 * nv_now);
          }
        }
        uint32_t hi[N][TOK / 2], lo[N][TOK / 2];
#pragma unroll
        for (int t = 0; t < N; ++t) {
          float mx = sc[t][0][0];
#pragma unroll
          for (int e = 1; e < TOK; ++e) mx = fmaxf(mx, sc[t][e / 4][e & 3]);
          const float m_new = fmaxf(m_run[t], row_max(mx) * p.scale_log2);
          const float m_use = (m_new == kNegInf) ? 0.f : m_new;
          if (!__all(m_new == m_run[t])) {
            const float alpha = fast_exp2(m_run[t] - m_use);
            l_run[t] *= alpha;
#pragma unroll
            for (int mt = 0; mt < NMT; ++mt) acc[t][mt] *= alpha;
            m_run[t] = m_new;
          }
          float ps = 0.f;
#pragma unroll
          for (int e = 0; e < TOK; e += 2) {
            float w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int at = e + i;
              w[i] = fast_exp2(fmaf(sc[t][at / 4][at & 3], p.scale_log2, -m_use));
              ps += w[i];
              if constexpr (F8) {
                const uint32_t ex = TOK == 16 ? vx[at / 4] : (qg & 1) ? vx[(2 + at / 4) & 3] : vx[at / 4 & 1];
                w[i] = __builtin_ldexpf(w[i], (int8_t)(ex >> (8 * (at & 3))));
              }
            }
            split_weights(w[0], w[1], hi[t][e / 2], lo[t][e / 2]);
          }
          l_run[t] += ps;
        }

        // ---- O^T ----
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt) {
          bf16x8 vf[PS];
          if constexpr (F8) {
            vf[0] = widen(vraw[mt][0], vraw[mt][1], 1.f);
            if constexpr (PS == 2) vf[1] = widen(vraw[mt][2], vraw[mt][3], 1.f);
          } else {
            vf[0] = __builtin_bit_cast(bf16x8, vraw[mt]);
          }
#pragma unroll
          for (int t = 0; t < N; ++t)
#pragma unroll
            for (int k = 0; k < PS; ++k) {
              const uint32_t *h = hi[t] + 4 * k, *l = lo[t] + 4 * k;
              acc[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  vf[k], __builtin_bit_cast(bf16x8, u32x4{h[0], h[1], h[2], h[3]}), acc[t][mt], 0, 0, 0);
              acc[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  vf[k], __builtin_bit_cast(bf16x8, u32x4{l[0], l[1], l[2], l[3]}), acc[t][mt], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (EARLY) {
          load_values(next);
        } else {
          take_ids(next);
          load_keys();
          fetch_ids(min(next + turns, steps - 1));
        }
      }
    };
    if constexpr (RT == 1) {
      run_steps(std::integral_constant<int, 1>{});
    } else {
      if (mine == 1) run_steps(std::integral_constant<int, 1>{});
      if (mine == 2) run_steps(std::integral_constant<int, 2>{});
      if constexpr (RT == 4) {
        if (mine == 3) run_steps(std::integral_constant<int, 3>{});
        if (mine == 4) run_steps(std::integral_constant<int, 4>{});
      }
    }

    // ---- merge the waves that took turns, in a fixed order ----
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      l_run[t] += __shfl_xor(l_run[t], 16);
      l_run[t] += __shfl_xor(l_run[t], 32);
    }
    // Halving: the upper half of the turns deposits, the lower half adds. A slot
    // holds a wave's row tiles: O [row][LDO], then (m, l) behind each row's O.
    for (int half = turns / 2; half >= 1; half /= 2) {
      const int slot = (turn % half) * share + wave % share;  // of 2 at most
      float* mine_o = so + slot * 16 * RT * LDO;
      __syncthreads();
      if (turn >= half && turn < 2 * half) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          if (t >= mine) break;
          float* o = mine_o + (t * 16 + r) * LDO;
#pragma unroll
          for (int mt = 0; mt < NMT; ++mt) *reinterpret_cast<f32x4*>(o + mt * 16 + 4 * qg) = acc[t][mt];
          if (qg == 0) *reinterpret_cast<float2*>(o + D) = make_float2(m_run[t], l_run[t]);
        }
      }
      __syncthreads();
      if (turn < half) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          if (t >= mine) break;
          const float* o = mine_o + (t * 16 + r) * LDO;
          const float2 ml = *reinterpret_cast<const float2*>(o + D);
          const float mn = fmaxf(m_run[t], ml.x);
          const float mu = (mn == kNegInf) ? 0.f : mn;
          const float wa = fast_exp2(m_run[t] - mu), wb = fast_exp2(ml.x - mu);
          l_run[t] = l_run[t] * wa + ml.y * wb;
          m_run[t] = mn;
#pragma unroll
          for (int mt = 0; mt < NMT; ++mt)
            acc[t][mt] = acc[t][mt] * wa + *reinterpret_cast<const f32x4*>(o + mt * 16 + 4 * qg) * wb;
        }
      }
    }

    // ---- out, or the unit's partial ----
    if (turn == 0) {
      const int first = ustart / per, last = (ustart + nb - 1) / per;
      if (lane == 0 && wave == 0 && wg == first)
        p.span[((size_t)b * p.Hkv + kvh) * p.max_passes + pass] = make_int2(first, last);
      const size_t part = part_row(p, s, kvh, pass, wg);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const int row = (t0 + t) * 16 + r;
        if (t >= mine || row >= rows) continue;
        if (first == last) {
          const int tok = (row_base + row) / G, h = row_base + row - tok * G;
          const float inv = l_run[t] > 0.f ? 1.f / l_run[t] : 0.f;
          uint16_t* o = p.out + ((size_t)(s.row0 + tok) * p.Hq + kvh * G + h) * D + 4 * qg;
#pragma unroll
          for (int mt = 0; mt < NMT; ++mt) {
            ushort4 v;
            v.x = f2bf(acc[t][mt][0] * inv);
            v.y = f2bf(acc[t][mt][1] * inv);
            v.z = f2bf(acc[t][mt][2] * inv);
            v.w = f2bf(acc[t][mt][3] * inv);
            *reinterpret_cast<ushort4*>(o + mt * 16) = v;
          }
        } else {
          float* o = p.part_o + (part + row) * D + 4 * qg;
#pragma unroll
          for (int mt = 0; mt < NMT; ++mt) *reinterpret_cast<f32x4*>(o + mt * 16) = acc[t][mt];
          if (qg == 0) *reinterpret_cast<float2*>(p.part_ml + (part + row) * 2) = make_float2(m_run[t], l_run[t]);
        }
      }
    }
  }
}

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
    const int row = tok * G + h, pass = row / kPassRows;
    const int2 sp = p.span[((size_t)b * p.Hkv + kvh) * p.max_passes + pass];
    if (sp.x == sp.y) continue;  // written by the first launch
    float M = kNegInf, L = 0.f;
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int w = sp.x; w <= sp.y; ++w) {
      const size_t at = part_row(p, s, kvh, pass, w) + (row - pass * kPassRows);
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

int row_tiles(const RowsShape& s) {
  const int rows = s.max_n * (s.Hq / s.Hkv);
  return rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
}

int resident(int tiles) {
  static std::atomic<int> cached{0};
  int cus = cached.load(std::memory_order_relaxed);
  if (cus == 0) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess ||
        hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
      cus = 256;
    cached.store(cus, std::memory_order_relaxed);
  }
  return cus * (tiles == 1 ? 3 : 2);
}

constexpr int kRowsUnitCost = 8;

int passes_bound(const RowsShape& s) {
  const int rows = s.max_n * (s.Hq / s.Hkv);
  return rows > 0 ? (rows + kPassRows - 1) / kPassRows : 1;
}

long long positions_bound(const RowsShape& s) {
  return (long long)s.B * s.Hkv * passes_bound(s) * ((s.max_ctx + 15) / 16 + kRowsUnitCost);
}

int rows_grid(const RowsShape& s) {
  const int least = (s.f8 ? 4 : 2) * kRowWaves;
  const long long P = (positions_bound(s) + least - 1) / least;
  const int most = resident(row_tiles(s));
  return (int)(P < 1 ? 1 : P < most ? P : most);
}

int pass_rows(const RowsShape& s) {
  const int rows = s.max_n * (s.Hq / s.Hkv);
  return rows < kPassRows ? rows : kPassRows;
}

size_t part_rows(const RowsShape& s) { return (size_t)s.T * s.Hq + (size_t)rows_grid(s) * pass_rows(s); }

template <int D, bool F8>
void launch_tiles(const RowsParams& p, int tiles, int P, hipStream_t stream) {
  if (tiles == 1)
    attn_rows_kernel<D, F8, 1, F8 ? 16 : 8><<<P, 64 * kRowWaves, 0, stream>>>(p);
  else if (tiles == 2)
    attn_rows_kernel<D, F8, 2, 8><<<P, 64 * kRowWaves, 0, stream>>>(p);
  else
    attn_rows_kernel<D, F8, 4, 8><<<P, 64 * kRowWaves, 0, stream>>>(p);
}

}  // namespace

bool rows_shape_fits(const RowsShape& s) {
  return (long long)s.B * s.Hkv * passes_bound(s) * ((s.max_ctx + 15) / 16 + 16) < (1ll << 30) &&
         (long long)s.T * s.Hq < (1ll << 30);
}

size_t rows_workspace_bytes(const RowsShape& s) {
  return align_up(part_rows(s) * s.D * sizeof(float), 256) + align_up(part_rows(s) * 2 * sizeof(float), 256) +
         align_up((size_t)s.B * s.Hkv * passes_bound(s) * sizeof(int2), 256);
}

hipError_t launch_attn_rows(const RowsShape& s, const RowsTensors& t, void* ws, hipStream_t stream) {
  if (s.T == 0 || s.max_n == 0) return hipSuccess;
  const int P = rows_grid(s), tiles = row_tiles(s);
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
  w += align_up(part_rows(s) * s.D * sizeof(float), 256);
  p.part_ml = reinterpret_cast<float*>(w);
  w += align_up(part_rows(s) * 2 * sizeof(float), 256);
  p.span = reinterpret_cast<int2*>(w);
  p.B = s.B;
  p.T = s.T;
  p.Hq = s.Hq;
  p.Hkv = s.Hkv;
  p.G = s.Hq / s.Hkv;
  p.max_n = s.max_n;
  p.max_passes = passes_bound(s);
  p.pass_rows = pass_rows(s);
  p.max_blocks = s.max_blocks;
  p.num_blocks = s.num_blocks;
  p.max_ctx = s.max_ctx;
  p.unit_cost = kRowsUnitCost;
  p.scale_log2 = (s.scale != 0.f ? s.scale : 1.0f / sqrtf((float)s.D)) * kLog2e;
  {
    ProfScope ps("attn_rows", stream);
    if (s.D == 128 && s.f8)
      launch_tiles<128, true>(p, tiles, P, stream);
    else if (s.D == 128)
      launch_tiles<128, false>(p, tiles, P, stream);
    else if (s.f8)
      launch_tiles<64, true>(p, tiles, P, stream);
    else
      launch_tiles<64, false>(p, tiles, P, stream);
  }
  if (P > 1) {  // one work-group cuts no unit
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
