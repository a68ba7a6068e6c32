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

__device__ __forceinline__ uint4 stream16(const uint8_t* p) {
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)));
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

// The first n of 16 bytes, zeros behind them (n may be <= 0).
__device__ __forceinline__ uint4 keep_bytes(uint4 v, int n) {
  const auto w = [n](uint32_t x, int at) {
    const int k = n - at;
    return k >= 4 ? x : k <= 0 ? 0u : x & ((1u << (8 * k)) - 1u);
  };
  return make_uint4(w(v.x, 0), w(v.y, 4), w(v.z, 8), w(v.w, 12));
}

__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) {
  return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
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

}  // namespace

// D, 8-bit cache or bf16, row tiles of a wave.
template <int D, bool F8, int RT>
__global__ __launch_bounds__(64 * kRowWaves, RT == 1 ? 3 : 2) void attn_rows_kernel(RowsParams p) {
  constexpr int NC = D / 32;          // k-chunks of the first product
  constexpr int NMT = D / 16;         // d-tiles of the second
  constexpr int SB = F8 ? 4 : 2;      // blocks of a step
  constexpr int KT = SB;              // its 16-token tiles in the first product
  constexpr int TOK = F8 ? 16 : 8;    // tokens of a lane in the second product
  constexpr int PS = TOK / 8;         // its 32-token slices
  constexpr int LDQ = D + 8;          // padded row of q in LDS
  constexpr int LDO = D + 4;          // row of a partial in LDS: O, then (m, l)
  constexpr int QROWS = RT == 4 ? kPassRows : 16 * RT;
  constexpr int kQBytes = QROWS * LDQ * 2;
  constexpr int kPartBytes = 2 * 16 * RT * LDO * 4;  // partials of two waves
  __shared__ __attribute__((aligned(16))) uint8_t sm[kQBytes > kPartBytes ? kQBytes : kPartBytes];
  uint16_t* sq = reinterpret_cast<uint16_t*>(sm);
  float* so = reinterpret_cast<float*>(sm);

  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lane = tid & 63;
  const int r = lane & 15, qg = lane >> 4;
  const int G = p.G, wg = blockIdx.x, P = gridDim.x;

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

    // ---- q into LDS: row i G + h of the pass is token i, head kvh G + h ----
    __syncthreads();
    for (int i = tid; i < tiles * 16 * (D / 8); i += 64 * kRowWaves) {
      const int row = i / (D / 8), c = i % (D / 8);
      uint4 v = make_uint4(0, 0, 0, 0);
      if (row < rows) {
        const int tok = (row_base + row) / G, h = row_base + row - tok * G;
        v = *reinterpret_cast<const uint4*>(p.q + ((size_t)(s.row0 + tok) * p.Hq + kvh * G + h) * D + c * 8);
      }
      *reinterpret_cast<uint4*>(sq + row * LDQ + c * 8) = v;
    }
    __syncthreads();

    float m_run[RT], l_run[RT];
    f32x4 acc[RT][NMT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      m_run[t] = kNegInf;
      l_run[t] = 0.f;
#pragma unroll
      for (int mt = 0; mt < NMT; ++mt) acc[t][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const int steps = (j1 - j0 + SB - 1) / SB;
    const int32_t* table = p.bt + (size_t)b * p.max_blocks;
    auto load_id = [&](int j) {
      const int id = j < j1 ? table[j] : -1;
      return id >= 0 && id < p.num_blocks ? id : -1;
    };
    // Block ids, 64 per wave register, the next ones loaded a register ahead.
    int my_id = load_id(j0 + lane), next_id = load_id(j0 + 64 + lane), chunk = 0;

    for (int st = turn; st < (mine > 0 ? steps : 0); st += turns) {
      if (st * SB / 64 != chunk) {
        chunk = st * SB / 64;
        my_id = next_id;
        next_id = load_id(j0 + (chunk + 1) * 64 + lane);
      }
      int id[SB];
#pragma unroll
      for (int i = 0; i < SB; ++i) id[i] = __builtin_amdgcn_readlane(my_id, (st * SB + i) & 63);
      const int jb = j0 + st * SB;
      // the block of the lane's key row, and that of its values
      int pk, pv, vb;
      if constexpr (F8) {
        pk = (r & 8) ? ((r & 4) ? id[3] : id[2]) : ((r & 4) ? id[1] : id[0]);
        pv = (qg & 2) ? ((qg & 1) ? id[3] : id[2]) : ((qg & 1) ? id[1] : id[0]);
        vb = qg;
      } else {
        pk = (r & 8) ? id[1] : id[0];
        pv = (qg & 2) ? id[1] : id[0];
        vb = qg >> 1;
      }
      const int tb = (jb + vb) * 16 + (F8 ? 0 : (qg & 1) * 8);  // place of the lane's first token
      const int nv = pv >= 0 ? s.ctx - tb : 0;                  // how many of them are cached

      // keys: tile t holds tokens of all SB blocks; the lane's row
      bf16x8 kf[KT][NC];
      if constexpr (F8) {
        float ks[KT] = {};
        if (pk >= 0) {
          const size_t tile = (size_t)pk * p.Hkv + kvh;
          const uint4 ex = *reinterpret_cast<const uint4*>(p.ke + tile * 32);
          const uint8_t* kb = p.kc + (tile * 16 + (r & 3)) * D + qg * 16;
          uint4 raw[KT][NC / 2];
#pragma unroll
          for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int c = 0; c < NC / 2; ++c) raw[t][c] = stream16(kb + 4 * t * D + c * 64);
#pragma unroll
          for (int t = 0; t < KT; ++t) {
            ks[t] = exp2_whole((int8_t)(word_of(ex, t) >> (8 * (r & 3))));
#pragma unroll
            for (int c = 0; c < NC / 2; ++c) {
              kf[t][2 * c] = widen(raw[t][c].x, raw[t][c].y, ks[t]);
              kf[t][2 * c + 1] = widen(raw[t][c].z, raw[t][c].w, ks[t]);
            }
          }
        } else {
#pragma unroll
          for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c) kf[t][c] = zero_bf16x8();
        }
      } else {
        if (pk >= 0) {
          const uint8_t* kb =
              p.kc + ((((size_t)pk * p.Hkv + kvh) * 16 + ((r >> 2) & 1) * 8 + (r & 3)) * D + qg * 8) * 2;
#pragma unroll
          for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c)
              kf[t][c] = __builtin_bit_cast(bf16x8, stream16(kb + (4 * t * D + c * 32) * 2));
        } else {
#pragma unroll
          for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c) kf[t][c] = zero_bf16x8();
        }
      }
      // values: zeros behind the context, so that 0 times what lies there is 0
      uint4 vraw[NMT];
      int vexp[F8 ? TOK : 1];
      if (pv >= 0) {
        const size_t tile = (size_t)pv * p.Hkv + kvh;
        const uint8_t* vbase = F8 ? p.vc + (tile * D + r) * 16 : p.vc + ((tile * D + r) * 16 + (qg & 1) * 8) * 2;
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt) vraw[mt] = stream16(vbase + mt * 16 * 16 * (F8 ? 1 : 2));
        if constexpr (F8) {
          const uint4 ex = *reinterpret_cast<const uint4*>(p.ke + tile * 32 + 16);
#pragma unroll
          for (int e = 0; e < TOK; ++e) vexp[e] = (int8_t)(word_of(ex, e / 4) >> (8 * (e & 3)));
        }
      } else {
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt) vraw[mt] = make_uint4(0, 0, 0, 0);
        if constexpr (F8) {
#pragma unroll
          for (int e = 0; e < TOK; ++e) vexp[e] = 0;
        }
      }
      if (nv < TOK) {
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt)
          vraw[mt] = F8 ? keep_bytes(vraw[mt], nv)
                        : __builtin_bit_cast(uint4, keep_first(__builtin_bit_cast(bf16x8, vraw[mt]), nv));
      }
      bf16x8 vf[PS][NMT];
#pragma unroll
      for (int mt = 0; mt < NMT; ++mt) {
        if constexpr (F8) {
          vf[0][mt] = widen(vraw[mt].x, vraw[mt].y, 1.f);
          vf[PS - 1][mt] = widen(vraw[mt].z, vraw[mt].w, 1.f);
        } else {
          vf[0][mt] = __builtin_bit_cast(bf16x8, vraw[mt]);
        }
      }
      // tokens that exist, as bits; whether the step reaches the drafts
      const uint32_t cached = nv >= TOK ? (1u << TOK) - 1u : nv <= 0 ? 0u : (1u << nv) - 1u;
      const bool open = (jb + SB) * 16 <= start;

#pragma unroll
      for (int t = 0; t < RT; ++t) {
        if (t >= mine) break;
        const int row = (t0 + t) * 16 + r;  // of the pass
        f32x4 sc[KT];
#pragma unroll
        for (int k = 0; k < KT; ++k) sc[k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const int d = F8 ? (c >> 1) * 64 + qg * 16 + (c & 1) * 8 : c * 32 + qg * 8;
          const bf16x8 qf = ld_bf16x8(sq + row * LDQ + d);
#pragma unroll
          for (int k = 0; k < KT; ++k) sc[k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[k][c], qf, sc[k], 0, 0, 0);
        }
        uint32_t seen = cached;
        if (!open) {
          uint64_t mask = 0;
          if (row < rows) {
            const int tok = (row_base + row) / G;
            mask = p.masks ? p.masks[s.row0 + tok] : (2ull << tok) - 1ull;
          }
          seen &= seen_bits(mask, tb, start);
        }
        float sv[TOK];
#pragma unroll
        for (int e = 0; e < TOK; ++e) sv[e] = (seen >> e & 1u) ? sc[e / 4][e & 3] * p.scale_log2 : kNegInf;
        float mx = sv[0];
#pragma unroll
        for (int e = 1; e < TOK; ++e) mx = fmaxf(mx, sv[e]);
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m_run[t], mx);
        const float m_use = (m_new == kNegInf) ? 0.f : m_new;
        const float alpha = fast_exp2(m_run[t] - m_use);
        m_run[t] = m_new;
        float ps = 0.f;
        bf16x8 hi[PS], lo[PS];
#pragma unroll
        for (int e = 0; e < TOK; ++e) {
          const float w = fast_exp2(sv[e] - m_use);
          ps += w;
          float u = w;
          if constexpr (F8) u = __builtin_ldexpf(w, vexp[e]);
          const __bf16 h = static_cast<__bf16>(u);
          hi[e / 8][e & 7] = h;
          lo[e / 8][e & 7] = static_cast<__bf16>(u - static_cast<float>(h));
        }
        l_run[t] = l_run[t] * alpha + ps;
#pragma unroll
        for (int mt = 0; mt < NMT; ++mt) {
          acc[t][mt] *= alpha;
#pragma unroll
          for (int k = 0; k < PS; ++k) {
            acc[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[k][mt], hi[k], acc[t][mt], 0, 0, 0);
            acc[t][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[k][mt], lo[k], acc[t][mt], 0, 0, 0);
          }
        }
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
    attn_rows_kernel<D, F8, 1><<<P, 64 * kRowWaves, 0, stream>>>(p);
  else if (tiles == 2)
    attn_rows_kernel<D, F8, 2><<<P, 64 * kRowWaves, 0, stream>>>(p);
  else
    attn_rows_kernel<D, F8, 4><<<P, 64 * kRowWaves, 0, stream>>>(p);
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
