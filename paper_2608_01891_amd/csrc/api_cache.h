// Checks that the entry points over paged caches share.
#pragma once
#include "api_common.h"

namespace aflex {

// Threads of a launch along one dimension, which have to stay below this.
constexpr long long kMostThreads = 1ll << 32;
constexpr long long kMostUnits = kMostThreads / 256;  // (sequence, kv head) pairs that get a work-group of 256 each

// Sizes that every entry point takes.
inline aflex_status check_pools(const char* who, int B, int Hkv, int D, int block_size, int max_blocks, int num_blocks) {
  REQUIRE(B >= 1 && Hkv >= 1 && D >= 1 && num_blocks >= 1 && max_blocks >= 1, AFLEX_ERR_INVALID_ARG,
          "%s: B, Hkv, D, num_blocks and max_blocks_per_seq must be positive", who);
  REQUIRE(D == 64 || D == 128, AFLEX_ERR_UNSUPPORTED, "%s: head_dim %d unsupported (64 or 128)", who, D);
  REQUIRE(block_size == 16, AFLEX_ERR_UNSUPPORTED, "%s: block_size %d unsupported (16)", who, block_size);
  REQUIRE(max_blocks <= (1 << 26), AFLEX_ERR_UNSUPPORTED, "%s: max_blocks_per_seq %d above 2^26", who, max_blocks);
  return AFLEX_OK;
}

inline aflex_status check_context(const char* who, int max_context_len, int max_blocks) {
  REQUIRE(max_context_len >= 0, AFLEX_ERR_INVALID_ARG, "%s: max_context_len < 0", who);
  REQUIRE((long long)max_context_len <= 16ll * max_blocks, AFLEX_ERR_INVALID_ARG,
          "%s: max_context_len %d exceeds the block table capacity %lld", who, max_context_len, 16ll * max_blocks);
  return AFLEX_OK;
}

inline aflex_status check_stride(const char* who, const char* name, int stride, long long row) {
  REQUIRE(stride == 0 || (stride % 8 == 0 && stride >= row), AFLEX_ERR_INVALID_ARG,
          "%s: %s %d must be 0 or a multiple of 8 of at least %lld", who, name, stride, row);
  return AFLEX_OK;
}

// Rotating cache writes, packed or a token per sequence, whatever the pools hold.
template <class Args>
aflex_status check_rope(const char* who, const Args* a, bool packed) {
  REQUIRE(a, AFLEX_ERR_INVALID_ARG, "%s: args is NULL", who);
  REQUIRE(a->q && a->k_new && a->v_new && a->q_out && a->k_cache && a->v_cache && a->block_table && a->context_lens &&
              (!packed || a->cu_seqlens) && (a->rotary_dim == 0 || a->rope),
          AFLEX_ERR_INVALID_ARG, "%s: NULL tensor pointer", who);
  aflex_status s = check_pools(who, a->B, a->Hkv, a->D, a->block_size, a->max_blocks_per_seq, a->num_blocks);
  if (s != AFLEX_OK) return s;
  REQUIRE(a->Hq >= 1, AFLEX_ERR_INVALID_ARG, "%s: Hq must be positive", who);
  REQUIRE(a->rotary_dim >= 0 && a->rotary_dim <= a->D && a->rotary_dim % 16 == 0, AFLEX_ERR_INVALID_ARG,
          "%s: rotary_dim %d must be a multiple of 16 in [0, %d]", who, a->rotary_dim, a->D);
  REQUIRE(a->rotary_dim == 0 || a->rope_len >= 1, AFLEX_ERR_INVALID_ARG, "%s: rope_len must be positive", who);
  REQUIRE((long long)a->Hq * a->D < (1ll << 30) && (long long)a->Hkv * a->D < (1ll << 30), AFLEX_ERR_UNSUPPORTED,
          "%s: rows of 2^30 elements or more", who);
  REQUIRE(packed || (long long)a->B * ((long long)a->Hq + a->Hkv) < (1ll << 30), AFLEX_ERR_UNSUPPORTED,
          "%s: B * (Hq + Hkv) must stay below 2^30", who);
  REQUIRE(packed || ((long long)a->B * a->Hkv + (long long)a->B * a->Hq * a->D / 1024 + 4) * 64 < kMostThreads,
          AFLEX_ERR_UNSUPPORTED, "%s: B * (Hkv + Hq * D / 1024) must stay below 2^26 - 4", who);
  if (packed) {
    REQUIRE(a->T >= 0 && a->max_seqlen >= 0, AFLEX_ERR_INVALID_ARG, "%s: T and max_seqlen must not be negative", who);
    REQUIRE(a->max_seqlen <= a->T, AFLEX_ERR_INVALID_ARG, "%s: max_seqlen %d exceeds T %d", who, a->max_seqlen, a->T);
    REQUIRE(a->B <= 65535, AFLEX_ERR_UNSUPPORTED, "%s: B %d above 65535", who, a->B);
    REQUIRE(((a->max_seqlen + 15ll) / 16 + 1) * 256 < kMostThreads, AFLEX_ERR_UNSUPPORTED,
            "%s: max_seqlen %d above 2^28 - 32", who, a->max_seqlen);
    REQUIRE(a->Hq <= 4096 && a->Hkv <= 4096, AFLEX_ERR_UNSUPPORTED, "%s: more than 4096 heads", who);
  }
  if ((s = check_stride(who, "q_stride", a->q_stride, (long long)a->Hq * a->D)) != AFLEX_OK) return s;
  if ((s = check_stride(who, "k_stride", a->k_stride, (long long)a->Hkv * a->D)) != AFLEX_OK) return s;
  if ((s = check_stride(who, "v_stride", a->v_stride, (long long)a->Hkv * a->D)) != AFLEX_OK) return s;
  REQUIRE(aligned16(a->q) && aligned16(a->k_new) && aligned16(a->v_new) && aligned16(a->q_out) &&
              aligned16(a->k_cache) && aligned16(a->v_cache) && (a->rotary_dim == 0 || aligned16(a->rope)),
          AFLEX_ERR_ALIGNMENT, "%s: tensors must be 16-byte aligned", who);
  REQUIRE(aligned4(a->block_table) && aligned4(a->context_lens) && (!packed || aligned4(a->cu_seqlens)) &&
              aligned4(a->positions),
          AFLEX_ERR_ALIGNMENT, "%s: index arrays must be 4-byte aligned", who);
  return AFLEX_OK;
}

}  // namespace aflex
