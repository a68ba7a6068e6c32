// C-ABI layer of the long-context operators: host-side validation, workspace
// queries, launches.
#include "aflex_longctx.h"
#include "api_common.h"
#include "kernels.h"

using aflex::aligned16;
using aflex::aligned4;
using aflex::check_ws;
using aflex::hip_status;

namespace {

// Threads of a launch along one dimension, which have to stay below this.
constexpr long long kMostThreads = 1ll << 32;
constexpr long long kMostUnits = kMostThreads / 256;  // (sequence, kv head) pairs that get a work-group of 256 each

// Sizes that every entry point takes.
aflex_status check_pools(const char* who, int B, int Hkv, int D, int block_size, int max_blocks, int num_blocks) {
  REQUIRE(B >= 1 && Hkv >= 1 && D >= 1 && num_blocks >= 1 && max_blocks >= 1, AFLEX_ERR_INVALID_ARG,
          "%s: B, Hkv, D, num_blocks and max_blocks_per_seq must be positive", who);
  REQUIRE(D == 64 || D == 128, AFLEX_ERR_UNSUPPORTED, "%s: head_dim %d unsupported (64 or 128)", who, D);
  REQUIRE(block_size == 16, AFLEX_ERR_UNSUPPORTED, "%s: block_size %d unsupported (16)", who, block_size);
  REQUIRE(max_blocks <= (1 << 26), AFLEX_ERR_UNSUPPORTED, "%s: max_blocks_per_seq %d above 2^26", who, max_blocks);
  return AFLEX_OK;
}

aflex_status check_context(const char* who, int max_context_len, int max_blocks) {
  REQUIRE(max_context_len >= 0, AFLEX_ERR_INVALID_ARG, "%s: max_context_len < 0", who);
  REQUIRE((long long)max_context_len <= 16ll * max_blocks, AFLEX_ERR_INVALID_ARG,
          "%s: max_context_len %d exceeds the block table capacity %lld", who, max_context_len, 16ll * max_blocks);
  return AFLEX_OK;
}

aflex_status check_stride(const char* who, const char* name, int stride, long long row) {
  REQUIRE(stride == 0 || (stride % 8 == 0 && stride >= row), AFLEX_ERR_INVALID_ARG,
          "%s: %s %d must be 0 or a multiple of 8 of at least %lld", who, name, stride, row);
  return AFLEX_OK;
}

aflex_status check_rope(const aflex_rope_args* a, bool packed) {
  const char* who = packed ? "rope_write" : "rope_append";
  REQUIRE(a, AFLEX_ERR_INVALID_ARG, "%s: args is NULL", who);
  REQUIRE(a->q && a->k_new && a->v_new && a->q_out && a->k_cache && a->v_cache && a->block_table && a->context_lens &&
              (!packed || a->cu_seqlens) && (a->rotary_dim == 0 || a->rope),
          AFLEX_ERR_INVALID_ARG, "%s: NULL tensor pointer", who);
  REQUIRE(!a->block_keys == !a->block_exp, AFLEX_ERR_INVALID_ARG,
          "%s: block_keys and block_exp must be given together", who);
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
              aligned16(a->k_cache) && aligned16(a->v_cache) && (a->rotary_dim == 0 || aligned16(a->rope)) &&
              aligned16(a->block_keys),
          AFLEX_ERR_ALIGNMENT, "%s: tensors must be 16-byte aligned", who);
  REQUIRE(aligned4(a->block_table) && aligned4(a->context_lens) && (!packed || aligned4(a->cu_seqlens)) &&
              aligned4(a->positions),
          AFLEX_ERR_ALIGNMENT, "%s: index arrays must be 4-byte aligned", who);
  return AFLEX_OK;
}

aflex_status check_select(const aflex_block_select_args* a) {
  const char* who = "block_select";
  REQUIRE(a, AFLEX_ERR_INVALID_ARG, "%s: args is NULL", who);
  REQUIRE(a->q && a->block_keys && a->block_exp && a->block_table && a->context_lens && a->selected,
          AFLEX_ERR_INVALID_ARG, "%s: NULL tensor pointer", who);
  aflex_status s = check_pools(who, a->B, a->Hkv, a->D, a->block_size, a->max_blocks_per_seq, a->num_blocks);
  if (s == AFLEX_OK) s = check_context(who, a->max_context_len, a->max_blocks_per_seq);
  if (s != AFLEX_OK) return s;
  REQUIRE(a->Hq >= 1 && a->Hq % a->Hkv == 0, AFLEX_ERR_INVALID_ARG, "%s: Hq (%d) not a positive multiple of Hkv (%d)",
          who, a->Hq, a->Hkv);
  REQUIRE(a->Hq / a->Hkv <= 16, AFLEX_ERR_UNSUPPORTED, "%s: %d query heads per kv head (max 16)", who,
          a->Hq / a->Hkv);
  REQUIRE(a->sink_blocks >= 0 && a->recent_blocks >= 1 &&
              (long long)a->sink_blocks + a->recent_blocks <= a->top_blocks,
          AFLEX_ERR_INVALID_ARG,
          "%s: need sink_blocks >= 0, recent_blocks >= 1 and their sum <= top_blocks (got %d, %d, %d)", who,
          a->sink_blocks, a->recent_blocks, a->top_blocks);
  // (the forms with larger work-groups have more than 1024 blocks, so fewer units)
  REQUIRE((long long)a->B * a->Hkv < kMostUnits, AFLEX_ERR_UNSUPPORTED, "%s: B * Hkv must stay below 2^24", who);
  REQUIRE((long long)a->B * a->Hkv * ((a->max_context_len + 15ll) / 16) < (1ll << 30) &&
              (long long)a->B * a->Hkv * a->top_blocks < (1ll << 30),
          AFLEX_ERR_UNSUPPORTED,
          "%s: B * Hkv times ceil(max_context_len / 16), and times top_blocks, must stay below 2^30", who);
  REQUIRE(aligned16(a->q) && aligned16(a->block_keys), AFLEX_ERR_ALIGNMENT,
          "%s: q and block_keys must be 16-byte aligned", who);
  REQUIRE(aligned4(a->block_table) && aligned4(a->context_lens) && aligned4(a->selected), AFLEX_ERR_ALIGNMENT,
          "%s: index arrays must be 4-byte aligned", who);
  return AFLEX_OK;
}

aflex_status check_sparse(const aflex_attn_sparse_args* a, bool need_out) {
  REQUIRE(a, AFLEX_ERR_INVALID_ARG, "attn_sparse: args is NULL");
  aflex_status s = aflex::check_attn(&a->attn, need_out);
  if (s != AFLEX_OK) return s;
  REQUIRE(a->selected, AFLEX_ERR_INVALID_ARG, "attn_sparse: selected is NULL");
  REQUIRE(a->top_blocks >= 1, AFLEX_ERR_INVALID_ARG, "attn_sparse: top_blocks must be positive");
  REQUIRE(a->attn.split_tokens == 0, AFLEX_ERR_UNSUPPORTED, "attn_sparse: split_tokens must be 0");
  REQUIRE((long long)a->attn.B * a->attn.Hkv < kMostUnits, AFLEX_ERR_UNSUPPORTED,
          "attn_sparse: B * Hkv must stay below 2^24");
  REQUIRE((long long)a->attn.B * a->attn.Hkv * a->top_blocks < (1ll << 30), AFLEX_ERR_UNSUPPORTED,
          "attn_sparse: B * Hkv * top_blocks must stay below 2^30");
  REQUIRE(aligned4(a->selected), AFLEX_ERR_ALIGNMENT, "attn_sparse: selected must be 4-byte aligned");
  return AFLEX_OK;
}

}  // namespace

extern "C" {

aflex_status aflex_rope_append(const aflex_rope_args* a, aflex_stream stream) {
  const aflex_status s = check_rope(a, false);
  if (s != AFLEX_OK) return s;
  return hip_status(aflex::launch_rope_append(*a, (hipStream_t)stream), "rope_append");
}

aflex_status aflex_rope_write(const aflex_rope_args* a, aflex_stream stream) {
  const aflex_status s = check_rope(a, true);
  if (s != AFLEX_OK) return s;
  return hip_status(aflex::launch_rope_write(*a, (hipStream_t)stream), "rope_write");
}

aflex_status aflex_block_summary(const aflex_block_summary_args* a, aflex_stream stream) {
  const char* who = "block_summary";
  REQUIRE(a, AFLEX_ERR_INVALID_ARG, "%s: args is NULL", who);
  REQUIRE(a->k_cache && a->block_keys && a->block_exp && a->block_table && a->context_lens, AFLEX_ERR_INVALID_ARG,
          "%s: NULL tensor pointer", who);
  aflex_status s = check_pools(who, a->B, a->Hkv, a->D, a->block_size, a->max_blocks_per_seq, a->num_blocks);
  if (s == AFLEX_OK) s = check_context(who, a->max_context_len, a->max_blocks_per_seq);
  if (s != AFLEX_OK) return s;
  REQUIRE(a->B <= 65535, AFLEX_ERR_UNSUPPORTED, "%s: B %d above 65535", who, a->B);
  REQUIRE((a->max_context_len / 16ll) * a->Hkv < (1ll << 30), AFLEX_ERR_UNSUPPORTED,
          "%s: max_context_len / 16 * Hkv must stay below 2^30", who);
  REQUIRE(aligned16(a->k_cache) && aligned16(a->block_keys), AFLEX_ERR_ALIGNMENT,
          "%s: k_cache and block_keys must be 16-byte aligned", who);
  REQUIRE(aligned4(a->block_table) && aligned4(a->context_lens), AFLEX_ERR_ALIGNMENT,
          "%s: index arrays must be 4-byte aligned", who);
  return hip_status(aflex::launch_block_summary(*a, (hipStream_t)stream), who);
}

aflex_status aflex_block_select_workspace(const aflex_block_select_args* a, size_t* bytes) {
  REQUIRE(bytes, AFLEX_ERR_INVALID_ARG, "block_select: bytes is NULL");
  const aflex_status s = check_select(a);
  if (s != AFLEX_OK) return s;
  *bytes = aflex::block_select_workspace_bytes(*a);
  return AFLEX_OK;
}

aflex_status aflex_block_select(const aflex_block_select_args* a, void* ws, size_t ws_bytes, aflex_stream stream) {
  aflex_status s = check_select(a);
  if (s != AFLEX_OK) return s;
  s = check_ws(ws, ws_bytes, aflex::block_select_workspace_bytes(*a), "block_select");
  if (s != AFLEX_OK) return s;
  return hip_status(aflex::launch_block_select(*a, ws, (hipStream_t)stream), "block_select");
}

aflex_status aflex_attn_sparse_decode_workspace(const aflex_attn_sparse_args* a, size_t* bytes) {
  REQUIRE(bytes, AFLEX_ERR_INVALID_ARG, "attn_sparse: bytes is NULL");
  const aflex_status s = check_sparse(a, false);
  if (s != AFLEX_OK) return s;
  *bytes = aflex::attn_workspace_bytes(a->attn, a->top_blocks);
  return AFLEX_OK;
}

aflex_status aflex_attn_sparse_decode(const aflex_attn_sparse_args* a, void* ws, size_t ws_bytes,
                                      aflex_stream stream) {
  aflex_status s = check_sparse(a, true);
  if (s != AFLEX_OK) return s;
  s = check_ws(ws, ws_bytes, aflex::attn_workspace_bytes(a->attn, a->top_blocks), "attn_sparse");
  if (s != AFLEX_OK) return s;
  return hip_status(aflex::launch_attn_sparse(*a, ws, (hipStream_t)stream), "attn_sparse");
}

}  // extern "C"
