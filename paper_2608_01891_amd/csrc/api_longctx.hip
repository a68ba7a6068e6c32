// C-ABI layer of the long-context operators: host-side validation, workspace
// queries, launches.
#include "aflex_longctx.h"
#include "api_cache.h"
#include "kernels.h"

using aflex::aligned16;
using aflex::aligned4;
using aflex::check_context;
using aflex::check_pools;
using aflex::check_ws;
using aflex::hip_status;
using aflex::kMostUnits;

namespace {

aflex_status check_rope(const aflex_rope_args* a, bool packed) {
  const char* who = packed ? "rope_write" : "rope_append";
  const aflex_status s = aflex::check_rope(who, a, packed);
  if (s != AFLEX_OK) return s;
  REQUIRE(!a->block_keys == !a->block_exp, AFLEX_ERR_INVALID_ARG,
          "%s: block_keys and block_exp must be given together", who);
  REQUIRE(aligned16(a->block_keys), AFLEX_ERR_ALIGNMENT, "%s: block_keys must be 16-byte aligned", who);
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
