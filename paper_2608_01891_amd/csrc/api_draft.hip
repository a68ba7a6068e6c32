// C-ABI layer of the 8-bit cache and of drafted tokens: host-side validation,
// workspace queries, launches.
#include <math.h>

#include "aflex_draft.h"
#include "api_cache.h"
#include "kernels.h"

using aflex::aligned16;
using aflex::aligned4;
using aflex::check_context;
using aflex::check_pools;
using aflex::check_ws;
using aflex::hip_status;
using aflex::RowsShape;
using aflex::RowsTensors;

namespace {

constexpr int kMostDrafts = 64;  // bits of a mask

aflex_status check_rope_f8(const aflex_rope_f8_args* a, bool packed) {
  const char* who = packed ? "rope_write_f8" : "rope_append_f8";
  const aflex_status s = aflex::check_rope(who, a, packed);
  if (s != AFLEX_OK) return s;
  REQUIRE(a->kv_exp, AFLEX_ERR_INVALID_ARG, "%s: kv_exp is NULL", who);
  REQUIRE(aligned16(a->kv_exp), AFLEX_ERR_ALIGNMENT, "%s: kv_exp must be 16-byte aligned", who);
  return AFLEX_OK;
}

// What the two attention calls have in common.
aflex_status check_rows(const char* who, const RowsShape& s, const RowsTensors& t, int block_size, bool need_out) {
  REQUIRE(t.q && t.k_cache && t.v_cache && t.block_table && t.context_lens && (!need_out || t.out),
          AFLEX_ERR_INVALID_ARG, "%s: NULL tensor pointer", who);
  aflex_status st = check_pools(who, s.B, s.Hkv, s.D, block_size, s.max_blocks, s.num_blocks);
  if (st == AFLEX_OK) st = check_context(who, s.max_ctx, s.max_blocks);
  if (st != AFLEX_OK) return st;
  REQUIRE(s.Hq >= 1 && s.Hq % s.Hkv == 0, AFLEX_ERR_INVALID_ARG, "%s: Hq (%d) not a positive multiple of Hkv (%d)",
          who, s.Hq, s.Hkv);
  REQUIRE(s.Hq / s.Hkv <= 16, AFLEX_ERR_UNSUPPORTED, "%s: %d query heads per kv head (max 16)", who, s.Hq / s.Hkv);
  REQUIRE(s.Hkv <= 65535, AFLEX_ERR_UNSUPPORTED, "%s: Hkv %d above 65535", who, s.Hkv);
  REQUIRE(isfinite(s.scale) && s.scale >= 0.f, AFLEX_ERR_INVALID_ARG, "%s: scale must be finite and >= 0", who);
  REQUIRE(s.T < (1 << 24), AFLEX_ERR_UNSUPPORTED, "%s: %d rows, 2^24 or more", who, s.T);
  REQUIRE(aflex::rows_shape_fits(s), AFLEX_ERR_UNSUPPORTED,
          "%s: B * Hkv * (ceil(max_context_len / 16) + 16) times the passes over its rows, and rows * Hq, must stay "
          "below 2^30",
          who);
  REQUIRE(aligned16(t.q) && aligned16(t.k_cache) && aligned16(t.v_cache) && aligned16(t.kv_exp) && aligned16(t.out),
          AFLEX_ERR_ALIGNMENT, "%s: tensors must be 16-byte aligned", who);
  REQUIRE(aligned4(t.block_table) && aligned4(t.context_lens) && aligned4(t.cu_seqlens), AFLEX_ERR_ALIGNMENT,
          "%s: index arrays must be 4-byte aligned", who);
  REQUIRE((reinterpret_cast<uintptr_t>(t.masks) & 7u) == 0, AFLEX_ERR_ALIGNMENT, "%s: masks must be 8-byte aligned",
          who);
  return AFLEX_OK;
}

aflex_status rows_of(const aflex_attn_f8_args* a, bool need_out, RowsShape& s, RowsTensors& t) {
  const char* who = "attn_decode_f8";
  REQUIRE(a, AFLEX_ERR_INVALID_ARG, "%s: args is NULL", who);
  REQUIRE(a->kv_exp, AFLEX_ERR_INVALID_ARG, "%s: kv_exp is NULL", who);
  s = {a->B, a->B, a->Hq, a->Hkv, a->D, 1, a->max_blocks_per_seq, a->num_blocks, a->max_context_len, a->scale, true};
  t = {a->q, a->k_cache, a->v_cache, a->kv_exp, a->block_table, a->context_lens, nullptr, nullptr, a->out};
  return check_rows(who, s, t, a->block_size, need_out);
}

aflex_status rows_of(const aflex_attn_tree_args* a, bool need_out, RowsShape& s, RowsTensors& t) {
  const char* who = "attn_tree";
  REQUIRE(a, AFLEX_ERR_INVALID_ARG, "%s: args is NULL", who);
  REQUIRE(a->cu_seqlens, AFLEX_ERR_INVALID_ARG, "%s: cu_seqlens is NULL", who);
  REQUIRE(a->T >= 0 && a->max_drafts >= 0, AFLEX_ERR_INVALID_ARG, "%s: T and max_drafts must not be negative", who);
  REQUIRE(a->max_drafts <= kMostDrafts, AFLEX_ERR_UNSUPPORTED, "%s: max_drafts %d above %d", who, a->max_drafts,
          kMostDrafts);
  REQUIRE((long long)a->T <= (long long)a->B * a->max_drafts, AFLEX_ERR_INVALID_ARG,
          "%s: T %d exceeds B * max_drafts", who, a->T);
  s = {a->B, a->T, a->Hq, a->Hkv, a->D, a->max_drafts, a->max_blocks_per_seq, a->num_blocks, a->max_context_len,
       a->scale, a->kv_exp != nullptr};
  t = {a->q, a->k_cache, a->v_cache, a->kv_exp, a->block_table, a->context_lens, a->cu_seqlens, a->masks, a->out};
  return check_rows(who, s, t, a->block_size, need_out);
}

template <class Args>
aflex_status rows_workspace(const Args* a, size_t* bytes, const char* who) {
  REQUIRE(bytes, AFLEX_ERR_INVALID_ARG, "%s: bytes is NULL", who);
  RowsShape s;
  RowsTensors t;
  const aflex_status st = rows_of(a, false, s, t);
  if (st != AFLEX_OK) return st;
  *bytes = aflex::rows_workspace_bytes(s);
  return AFLEX_OK;
}

template <class Args>
aflex_status rows_call(const Args* a, void* ws, size_t ws_bytes, aflex_stream stream, const char* who) {
  RowsShape s;
  RowsTensors t;
  aflex_status st = rows_of(a, true, s, t);
  if (st != AFLEX_OK) return st;
  st = check_ws(ws, ws_bytes, aflex::rows_workspace_bytes(s), who);
  if (st != AFLEX_OK) return st;
  return hip_status(aflex::launch_attn_rows(s, t, ws, (hipStream_t)stream), who);
}

}  // namespace

extern "C" {

aflex_status aflex_rope_append_f8(const aflex_rope_f8_args* a, aflex_stream stream) {
  const aflex_status s = check_rope_f8(a, false);
  if (s != AFLEX_OK) return s;
  return hip_status(aflex::launch_rope_append_f8(*a, (hipStream_t)stream), "rope_append_f8");
}

aflex_status aflex_rope_write_f8(const aflex_rope_f8_args* a, aflex_stream stream) {
  const aflex_status s = check_rope_f8(a, true);
  if (s != AFLEX_OK) return s;
  return hip_status(aflex::launch_rope_write_f8(*a, (hipStream_t)stream), "rope_write_f8");
}

aflex_status aflex_attn_decode_f8_workspace(const aflex_attn_f8_args* a, size_t* bytes) {
  return rows_workspace(a, bytes, "attn_decode_f8");
}

aflex_status aflex_attn_decode_f8(const aflex_attn_f8_args* a, void* ws, size_t ws_bytes, aflex_stream stream) {
  return rows_call(a, ws, ws_bytes, stream, "attn_decode_f8");
}

aflex_status aflex_attn_tree_workspace(const aflex_attn_tree_args* a, size_t* bytes) {
  return rows_workspace(a, bytes, "attn_tree");
}

aflex_status aflex_attn_tree(const aflex_attn_tree_args* a, void* ws, size_t ws_bytes, aflex_stream stream) {
  return rows_call(a, ws, ws_bytes, stream, "attn_tree");
}

aflex_status aflex_cache_accept(const aflex_cache_accept_args* a, aflex_stream stream) {
  const char* who = "cache_accept";
  REQUIRE(a, AFLEX_ERR_INVALID_ARG, "%s: args is NULL", who);
  REQUIRE(a->k_cache && a->v_cache && a->block_table && a->context_lens && a->cu_seqlens && a->accepted &&
              a->accepted_counts && a->context_out,
          AFLEX_ERR_INVALID_ARG, "%s: NULL tensor pointer", who);
  const aflex_status s = check_pools(who, a->B, a->Hkv, a->D, a->block_size, a->max_blocks_per_seq, a->num_blocks);
  if (s != AFLEX_OK) return s;
  REQUIRE(a->max_accepted >= 1, AFLEX_ERR_INVALID_ARG, "%s: max_accepted must be positive", who);
  REQUIRE(a->max_accepted <= kMostDrafts, AFLEX_ERR_UNSUPPORTED, "%s: max_accepted %d above %d", who, a->max_accepted,
          kMostDrafts);
  REQUIRE(a->B <= 65535 && a->Hkv <= 65535, AFLEX_ERR_UNSUPPORTED, "%s: B (%d) or Hkv (%d) above 65535", who, a->B,
          a->Hkv);
  REQUIRE(aligned16(a->k_cache) && aligned16(a->v_cache) && aligned16(a->kv_exp), AFLEX_ERR_ALIGNMENT,
          "%s: pools must be 16-byte aligned", who);
  REQUIRE(aligned4(a->block_table) && aligned4(a->context_lens) && aligned4(a->cu_seqlens) && aligned4(a->accepted) &&
              aligned4(a->accepted_counts) && aligned4(a->context_out),
          AFLEX_ERR_ALIGNMENT, "%s: index arrays must be 4-byte aligned", who);
  // (each work-group of a sequence reads them, while the first writes context_out)
  const auto apart = [a](const int32_t* p, long long n) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a->context_out), y = reinterpret_cast<uintptr_t>(p);
    return x + a->B * sizeof(int32_t) <= y || y + n * sizeof(int32_t) <= x;
  };
  REQUIRE(apart(a->context_lens, a->B) && apart(a->cu_seqlens, a->B + 1ll) && apart(a->accepted_counts, a->B) &&
              apart(a->accepted, (long long)a->B * a->max_accepted) &&
              apart(a->block_table, (long long)a->B * a->max_blocks_per_seq),
          AFLEX_ERR_INVALID_ARG, "%s: context_out must not overlap the index arrays", who);
  return hip_status(aflex::launch_cache_accept(*a, (hipStream_t)stream), who);
}

}  // extern "C"
