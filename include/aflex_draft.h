/*
 * aflex_draft.h -- the 8-bit KV cache and drafted tokens: operators of libaflex
 * over the paged caches of aflex.h.
 *
 *   aflex_rope_append_f8   rotate one token's q and k per sequence, append K/V in 8 bits
 *   aflex_rope_write_f8    the same for packed prompts, chunks or drafts
 *   aflex_attn_decode_f8   decode attention over the 8-bit cache
 *   aflex_attn_tree        attention of trees of drafted tokens, 8-bit or bf16 cache
 *   aflex_cache_accept     the accepted drafts' cache entries to their places
 *
 * A step that verifies drafts is a write of the drafts (aflex_rope_write_f8, or
 * aflex_rope_write of aflex_longctx.h without summaries, with the drafts' depths
 * as positions), aflex_attn_tree in every layer, the program's own choice of the
 * accepted drafts, and aflex_cache_accept in every layer. The conventions of
 * aflex.h hold (device pointers, alignment, streams, workspaces, validation
 * before launch, errors); strides are counted in elements. The two attention
 * calls may be two launches that communicate through the workspace: calls that
 * share one run on one stream, and are made by one host thread at a time.
 *
 * The 8-bit cache. A cached row x [D] (the key or the value of a token and kv
 * head) is held as codes c [D], floats of 8 bits (e4m3: 4 exponent and 3
 * mantissa bits, largest 448, one NaN, no infinities), and an exponent e:
 *   e = least whole number >= -100 with |x_d| <= 448 2^e for all finite x_d
 *   c_d = x_d 2^-e rounded to e4m3 (to nearest, ties to even); NaN for a
 *         non-finite x_d
 * and stands for c 2^e. Every step but the one rounding is exact. (A row with
 * values of 1.9375 2^127 or more may stand for an infinity.) Exponents lie in
 * [-100, 120]; others are read for tokens that nothing attends only. Pools of a
 * cache:
 *   k_cache [num_blocks, Hkv, 16, D] codes
 *   v_cache [num_blocks, Hkv, D, 16] codes (token fastest)
 *   kv_exp  [num_blocks, Hkv, 2, 16] exponents: the 16 keys', the 16 values'
 */
#ifndef AFLEX_DRAFT_H
#define AFLEX_DRAFT_H

#include "aflex.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef uint8_t aflex_f8; /* e4m3 bits */

/* ------------------------------------------------------------------------ */
/* aflex_rope_append / aflex_rope_write (aflex_longctx.h) into an 8-bit        */
/* cache: the same rotation, slots, positions and strides. q is rotated and    */
/* rounded to bf16; a key row is the rotated row in fp32 (each operation       */
/* rounded), a value row the row as given, each turned into codes and an       */
/* exponent as above (one rounding).                                           */
/* ------------------------------------------------------------------------ */
typedef struct aflex_rope_f8_args {
  const aflex_bf16 *q;         /* [T, Hq, D], rows q_stride apart */
  const aflex_bf16 *k_new;     /* [T, Hkv, D], rows k_stride apart */
  const aflex_bf16 *v_new;     /* [T, Hkv, D], rows v_stride apart */
  const float *rope;           /* [rope_len, rotary_dim]: cosines, then sines (unread if rotary_dim = 0) */
  const int32_t *positions;    /* [T] rows of rope, or NULL: the token's place in its sequence */
  const int32_t *cu_seqlens;   /* [B+1] as in aflex_kv_write (aflex_rope_append_f8: unread) */
  aflex_bf16 *q_out;           /* [T, Hq, D] dense (written) */
  aflex_f8 *k_cache;           /* (written) */
  aflex_f8 *v_cache;           /* (written) */
  int8_t *kv_exp;              /* (written) */
  const int32_t *block_table;  /* [B, max_blocks_per_seq] */
  const int32_t *context_lens; /* [B], including the new tokens */
  int32_t B, T;                /* sequences, new tokens (aflex_rope_append_f8: T is unread, B) */
  int32_t Hq, Hkv, D;
  int32_t rotary_dim;          /* a multiple of 16 in [0, D] */
  int32_t interleaved;         /* 0: pairs (i, i + rotary_dim / 2); else (2i, 2i + 1) */
  int32_t rope_len;            /* rows of rope (unread if rotary_dim = 0) */
  int32_t max_seqlen;          /* host-known bound on n_b (aflex_rope_append_f8: unread) */
  int32_t block_size;          /* must be 16 */
  int32_t max_blocks_per_seq, num_blocks;
  int32_t q_stride, k_stride, v_stride; /* as in aflex_rope_args */
} aflex_rope_f8_args;

/* Supported and clamped as aflex_rope_append and aflex_rope_write. No workspace. */
/* aflex_rope_write_f8 may read and write back the values' codes of the other      */
/* slots of a block that it writes: no other call writes that block meanwhile.     */
aflex_status aflex_rope_append_f8(const aflex_rope_f8_args *a, aflex_stream stream);
aflex_status aflex_rope_write_f8(const aflex_rope_f8_args *a, aflex_stream stream);

/* ------------------------------------------------------------------------ */
/* aflex_attn_decode over an 8-bit cache, with k_j and v_j the rows that the   */
/* codes and exponents stand for.                                              */
/* ------------------------------------------------------------------------ */
typedef struct aflex_attn_f8_args {
  const aflex_bf16 *q;         /* [B, Hq, D] */
  const aflex_f8 *k_cache;
  const aflex_f8 *v_cache;
  const int8_t *kv_exp;
  const int32_t *block_table;  /* [B, max_blocks_per_seq] */
  const int32_t *context_lens; /* [B] */
  aflex_bf16 *out;             /* [B, Hq, D] */
  int32_t B, Hq, Hkv, D;
  int32_t block_size;          /* must be 16 */
  int32_t max_blocks_per_seq, num_blocks;
  int32_t max_context_len;     /* as in aflex_attn_args */
  float scale;                 /* softmax scale; 0 selects 1/sqrt(D) */
} aflex_attn_f8_args;

/* Supported: D in {64, 128}, block_size == 16, Hq % Hkv == 0, Hq / Hkv <= 16, */
/* B * Hkv * (ceil(max_context_len / 16) + 16) < 2^30. Contexts are clamped    */
/* to [0, max_context_len]; a context of 0 yields out = 0; tokens of block ids */
/* outside [0, num_blocks) are masked. The workspace needs no initialisation.  */
/* The same result on every call with the same inputs (bitwise).               */
aflex_status aflex_attn_decode_f8_workspace(const aflex_attn_f8_args *a, size_t *bytes);
aflex_status aflex_attn_decode_f8(const aflex_attn_f8_args *a, void *workspace, size_t workspace_bytes,
                                  aflex_stream stream);

/* ------------------------------------------------------------------------ */
/* Attention of drafted tokens. Sequence b has n_b = cu_seqlens[b+1] -         */
/* cu_seqlens[b] drafts, whose keys and values are the newest n_b tokens of    */
/* its context: draft j sits at place s_b + j, s_b = context_lens[b] - n_b.    */
/* Row cu_seqlens[b] + i of q is draft i; it attends                           */
/*   the places before s_b, and                                                */
/*   place s_b + j for each j < n_b whose bit j of masks[cu_seqlens[b] + i] is */
/*   set (its ancestors and itself; any set is allowed). masks NULL: j <= i    */
/*   (a chain: the drafts follow each other, or are the tokens of a chunk).    */
/* A row that attends nothing yields 0, and what a row does not attend does    */
/* not change it, whatever its keys and values hold. One draft per sequence    */
/* that sees itself is decode attention.                                       */
/* ------------------------------------------------------------------------ */
typedef struct aflex_attn_tree_args {
  const aflex_bf16 *q;         /* [T, Hq, D] */
  const void *k_cache;         /* aflex_f8 pools with kv_exp, or bf16 pools as in aflex_attn_args */
  const void *v_cache;
  const int8_t *kv_exp;        /* NULL: the pools hold bf16 */
  const int32_t *block_table;  /* [B, max_blocks_per_seq] */
  const int32_t *context_lens; /* [B], including the drafts */
  const int32_t *cu_seqlens;   /* [B+1] device, nondecreasing, cu[0] = 0, cu[B] = T */
  const uint64_t *masks;       /* [T], or NULL */
  aflex_bf16 *out;             /* [T, Hq, D] */
  int32_t B, T, Hq, Hkv, D;
  int32_t max_drafts;          /* host-known bound on n_b, in [0, 64] */
  int32_t block_size;          /* must be 16 */
  int32_t max_blocks_per_seq, num_blocks;
  int32_t max_context_len;     /* as in aflex_attn_args */
  float scale;                 /* softmax scale; 0 selects 1/sqrt(D) */
} aflex_attn_tree_args;

/* Supported: D in {64, 128}, block_size == 16, Hq % Hkv == 0, Hq / Hkv <= 16, */
/* max_drafts <= 64, T <= B * max_drafts, B * Hkv * (ceil(max_context_len /    */
/* 16) + 16) * ceil(max_drafts * (Hq / Hkv) / 128) < 2^30, T * Hq < 2^30,      */
/* T < 2^24, Hkv <= 65535. */
/* Device-side values are clamped: rows to [0, T], contexts to [0,             */
/* max_context_len] (s_b then counts from the clamped length; places below 0   */
/* do not exist, and the drafts there are not seen); rows of a sequence beyond */
/* max_drafts are not written. A context of 0 yields 0. Tokens of block ids    */
/* outside [0, num_blocks) are masked. The workspace needs no initialisation.  */
/* The same result on every call with the same inputs (bitwise). Values of a   */
/* bf16 cache below 2^-113 in magnitude lose bits.                             */
aflex_status aflex_attn_tree_workspace(const aflex_attn_tree_args *a, size_t *bytes);
aflex_status aflex_attn_tree(const aflex_attn_tree_args *a, void *workspace, size_t workspace_bytes,
                             aflex_stream stream);

/* ------------------------------------------------------------------------ */
/* The accepted drafts to their places. With n_b and s_b as above, N_b the     */
/* leading entries of accepted[b] that ascend strictly and lie in [0, n_b),    */
/* at most accepted_counts[b] and max_accepted of them: the cache entries      */
/* (keys, values, exponents) of place s_b + accepted[b][i] are copied to place */
/* s_b + i, all read before they are overwritten, and                          */
/*   context_out[b] = s_b + N_b.                                               */
/* Places behind keep what they hold.                                          */
/* ------------------------------------------------------------------------ */
typedef struct aflex_cache_accept_args {
  void *k_cache;               /* pools as in aflex_attn_tree_args (updated in place) */
  void *v_cache;
  int8_t *kv_exp;              /* NULL: the pools hold bf16 */
  const int32_t *block_table;  /* [B, max_blocks_per_seq] */
  const int32_t *context_lens; /* [B], including the drafts */
  const int32_t *cu_seqlens;   /* [B+1] device, as in aflex_attn_tree_args */
  const int32_t *accepted;     /* [B, max_accepted] drafts, ascending */
  const int32_t *accepted_counts; /* [B] */
  int32_t *context_out;        /* [B] (written; overlaps none of the arrays above) */
  int32_t B, Hkv, D;
  int32_t max_accepted;        /* row stride of accepted, in [1, 64] */
  int32_t block_size;          /* must be 16 */
  int32_t max_blocks_per_seq, num_blocks;
} aflex_cache_accept_args;

/* Supported: D in {64, 128}, block_size == 16, max_accepted <= 64, B <= 65535, */
/* Hkv <= 65535. Device-side values are clamped: a sequence with context_lens   */
/* outside [1, capacity] or with n_b outside [0, context_lens[b]] moves nothing */
/* and gets context_out[b] = context_lens[b]; entries whose source or target    */
/* block id is outside [0, num_blocks) are not copied. A block must not appear  */
/* twice among the slots written. No workspace.                                 */
/* Block summaries (aflex_longctx.h) do not follow: blocks that drafts fill have */
/* none, and those that the move changes have none of their new keys. Behind it, */
/* aflex_block_summary with the new lengths makes them for the next              */
/* aflex_block_select.                                                           */
aflex_status aflex_cache_accept(const aflex_cache_accept_args *a, aflex_stream stream);

/* Kernel names for aflex_profile_start: rope_append_f8, rope_write_f8,        */
/* attn_rows, attn_rows_merge, cache_accept.                                   */

#ifdef __cplusplus
}
#endif
#endif /* AFLEX_DRAFT_H */
