/*
 * aflex_longctx.h -- long-context operators of libaflex over the paged KV
 * cache of aflex.h: the position rotation on the way into the cache, a
 * whole-number summary of each block's keys, the choice of the blocks that a
 * query attends, and decode attention over the chosen blocks.
 *
 *   aflex_rope_append         rotate one token's q and k per sequence, append K/V
 *   aflex_rope_write          the same for packed prompts or chunks
 *   aflex_block_summary       summaries of the blocks of a cache written otherwise
 *   aflex_block_select        the blocks that each (sequence, kv head) attends
 *   aflex_attn_sparse_decode  decode attention over those blocks
 *
 * A decode step is rope_append, block_select, attn_sparse_decode. A context of
 * n tokens then costs its attention min(n, 16 top_blocks) cached tokens and
 * the choice D + 1 bytes per 16 tokens and kv head, a 64th of the K and V of
 * those tokens. The conventions of aflex.h hold (device pointers, alignment,
 * streams, workspaces, validation before launch, errors); strides are counted
 * in elements. block_select and attn_sparse_decode may be several launches that
 * communicate through the workspace: calls that share one run on one stream,
 * and are made by one host thread at a time.
 */
#ifndef AFLEX_LONGCTX_H
#define AFLEX_LONGCTX_H

#include "aflex.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------ */
/* Rotation and cache write. Channels come in rotary_dim / 2 pairs (a, b):   */
/* channels i and i + rotary_dim / 2, or 2i and 2i + 1 (interleaved). With    */
/* c = rope[p][i], s = rope[p][rotary_dim / 2 + i] at position p:             */
/*   a' = a c - b s,   b' = b c + a s    (fp32, each operation rounded; bf16) */
/* channels from rotary_dim on are copied. q rows are rotated into q_out, k   */
/* rows into the K pool (there alone), v rows are copied into the V pool, at  */
/* the slots of aflex_kv_append / aflex_kv_write: token i of sequence b's n_b */
/* new tokens sits at j = context_lens[b] - n_b + i. p = j unless positions   */
/* is given.                                                                  */
/*                                                                            */
/* Summaries (block_keys / block_exp, both or neither): whenever a write      */
/* fills a block's last slot, the block's summary is made from its 16 cached  */
/* keys (the older ones read back from the K pool). For kv head g:            */
/*   e = least whole number >= -100 with |k| < 2^e for all 16 D values        */
/*   S_d = sum over the keys of rne(k_d 2^(14 - e))     (whole numbers)       */
/*   r = max(0, bits(max_d |S_d|) - 7)                                        */
/*   block_keys[d] = clamp(rne(S_d 2^-r), -127, 127),  block_exp = e - 18 + r */
/* so that the mean key is about block_keys 2^block_exp. A block that holds   */
/* an infinity or NaN gets block_exp = 127 and zero codes. Every value is     */
/* exact, whatever the order of the sum: equal keys give equal summaries.     */
/* ------------------------------------------------------------------------ */
typedef struct aflex_rope_args {
  const aflex_bf16 *q;         /* [T, Hq, D], rows q_stride apart */
  const aflex_bf16 *k_new;     /* [T, Hkv, D], rows k_stride apart */
  const aflex_bf16 *v_new;     /* [T, Hkv, D], rows v_stride apart */
  const float *rope;           /* [rope_len, rotary_dim]: cosines, then sines (unread if rotary_dim = 0) */
  const int32_t *positions;    /* [T] rows of rope, or NULL: the token's place in its sequence */
  const int32_t *cu_seqlens;   /* [B+1] as in aflex_kv_write (aflex_rope_append: unread) */
  aflex_bf16 *q_out;           /* [T, Hq, D] dense (written) */
  aflex_bf16 *k_cache;         /* [num_blocks, Hkv, block_size, D] (written) */
  aflex_bf16 *v_cache;         /* [num_blocks, Hkv, D, block_size] (written) */
  int8_t *block_keys;          /* [num_blocks, Hkv, D] (written), or NULL */
  int8_t *block_exp;           /* [num_blocks, Hkv] (written), or NULL */
  const int32_t *block_table;  /* [B, max_blocks_per_seq] */
  const int32_t *context_lens; /* [B], including the new tokens */
  int32_t B, T;                /* sequences, new tokens (aflex_rope_append: T is unread, B) */
  int32_t Hq, Hkv, D;
  int32_t rotary_dim;          /* a multiple of 16 in [0, D] */
  int32_t interleaved;         /* 0: pairs (i, i + rotary_dim / 2); else (2i, 2i + 1) */
  int32_t rope_len;            /* rows of rope (unread if rotary_dim = 0) */
  int32_t max_seqlen;          /* host-known bound on n_b (aflex_rope_append: unread) */
  int32_t block_size;          /* must be 16 */
  int32_t max_blocks_per_seq, num_blocks;
  int32_t q_stride, k_stride, v_stride; /* elements from one token's row to the next, multiples of 8
                                  of at least H D; 0: dense */
} aflex_rope_args;

/* Supported: D in {64, 128}, block_size == 16, rows of fewer than 2^30     */
/* elements; for aflex_rope_append B (Hq + Hkv) < 2^30 and B (Hkv + Hq D /  */
/* 1024) < 2^26 - 4; for aflex_rope_write B <= 65535, at most 4096 heads,   */
/* max_seqlen <= T and max_seqlen <= 2^28 - 32. No workspace. Device-side   */
/* values are clamped as in aflex_kv_append and aflex_kv_write: sequences   */
/* with context_lens outside [1, capacity], tokens before place 0 and, with */
/* rotary_dim > 0, tokens whose position is outside [0, rope_len) are left  */
/* alone (neither q_out nor the cache is written for them); for a block id  */
/* outside [0, num_blocks) only q_out is written. A block must not appear   */
/* twice among the slots written. Tokens beyond max_seqlen may be left      */
/* alone.                                                                   */
aflex_status aflex_rope_append(const aflex_rope_args *a, aflex_stream stream);
aflex_status aflex_rope_write(const aflex_rope_args *a, aflex_stream stream);

/* Summaries, as above, of every full block of the B sequences (blocks         */
/* j < context_lens / 16): for caches filled by aflex_kv_append, aflex_kv_write */
/* or another program. Blocks that are not full keep what they hold.           */
typedef struct aflex_block_summary_args {
  const aflex_bf16 *k_cache;   /* [num_blocks, Hkv, block_size, D] */
  int8_t *block_keys;          /* [num_blocks, Hkv, D] (written) */
  int8_t *block_exp;           /* [num_blocks, Hkv] (written) */
  const int32_t *block_table;  /* [B, max_blocks_per_seq] */
  const int32_t *context_lens; /* [B] */
  int32_t B, Hkv, D;
  int32_t block_size;          /* must be 16 */
  int32_t max_blocks_per_seq, num_blocks;
  int32_t max_context_len;     /* host-known bound on the context lengths; larger device values are clamped */
} aflex_block_summary_args;

/* Supported: D in {64, 128}, block_size == 16, B <= 65535,                    */
/* max_context_len / 16 * Hkv < 2^30. No workspace.                            */
aflex_status aflex_block_summary(const aflex_block_summary_args *a, aflex_stream stream);

/* ------------------------------------------------------------------------ */
/* Choice of blocks for one new token per sequence. With n_b =                */
/* ceil(context_lens[b] / 16) blocks and N = min(top_blocks, n_b), row (b, g) */
/* of `selected` gets N block numbers (indices into b's block table, not pool */
/* ids) in ascending order, then -1: the first sink_blocks, the last           */
/* recent_blocks (the block being filled is one of them), and those of the     */
/* others that score highest, the lower number first among equals.             */
/* Each query head h of group g is rounded to whole numbers like a summary:    */
/*   e_h least whole number >= -100 with |q_d| < 2^e_h for all finite q_d      */
/*   c_hd = clamp(rne(q_d 2^(7 - e_h)), -127, 127)   (0 for non-finite q_d)    */
/*   score_j = max over h of 2^(e_h - 7 + block_exp_j) sum_d c_hd block_keys_jd */
/* in fp32; +infinity where block_exp_j = 127. The sum is over whole numbers,  */
/* so the choice does not depend on how the work is split. Blocks whose id is  */
/* outside [0, num_blocks) come last.                                          */
/* ------------------------------------------------------------------------ */
typedef struct aflex_block_select_args {
  const aflex_bf16 *q;         /* [B, Hq, D] (rotated) */
  const int8_t *block_keys;    /* [num_blocks, Hkv, D] */
  const int8_t *block_exp;     /* [num_blocks, Hkv] */
  const int32_t *block_table;  /* [B, max_blocks_per_seq] */
  const int32_t *context_lens; /* [B] */
  int32_t *selected;           /* [B, Hkv, top_blocks] (written) */
  int32_t B, Hq, Hkv, D;
  int32_t block_size;          /* must be 16 */
  int32_t max_blocks_per_seq, num_blocks;
  int32_t max_context_len;     /* as in aflex_attn_args */
  int32_t top_blocks;          /* blocks per (sequence, kv head), >= sink_blocks + recent_blocks */
  int32_t sink_blocks;         /* >= 0 */
  int32_t recent_blocks;       /* >= 1 */
} aflex_block_select_args;

/* Supported: D in {64, 128}, block_size == 16, Hq % Hkv == 0,                 */
/* Hq / Hkv <= 16, B * Hkv < 2^24,                                             */
/* B * Hkv * ceil(max_context_len / 16) < 2^30,                                */
/* B * Hkv * top_blocks < 2^30. The workspace needs no initialisation.         */
aflex_status aflex_block_select_workspace(const aflex_block_select_args *a, size_t *bytes);
aflex_status aflex_block_select(const aflex_block_select_args *a, void *workspace, size_t workspace_bytes,
                                aflex_stream stream);

/* ------------------------------------------------------------------------ */
/* Decode attention over chosen blocks: aflex_attn_decode restricted, for kv   */
/* head g of sequence b, to the tokens of blocks selected[b][g][0 .. N),       */
/* N = min(top_blocks, ceil(context_lens[b] / 16)). Rows must ascend: an entry */
/* that is not greater than the one before it, or outside the sequence's       */
/* blocks, contributes nothing. A row without a valid entry yields out = 0.    */
/* ------------------------------------------------------------------------ */
typedef struct aflex_attn_sparse_args {
  aflex_attn_args attn;        /* split_tokens must be 0 */
  const int32_t *selected;     /* [B, Hkv, top_blocks] */
  int32_t top_blocks;          /* >= 1 */
} aflex_attn_sparse_args;

/* Supported: as aflex_attn_decode, and B * Hkv < 2^24, B * Hkv *           */
/* top_blocks < 2^30. The same result on every call with the same inputs    */
/* (bitwise). The softmax weights keep 16 bits (two bf16 values) in the     */
/* product with the values and are summed as rounded; scores, sums and the  */
/* merge of split lists are fp32.                                           */
aflex_status aflex_attn_sparse_decode_workspace(const aflex_attn_sparse_args *a, size_t *bytes);
aflex_status aflex_attn_sparse_decode(const aflex_attn_sparse_args *a, void *workspace, size_t workspace_bytes,
                                      aflex_stream stream);

/* Kernel names for aflex_profile_start: rope_append, rope_write,              */
/* block_summary, block_select, block_score, block_pick, attn_sparse,         */
/* attn_merge.                                                                */

#ifdef __cplusplus
}
#endif
#endif /* AFLEX_LONGCTX_H */
