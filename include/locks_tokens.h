/*
 * locks_tokens.h -- C ABI of the calls on single tokens of the paged KV cache: several new
 * tokens of a sequence attended at once (a tree of drafted ones, or a run of a prompt), the
 * attention weight that every cached token collects, the tokens to keep by it, and kept
 * tokens moved together.  Part of liblocks; the conventions of locks.h (device pointers
 * owned by the caller, no allocation, no synchronisation, work enqueued on `stream`, host
 * checks before any launch, status codes, layouts) hold here too.
 *
 *   speculative decoding   locks_rope_append_kv (all drafts, positions by depth),
 *                          locks_tree_attend, [the caller accepts a branch],
 *                          locks_keep_tokens
 *   a bounded cache        an attention with out_lse, locks_token_mass, and when the cache
 *                          is full locks_pick_tokens and locks_keep_tokens
 *
 * Pointers to rows, caches and outputs must be 16-byte aligned and row strides a multiple of
 * 16 bytes; LOCKS_E_INVAL otherwise.  Lengths are held to [0, B * max_pages_per_seq] and row
 * ranges to [0, n_tokens] by the kernels (of cu_tokens that do not ascend rows may be wrong
 * or not written, but nothing outside the buffers is accessed); a page whose block lies
 * outside [0, num_blocks) is read as block 0 by locks_tree_attend (with table checks on it is
 * reported, see locks_set_table_checks) and left out by locks_token_mass and
 * locks_keep_tokens.  The calls touch no summaries, so they take caches whose summary store
 * would be too large too.
 *
 * Lengths are known on the device only, so where kernels differ for short sequences they are
 * chosen by the tables' width, max_pages_per_seq.  In tables much wider than the sequences
 * attention over up to 512 tokens takes 1.4 times as long, picks of up to 32,768 tokens two to
 * four times, masses of many new tokens over few four to five times.
 */
#ifndef LOCKS_TOKENS_H
#define LOCKS_TOKENS_H

#include "locks.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The new tokens of every sequence, whose keys and values are in the cache already (the
 * last ones of each sequence, counted by seq_lens).  With cu_tokens (device
 * [num_seqs + 1], ascending from 0) sequence s's are rows [cu_tokens[s], cu_tokens[s + 1]);
 * it may have none, and rows from cu_tokens[num_seqs] on are padding: any values, and the
 * outputs' rows there are left as they were.  Without it, row s is the newest token of
 * sequence s and n_tokens must be num_seqs.
 *
 * With n new tokens, new token i (of the sequence's) sees every token below seq_lens[s] - n,
 * and of the new ones:
 *   mask NULL   tokens 0 .. i (a run)
 *   mask        token j where bit j % 32 of word mask[row][j / 32] is set; none from
 *               32 * mask_words on.  A tree's row holds its ancestors' bits and its own. */
typedef struct locks_draft {
  const void* q;             /* [n_tokens][H_q][128] (q_dtype), already rotated            */
  const int32_t* cu_tokens;  /* or NULL                                                    */
  const uint32_t* mask;      /* device [n_tokens][mask_words], or NULL                     */
  int64_t q_stride;          /* elements between tokens, at least a row's                  */
  int32_t n_tokens;          /* >= 0                                                       */
  int32_t mask_words;        /* >= 1 where there is a mask, else not read                  */
} locks_draft_t;

/* Bytes of workspace for locks_tree_attend with cfg and n_tokens new tokens, and with fewer
 * of them or fewer sequences (num_seqs); at least locks_workspace_bytes(cfg) (whose
 * table-check word it holds too).  0 if one is invalid. */
size_t locks_tree_workspace_bytes(const locks_cfg_t* cfg, int32_t n_tokens);

/* Attention of every new token's query heads over the tokens that it sees,
 *   o = sum_t softmax_t(q . k_t / sqrt(128)) v_t.
 *   out      [n_tokens][H_q][128] of out_dtype (LOCKS_BF16 or LOCKS_FP32)
 *   out_lse  nullable float [n_tokens][H_q], log of the softmax denominator
 * A token that sees nothing gets out = 0 and out_lse = -inf; a NaN in a query, or in a key
 * that it sees, makes its out and out_lse NaN.  Tokens that a row does not see do not reach
 * it, whatever their keys and values hold; nor do rows past a sequence's end.
 * Logits, maxima and sums are fp32.  Over bf16 queries and caches the softmax weights enter
 * the product with the values as sums of bf16 terms: three for fp32 outputs (2^-24 of a
 * weight), two for bf16 ones (2^-16), whatever the batch; other types are computed in fp32
 * throughout.
 * Returns LOCKS_E_INVAL for a null or misaligned pointer, a bad stride or count or out == q,
 * and LOCKS_E_UNSUPPORTED for another out_dtype, for n_tokens * H_q of 2^31 or more, the
 * tables' tokens over all sequences and KV heads of 2^31 - 4,096 or more, masks of more than
 * 2^25 words a row, or a block of 4 GiB or more (all KV heads of a page). */
int locks_tree_attend(const locks_cfg_t* cfg, const locks_draft_t* draft, const void* k_cache,
                      const void* v_cache, const int32_t* page_table, const int32_t* seq_lens,
                      void* out, int32_t out_dtype, float* out_lse, void* ws, size_t ws_bytes,
                      void* stream);

/* Adds up the attention that every token gets from the new ones, per KV head h:
 *   mass[s][h][t] = decay * mass[s][h][t] + sum over new tokens i that see t and heads g of
 *                   the group of exp(q_ig . k_t / sqrt(128) - lse[i][g])
 * for t < seq_lens[s]; the old value of the new tokens themselves counts as 0 (their slots
 * may hold that of others), and entries from seq_lens[s] on are left as they were.  A row
 * whose lse is -inf adds nothing.  `lse` [n_tokens][H_q] is what the attention over the same
 * tokens returned (of one over fewer, such as locks_sparse_attend, weights are relative to
 * its own sum).  The sums are fp32 and always added in the same order.
 *   mass  float [S][H_kv][B * max_pages_per_seq]
 * Sequences without new tokens are left as they were.  Errors as in locks_tree_attend, and
 * LOCKS_E_INVAL unless decay is finite. */
int locks_token_mass(const locks_cfg_t* cfg, const locks_draft_t* draft, const float* lse,
                     const void* k_cache, const int32_t* page_table, const int32_t* seq_lens,
                     float decay, float* mass, void* stream);

/* Bytes of workspace for locks_pick_tokens with cfg, and with fewer sequences (0 if cfg is
 * invalid). */
size_t locks_pick_workspace_bytes(const locks_cfg_t* cfg);

/* The n_keep tokens of every sequence and KV head to keep: the first n_sink, the last
 * n_recent, and of the others those of largest mass, the lower index first where masses are
 * equal (0 and -0 are; a NaN counts as less than everything).  A sequence of at most n_keep
 * tokens keeps all of them.
 *   out_ids  int32 [S][H_kv][n_keep], ascending, padded with -1
 * Returns LOCKS_E_INVAL for a null pointer, n_keep < 1, negative counts or
 * n_sink + n_recent > n_keep; LOCKS_E_UNSUPPORTED for 2^31 entries or more of mass or
 * out_ids; LOCKS_E_WORKSPACE as elsewhere. */
int locks_pick_tokens(const locks_cfg_t* cfg, const float* mass, const int32_t* seq_lens,
                      int32_t n_keep, int32_t n_sink, int32_t n_recent, int32_t* out_ids, void* ws,
                      size_t ws_bytes, void* stream);

/* Moves kept tokens together, in place: with a = start[s] (0 where start is NULL) and
 * src = kept[s][h][i], the key, value and mass of token src become those of token a + i, for
 * every i before the list's first negative entry.  Nothing else is written: tokens below a
 * and the rows behind the last one moved stay as they were.  Lists need not ascend, but a
 * token may only move to the front: an entry src < a + i is left out (that row stays as it
 * was), and so is one whose own or new place lies outside the tables.
 *   kept      int32 [S][heads][n_keep], heads = H_kv, or 1: one list for all KV heads
 *   mass      nullable float [S][H_kv][B * max_pages_per_seq]
 *   out_lens  nullable int32 [S]: a + the entries of the sequence's first list; may be the
 *             caller's seq_lens, but not `start`
 * A block that tokens are moved into must belong to one sequence.  Summaries of the pages
 * that change have to be built again (locks_build_summaries).  Positions stay with the
 * tokens: keys are moved as rotated.
 * Returns LOCKS_E_INVAL for a null or misaligned cache, a null list or table, n_keep < 0,
 * heads other than 1 or H_kv, or out_lens == start. */
int locks_keep_tokens(const locks_cfg_t* cfg, const int32_t* kept, int32_t heads, int32_t n_keep,
                      const int32_t* start, void* k_cache, void* v_cache, float* mass,
                      const int32_t* page_table, int32_t* out_lens, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LOCKS_TOKENS_H */
