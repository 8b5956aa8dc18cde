/*
 * locks_cache.h -- C ABI of the paged KV cache around the decode step: new tokens
 * rotated by their positions and appended, a cache held in 8 bits, and decode
 * attention over it.  Part of liblocks; the conventions of locks.h (device pointers
 * owned by the caller, no allocation, no synchronisation, work enqueued on `stream`,
 * host checks before any launch, status codes, layouts, the workspace and the table
 * checks) hold here too.
 *
 * Pointers to rows, caches, stores and outputs must be 16-byte aligned and row strides a
 * multiple of 16 bytes; LOCKS_E_INVAL otherwise.  Where a call trusts page tables (table checks
 * off, or a call without a workspace), the appends still leave out every token whose
 * page, block, input row or position lies outside its table: nothing of it is written.
 * The appends and the attentions touch no summaries, so they take caches whose summary store
 * would be too large too.
 */
#ifndef LOCKS_CACHE_H
#define LOCKS_CACHE_H

#include "locks.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rotary positions.  Pair i (0 <= i < rot_dim / 2) of a row is elements (i, i + rot_dim / 2),
 * or (2 i, 2 i + 1) where `interleaved`; elements from rot_dim on are not rotated.  With the
 * entries c = table[p][i] and s = table[p][rot_dim / 2 + i] of the token's position p, the
 * pair (a, b) becomes (a c - b s, b c + a s): fp32, each product and the sum rounded, the
 * result rounded once to the row's type (or quantised).
 * With several axes (time, height, width) the pairs are split in order, axis_pairs[a] of
 * them for axis a, and a pair reads its own axis's position. */
typedef struct locks_rope {
  const float* table;        /* device [n_pos][rot_dim]; NULL: no rotation, the other
                                fields are not read                                       */
  const int32_t* positions;  /* device [n_axes][n_tokens], or NULL (one axis only): a
                                token's index in its sequence                              */
  int32_t n_pos;             /* rows of the table, >= 1                                    */
  int32_t rot_dim;           /* a multiple of 16 in [16, 128], else LOCKS_E_UNSUPPORTED    */
  int32_t interleaved;       /* 0 or 1                                                     */
  int32_t n_axes;            /* 1, 2 or 3                                                  */
  int32_t axis_pairs[3];     /* >= 0, the first n_axes summing to rot_dim / 2              */
} locks_rope_t;

/* The rows of a step's new tokens.  With cu_tokens (device [num_seqs + 1], ascending from
 * 0) sequence s's new tokens are rows [cu_tokens[s], cu_tokens[s + 1]) and are its last
 * ones, seq_lens[s] counting them; a sequence may have none, and rows from
 * cu_tokens[num_seqs] (at most n_tokens) on are padding: any values, and q_out's rows there
 * are left as they were.  Without it, row s is the newest token of sequence s and n_tokens must be num_seqs
 * (a sequence of length 0 has none).
 * Row t, head h of a tensor starts stride * t + 128 * h elements from its pointer. */
typedef struct locks_rows {
  const void* q;             /* [n_tokens][H_q][128] (q_dtype), or NULL: no queries        */
  const void* k;             /* [n_tokens][H_kv][128] (kv_dtype)                           */
  const void* v;
  void* q_out;               /* rotated queries; may be q itself with the same stride      */
  const int32_t* cu_tokens;  /* or NULL                                                    */
  int64_t q_stride, k_stride, v_stride, q_out_stride;  /* elements between tokens, at least
                                a row's                                                    */
  int32_t n_tokens;          /* >= 0                                                       */
} locks_rows_t;

/* Rotates the new tokens' queries and keys and writes keys and values into the paged
 * caches (locks_append_kv with positions, for any number of tokens): one launch.  `rope`
 * NULL rotates nothing.  A block that receives tokens must belong to one sequence.
 * Returns LOCKS_E_INVAL for a null or misaligned pointer, a bad stride, count or axis
 * split, LOCKS_E_UNSUPPORTED for another rot_dim. */
int locks_rope_append_kv(const locks_cfg_t* cfg, const locks_rows_t* rows,
                         const locks_rope_t* rope, void* k_cache, void* v_cache,
                         const int32_t* page_table, const int32_t* seq_lens, void* stream);

/* A paged cache in 8 bits: codes in the caches' layout and one scale per block and KV
 * head, for keys and for values.  An element is code * scale.
 *   LOCKS_Q8_INT8  two's complement in [-127, 127], scale = largest magnitude / 127
 *   LOCKS_Q8_E4M3  OCP e4m3 (largest 448), scale the least power of two that keeps the
 *                  largest magnitude within 448 scale, so that a page whose scale grows
 *                  moves its codes without rounding (but for codes that become subnormal) */
enum { LOCKS_Q8_INT8 = 0, LOCKS_Q8_E4M3 = 1 };
typedef struct locks_q8 {
  void* k;                   /* uint8 [num_blocks][num_kv_heads][B][128]                   */
  void* v;
  float* k_scale;            /* [num_blocks][num_kv_heads]                                 */
  float* v_scale;
  int32_t code;              /* LOCKS_Q8_INT8 or LOCKS_Q8_E4M3, else LOCKS_E_UNSUPPORTED   */
} locks_q8_t;

/* locks_rope_append_kv into an 8-bit cache, quantised from the rotated fp32 values.  Of a
 * page, KV head and tensor let A be the largest magnitude of the call's new rows (0 if it
 * is under 2^-100).  A page that the call begins takes A's scale, one with earlier rows
 * keeps its own unless A's is larger than its magnitude; then it takes A's, and the earlier
 * rows' codes become Q(code * old scale * (1 / new scale)).  New codes are Q(x * (1 / scale)),
 * 0 where the scale is 0, Q rounding to the nearest code, ties to even, and saturating.
 * Elements that are not finite do not count for A: an infinity takes the largest code whatever
 * the scale (with the sign that keeps its own), a NaN becomes 0 (int8) or NaN (e4m3).
 * Scales and codes of rows past the sequence's end are left as they were, except that the
 * page's scale is theirs too.  Appending the same rows again changes nothing.
 * cfg->kv_dtype is the type of the rows.  Errors as in locks_rope_append_kv. */
int locks_q8_append_kv(const locks_cfg_t* cfg, const locks_rows_t* rows,
                       const locks_rope_t* rope, const locks_q8_t* cache,
                       const int32_t* page_table, const int32_t* seq_lens, void* stream);

/* locks_build_summaries from the keys of an 8-bit cache: the summaries that the fp32 keys
 * code * scale have, bit for bit, so that locks_select serves a sequence whose cache is
 * held in 8 bits (cfg->kv_dtype is not used).  Arguments and errors as there. */
int locks_q8_build_summaries(const locks_cfg_t* cfg, const locks_q8_t* cache,
                             const int32_t* page_table, const int32_t* seq_lens,
                             const int32_t* build_list, int32_t n_build, void* summaries,
                             void* stream);

/* locks_dense_attend and locks_sparse_attend over an 8-bit cache (q [S][H_q][128] of
 * q_dtype, already rotated; cfg->kv_dtype is not used): same arguments, outputs, workspace
 * and table checks.  Rows past a sequence's end may hold any codes, and so may blocks that
 * its table does not reach.  A NaN in a query or in a scale of a live page gives NaN in its
 * outputs.
 * Sums, maxima and outputs are fp32 (weights times values are summed before the division by
 * the weights' sum, at most the tokens' number, and have to stay finite).  Codes enter as they
 * are; queries and weights (the softmax weight times its value scale) as f16 terms: a bf16
 * query element in one, exact but for 2^-39 of its head's largest; an fp32 one, and a weight,
 * in two, off by at most 2^-23 of itself or 2^-39 of the head's largest element or the largest
 * value scale, whichever is more.
 * Returns LOCKS_E_INVAL for a null or misaligned pointer, LOCKS_E_UNSUPPORTED for
 * tables of 2^31 sixteen-token units or more over all sequences and KV heads. */
int locks_q8_dense_attend(const locks_cfg_t* cfg, const void* q, const locks_q8_t* cache,
                          const int32_t* page_table, const int32_t* seq_lens, float* out,
                          float* out_lse, void* ws, size_t ws_bytes, void* stream);
int locks_q8_sparse_attend(const locks_cfg_t* cfg, const void* q, const locks_q8_t* cache,
                           const int32_t* page_table, const int32_t* seq_lens,
                           const int32_t* page_ids, float* out, float* out_lse, void* ws,
                           size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LOCKS_CACHE_H */
