// Host side of the C ABI declared in include/locks_tokens.h: argument checks and
// stream-ordered launches.
#include <math.h>

#include "tokens_internal.h"

namespace locks {
namespace {

bool aligned16(const void* p) { return !(reinterpret_cast<uintptr_t>(p) & 15); }

// Checks the new tokens against the configuration and lays them out for the kernels.
int draft_args(const locks_cfg_t* c, const locks_draft_t* d, const int32_t* page_table,
               const int32_t* seq_lens, DraftArgs* a) {
  const int rc = validate(c, false);
  if (rc) return rc;
  if (!d || !page_table || !seq_lens || d->n_tokens < 0) return LOCKS_E_INVAL;
  if (!d->cu_tokens && d->n_tokens != c->num_seqs) return LOCKS_E_INVAL;
  if (d->mask && d->mask_words < 1) return LOCKS_E_INVAL;
  const int qb = c->q_dtype == LOCKS_BF16 ? 2 : 4;
  if (d->n_tokens > 0 &&
      (!d->q || !aligned16(d->q) || d->q_stride < (int64_t)c->num_q_heads * kDim ||
       d->q_stride * qb % 16 != 0 || d->q_stride > (int64_t)1 << 40))
    return LOCKS_E_INVAL;
  // (a sequence's tokens are rounded up to whole units in 32 bits)
  if ((int64_t)d->n_tokens * c->num_q_heads > 0x7fffffffL ||
      (int64_t)c->max_pages_per_seq * c->page_size * c->num_kv_heads >
          (0x7fffffffL - 4096) / (c->num_seqs ? c->num_seqs : 1) ||
      (int64_t)c->num_kv_heads * c->page_size * kDim * (c->kv_dtype == LOCKS_BF16 ? 2 : 4) > 0xffffffffL ||
      (d->mask && d->mask_words > 1 << 25))
    return LOCKS_E_UNSUPPORTED;
  *a = DraftArgs{d->q, d->cu_tokens, d->mask, page_table, seq_lens, (long)d->q_stride, d->n_tokens,
                 d->mask ? d->mask_words : 0, c->num_seqs, c->num_kv_heads,
                 c->num_q_heads / c->num_kv_heads, c->page_size, c->max_pages_per_seq, c->num_blocks};
  return LOCKS_OK;
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

}  // namespace
}  // namespace locks

using namespace locks;

extern "C" {

size_t locks_tree_workspace_bytes(const locks_cfg_t* cfg, int32_t n_tokens) {
  if (validate(cfg, false) || n_tokens < 0) return 0;
  // the attention calls' part of fewer sequences can be larger too
  locks_cfg_t fewer = *cfg;
  size_t most = plan_workspace(*cfg).total;
  for (fewer.num_seqs = 1; fewer.num_seqs < cfg->num_seqs; ++fewer.num_seqs) {
    const size_t n = plan_workspace(fewer).total;
    if (n > most) most = n;
  }
  return align256(most) + tree_scratch_most(*cfg, n_tokens);
}

int locks_tree_attend(const locks_cfg_t* cfg, const locks_draft_t* draft, const void* k_cache,
                      const void* v_cache, const int32_t* page_table, const int32_t* seq_lens,
                      void* out, int32_t out_dtype, float* out_lse, void* ws, size_t ws_bytes,
                      void* stream) {
  DraftArgs a;
  int rc = draft_args(cfg, draft, page_table, seq_lens, &a);
  if (rc) return rc;
  if (out_dtype != LOCKS_BF16 && out_dtype != LOCKS_FP32) return LOCKS_E_UNSUPPORTED;
  if (!k_cache || !v_cache || !aligned16(k_cache) || !aligned16(v_cache)) return LOCKS_E_INVAL;
  if (draft->n_tokens > 0 && (!out || !aligned16(out) || out == draft->q)) return LOCKS_E_INVAL;
  if ((rc = check_ws(cfg, ws, ws_bytes))) return rc;
  const size_t scratch = align256(plan_workspace(*cfg).total);
  if (ws_bytes < scratch + tree_scratch_bytes(*cfg, draft->n_tokens)) return LOCKS_E_WORKSPACE;
  if (cfg->num_seqs == 0 || draft->n_tokens == 0) return LOCKS_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if ((rc = checked_tables(*cfg, ws, a.page_table, a.seq_lens, st))) return rc;
  return hip_status(launch_tree_attend(*cfg, a, k_cache, v_cache, out, out_dtype == LOCKS_BF16, out_lse,
                                       static_cast<char*>(ws) + scratch, st));
}

int locks_token_mass(const locks_cfg_t* cfg, const locks_draft_t* draft, const float* lse,
                     const void* k_cache, const int32_t* page_table, const int32_t* seq_lens,
                     float decay, float* mass, void* stream) {
  DraftArgs a;
  const int rc = draft_args(cfg, draft, page_table, seq_lens, &a);
  if (rc) return rc;
  if (!k_cache || !aligned16(k_cache) || !mass || !aligned16(mass) || !isfinite(decay))
    return LOCKS_E_INVAL;
  if (draft->n_tokens > 0 && !lse) return LOCKS_E_INVAL;
  if (cfg->num_seqs == 0 || draft->n_tokens == 0) return LOCKS_OK;
  return hip_status(launch_token_mass(*cfg, a, lse, k_cache, decay, mass, static_cast<hipStream_t>(stream)));
}

size_t locks_pick_workspace_bytes(const locks_cfg_t* cfg) {
  if (validate(cfg, false)) return 0;
  return pick_scratch_most(*cfg);
}

int locks_pick_tokens(const locks_cfg_t* cfg, const float* mass, const int32_t* seq_lens,
                      int32_t n_keep, int32_t n_sink, int32_t n_recent, int32_t* out_ids, void* ws,
                      size_t ws_bytes, void* stream) {
  const int rc = validate(cfg, false);
  if (rc) return rc;
  if (!mass || !aligned16(mass) || !seq_lens || !out_ids || n_keep < 1 || n_sink < 0 || n_recent < 0 ||
      n_recent > n_keep || n_sink > n_keep - n_recent)
    return LOCKS_E_INVAL;
  const int64_t lists = (int64_t)cfg->num_seqs * cfg->num_kv_heads;
  const int64_t width = (int64_t)cfg->max_pages_per_seq * cfg->page_size;
  if (lists > 0x7fffffffL || (lists && (width > 0x7fffffffL / lists || n_keep > 0x7fffffffL / lists)))
    return LOCKS_E_UNSUPPORTED;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255) || ws_bytes < pick_scratch_bytes(*cfg))
    return LOCKS_E_WORKSPACE;
  if (lists == 0) return LOCKS_OK;
  return hip_status(launch_pick_tokens(*cfg, mass, seq_lens, n_keep, n_sink, n_recent, out_ids, ws,
                                       static_cast<hipStream_t>(stream)));
}

int locks_keep_tokens(const locks_cfg_t* cfg, const int32_t* kept, int32_t heads, int32_t n_keep,
                      const int32_t* start, void* k_cache, void* v_cache, float* mass,
                      const int32_t* page_table, int32_t* out_lens, void* stream) {
  const int rc = validate(cfg, false);
  if (rc) return rc;
  if (!k_cache || !v_cache || !aligned16(k_cache) || !aligned16(v_cache) || !page_table || n_keep < 0 ||
      (heads != 1 && heads != cfg->num_kv_heads) || (n_keep > 0 && !kept) ||
      (out_lens && out_lens == start))
    return LOCKS_E_INVAL;
  const int64_t lists = (int64_t)cfg->num_seqs * cfg->num_kv_heads;
  if (lists > 0x7fffffffL || (lists && n_keep > 0x7fffffffL / lists) ||
      (int64_t)cfg->max_pages_per_seq * cfg->page_size > 0x7fffffffL)
    return LOCKS_E_UNSUPPORTED;
  if (cfg->num_seqs == 0) return LOCKS_OK;
  return hip_status(launch_keep_tokens(*cfg, kept, heads, n_keep, start, k_cache, v_cache, mass, page_table,
                                       out_lens, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
