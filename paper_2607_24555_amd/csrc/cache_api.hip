// Host side of the C ABI declared in include/locks_cache.h: argument checks, split planning
// and stream-ordered launches.
#include "cache_internal.h"

namespace locks {
namespace {

bool aligned16(const void* p) { return !(reinterpret_cast<uintptr_t>(p) & 15); }

int q8_valid(const locks_q8_t* q8) {
  if (!q8) return LOCKS_E_INVAL;
  if (q8->code != LOCKS_Q8_INT8 && q8->code != LOCKS_Q8_E4M3) return LOCKS_E_UNSUPPORTED;
  if (!q8->k || !q8->v || !q8->k_scale || !q8->v_scale) return LOCKS_E_INVAL;
  if (!aligned16(q8->k) || !aligned16(q8->v)) return LOCKS_E_INVAL;
  return LOCKS_OK;
}

// A rows tensor: pointer and stride (elements of `bytes` bytes, rows of `heads` heads).
bool rows_valid(const void* p, int64_t stride, int heads, int bytes) {
  return p && aligned16(p) && stride >= (int64_t)heads * kDim && stride * bytes % 16 == 0 &&
         stride <= (int64_t)1 << 40;
}

// Checks the rows and the rotation of an append and lays them out for the kernels.
int append_args(const locks_cfg_t* c, const locks_rows_t* rows, const locks_rope_t* rope,
                const int32_t* page_table, const int32_t* seq_lens, RowArgs* a, RopeArgs* r) {
  int rc = validate(c, false);
  if (rc) return rc;
  if (!rows || !page_table || !seq_lens || rows->n_tokens < 0) return LOCKS_E_INVAL;
  if (!rows->cu_tokens && rows->n_tokens != c->num_seqs) return LOCKS_E_INVAL;
  const int kb = c->kv_dtype == LOCKS_BF16 ? 2 : 4, qb = c->q_dtype == LOCKS_BF16 ? 2 : 4;
  const bool any = rows->n_tokens > 0;  // (no rows: their pointers are not looked at)
  if (any && (!rows_valid(rows->k, rows->k_stride, c->num_kv_heads, kb) ||
              !rows_valid(rows->v, rows->v_stride, c->num_kv_heads, kb)))
    return LOCKS_E_INVAL;
  if (any && rows->q && (!rows_valid(rows->q, rows->q_stride, c->num_q_heads, qb) ||
                  !rows_valid(rows->q_out, rows->q_out_stride, c->num_q_heads, qb)))
    return LOCKS_E_INVAL;
  if (rows->q && rows->q == rows->q_out && rows->q_stride != rows->q_out_stride) return LOCKS_E_INVAL;
  *a = RowArgs{rows->q, rows->k, rows->v, rows->q_out, rows->cu_tokens, (long)rows->q_stride,
               (long)rows->k_stride, (long)rows->v_stride, (long)rows->q_out_stride, rows->n_tokens};
  *r = RopeArgs{};
  r->n_tokens = rows->n_tokens;
  if (rope && rope->table) {
    if (rope->rot_dim < 16 || rope->rot_dim > kDim || rope->rot_dim % 16) return LOCKS_E_UNSUPPORTED;
    if (!aligned16(rope->table) || rope->n_pos < 1 || rope->n_axes < 1 || rope->n_axes > 3 ||
        (rope->interleaved != 0 && rope->interleaved != 1) || (rope->n_axes > 1 && !rope->positions))
      return LOCKS_E_INVAL;
    int sum = 0;
    for (int i = 0; i < rope->n_axes; ++i) {
      if (rope->axis_pairs[i] < 0 || rope->axis_pairs[i] > kDim) return LOCKS_E_INVAL;
      sum += rope->axis_pairs[i];
    }
    if (sum != rope->rot_dim / 2) return LOCKS_E_INVAL;
    r->table = rope->table;
    r->positions = rope->positions;
    r->n_pos = rope->n_pos;
    r->half = rope->rot_dim / 2;
    r->interleaved = rope->interleaved;
    r->n_axes = rope->n_axes;
    r->axis1 = rope->axis_pairs[0];
    r->axis2 = r->axis1 + (rope->n_axes > 1 ? rope->axis_pairs[1] : 0);
  }
  return LOCKS_OK;
}

// Equal shares for 512 blocks, two of the three that a compute unit holds (8 ragged sequences,
// 272K tokens, 8 heads: 98 us; 256 blocks 111, 640 110, 768 100, 1,024 101), but for 256 where
// a share is 8 to 64 units and there are no more lists than that (65K tokens of one head 13.8
// us against 16.6, of eight 29.8 against 28.8); as many blocks as lists between 512 and 1,024
// of them; fewer where the workspace holds fewer partials (they may take it up to the checked
// tables).
// A block per list, without partials, up to the widths where that was no slower: 32 units with
// few lists (64 lists: 9.3 us against 10.4, at 64 units 14.9 against 12.8), 64 from 128 lists
// (15.1 against 16.0, at 128 units 23.9 against 20.3) and 256 from 512 (103 against 112).
Q8Plan q8_plan(const locks_cfg_t& c, long list_units, bool listed) {
  const WsPlan p = plan_workspace(c);
  const long lists = (long)c.num_seqs * c.num_kv_heads;
  const size_t slot = (size_t)(c.num_q_heads / c.num_kv_heads) * (kDim + 2) * sizeof(float);
  const long room = (long)(p.chk_pt_off / slot) - lists;
  list_units = (list_units + 7) / 8 * 8;  // (as the kernel counts a list)
  const long all = lists * list_units, most = lists < 512 ? 512 : lists < 1024 ? lists : 1024;
  long blocks = all / 8 < most ? all / 8 : most;
  blocks = blocks < room ? blocks : room;
  if (list_units <= (lists >= 512 ? 256 : lists >= 128 ? 64 : 32) || blocks < 1)
    return Q8Plan{(int)lists, 0, 0};
  const long few = lists <= 256 && blocks > 256 ? 256 : blocks;
  const long share = q8_share((unsigned)all, (unsigned)blocks, (unsigned)few);
  return Q8Plan{(int)(listed ? (all + share - 1) / share : blocks), (int)blocks, (int)few};
}

int q8_attend(const locks_cfg_t* cfg, const void* q, const locks_q8_t* cache,
              const int32_t* page_table, const int32_t* seq_lens, const int32_t* page_ids,
              bool listed, float* out, float* out_lse, void* ws, size_t ws_bytes, void* stream) {
  int rc = validate(cfg, false);
  if (rc) return rc;
  if ((rc = q8_valid(cache))) return rc;
  if (!q || !aligned16(q) || !page_table || !seq_lens || !out || !aligned16(out) ||
      (listed && !page_ids))
    return LOCKS_E_INVAL;
  if ((rc = check_ws(cfg, ws, ws_bytes))) return rc;
  if (cfg->num_seqs == 0) return LOCKS_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const long units = (long)(listed ? page_budget(*cfg) : cfg->max_pages_per_seq) << sub_page_log2(*cfg);
  if ((units + 7) * cfg->num_seqs * cfg->num_kv_heads > 0x7fffffffL) return LOCKS_E_UNSUPPORTED;
  if ((rc = checked_tables(*cfg, ws, page_table, seq_lens, st))) return rc;
  return hip_status(launch_q8_attend(*cfg, q, *cache, page_table, seq_lens, page_ids,
                                     q8_plan(*cfg, units, listed), static_cast<float*>(ws), out, out_lse, st));
}

}  // namespace
}  // namespace locks

using namespace locks;

extern "C" {

int locks_rope_append_kv(const locks_cfg_t* cfg, const locks_rows_t* rows,
                         const locks_rope_t* rope, void* k_cache, void* v_cache,
                         const int32_t* page_table, const int32_t* seq_lens, void* stream) {
  RowArgs a;
  RopeArgs r;
  const int rc = append_args(cfg, rows, rope, page_table, seq_lens, &a, &r);
  if (rc) return rc;
  if (!k_cache || !v_cache || !aligned16(k_cache) || !aligned16(v_cache)) return LOCKS_E_INVAL;
  if (cfg->num_seqs == 0 || rows->n_tokens == 0) return LOCKS_OK;
  return hip_status(launch_rope_append(*cfg, a, r, k_cache, v_cache, page_table, seq_lens,
                                       static_cast<hipStream_t>(stream)));
}

int locks_q8_append_kv(const locks_cfg_t* cfg, const locks_rows_t* rows,
                       const locks_rope_t* rope, const locks_q8_t* cache,
                       const int32_t* page_table, const int32_t* seq_lens, void* stream) {
  RowArgs a;
  RopeArgs r;
  int rc = append_args(cfg, rows, rope, page_table, seq_lens, &a, &r);
  if (rc) return rc;
  if ((rc = q8_valid(cache))) return rc;
  if (cfg->num_seqs == 0 || rows->n_tokens == 0) return LOCKS_OK;
  return hip_status(launch_q8_append(*cfg, a, r, *cache, page_table, seq_lens,
                                     static_cast<hipStream_t>(stream)));
}

int locks_q8_build_summaries(const locks_cfg_t* cfg, const locks_q8_t* cache,
                             const int32_t* page_table, const int32_t* seq_lens,
                             const int32_t* build_list, int32_t n_build, void* summaries,
                             void* stream) {
  int rc = validate(cfg);
  if (rc) return rc;
  if ((rc = q8_valid(cache))) return rc;
  if (!page_table || !seq_lens || !summaries || n_build < 0 || (!build_list && n_build > 0))
    return LOCKS_E_INVAL;
  if (cfg->num_seqs == 0) return LOCKS_OK;
  const bool all = build_list == nullptr;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (cfg->page_size != kPage)
    return hip_status(launch_build_page(*cfg, cache->k, page_table, seq_lens, build_list, n_build, all,
                                        summaries, nullptr, nullptr, nullptr, nullptr, st,
                                        cache->k_scale, cache->code));
  return hip_status(launch_build(*cfg, cache->k, page_table, seq_lens, build_list, n_build, all, summaries,
                                 nullptr, nullptr, nullptr, nullptr, st, kBuildAll, nullptr,
                                 cache->k_scale, cache->code));
}

int locks_q8_dense_attend(const locks_cfg_t* cfg, const void* q, const locks_q8_t* cache,
                          const int32_t* page_table, const int32_t* seq_lens, float* out,
                          float* out_lse, void* ws, size_t ws_bytes, void* stream) {
  return q8_attend(cfg, q, cache, page_table, seq_lens, nullptr, false, out, out_lse, ws, ws_bytes,
                   stream);
}

int locks_q8_sparse_attend(const locks_cfg_t* cfg, const void* q, const locks_q8_t* cache,
                           const int32_t* page_table, const int32_t* seq_lens,
                           const int32_t* page_ids, float* out, float* out_lse, void* ws,
                           size_t ws_bytes, void* stream) {
  return q8_attend(cfg, q, cache, page_table, seq_lens, page_ids, true, out, out_lse, ws, ws_bytes,
                   stream);
}

}  // extern "C"
