// Internal declarations of the paged-cache calls (include/locks_cache.h).
#pragma once

#include "../../include/locks_cache.h"
#include "locks_internal.h"

namespace locks {

// Rotation as the kernels take it: pair i reads axis 0 below axis1, axis 1 below axis2,
// else axis 2.  half = 0: no rotation.
struct RopeArgs {
  const float* table;
  const int32_t* positions;
  int n_pos, half, interleaved, n_axes, axis1, axis2, n_tokens;
};
struct RowArgs {
  const void *q, *k, *v;
  void* q_out;
  const int32_t* cu;
  long q_stride, k_stride, v_stride, q_out_stride;
  int n_tokens;
};

hipError_t launch_rope_append(const locks_cfg_t& c, const RowArgs& a, const RopeArgs& r,
                              void* k_cache, void* v_cache, const int32_t* page_table,
                              const int32_t* seq_lens, hipStream_t st);
hipError_t launch_q8_append(const locks_cfg_t& c, const RowArgs& a, const RopeArgs& r,
                            const locks_q8_t& cache, const int32_t* page_table,
                            const int32_t* seq_lens, hipStream_t st);
// How an attention over an 8-bit cache is split over blocks: `blocks` equal shares of all
// lists' units, each of `share` units or (0) as many as the lengths come to; blocks = 0: one
// block a list.
struct Q8Plan {
  int blocks, share;
};
// page_ids == nullptr: every page.  partial: blocks + lists slots of [G][130] floats.
hipError_t launch_q8_attend(const locks_cfg_t& c, const void* q, const locks_q8_t& cache,
                            const int32_t* page_table, const int32_t* seq_lens,
                            const int32_t* page_ids, const Q8Plan& plan, float* partial, float* out,
                            float* out_lse, hipStream_t st);

}  // namespace locks
