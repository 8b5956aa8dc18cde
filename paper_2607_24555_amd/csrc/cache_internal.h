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
// How an attention over an 8-bit cache is split: the lists' units, in order, in equal shares
// for at most `blocks` blocks, of which `grid` are launched (fewer where the units are known);
// blocks = 0: one block a list.
struct Q8Plan {
  int grid, blocks, few;
};
// Units of a share, a multiple of 8 (a pair per wave): 8 for up to 320 blocks, then what `few`
// blocks need (few <= blocks), but from 64 units on no more than `blocks` need.
// ceil(units / share) <= blocks.
// 320 stands between two kinds of batch, with blocks of 8 units against the 256 of `few`: eight
// lists take 11.1 us against 12.7 at 264 blocks and 11.3 against 13.3 at 312, and still 11.4
// against 13.1 at 328, from 352 on the same; one long list 14.2 against 12.9 at 275, 14.7 against
// 13.6 at 313 and 15.0 against 13.6 at 338; 64 short ones 11.0 against 10.7 at 384.
__host__ __device__ inline unsigned q8_share(unsigned units, unsigned blocks, unsigned few) {
  if (units <= 8 * blocks && units <= 8 * 320) return 8;
  const unsigned least = (units + blocks - 1) / blocks, cap = least < 64 ? 64 : least;
  const unsigned share = (units + few - 1) / few;
  return ((share < cap ? share : cap) + 7) / 8 * 8;  // (>= 8: units > 0 here)
}
// page_ids == nullptr: every page.  partial: plan.blocks + lists slots of [G][130] floats.
hipError_t launch_q8_attend(const locks_cfg_t& c, const void* q, const locks_q8_t& cache,
                            const int32_t* page_table, const int32_t* seq_lens,
                            const int32_t* page_ids, const Q8Plan& plan, float* partial, float* out,
                            float* out_lse, hipStream_t st);

}  // namespace locks
