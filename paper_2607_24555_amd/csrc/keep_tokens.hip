// Kept tokens moved together at the front of their sequence, in place: row a + i becomes row
// src_i, for keys, values and masses.
//
// As src_i >= a + i, row a + i may only be written once every entry up to i has been read; no
// entry after i reads it.  A block owns a list's column of 16 bytes times kLanes and goes
// through the list in order, a round of rows read by all its threads before any is written.
#include "tokens_internal.h"

namespace locks {
namespace {

constexpr int kKeepBlock = 256;

// A token's row in the cache, or -1 where its page is not a page.
__device__ __forceinline__ long row_of(const int32_t* table, int t, int pgsz, int max_pages,
                                       int num_blocks, int H, int h) {
  const int page = t / pgsz;
  if (t < 0 || page >= max_pages) return -1;
  const int blk = table[page];
  if ((unsigned)blk >= (unsigned)num_blocks) return -1;
  return ((long)blk * H + h) * pgsz + t % pgsz;
}

// grid (list, K or V, eight 16-byte lanes of a row)
__global__ __launch_bounds__(kKeepBlock) void keep_kernel(
    const int32_t* __restrict__ kept, int heads, int n_keep, const int32_t* __restrict__ start,
    uint4* __restrict__ k_cache, uint4* __restrict__ v_cache, float* __restrict__ mass,
    const int32_t* __restrict__ page_table, int32_t* __restrict__ out_lens, int H, int row_lanes, int pgsz,
    int max_pages, int num_blocks) {
  __shared__ int s_end;
  const int s = blockIdx.x / H, h = blockIdx.x % H, tid = threadIdx.x;
  const int32_t* ids = kept + ((long)s * heads + (heads > 1 ? h : 0)) * n_keep;
  const int32_t* table = page_table + (long)s * max_pages;
  uint4* cache = blockIdx.y ? v_cache : k_cache;
  const int lane = blockIdx.z * 8 + (tid & 7), a = start ? start[s] : 0;
  const bool with_mass = mass && blockIdx.z == 0 && blockIdx.y == 0 && (tid & 7) == 0;
  float* m = mass + ((long)s * H + h) * max_pages * pgsz;
  if (tid == 0) s_end = n_keep;
  __syncthreads();
  int i0 = 0;
  for (; i0 < n_keep; i0 += kKeepBlock / 8) {
    const int i = i0 + tid / 8;
    const int src = i < n_keep ? ids[i] : 0;
    if (src < 0 && i < n_keep) atomicMin(&s_end, i);
    __syncthreads();
    const int end = s_end;
    uint4 x = {};
    float y = 0.0f;
    long from = -1, to = -1;
    if (i < end && src >= (long)a + i) {
      from = row_of(table, src, pgsz, max_pages, num_blocks, H, h);
      to = row_of(table, a + i, pgsz, max_pages, num_blocks, H, h);
    }
    const bool move = from >= 0 && to >= 0 && from != to;
    if (move) {
      x = cache[from * row_lanes + lane];
      if (with_mass) y = m[src];
    }
    __syncthreads();
    if (move) {
      cache[to * row_lanes + lane] = x;
      if (with_mass) m[a + i] = y;
    }
    if (end < i0 + kKeepBlock / 8) break;
  }
  if (out_lens && blockIdx.z == 0 && blockIdx.y == 0 && h == 0 && tid == 0) out_lens[s] = a + s_end;
}

}  // namespace

hipError_t launch_keep_tokens(const locks_cfg_t& c, const int32_t* kept, int heads, int n_keep,
                              const int32_t* start, void* k_cache, void* v_cache, float* mass,
                              const int32_t* page_table, int32_t* out_lens, hipStream_t st) {
  const int row_lanes = kDim * (c.kv_dtype == LOCKS_BF16 ? 2 : 4) / 16;
  hipLaunchKernelGGL(keep_kernel, dim3((unsigned)(c.num_seqs * c.num_kv_heads), 2, row_lanes / 8),
                     dim3(kKeepBlock), 0, st, kept, heads, n_keep, start, static_cast<uint4*>(k_cache),
                     static_cast<uint4*>(v_cache), mass, page_table, out_lens, c.num_kv_heads, row_lanes,
                     c.page_size, c.max_pages_per_seq, c.num_blocks);
  return hipGetLastError();
}

}  // namespace locks
