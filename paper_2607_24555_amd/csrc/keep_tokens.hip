// Kept tokens moved together at the front of their sequence, in place: row a + i becomes row
// src_i, for keys, values and masses.
//
// As src_i >= a + i, row a + i may only be written once every entry up to i has been read, and
// no entry after i reads it.  So a block takes a slice of 16 kLanes bytes of a list's rows and
// goes through the list in rounds: the round's rows are in registers (all waves', by the
// barrier) before any is written, and the next round's are requested before that.  Slices are
// independent; there are as many as fill the chip, down to 32 bytes (4 sequences x 8 heads,
// 4,096 rows of 256 bytes each, K and V).
#include "tokens_internal.h"

namespace locks {
namespace {

constexpr int kKeepRows = 4;  // rows of a thread in a round

struct KeepArgs {
  const int32_t* kept;
  const int32_t* start;
  const int32_t* table;
  void *k, *v;
  float* mass;
  int32_t* out_lens;
  int heads, n_keep, H, pgsz, max_pages, num_blocks, row_lanes;
};

// A token's row in the cache, or -1 where its page is not a page.
__device__ __forceinline__ long row_of(const KeepArgs& a, const int32_t* table, int t, int h) {
  if (t < 0 || t / a.pgsz >= a.max_pages) return -1;
  const int blk = table[t / a.pgsz];
  if ((unsigned)blk >= (unsigned)a.num_blocks) return -1;
  return ((long)blk * a.H + h) * a.pgsz + t % a.pgsz;
}

// One list's slice (T: 16 bytes, or a mass); kLanes threads a row, `lane` this thread's part.
template <typename T, int kLanes, int kBlock>
__device__ __forceinline__ void move_rows(const KeepArgs& a, T* data, bool cache, int s, int h, long a0,
                                          int row_lanes, int lane, int& s_end) {
  constexpr int kStep = kBlock / kLanes, kRound = kStep * kKeepRows;
  const int32_t* ids = a.kept + ((long)s * a.heads + (a.heads > 1 ? h : 0)) * a.n_keep;
  const int32_t* table = a.table + (long)s * a.max_pages;
  const int me = threadIdx.x / kLanes;
  struct Place {
    long from[kKeepRows], to[kKeepRows];
  };
  // where a round's rows come from and go to; -1: nothing moves
  auto places = [&](int i0, Place& p) {
    int src[kKeepRows];
#pragma unroll
    for (int e = 0; e < kKeepRows; ++e) {
      const int i = i0 + e * kStep + me;
      src[e] = i < a.n_keep ? ids[i] : 0;
      if (src[e] < 0 && i < a.n_keep) atomicMin(&s_end, i);
    }
#pragma unroll
    for (int e = 0; e < kKeepRows; ++e) {
      const long i = i0 + e * kStep + me, dst = a0 + i;
      p.from[e] = p.to[e] = -1;
      if (i < a.n_keep && src[e] > dst && dst >= 0) {
        const long f = row_of(a, table, src[e], h), t = row_of(a, table, (int)dst, h);
        if (f >= 0 && t >= 0) {
          p.from[e] = cache ? f : src[e];
          p.to[e] = cache ? t : dst;
        }
      }
    }
  };
  Place p;
  T x[kKeepRows];
  auto read = [&](int i0, int end) {
#pragma unroll
    for (int e = 0; e < kKeepRows; ++e) {
      if (i0 + e * kStep + me >= end) p.to[e] = -1;
      if (p.to[e] >= 0) x[e] = data[p.from[e] * row_lanes + lane];
    }
  };
  places(0, p);
  __syncthreads();
  int end = s_end;  // (the list's end, or one behind this round)
  read(0, end);
  for (int i0 = 0; i0 < min(a.n_keep, end); i0 += kRound) {
    Place next;
    places(i0 + kRound, next);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this round's rows are here
    __syncthreads();
    end = s_end;
    long to[kKeepRows];
    T y[kKeepRows];
#pragma unroll
    for (int e = 0; e < kKeepRows; ++e) to[e] = p.to[e], y[e] = x[e];
    p = next;
    read(i0 + kRound, end);
#pragma unroll
    for (int e = 0; e < kKeepRows; ++e)
      if (to[e] >= 0) data[to[e] * row_lanes + lane] = y[e];
  }
}

// grid (list, K / V / mass, slice)
template <int kLanes, int kBlock>
__global__ __launch_bounds__(kBlock) void keep_kernel(KeepArgs a) {
  __shared__ int s_end;
  const int s = blockIdx.x / a.H, h = blockIdx.x % a.H, tid = threadIdx.x;
  const long a0 = a.start ? a.start[s] : 0;
  if (tid == 0) s_end = a.n_keep;
  __syncthreads();
  if (blockIdx.y == 2) {
    if (blockIdx.z == 0 && a.mass)
      move_rows<float, 1, kBlock>(a, a.mass + ((long)s * a.H + h) * a.max_pages * a.pgsz, false, s, h, a0, 1, 0, s_end);
    return;
  }
  typedef uint32_t u4 __attribute__((ext_vector_type(4)));
  move_rows<u4, kLanes, kBlock>(a, static_cast<u4*>(blockIdx.y ? a.v : a.k), true, s, h, a0, a.row_lanes,
                        blockIdx.z * kLanes + tid % kLanes, s_end);
  if (a.out_lens && blockIdx.z == 0 && blockIdx.y == 0 && h == 0) {
    __syncthreads();
    if (tid == 0) a.out_lens[s] = (int)a0 + s_end;
  }
}

}  // namespace

hipError_t launch_keep_tokens(const locks_cfg_t& c, const int32_t* kept, int heads, int n_keep,
                              const int32_t* start, void* k_cache, void* v_cache, float* mass,
                              const int32_t* page_table, int32_t* out_lens, hipStream_t st) {
  const int row_lanes = kDim * (c.kv_dtype == LOCKS_BF16 ? 2 : 4) / 16;
  const KeepArgs a{kept,   start,  page_table, k_cache,     v_cache,             mass,         out_lens, heads,
                   n_keep, c.num_kv_heads, c.page_size, c.max_pages_per_seq, c.num_blocks, row_lanes};
  const long lists = (long)c.num_seqs * c.num_kv_heads;
  int lanes = 16;  // of a slice
  while (lanes > 2 && lists * 2 * (row_lanes / lanes) < 256) lanes /= 2;
  // (short lists: a block of 256 threads reads them in one round)
  const bool few = (long)n_keep * lanes <= 256 * kKeepRows;
  const dim3 grid((unsigned)lists, mass ? 3 : 2, row_lanes / lanes), block(few ? 256 : 1024);
#define KEEP(N)                                                        \
  if (few) hipLaunchKernelGGL((keep_kernel<N, 256>), grid, block, 0, st, a); \
  else hipLaunchKernelGGL((keep_kernel<N, 1024>), grid, block, 0, st, a)
  if (lanes == 16) { KEEP(16); }
  else if (lanes == 8) { KEEP(8); }
  else if (lanes == 4) { KEEP(4); }
  else { KEEP(2); }
#undef KEEP
  return hipGetLastError();
}

}  // namespace locks
