// Kept tokens moved together at the front of their sequence, in place: row a + i becomes row
// src_i, for keys, values and masses.
//
// As src_i >= a + i, row a + i may only be written once every entry up to i has been read, and
// no entry after i reads it.  So a block takes a slice of 16 kLanes bytes of a list's rows and
// goes through the list in rounds: a round's rows are in registers (all waves', by the barrier)
// before any is written.  Of the rounds behind it one has its rows on their way, one its page
// table entries and one its list entries, so that a round waits for one memory latency (4,096
// rows: 36 us; with the list and the table of the next round read in turn 44).  Slices are
// independent; there are as many as fill the chip, down to 32 bytes (4 sequences of 8 heads: 64
// bytes 36 us, 128 bytes 39, 32 bytes 44).
#include "tokens_internal.h"

namespace locks {
namespace {

struct KeepArgs {
  const int32_t* kept;
  const int32_t* start;
  const int32_t* table;
  void *k, *v;
  float* mass;
  int32_t* out_lens;
  int heads, n_keep, H, pgsz, max_pages, num_blocks, row_lanes;
};

// One list's slice (T: 16 bytes, or a mass); kLanes threads a row, `lane` this thread's part.
template <typename T, int kLanes, int kBlock, int kRows>
__device__ __forceinline__ void move_rows(const KeepArgs& a, T* data, bool cache, int s, int h, long a0,
                                          int row_lanes, int lane, int& s_end) {
  constexpr int kStep = kBlock / kLanes, kRound = kStep * kRows;
  const int32_t* ids = a.kept + ((long)s * a.heads + (a.heads > 1 ? h : 0)) * a.n_keep;
  const int32_t* table = a.table + (long)s * a.max_pages;
  const int me = threadIdx.x / kLanes;
  const int lgP = a.pgsz == 64 ? 6 : a.pgsz == 32 ? 5 : 4;
  struct Round {
    int src[kRows];                  // list entries
    int from[kRows], to[kRows];  // blocks of the row's old and new page; -1: nothing moves
  };
  // (rounds are counted in 64 bits: those requested ahead may begin past 2^31)
  auto entries = [&](long i0, Round& r) {
#pragma unroll
    for (int e = 0; e < kRows; ++e) {
      const long i = i0 + e * kStep + me;
      r.src[e] = i < a.n_keep ? ids[i] : 0;
    }
  };
  // (once the entries are here) the list's end, and the pages
  auto ends = [&](long i0, const Round& r) {
#pragma unroll
    for (int e = 0; e < kRows; ++e) {
      const long i = i0 + e * kStep + me;
      if (r.src[e] < 0 && i < a.n_keep) atomicMin(&s_end, (int)i);
    }
  };
  auto pages = [&](long i0, Round& r) {
#pragma unroll
    for (int e = 0; e < kRows; ++e) {
      const long i = i0 + e * kStep + me, dst = a0 + i;
      r.from[e] = r.to[e] = -1;
      if (i < a.n_keep && r.src[e] > dst && dst >= 0 && r.src[e] >> lgP < a.max_pages) {
        r.from[e] = table[r.src[e] >> lgP];
        r.to[e] = table[dst >> lgP];
      }
    }
  };
  // (once those are here) the rows, and where they go
  auto read = [&](long i0, const Round& r, int end, T (&x)[kRows], long (&to)[kRows]) {
#pragma unroll
    for (int e = 0; e < kRows; ++e) {
      const long i = i0 + e * kStep + me, dst = a0 + i;
      to[e] = -1;
      if (i < end && (unsigned)r.from[e] < (unsigned)a.num_blocks && (unsigned)r.to[e] < (unsigned)a.num_blocks) {
        auto at = [&](int blk, long t) {
          return cache ? (((long)blk * a.H + h) * a.pgsz + (t & (a.pgsz - 1))) * row_lanes + lane : t;
        };
        x[e] = data[at(r.from[e], r.src[e])];
        to[e] = at(r.to[e], dst);
      }
    }
  };
  auto arrived = [] { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };
  Round r1, r2, r3;  // of the round at hand, the next, the one after
  T x[kRows];
  long to[kRows];
  entries(0, r1);
  entries(kRound, r2);
  ends(0, r1);
  ends(kRound, r2);
  pages(0, r1);
  pages(kRound, r2);
  entries(2 * kRound, r3);
  __syncthreads();
  int end = s_end;
  read(0, r1, end, x, to);
  for (long i0 = 0; i0 < min(a.n_keep, end); i0 += kRound) {
    arrived();
    ends(i0 + 2 * kRound, r3);
    __syncthreads();  // this round's rows are in registers, the list is known up to r3
    end = s_end;
    T y[kRows];
    long at[kRows];
#pragma unroll
    for (int e = 0; e < kRows; ++e) y[e] = x[e], at[e] = to[e];
    read(i0 + kRound, r2, end, x, to);
    r2 = r3;
    pages(i0 + 2 * kRound, r2);
    entries(i0 + 3 * kRound, r3);
#pragma unroll
    for (int e = 0; e < kRows; ++e)
      if (at[e] >= 0) data[at[e]] = y[e];
  }
}

// grid (list, K / V / mass, slice)
template <int kLanes, int kBlock, int kRows>
__global__ __launch_bounds__(kBlock) void keep_kernel(KeepArgs a) {
  __shared__ int s_end;
  const int s = blockIdx.x / a.H, h = blockIdx.x % a.H, tid = threadIdx.x;
  const long a0 = a.start ? a.start[s] : 0;
  if (tid == 0) s_end = a.n_keep;
  __syncthreads();
  if (blockIdx.y == 2) {
    if (blockIdx.z == 0 && a.mass)
      move_rows<float, 1, kBlock, kRows>(a, a.mass + ((long)s * a.H + h) * a.max_pages * a.pgsz, false, s, h, a0, 1, 0, s_end);
    return;
  }
  typedef uint32_t u4 __attribute__((ext_vector_type(4)));
  move_rows<u4, kLanes, kBlock, kRows>(a, static_cast<u4*>(blockIdx.y ? a.v : a.k), true, s, h, a0, a.row_lanes,
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
  // short lists: 256 threads, a row each (64 lists of up to 8: 6.2 us, with four rows 7.9)
  const bool few = (long)n_keep * lanes <= 512;
  const dim3 grid((unsigned)lists, mass ? 3 : 2, row_lanes / lanes), block(few ? 256 : 1024);
#define KEEP(N)                                                        \
  if (few) hipLaunchKernelGGL((keep_kernel<N, 256, 1>), grid, block, 0, st, a); \
  else hipLaunchKernelGGL((keep_kernel<N, 1024, 4>), grid, block, 0, st, a)
  if (lanes == 16) { KEEP(16); }
  else if (lanes == 8) { KEEP(8); }
  else if (lanes == 4) { KEEP(4); }
  else { KEEP(2); }
#undef KEEP
  return hipGetLastError();
}

}  // namespace locks
