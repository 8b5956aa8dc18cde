// The tokens of a list (sequence, KV head) to keep: the first n_sink, the last n_recent and
// the others of largest mass, in order.
//
// With the masses as unsigned keys of the same order, the key of the last token kept is found
// digit by digit (radix select, 8 bits a pass, histograms in LDS), then the tokens above it and
// the first ones equal to it are written at their ranks.  One block per list.
#include "tokens_internal.h"

namespace locks {
namespace {

constexpr int kPickBlock = 1024;

// Unsigned key of a mass: order as the values', -0 as 0, NaN below everything.
__device__ __forceinline__ uint32_t mass_key(float x) {
  if (x != x) return 0;
  return f32_order_key(x + 0.0f);
}

// Exclusive prefix sum of a value per thread over the block; total in `sum`.
__device__ __forceinline__ int block_scan(int v, int* lds, int& sum) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  int before = 0;
  sum = 0;
  for (int w = 0; w < kPickBlock / 64; ++w) {
    if (w < wave) before += lds[w];
    sum += lds[w];
  }
  return before + x - v;
}

__global__ __launch_bounds__(kPickBlock) void pick_kernel(const float* __restrict__ mass,
                                                          const int32_t* __restrict__ seq_lens, int H,
                                                          int width, int n_keep, int n_sink,
                                                          int n_recent, int32_t* __restrict__ out_ids) {
  __shared__ int hist[256], waves[kPickBlock / 64], s_bin, s_left;
  const long list = blockIdx.x;
  const int L = min(max(seq_lens[list / H], 0), width), tid = threadIdx.x;
  const float* x = mass + list * width;
  int32_t* out = out_ids + list * n_keep;
  if (L <= n_keep) {
    for (int i = tid; i < n_keep; i += kPickBlock) out[i] = i < L ? i : -1;
    return;
  }
  const int lo = n_sink, hi = L - n_recent;  // the candidates (lo < hi as L > n_keep)
  int left = n_keep - n_sink - n_recent;     // of which so many are kept
  uint32_t prefix = 0;
  if (left > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int b = tid; b < 256; b += kPickBlock) hist[b] = 0;
      __syncthreads();
      for (int i = lo + tid; i < hi; i += kPickBlock) {
        const uint32_t k = mass_key(x[i]);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[k >> shift & 255], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int b = 255, above = 0;
        while (above + hist[b] < left) above += hist[b--];
        s_bin = b;
        s_left = left - above;
      }
      __syncthreads();
      prefix |= (uint32_t)s_bin << shift;
      left = s_left;
      __syncthreads();
    }
  }
  // ranks: a token is kept if forced, above the key, or among the first `left` equal to it
  const bool none = n_keep == n_sink + n_recent;
  int base = 0, ties = 0;
  for (int i0 = 0; i0 < L; i0 += kPickBlock) {
    const int i = i0 + tid;
    const bool forced = i < L && (i < lo || i >= hi);
    const uint32_t k = i < L ? mass_key(x[i]) : 0;
    const bool open = i < L && !forced && !none;
    const int tie = open && k == prefix;
    int n_tie, n_new;
    const int before = ties + block_scan(tie, waves, n_tie);
    const int take = forced || (open && k > prefix) || (tie && before < left);
    const int at = base + block_scan(take, waves, n_new);
    if (take) out[at] = i;
    base += n_new;
    ties += n_tie;
  }
}

}  // namespace

size_t pick_scratch_bytes(const locks_cfg_t&) { return 256; }

hipError_t launch_pick_tokens(const locks_cfg_t& c, const float* mass, const int32_t* seq_lens,
                              int n_keep, int n_sink, int n_recent, int32_t* out_ids, void*,
                              hipStream_t st) {
  hipLaunchKernelGGL(pick_kernel, dim3((unsigned)(c.num_seqs * c.num_kv_heads)), dim3(kPickBlock), 0, st, mass,
                     seq_lens, c.num_kv_heads, c.max_pages_per_seq * c.page_size, n_keep, n_sink, n_recent,
                     out_ids);
  return hipGetLastError();
}

}  // namespace locks
