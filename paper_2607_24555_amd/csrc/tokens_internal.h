// Internal declarations of the calls on single tokens (include/locks_tokens.h).
#pragma once

#include "../../include/locks_tokens.h"
#include "locks_internal.h"

namespace locks {

// The new tokens and the cache as the kernels take them.
struct DraftArgs {
  const void* q;
  const int32_t* cu;
  const uint32_t* mask;
  const int32_t* page_table;
  const int32_t* seq_lens;
  long q_stride;
  int n_tokens, words;
  int S, H, G, pgsz, max_pages, num_blocks;
};

// A sequence's rows of the new tokens, held to [0, n_tokens].
__device__ __forceinline__ int2 draft_rows(const DraftArgs& a, int s) {
  if (!a.cu) return make_int2(s, s + 1);
  const int b = min(max(a.cu[s], 0), a.n_tokens), e = min(max(a.cu[s + 1], 0), a.n_tokens);
  return make_int2(b, max(b, e));
}
// (the loads together, so that one wait covers them)
struct DraftSeq {
  int row0, n, L;
};
__device__ __forceinline__ DraftSeq draft_seq(const DraftArgs& a, int s) {
  int b = s, e = s + 1;
  const int len = a.seq_lens[s];
  if (a.cu) b = a.cu[s], e = a.cu[s + 1];
  b = min(max(b, 0), a.n_tokens), e = min(max(e, 0), a.n_tokens);
  return DraftSeq{b, max(e - b, 0), min(max(len, 0), a.max_pages * a.pgsz)};
}
__device__ __forceinline__ int draft_len(const DraftArgs& a, int s) {
  return min(max(a.seq_lens[s], 0), a.max_pages * a.pgsz);
}
// Which of the 32 tokens from new token j0 on (j0 > -32) new token i (mask row `row`) sees, `left`
// of them up to the sequence's end.
__device__ __forceinline__ uint32_t draft_window(const DraftArgs& a, int row, int i, int j0, int left) {
  if (left <= 0) return 0u;
  uint32_t seen = j0 < 0 ? (1u << -j0) - 1u : 0u;
  if (a.mask) {
    const uint32_t* mask = a.mask + (long)row * a.words;
    const int w = j0 >> 5, sh = j0 & 31;
    const uint32_t lo = (unsigned)w < (unsigned)a.words ? mask[w] : 0u;
    const uint32_t hi = (unsigned)(w + 1) < (unsigned)a.words ? mask[w + 1] : 0u;
    seen |= sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
  } else if (i >= j0) {
    seen |= i - j0 >= 31 ? ~0u : (2u << (i - j0)) - 1u;
  }
  return left >= 32 ? seen : seen & ((1u << left) - 1u);
}

// Exclusive prefix sum of one value a thread over a block of kWaves waves; total in `sum`.
template <int kWaves, typename T>
__device__ __forceinline__ T scan_block(T v, T* lds, T& sum) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T x = v;
  for (int o = 1; o < 64; o <<= 1) {
    const T y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  T before = 0;
  sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += lds[w];
    sum += lds[w];
  }
  return before + x - v;
}

// Position of a 16-byte piece within a token's row in LDS: an exclusive or with this.  Any 8
// tokens in a row differ in the lower three bits (row reads), any 4 in bits 1 and 2 (transposed
// reads of two pieces each).
__device__ __forceinline__ int piece_xor(int tok) { return ((tok & 3) << 1) | ((tok >> 2) & 1) | (tok & 8); }

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

size_t tree_scratch_bytes(const locks_cfg_t& c, int n_tokens);
size_t tree_scratch_most(const locks_cfg_t& c, int n_tokens);
hipError_t launch_tree_attend(const locks_cfg_t& c, const DraftArgs& a, const void* k_cache,
                              const void* v_cache, void* out, bool out_bf16, float* out_lse,
                              void* scratch, hipStream_t st);
hipError_t launch_token_mass(const locks_cfg_t& c, const DraftArgs& a, const float* lse,
                             const void* k_cache, float decay, float* mass, hipStream_t st);
size_t pick_scratch_bytes(const locks_cfg_t& c);
size_t pick_scratch_most(const locks_cfg_t& c);
hipError_t launch_pick_tokens(const locks_cfg_t& c, const float* mass, const int32_t* seq_lens,
                              int n_keep, int n_sink, int n_recent, int32_t* out_ids, void* scratch,
                              hipStream_t st);
hipError_t launch_keep_tokens(const locks_cfg_t& c, const int32_t* kept, int heads, int n_keep,
                              const int32_t* start, void* k_cache, void* v_cache, float* mass,
                              const int32_t* page_table, int32_t* out_lens, hipStream_t st);

}  // namespace locks
