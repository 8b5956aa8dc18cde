// Attention of several new tokens of a sequence over the paged cache:
//   o_i = sum_{t seen by i} softmax_t(q_i . k_t / sqrt d) v_t.
// One wave per (new token, query head), a token after the other, two dimensions a lane, with
// the running maximum and sum of an online softmax in fp32.
#include "tokens_internal.h"

namespace locks {
namespace {

template <typename TQ, typename TK>
__global__ __launch_bounds__(256) void tree_simple_kernel(DraftArgs a, const TK* __restrict__ k_cache,
                                                          const TK* __restrict__ v_cache,
                                                          void* __restrict__ out, int out_bf16,
                                                          float* __restrict__ out_lse) {
  const int Hq = a.H * a.G, lane = threadIdx.x & 63;
  const long unit = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int row = (int)(unit / Hq), hq = (int)(unit % Hq), h = hq / a.G;
  if (row >= a.n_tokens) return;
  int s = 0;
  while (s < a.S && draft_rows(a, s).y <= row) ++s;
  if (s == a.S || draft_rows(a, s).x > row) return;  // padding
  const int2 rows = draft_rows(a, s);
  const int i = row - rows.x, L = draft_len(a, s), first = L - (rows.y - rows.x);
  const TQ* q = static_cast<const TQ*>(a.q) + (long)row * a.q_stride + hq * kDim + 2 * lane;
  const float q0 = load_elem(q, 0), q1 = load_elem(q, 1), scale = 1.0f / sqrtf((float)kDim);
  float m = -INFINITY, l = 0.0f, o0 = 0.0f, o1 = 0.0f;
  for (int t = 0; t < L; ++t) {
    if (!draft_sees(a, row, i, t, first)) continue;
    int blk = a.page_table[(long)s * a.max_pages + t / a.pgsz];
    if ((unsigned)blk >= (unsigned)a.num_blocks) blk = 0;
    const long at = (((long)blk * a.H + h) * a.pgsz + t % a.pgsz) * kDim + 2 * lane;
    const float z = warp_sum(fmaf(q0, load_elem(k_cache + at, 0), q1 * load_elem(k_cache + at, 1))) * scale;
    const float mx = fmaxf(m, z);
    const float sc = m == -INFINITY ? 0.0f : expf(m - mx), w = z == -INFINITY ? 0.0f : expf(z - mx);
    l = fmaf(l, sc, w);
    o0 = fmaf(o0, sc, w * load_elem(v_cache + at, 0));
    o1 = fmaf(o1, sc, w * load_elem(v_cache + at, 1));
    m = mx;
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  const long to = ((long)row * Hq + hq) * kDim + 2 * lane;
  if (out_bf16) {
    static_cast<__bf16*>(out)[to] = (__bf16)(o0 * inv);
    static_cast<__bf16*>(out)[to + 1] = (__bf16)(o1 * inv);
  } else {
    static_cast<float*>(out)[to] = o0 * inv;
    static_cast<float*>(out)[to + 1] = o1 * inv;
  }
  if (out_lse && lane == 0) out_lse[(long)row * Hq + hq] = l > 0.0f ? m + logf(l) : -INFINITY;
}

}  // namespace

size_t tree_scratch_bytes(const locks_cfg_t&, int) { return 0; }

hipError_t launch_tree_attend(const locks_cfg_t& c, const DraftArgs& a, const void* k_cache,
                              const void* v_cache, void* out, bool out_bf16, float* out_lse,
                              void*, hipStream_t st) {
  const dim3 grid((unsigned)(((long)a.n_tokens * c.num_q_heads + 3) / 4)), block(256);
#define TREE(TQ, TK)                                                                             \
  hipLaunchKernelGGL((tree_simple_kernel<TQ, TK>), grid, block, 0, st, a,                        \
                     static_cast<const TK*>(k_cache), static_cast<const TK*>(v_cache), out,      \
                     out_bf16 ? 1 : 0, out_lse)
  if (c.q_dtype == LOCKS_BF16 && c.kv_dtype == LOCKS_BF16) TREE(uint16_t, uint16_t);
  else if (c.q_dtype == LOCKS_BF16) TREE(uint16_t, float);
  else if (c.kv_dtype == LOCKS_BF16) TREE(float, uint16_t);
  else TREE(float, float);
#undef TREE
  return hipGetLastError();
}

}  // namespace locks
