// The attention weight that every cached token gets from the new ones, added to what it had:
//   mass_t = decay mass_t + sum_{i sees t, g} exp(q_ig . k_t / sqrt d - lse_ig).
// One wave per (sequence, KV head, token), the rows one after the other.
#include "tokens_internal.h"

namespace locks {
namespace {

template <typename TQ, typename TK>
__global__ __launch_bounds__(256) void mass_simple_kernel(DraftArgs a, const float* __restrict__ lse,
                                                          const TK* __restrict__ k_cache, float decay,
                                                          float* __restrict__ mass) {
  const int h = blockIdx.y, s = blockIdx.z, lane = threadIdx.x & 63;
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int2 rows = draft_rows(a, s);
  const int n = rows.y - rows.x, L = draft_len(a, s), first = L - n;
  if (t >= L || n == 0) return;
  const int blk = a.page_table[(long)s * a.max_pages + t / a.pgsz];
  if ((unsigned)blk >= (unsigned)a.num_blocks) return;
  const TK* k = k_cache + (((long)blk * a.H + h) * a.pgsz + t % a.pgsz) * kDim + 2 * lane;
  const float k0 = load_elem(k, 0), k1 = load_elem(k, 1), scale = 1.0f / sqrtf((float)kDim);
  float sum = 0.0f;
  for (int i = 0; i < n; ++i) {
    if (!draft_sees(a, rows.x + i, i, t, first)) continue;
    for (int g = 0; g < a.G; ++g) {
      const float e = lse[(long)(rows.x + i) * a.H * a.G + h * a.G + g];
      const TQ* q = static_cast<const TQ*>(a.q) + (long)(rows.x + i) * a.q_stride + (h * a.G + g) * kDim + 2 * lane;
      const float z = warp_sum(fmaf(load_elem(q, 0), k0, load_elem(q, 1) * k1)) * scale;
      if (e != -INFINITY) sum += expf(z - e);
    }
  }
  const long at = ((long)s * a.H + h) * a.max_pages * a.pgsz + t;
  if (lane == 0) mass[at] = (t < first ? decay * mass[at] : 0.0f) + sum;
}

}  // namespace

hipError_t launch_token_mass(const locks_cfg_t& c, const DraftArgs& a, const float* lse,
                             const void* k_cache, float decay, float* mass, hipStream_t st) {
  const dim3 grid((unsigned)(((long)a.max_pages * a.pgsz + 3) / 4), a.H, a.S), block(256);
#define MASS(TQ, TK)                                                                            \
  hipLaunchKernelGGL((mass_simple_kernel<TQ, TK>), grid, block, 0, st, a, lse,                  \
                     static_cast<const TK*>(k_cache), decay, mass)
  if (c.q_dtype == LOCKS_BF16 && c.kv_dtype == LOCKS_BF16) MASS(uint16_t, uint16_t);
  else if (c.q_dtype == LOCKS_BF16) MASS(uint16_t, float);
  else if (c.kv_dtype == LOCKS_BF16) MASS(float, uint16_t);
  else MASS(float, float);
#undef MASS
  return hipGetLastError();
}

}  // namespace locks
