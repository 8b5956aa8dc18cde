// New tokens of a step, rotated and appended to the paged caches (locks_rope_append_kv):
// query rows from q to q_out, key and value rows into their slots, in one launch.
//
// A wave moves rows of one token, four at a time with 16 lanes each.  A lane holds both
// elements of its pairs, its four angles are loaded once and serve every row of the wave, and
// the first rows are requested before the token's place is known.
// Prompts are bound by HBM: 15K bf16 tokens of 32 + 2 x 8 heads take 67.5 us, 5.7 TB/s of what
// they read and write (counted traffic is that to 1%; a large copy reaches 5.1); 6K fp32 tokens
// of 28 + 2 x 4 heads with three axes 42.9 us, 5.3 TB/s.  A few tokens are bound by the chain
// length -> table entry -> store: 1 token 2.8 us, 64 tokens 3.0, an empty launch 1.9.
#include "rope.h"

namespace locks {
namespace {

constexpr int kRows = 4;  // rows in flight per 16 lanes

// From this many written bytes on (more than the L2s hold), rows pass the caches' replacement.
// Alone, and with a copy of q_out behind it as its reader, cached against streamed:
// 1,024 bf16 tokens of 48 heads 8.2 / 11.9 us against 7.0 / 13.3; 4,096 (50 MB) 24.7 / 36.1
// against 20.2 / 34.9; 8,192 43.2 / 66.7 against 37.7 / 65.0; 16,384 of 10 heads (42 MB)
// 27.2 / 38.3 against 25.6 / 40.0.
constexpr long kStreamBytes = 48L << 20;

// Wave (token, part), a token's parts in a row (15K prompt tokens of 48 heads, cached stores:
// 71.2 us, with a part's tokens in a row 75.8): q_parts of `rows` query rows, then of `rows` key
// and value rows (keys first).
template <typename QT, typename KT, bool kStream>
__global__ __launch_bounds__(256) void rope_append_kernel(
    RowArgs a, RopeArgs rope, KT* __restrict__ k_cache, KT* __restrict__ v_cache,
    const int32_t* __restrict__ page_table, const int32_t* __restrict__ seq_lens, int S, int H_q,
    int H_kv, int max_pages, int num_blocks, int pgsz, unsigned parts, int q_parts,
    int rows) {
  const unsigned id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = (int)(id / parts), part = (int)(id % parts);
  if (row >= a.n_tokens) return;
  const int lane = threadIdx.x & 63;
  const bool is_q = part < q_parts;

  const int r0 = (is_q ? part : part - q_parts) * rows;
  const int r1 = min(r0 + rows, is_q ? H_q : 2 * H_kv);
  const Lane ln = lane_of(rope, lane & 15);
  const int tg = lane >> 4;
  const QT* q = static_cast<const QT*>(a.q) + row * a.q_stride;
  const KT* k = static_cast<const KT*>(a.k) + row * a.k_stride;
  const KT* v = static_cast<const KT*>(a.v) + row * a.v_stride;
  auto q_src = [&](int r) { return q + r * kDim; };
  auto kv_src = [&](int r) { return r < H_kv ? k + r * kDim : v + (r - H_kv) * kDim; };
  Mover<QT, kRows, kStream> mq;
  Mover<KT, kRows, kStream> mk;
  if (is_q) mq.begin(ln, r0 + tg, r1, q_src);
  else mk.begin(ln, r0 + tg, r1, kv_src);

  const NewTokens t = tokens_of_row(a, seq_lens, S, row);
  if (t.s < 0) return;
  const int tok = t.tok0 + (row - t.row0);
  if (row - t.row0 >= t.n || tok < 0 || tok / pgsz >= max_pages) return;
  const long blk = page_table[(long)t.s * max_pages + tok / pgsz];
  Positions pos;
  if (!positions_of(rope, row, tok, pos)) return;
  Angles A;
  load_angles(rope, ln, pos, A);
  if (blk < 0 || blk >= num_blocks) return;
  if (is_q) {
    QT* out = static_cast<QT*>(a.q_out) + row * a.q_out_stride;
    mq.move(rope, ln, A, tg, r0, r1, H_q, q_src, [&](int r) { return out + r * kDim; });
  } else {
    const long at = (blk * H_kv * pgsz + tok % pgsz) * kDim, head = (long)pgsz * kDim;
    mk.move(rope, ln, A, tg, r0, r1, H_kv, kv_src, [&](int r) {
      return r < H_kv ? k_cache + at + r * head : v_cache + at + (r - H_kv) * head;
    });
  }
}

template <typename QT, typename KT>
hipError_t launch_typed(const locks_cfg_t& c, const RowArgs& a, const RopeArgs& r, void* k_cache,
                        void* v_cache, const int32_t* page_table, const int32_t* seq_lens,
                        hipStream_t st) {
  // rows per wave: as many as 4 kRows while 4,096 waves remain
  const int hq = a.q ? c.num_q_heads : 0, hkv = 2 * c.num_kv_heads;
  int per = 4 * kRows;
  while (per > 4 && (long)a.n_tokens * ((hq + per - 1) / per + (hkv + per - 1) / per) < 4096) per /= 2;
  const int q_parts = (hq + per - 1) / per, kv_parts = (hkv + per - 1) / per;
  const long waves = (long)a.n_tokens * (q_parts + kv_parts);
  if (waves + 3 > 0x7fffffffL) return hipErrorInvalidConfiguration;
  const long bytes = (long)a.n_tokens * kDim * (hq * (long)sizeof(QT) + hkv * (long)sizeof(KT));
  auto* kernel = bytes >= kStreamBytes ? rope_append_kernel<QT, KT, true> : rope_append_kernel<QT, KT, false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, st, a, r,
                     static_cast<KT*>(k_cache), static_cast<KT*>(v_cache), page_table, seq_lens,
                     c.num_seqs, hq, c.num_kv_heads, c.max_pages_per_seq, c.num_blocks, c.page_size,
                     (unsigned)(q_parts + kv_parts), q_parts, per);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_append(const locks_cfg_t& c, const RowArgs& a, const RopeArgs& r,
                              void* k_cache, void* v_cache, const int32_t* page_table,
                              const int32_t* seq_lens, hipStream_t st) {
  const bool qb = !a.q || c.q_dtype == LOCKS_BF16, kb = c.kv_dtype == LOCKS_BF16;
  if (qb && kb)
    return launch_typed<uint16_t, uint16_t>(c, a, r, k_cache, v_cache, page_table, seq_lens, st);
  if (qb) return launch_typed<uint16_t, float>(c, a, r, k_cache, v_cache, page_table, seq_lens, st);
  if (kb) return launch_typed<float, uint16_t>(c, a, r, k_cache, v_cache, page_table, seq_lens, st);
  return launch_typed<float, float>(c, a, r, k_cache, v_cache, page_table, seq_lens, st);
}

}  // namespace locks
