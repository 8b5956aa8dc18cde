// New tokens of a step, rotated, quantised and appended to the 8-bit cache
// (locks_q8_append_kv), the rotated queries copied beside them in the same launch.
//
// A unit of the grid is a page that receives tokens, keys or values, and a few KV heads;
// 16 tokens of it a wave (one, two or four waves), 16 lanes a token, eight elements a lane.
// The wave keeps its tokens' angles in registers for all its heads and holds a head's new rows
// as rotated fp32 values, so that a page's largest magnitude, its scale and its codes come
// from one read; the next head's rows are in flight meanwhile.  Only where the scale of a page
// with earlier rows grows are those rows read and rounded again.
// Prompts are bound by HBM: 15K bf16 tokens of 32 + 2 x 8 heads take 72.2 us, 4.9 TB/s (VALU
// busy 0.32, three waves a SIMD); as many of 32 + 2 x 2 heads in 64-token pages 57.8 us, 4.6
// TB/s.  The queries' rows stay cached: streamed past the caches, 8K tokens of 32 heads took
// 42.1 us instead of 45.4, but with a reader behind them 69.9 instead of 67.2.  64 single tokens
// are bound by latency: 4.5 us where the pages' scales hold, of which an empty launch is 1.9 and
// the rest the chain length -> table -> the page's scale -> codes written.  Where scales grow, the
// earlier codes are one more round trip: as kernels on their own, after a copy that sets the cache
// back, 6.8 us where a third of the pages grow and 7.1 where all do against 5.2 to 6.0 where none
// does.
#include <type_traits>

#include "rope.h"

namespace locks {
namespace {

constexpr float kTiny = 7.888609052210118e-31f;  // 2^-100: smaller pages are stored as zeros

// The scale of a page whose largest magnitude is amax.
template <int kCode>
__device__ __forceinline__ float page_scale(float amax) {
  if (!(amax >= kTiny)) return 0.0f;
  if constexpr (kCode == LOCKS_Q8_INT8) {
    return amax / 127.0f;
  } else {
    // 2^e with amax <= 448 2^e = 1.75 2^(e + 8): from amax's exponent, one more where its
    // mantissa passes 1.75
    const uint32_t u = __float_as_uint(amax);
    return __uint_as_float(((u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0)) << 23);
  }
}

// Codes of eight scaled elements, none of them NaN.
template <int kCode>
__device__ __forceinline__ uint2 codes_of(const float (&x)[8]) {
  constexpr float kMost = kCode == LOCKS_Q8_INT8 ? 127.0f : 448.0f;
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = __builtin_amdgcn_fmed3f(x[e], -kMost, kMost);
  if constexpr (kCode == LOCKS_Q8_INT8) {
    // 1.5 2^23 + y rounds y to an integer, ties to even, in the low bits
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = __float_as_uint(y[e] + 12582912.0f);
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_perm(b[2 * e + 1], b[2 * e], 0x0c0c0400u);
    return make_uint2(__builtin_amdgcn_perm(w[1], w[0], 0x05040100u), __builtin_amdgcn_perm(w[3], w[2], 0x05040100u));
  } else {
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
    int hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
    return make_uint2((uint32_t)lo, (uint32_t)hi);
  }
}

// The same where there may be NaN among them: 0 (int8) or e4m3's NaN.  (Infinities saturate.)
template <int kCode>
__device__ __forceinline__ uint2 codes_of_any(const float (&x)[8]) {
  float y[8];
  uint32_t keep[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y[e] = x[e] == x[e] ? x[e] : 0.0f;
    keep[e >> 2] |= x[e] == x[e] ? 0xffu << (8 * (e & 3)) : 0u;
  }
  const uint2 c = codes_of<kCode>(y);
  const uint32_t nan = kCode == LOCKS_Q8_INT8 ? 0u : 0x7f7f7f7fu;
  return make_uint2((c.x & keep[0]) | (nan & ~keep[0]), (c.y & keep[1]) | (nan & ~keep[1]));
}

// Max over the wave.
__device__ __forceinline__ float wave_max(float v) {
  auto dpp = [](float x, auto ctl) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), decltype(ctl)::value, 0xf, 0xf, true));
  };
  v = fmaxf(v, dpp(v, std::integral_constant<int, 0xB1>{}));   // quad xor 1, xor 2
  v = fmaxf(v, dpp(v, std::integral_constant<int, 0x4E>{}));
  v = fmaxf(v, dpp(v, std::integral_constant<int, 0x141>{}));  // half-row and row mirrors
  v = fmaxf(v, dpp(v, std::integral_constant<int, 0x140>{}));
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

template <int kCode>
__device__ __forceinline__ void values_of(uint2 w, float (&x)[8]) {
  if constexpr (kCode == LOCKS_Q8_INT8) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = (float)(int8_t)(w.x >> (8 * e));
      x[4 + e] = (float)(int8_t)(w.y >> (8 * e));
    }
  } else {
    x[0] = __builtin_amdgcn_cvt_f32_fp8(w.x, 0); x[1] = __builtin_amdgcn_cvt_f32_fp8(w.x, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8(w.x, 2); x[3] = __builtin_amdgcn_cvt_f32_fp8(w.x, 3);
    x[4] = __builtin_amdgcn_cvt_f32_fp8(w.y, 0); x[5] = __builtin_amdgcn_cvt_f32_fp8(w.y, 1);
    x[6] = __builtin_amdgcn_cvt_f32_fp8(w.y, 2); x[7] = __builtin_amdgcn_cvt_f32_fp8(w.y, 3);
  }
}

constexpr int kRows = 4;  // query rows in flight per 16 lanes

// kWaves: waves per page (B / 16).  Blocks below page_blocks hold 4 / kWaves units of `heads`
// KV heads each, head_parts units a page and tensor; the others q_rows query rows of one token
// a wave, q_parts waves a token.
template <typename QT, typename KT, int kCode, int kWaves>
__global__ __launch_bounds__(256) void q8_append_kernel(
    RowArgs a, RopeArgs rope, uint8_t* __restrict__ k_codes, uint8_t* __restrict__ v_codes,
    float* __restrict__ k_scale, float* __restrict__ v_scale, const int32_t* __restrict__ page_table,
    const int32_t* __restrict__ seq_lens, int S, int H_q, int H_kv, int max_pages, int num_blocks,
    unsigned n_units, unsigned page_blocks, int heads, unsigned head_parts, unsigned q_parts, int q_rows) {
  constexpr int P = 16 * kWaves;
  __shared__ float s_max[2][4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, tg = lane >> 4;
  const Lane ln = lane_of(rope, lane & 15);

  if (blockIdx.x >= page_blocks) {  // query rows
    const unsigned id = (blockIdx.x - page_blocks) * 4 + wave;
    const int row = (int)(id / q_parts), part = (int)(id % q_parts);
    if (row >= a.n_tokens) return;
    const int r0 = part * q_rows, r1 = min(r0 + q_rows, H_q);
    const QT* q = static_cast<const QT*>(a.q) + row * a.q_stride;
    auto src = [&](int r) { return q + r * kDim; };
    Mover<QT, kRows, false> mq;
    mq.begin(ln, r0 + tg, r1, src);
    const NewTokens t = tokens_of_row(a, seq_lens, S, row);
    if (t.s < 0) return;
    const int tok = t.tok0 + (row - t.row0);
    if (row - t.row0 >= t.n || tok < 0 || tok / P >= max_pages) return;
    const int blk = page_table[(long)t.s * max_pages + tok / P];
    Positions pos;
    if (!positions_of(rope, row, tok, pos)) return;
    Angles A;
    load_angles(rope, ln, pos, A);
    if (blk < 0 || blk >= num_blocks) return;
    QT* out = static_cast<QT*>(a.q_out) + row * a.q_out_stride;
    mq.move(rope, ln, A, tg, r0, r1, H_q, src, [&](int r) { return out + r * kDim; });
    return;
  }

  // ---- which (sequence, page, tensor, KV heads) this wave belongs to
  const unsigned unit = blockIdx.x * (4 / kWaves) + wave / kWaves;
  bool live = unit < n_units;
  const int h0 = (int)(unit % head_parts) * heads, h1 = min(h0 + heads, H_kv);
  const int kv = (int)(unit / head_parts % 2);
  const int slot = (int)(unit / (2 * head_parts));
  // pages by slots: sequence s's begin at slot cu[s] / P + 2 s (it touches at most
  // n / P + 2 pages); without cu one slot a sequence
  NewTokens t{-1, 0, 0, 0};
  int ahead = 0;
  if (live) {
    if (a.cu) {
      t = find_tokens(a, seq_lens, S, slot, [](int c, int i) { return (long)(c / P) + 2 * i; });
      ahead = (int)(slot - (t.row0 / P + 2 * (long)t.s));
    } else {
      t = one_token(seq_lens, slot);
    }
  }
  const int first = max(t.tok0, 0), L = t.tok0 + t.n;  // tokens [first, L) are new
  const int j = first / P + ahead;
  live = live && t.s >= 0 && t.n > 0 && ahead >= 0 && j < max_pages && (long)j * P < L;
  // (the same for the block's waves of a page, so a page's waves leave together; pages of
  // several waves meet at the barriers below)
  if (kWaves == 1 && !live) return;
  const int blk = live ? page_table[(long)t.s * max_pages + j] : 0;  // looked at where it is used

  // ---- this wave's 16 tokens: where they are in the input, and their angles
  const int i0 = 16 * (wave % kWaves) + tg;  // token row of the page, + 4 u
  const int earlier = max(first - j * P, 0);  // rows of the page that were there before
  const KT* src = static_cast<const KT*>(kv ? a.v : a.k);
  const long stride = kv ? a.v_stride : a.k_stride;
  long from[4];
  bool on[4];
  Row8<KT> w[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int T = j * P + i0 + 4 * u;
    on[u] = live && T >= first && T < L;
    from[u] = on[u] ? (t.row0 + (T - t.tok0)) * stride : 0;
    w[u].load(src + from[u] + h0 * kDim, ln.a, ln.b);
  }
  Angles A[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int T = j * P + i0 + 4 * u;
    if (!on[u]) continue;
    Positions pos;
    on[u] = positions_of(rope, t.row0 + (T - t.tok0), T, pos);  // a position outside: left out
    if (kv == 0 && on[u]) load_angles(rope, ln, pos, A[u]);
  }
  live = live && blk >= 0 && blk < num_blocks;
  for (int h = h0; h < h0 + heads; ++h) {  // (as many rounds for every wave)
    float x[4][8];
    float big = -1.0f;  // stays so where no row is placed
    bool nan = false;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      w[u].to(x[u]);
      if (kv == 0) rotate(rope, ln, A[u], x[u]);
      if (on[u]) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          big = fmaxf(fmaxf(big, fabsf(x[u][e])), fabsf(x[u][e + 1]));
          nan |= __builtin_isunordered(x[u][e], x[u][e + 1]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) w[u].load(src + from[u] + min(h + 1, h1 - 1) * kDim, ln.a, ln.b);
    big = wave_max(big);
    const bool odd = __any(nan) || big > 3.402823466e38f;  // (rare) elements that are not finite
    if (odd) {
      big = -1.0f;
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float m = fabsf(x[u][e]);
          if (on[u]) big = fmaxf(big, m <= 3.402823466e38f ? m : 0.0f);
        }
      big = wave_max(big);
    }
    const long at = (long)(live ? blk : 0) * H_kv + min(h, h1 - 1);
    float* scale_at = (kv ? v_scale : k_scale) + at;
    const float before = live && earlier > 0 ? *scale_at : 0.0f;
    if constexpr (kWaves > 1) {  // every wave has read the old scale before it is replaced
      if (lane == 0) s_max[h & 1][wave] = big;
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kWaves; ++u) big = fmaxf(big, s_max[h & 1][wave / kWaves * kWaves + u]);
    }
    if (!live || big < 0.0f || h >= h1) continue;
    // (a page's scale may have either sign: its magnitude is what rows have to fit)
    float scale = page_scale<kCode>(big);
    const bool grew = earlier > 0 && scale > fabsf(before);
    if (earlier > 0 && !grew) scale = before;
    const float inv = fabsf(scale) > 0.0f ? 1.0f / scale : 0.0f;
    uint8_t* codes = (kv ? v_codes : k_codes) + at * (P * kDim);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      uint8_t* to = codes + (i0 + 4 * u) * kDim;
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = x[u][e] * inv;
      uint2 c = codes_of<kCode>(y);
      if (odd) {
        // an infinity stays one where the page has no scale, whose inverse is 0 here
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = inv == 0.0f && __builtin_isinf(x[u][e]) ? x[u][e] : y[e];
        c = codes_of_any<kCode>(y);
      }
      bool put = on[u];
      if (grew && i0 + 4 * u < earlier) {  // an earlier row under the larger scale
        values_of<kCode>(make_uint2(*reinterpret_cast<uint32_t*>(to + ln.a), *reinterpret_cast<uint32_t*>(to + ln.b)), y);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = y[e] * before * inv;
        c = codes_of_any<kCode>(y);
        put = true;
      }
      if (put) {
        *reinterpret_cast<uint32_t*>(to + ln.a) = c.x;
        *reinterpret_cast<uint32_t*>(to + ln.b) = c.y;
      }
    }
    if (wave % kWaves == 0 && lane == 0) *scale_at = scale;
  }
}

template <typename QT, typename KT, int kCode>
hipError_t launch_typed(const locks_cfg_t& c, const RowArgs& a, const RopeArgs& r,
                        const locks_q8_t& cache, const int32_t* page_table,
                        const int32_t* seq_lens, hipStream_t st) {
  const int hq = a.q ? c.num_q_heads : 0, P = c.page_size, waves = P / 16;
  const long slots = a.cu ? a.n_tokens / P + 2L * c.num_seqs : c.num_seqs;
  // heads per unit: up to 4 while 4,096 waves with tokens remain
  const long busy = a.cu ? a.n_tokens / 16 + c.num_seqs : c.num_seqs;
  int heads = c.num_kv_heads < 4 ? c.num_kv_heads : 4;
  while (heads > 1 && busy * 2 * ((c.num_kv_heads + heads - 1) / heads) < 4096) --heads;
  const int head_parts = (c.num_kv_heads + heads - 1) / heads;
  const long units = slots * 2 * head_parts;
  const long page_blocks = (units + 4 / waves - 1) / (4 / waves);
  int per = 16;
  while (per > 4 && (long)a.n_tokens * ((hq + per - 1) / per) < 4096) per /= 2;
  const int q_parts = (hq + per - 1) / per;
  const long q_blocks = ((long)a.n_tokens * q_parts + 3) / 4;
  if (4 * (page_blocks + q_blocks) > 0x7fffffffL) return hipErrorInvalidConfiguration;
#define LOCKS_Q8_APPEND(W)                                                                        \
  hipLaunchKernelGGL((q8_append_kernel<QT, KT, kCode, W>), dim3((unsigned)(page_blocks + q_blocks)), \
                     dim3(256), 0, st, a, r, static_cast<uint8_t*>(cache.k),                       \
                     static_cast<uint8_t*>(cache.v), cache.k_scale, cache.v_scale, page_table,    \
                     seq_lens, c.num_seqs, hq, c.num_kv_heads, c.max_pages_per_seq, c.num_blocks, \
                     (unsigned)units, (unsigned)page_blocks, heads, head_parts, q_parts, per)
  if (waves == 1) LOCKS_Q8_APPEND(1);
  else if (waves == 2) LOCKS_Q8_APPEND(2);
  else LOCKS_Q8_APPEND(4);
#undef LOCKS_Q8_APPEND
  return hipGetLastError();
}

}  // namespace

hipError_t launch_q8_append(const locks_cfg_t& c, const RowArgs& a, const RopeArgs& r,
                            const locks_q8_t& cache, const int32_t* page_table,
                            const int32_t* seq_lens, hipStream_t st) {
  const bool qb = !a.q || c.q_dtype == LOCKS_BF16, kb = c.kv_dtype == LOCKS_BF16;
#define LOCKS_Q8_TYPES(C)                                                                          \
  if (qb && kb) return launch_typed<uint16_t, uint16_t, C>(c, a, r, cache, page_table, seq_lens, st); \
  if (qb) return launch_typed<uint16_t, float, C>(c, a, r, cache, page_table, seq_lens, st);       \
  if (kb) return launch_typed<float, uint16_t, C>(c, a, r, cache, page_table, seq_lens, st);       \
  return launch_typed<float, float, C>(c, a, r, cache, page_table, seq_lens, st)
  if (cache.code == LOCKS_Q8_INT8) {
    LOCKS_Q8_TYPES(LOCKS_Q8_INT8);
  }
  LOCKS_Q8_TYPES(LOCKS_Q8_E4M3);
#undef LOCKS_Q8_TYPES
}

}  // namespace locks
