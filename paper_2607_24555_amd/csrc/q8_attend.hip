// Decode attention over a paged cache held in 8 bits (locks_q8_dense_attend,
// locks_q8_sparse_attend): with ck, cv the codes and sk, sv the scales of token i's page,
//   o_g = sum_i softmax_i(sk q_g^T ck_i / sqrt d) sv cv_i
// over the listed pages' tokens (page_ids == nullptr: every page).
//
// A list is one (sequence, KV head); its units are 16 tokens each.  The units of all lists in
// order are cut into equal shares, one a block, by the lengths themselves (read on the device:
// a table's width says little about them), so a block's share may end one list and begin
// others.  Its four waves take consecutive quarters of each list's piece, and the piece leaves
// one partial (o, max, sum) in slot block + list -- either grows from piece to piece, and a
// list's slots are consecutive -- merged afterwards.  Many short lists take a block each and no
// merge.  A wave
// takes two units a step on the matrix cores.  Codes are exact in f16 (int8: 7 bits and sign;
// e4m3: 4 bits), the key scale multiplies the logits, the value scale the weights, which enter
// as f16 hi + lo, both rounded to nearest: off by at most 2^-23, twice what a float is,
// and to no side.  (Rounded toward zero, 2^-21, outputs were 2^-23 too small on average; bf16
// hi + lo, 16 bits, cost ten times the error over tables of 256 tokens.)
//
// Long caches are bound by HBM, 256 bytes a token and head: 8 x 128K tokens of 8 heads 357 us,
// 6.0 TB/s; 8 ragged sequences (272K tokens) 100.6 us, 5.6 TB/s; 1M tokens of two heads of 16
// queries 94 us, 5.7 TB/s (VALU busy 0.31 to 0.38, matrix cores 0.11; a large copy reaches 5.1).
// Many sequences in a table far wider than they are cost more, every block and row summing the
// lengths: 512 of 512 tokens, 8 heads, 133 us (in a table of their width 112, their bytes 104),
// 4,096 of 256 tokens, one head, 148 (70, 52).
// Tables and short caches are bound by latency, the chain length -> table -> page -> codes and
// scale -> combine, and a merge where a list is split: 4,099 tokens of 8 heads 10.7 us, 2,048
// tokens of 8 x 8 lists 12.8 us (attention 10.2 and merge 4.0 alone).
#include "cache_internal.h"

namespace locks {
namespace {

typedef _Float16 h8v __attribute__((ext_vector_type(8)));
typedef _Float16 h2v __attribute__((ext_vector_type(2)));
typedef float f2v __attribute__((ext_vector_type(2)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef uint32_t u4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ h8v as_h8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(h8v, make_uint4(a, b, c, d));
}
// Two floats as f16 halves of a word, rounded to nearest, and what that leaves of them (of 24
// bits at most 12 and a sign: the second term keeps 11 of them).
__device__ __forceinline__ uint32_t split_h2(float& a, float& b) {
  const h2v h = __builtin_convertvector((f2v{a, b}), h2v);
  a -= (float)h[0];
  b -= (float)h[1];
  return __builtin_bit_cast(uint32_t, h);
}

// Codes widen to f16 exactly, times kUnit: int8 c as c 2^-9, e4m3 as itself.
template <int kCode>
constexpr float kUnit = kCode == LOCKS_Q8_INT8 ? 512.0f : 1.0f;  // what a widened 1 stands for

// int8: excess-128 bytes u in the low halves' low bytes are the f16 subnormals u 2^-24, and
// one packed multiply-add makes (u - 128) 2^-9 of them.
__device__ __forceinline__ uint32_t int8_h2(uint32_t w) {
  const h2v x = __builtin_bit_cast(h2v, w);
  const h2v y = __builtin_elementwise_fma(x, h2v{(_Float16)32768.0f, (_Float16)32768.0f},
                                          h2v{(_Float16)-0.25f, (_Float16)-0.25f});
  return __builtin_bit_cast(uint32_t, y);
}
// e4m3: bytes 0 and 1 (kHigh: 2 and 3) of w.
template <bool kHigh>
__device__ __forceinline__ uint32_t e4m3_h2(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, kHigh));
}

// Four codes (one word) as two words of f16 pairs, in order.
template <int kCode>
__device__ __forceinline__ void widen(uint32_t w, uint32_t& a, uint32_t& b) {
  if constexpr (kCode == LOCKS_Q8_INT8) {
    w ^= 0x80808080u;
    a = int8_h2(__builtin_amdgcn_perm(0u, w, 0x0c010c00u));
    b = int8_h2(__builtin_amdgcn_perm(0u, w, 0x0c030c02u));
  } else {
    a = e4m3_h2<false>(w);
    b = e4m3_h2<true>(w);
  }
}

// Codes of four tokens (words t0 .. t3 hold four elements each) as, per element e, the
// f16 pairs (t0, t1) in p[e] and (t2, t3) in q[e].
template <int kCode>
__device__ __forceinline__ void widen_across(uint32_t t0, uint32_t t1, uint32_t t2, uint32_t t3,
                                             uint32_t (&p)[4], uint32_t (&q)[4]) {
  if constexpr (kCode == LOCKS_Q8_INT8) {
    t0 ^= 0x80808080u;
    t1 ^= 0x80808080u;
    t2 ^= 0x80808080u;
    t3 ^= 0x80808080u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      p[e] = int8_h2(__builtin_amdgcn_perm(t1, t0, 0x0c040c00u + 0x00010001u * e));
      q[e] = int8_h2(__builtin_amdgcn_perm(t3, t2, 0x0c040c00u + 0x00010001u * e));
    }
  } else {
    // element 0 of two tokens, then element 1 (then 2 and 3): pairs the conversion widens
    widen<kCode>(__builtin_amdgcn_perm(t1, t0, 0x05010400u), p[0], p[1]);
    widen<kCode>(__builtin_amdgcn_perm(t1, t0, 0x07030602u), p[2], p[3]);
    widen<kCode>(__builtin_amdgcn_perm(t3, t2, 0x05010400u), q[0], q[1]);
    widen<kCode>(__builtin_amdgcn_perm(t3, t2, 0x07030602u), q[2], q[3]);
  }
}

// Max over the lanes {l, l^16, l^32, l^48} (the four 16-lane rows).
__device__ __forceinline__ float rows_max(float v) {
  auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float rows_sum(float v) {
  auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A read of codes.  kStream: past the cache levels' replacement.  Faster where the codes come
// from HBM (8 x 128K tokens, a whole cache: 383 -> 356 us, 6.0 TB/s; 16 x 4K in 8 copies in
// turn: 33.4 -> 31.5; 64 lists' tables, 35 of 34 MB in turn: 15.0 -> 14.3), slower where the last
// level (256 MB) still holds them (16 x 4K again and again: 27.9 -> 30.6; 3 such tables in turn:
// 13.2 -> 13.9).  A whole cache that fits there is small work and does not stay there beside a
// model's weights; a table's pages are few and mostly the ones of the step before, so those
// are left to the caches.
template <bool kStream, typename V>
__device__ __forceinline__ V load_codes(const uint8_t* p) {
  if constexpr (kStream) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  else return *reinterpret_cast<const V*>(p);
}

// Power of two, exponent clamped to what a float holds.
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(min(max(e, -126), 127) + 127) << 23); }
__device__ __forceinline__ int exponent(float v) { return (int)(__float_as_uint(v) >> 23 & 255u) - 127; }

// How the lists' units are cut (see Q8Plan).
struct Cut {
  int fixed_units;  // units of every list (a table's), or 0: the sequence's own
  int blocks, few;
};
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int units_of(int len) { return max((len + kPage - 1) / kPage, 0); }
__device__ __forceinline__ int wave_scan(int v) {  // inclusive sums over the wave
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast 15, 31
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}
// The sequences' lengths and places in the lists' order (units of all lists fit 31 bits, which
// the host checks).  Up to 64 sequences are one load and one scan, kept in a register.
// A list counts as a multiple of 8 units, so that at the smallest share no block holds a piece
// of two lists, one after the other (8 heads over 4,099 tokens: 13.0 -> 11.2 us).
struct Order {
  const int32_t* seq_lens;
  int S, H_kv, fixed;
  int len, end;    // S <= 64, lane i: sequence i's length; units of one KV head up to and with it
  unsigned units;  // of all sequences and KV heads
  unsigned share;
  __device__ __forceinline__ Order(const Cut& cut, const int32_t* sl, int S_, int H)
      : seq_lens(sl), S(S_), H_kv(H), fixed(cut.fixed_units) {
    const int lane = threadIdx.x & 63;
    len = S <= 64 && lane < S ? seq_lens[lane] : 0;
    end = 0;
    units = share = 0;
    if (!cut.blocks) return;  // a block a list: no shares (4,096 sequences: 140 -> 70 us)
    int sum = S * padded(fixed);
    if (!fixed) {
      if (S <= 64) {
        end = scan(len, 0);
        sum = __builtin_amdgcn_readlane(end, 63);
      } else {
        sum = 0;
#pragma unroll 4
        for (int i = lane; i < S; i += 64) sum += padded(units_of(seq_lens[i]));
        sum = __builtin_amdgcn_readlane(wave_scan(sum), 63);
      }
    }
    units = (unsigned)sum * H_kv;
    share = q8_share(units, cut.blocks, cut.few);
  }
  static __device__ __forceinline__ int padded(int n) { return (n + 7) & ~7; }
  // Units of one KV head up to and with each lane's sequence, `sum` of them before the first's.
  static __device__ __forceinline__ int scan(int lane_len, int sum) { return sum + wave_scan(padded(units_of(lane_len))); }
  __device__ __forceinline__ int load(int s0) const {
    const int i = s0 + (threadIdx.x & 63);
    return i < S ? seq_lens[i] : 0;
  }
  // s is wave-uniform
  __device__ __forceinline__ int length(int s) const {
    return S <= 64 ? __builtin_amdgcn_readlane(len, s) : seq_lens[s];
  }
  __device__ __forceinline__ int list_units(int s) const { return padded(fixed ? fixed : units_of(length(s))); }
  // Units of one KV head before sequence s.
  __device__ __forceinline__ int before(int s) const {
    if (fixed) return s * padded(fixed);
    int e = end, sum = 0;
    if (S > 64) {
      for (int i = threadIdx.x & 63; i < (s & ~63); i += 64) sum += padded(units_of(seq_lens[i]));
      sum = __builtin_amdgcn_readlane(wave_scan(sum), 63);
      e = scan(load(s & ~63), sum);
    }
    return (s & 63) ? __builtin_amdgcn_readlane(e, (s & 63) - 1) : sum;
  }
  // The sequence that unit u of the lists belongs to (u < units), and before() of it.
  __device__ __forceinline__ int find(unsigned u, int& bef) const {
    if (fixed) {
      const int s = (int)(u / ((unsigned)padded(fixed) * H_kv));
      bef = s * padded(fixed);
      return s;
    }
    int e = end, sum = 0, next = S > 64 ? load(0) : 0;
    for (int s0 = 0; s0 < S; s0 += 64) {
      if (S > 64) {
        const int now = next;
        next = load(s0 + 64);  // (zeros past the last)
        e = scan(now, sum);
      }
      const unsigned long long past = __ballot((unsigned)e * H_kv > u);
      if (past) {
        const int i = __ffsll(past) - 1;
        bef = i > 0 ? __builtin_amdgcn_readlane(e, i - 1) : sum;
        return s0 + i;
      }
      sum = __builtin_amdgcn_readlane(e, 63);
    }
    bef = sum;
    return S - 1;
  }
};

// Lane layout (l = 16 r + c):
//   S^T = K Q^T  (mfma 16x16x32, M = token, N = head; step 2 a + b holds dims
//                 64 a + 16 r + 8 b + e): lane holds S^T[4 r + j][c] of each unit
//   O^T += V^T P (mfma 16x16x32, M = dim, N = head, K = (r, 4 u + j) = token 4 r + j of
//                 unit u; tile n covers dims 8 m + n): P is the B operand exactly as S^T
//                 left it, and lane holds O^T for head c, dims 32 r + 8 j + n.
// Codes of two units, lane (c, r): k[u][a] token c, dims 64 a + 16 r .. + 15; v[u][j] token
// 4 r + j, dims 8 c .. + 7.  Each half of the next pair is requested as soon as its registers
// are free: the keys after the logits' products, the values after the outputs'.
// kAll: the whole cache, else page_ids' pages.
template <typename QT, int kCode, bool kAll>
__global__ __launch_bounds__(256, 3) void q8_attend_kernel(
    int S, int H_q, int H_kv, int max_pages, int k_list, int pgsz, int lg_sub, const QT* __restrict__ q,
    const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ v_codes,
    const float* __restrict__ k_scale, const float* __restrict__ v_scale,
    const int32_t* __restrict__ page_table, const int32_t* __restrict__ seq_lens,
    const int32_t* __restrict__ page_ids, Cut cut, float* __restrict__ partial, float* __restrict__ out,
    float* __restrict__ out_lse) {
  constexpr int kTerms = sizeof(QT) == 2 ? 1 : 2;
  __shared__ float sO[4][kDim][kMaxGroup + 1];
  __shared__ float sM[4][kMaxGroup], sL[4][kMaxGroup];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int c16 = lane & 15, r4 = lane >> 4;
  const int G = H_q / H_kv;
  const long page_bytes = (long)pgsz * kDim;
  const int k_off = c16 * kDim + 16 * r4, v_off = 4 * r4 * kDim + 8 * c16;

  // ---- the block's share of the units (wave-uniform, on the scalar unit)
  const Order order(cut, seq_lens, S, H_kv);
  int s, h, at = 0, left;  // list (s, h), first unit within it, units of the share still to do
  const bool whole = cut.blocks == 0;
  if (whole) {
    s = blockIdx.x / H_kv;
    h = blockIdx.x % H_kv;
    left = order.list_units(s);
  } else {
    const unsigned share = order.share, u0 = blockIdx.x * share;
    if (u0 >= order.units) return;
    left = uniform((int)min(share, order.units - u0));
    int before;
    s = uniform(order.find(u0, before));
    const unsigned n = order.list_units(s), in = u0 - (unsigned)before * H_kv;
    h = uniform((int)(in / n));
    at = uniform((int)(in - h * n));
  }

  while (true) {  // one piece: units [at, at + n) of list (s, h)
  // (of a table's list the length is only waited for once its pages are on their way: 13.0 ->
  // 12.75 us of 64 lists)
  int L = kAll ? uniform(order.length(s)) : 0;
  const int real = kAll ? units_of(L) : order.fixed;
  const int taken = min(left, order.padded(real) - at), n = min(taken, real - at);
  const bool complete = taken == order.padded(real);  // the whole list: its output is formed here
  const int per_wave = ((n + 3) / 4 + 1) & ~1;
  const int w_begin = min(wave * per_wave, n), w_end = min(w_begin + per_wave, n);

  // ---- queries: B operand of step 2 a + b, as stored until the first codes are on their way
  uint4 qb[kTerms][4];
  {
    const QT* row = q + ((long)s * H_q + h * G + min(c16, G - 1)) * kDim + 16 * r4;
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int u = 0; u < kTerms; ++u)
        qb[u][st] = reinterpret_cast<const uint4*>(row + 64 * (st >> 1) + 8 * (st & 1))[u];
  }
  // Then scaled by a power of two per head so that the largest element is in [2^14, 2^15): f16's
  // smallest step, 2^-24, is then at most 2^-38 of the largest.  A bf16 element is exact but for
  // half of that step, 2^-39 of the largest; a float in two terms is held to 2^-23 of itself or to
  // that, whichever is more.
  bool scaled = false;
  float head_scale = 0.0f;  // logits in log2 units = products * head_scale * key scale
  auto scale_queries = [&]() {
    auto element = [&](int st, int e) {
      if constexpr (sizeof(QT) == 2) {
        const uint4 w = qb[0][st];
        const uint32_t y = e < 2 ? w.x : (e < 4 ? w.y : (e < 6 ? w.z : w.w));
        return __uint_as_float((e & 1) ? y & 0xffff0000u : y << 16);
      } else {
        const uint4 w = qb[e >> 2][st];
        return __uint_as_float((e & 3) == 0 ? w.x : ((e & 3) == 1 ? w.y : ((e & 3) == 2 ? w.z : w.w)));
      }
    };
    float big = 0.0f;
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int e = 0; e < 8; ++e) big = fmaxf(big, fabsf(element(st, e)));
    const int e2 = min(14 - exponent(rows_max(big)), 126);
    const float up = pow2(e2);
    head_scale = pow2(-e2) * (kUnit<kCode> * kLog2e / 11.313708498984761f);  // / sqrt(128)
#pragma unroll
    for (int st = 0; st < 4; ++st) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = element(st, e) * up;
#pragma unroll
      for (int m = 0; m < kTerms; ++m) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = split_h2(x[2 * e], x[2 * e + 1]);
        qb[m][st] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    scaled = true;
  };
  float m = -INFINITY, l = 0.0f;  // l: this lane's tokens only
  int ve = -126;                  // o is in units of 2^ve (times 2^-15 and the codes' unit)
  f4v o[8];
#pragma unroll
  for (int n = 0; n < 8; ++n) o[n] = f4v{0.0f, 0.0f, 0.0f, 0.0f};

  // 64 units a round.  Lane j: the round's unit j (first token, or -1: nothing to attend), its
  // codes and scales
  for (int i0 = w_begin; i0 < w_end; i0 += 64) {
  const int t = at + i0 + lane, entry = t >> lg_sub;
  const bool mine = i0 + lane < w_end;
  int id = entry;
  if constexpr (!kAll) {
    id = mine && entry < k_list ? page_ids[((long)s * H_kv + h) * k_list + entry] : -1;
    L = uniform(order.length(s));
  }
  int my_tok = -1, my_blk = 0;
  float my_ks = 0.0f, my_vs = 0.0f;
  if (mine && id >= 0 && id < (L + pgsz - 1) / pgsz) {
    const int tok0 = id * pgsz + (t & ((1 << lg_sub) - 1)) * kPage;
    if (tok0 < L) {
      my_tok = tok0;
      my_blk = page_table[(long)s * max_pages + id];
      my_ks = k_scale[(long)my_blk * H_kv + h];
      my_vs = v_scale[(long)my_blk * H_kv + h];
    }
  }
  const unsigned long long live = __ballot(my_tok >= 0);
  if (!live) continue;
  const int cnt = 64 - __clzll(live);     // units up to the last one with tokens
  const int spare = __ffsll(live) - 1;    // an empty unit's loads read another unit

  auto unit_at = [&](int j) -> long {
    const int i = j < cnt && ((live >> j) & 1) ? j : spare;
    const long blk = __builtin_amdgcn_readlane(my_blk, i);
    const int tok0 = __builtin_amdgcn_readlane(my_tok, i);
    return (blk * H_kv + h) * page_bytes + (long)(tok0 & (pgsz - 1)) * kDim;
  };
  u4v kc[2][2];
  u2v vc[2][4];
  auto load_k = [&](int u, long base) {
#pragma unroll
    for (int a = 0; a < 2; ++a) kc[u][a] = load_codes<kAll, u4v>(k_codes + base + k_off + 64 * a);
  };
  auto load_v = [&](int u, long base) {
#pragma unroll
    for (int j = 0; j < 4; ++j) vc[u][j] = load_codes<kAll, u2v>(v_codes + base + v_off + j * kDim);
  };
  {
    const long b0 = unit_at(0), b1 = unit_at(1);
    load_k(0, b0);
    load_k(1, b1);
    load_v(0, b0);
    load_v(1, b1);
  }
  if (!scaled) scale_queries();
  // weights enter as f16 hi + lo of p * value scale, scaled so that the largest scale so far lies
  // in [2^14, 2^15): a weight is held to 2^-23 of itself or to half of f16's smallest step, 2^-39 of
  // that scale, whichever is more
  {
    const int e = exponent(warp_max(fabsf(my_vs))) + 1;
    if (e > ve) {
      const float down = ldexpf(1.0f, ve - e);
#pragma unroll
      for (int x = 0; x < 8; ++x) o[x] *= down;
      ve = e;
    }
    my_vs = ldexpf(my_vs, 15 - ve);  // (2^-ve alone may be too small for a float)
  }

  for (int j = 0; j < cnt; j += 2) {
    float z[2][4], vs[2];
    int valid[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int i = min(j + u, 63);
      const int tok0 = __builtin_amdgcn_readlane(my_tok, i);
      valid[u] = j + u < cnt && tok0 >= 0 ? min(kPage, L - tok0) : 0;
      const float ks = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_ks), i)) * head_scale;
      vs[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_vs), i));
      f4v st = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const uint32_t w[4] = {kc[u][a].x, kc[u][a].y, kc[u][a].z, kc[u][a].w};
        uint32_t b[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) widen<kCode>(w[e], b[2 * e], b[2 * e + 1]);
#pragma unroll
        for (int mt = kTerms - 1; mt >= 0; --mt) {
          st = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(b[0], b[1], b[2], b[3]),
                                                      __builtin_bit_cast(h8v, qb[mt][2 * a]), st, 0, 0, 0);
          st = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(b[4], b[5], b[6], b[7]),
                                                      __builtin_bit_cast(h8v, qb[mt][2 * a + 1]), st, 0, 0, 0);
        }
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) z[u][n] = st[n] * ks;
      if (valid[u] < kPage) {  // uniform: an empty or partial unit; its codes may be anything
#pragma unroll
        for (int n = 0; n < 4; ++n)
          if (4 * r4 + n >= valid[u]) {
            z[u][n] = -INFINITY;
            vc[u][n] = u2v{0u, 0u};
          }
        if (valid[u] == 0) vs[u] = 0.0f;
      }
    }
    const bool more = j + 2 < cnt;
    long b0 = 0, b1 = 0;
    if (more) {
      b0 = unit_at(j + 2);
      b1 = unit_at(j + 3);
      load_k(0, b0);
      load_k(1, b1);
    }
    const float pm = rows_max(fmaxf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])),
                                    fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3]))));
    const float mn = fmaxf(m, pm);
    const float at = fmaxf(mn, -3.0e38f);  // a finite origin while every weight is zero
    const float sc = __builtin_amdgcn_exp2f(m - at);
    m = mn;
    uint32_t ph[4], pl[4];
    float ps = 0.0f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float p0 = __builtin_amdgcn_exp2f(z[u][2 * n] - at), p1 = __builtin_amdgcn_exp2f(z[u][2 * n + 1] - at);
        ps += p0 + p1;
        float w0 = p0 * vs[u], w1 = p1 * vs[u];
        ph[2 * u + n] = split_h2(w0, w1);
        pl[2 * u + n] = split_h2(w0, w1);
      }
    l = fmaf(l, sc, ps);
    if (__any(sc != 1.0f)) {
#pragma unroll
      for (int n = 0; n < 8; ++n) o[n] *= sc;
    }
    const h8v bh = as_h8(ph[0], ph[1], ph[2], ph[3]), bl = as_h8(pl[0], pl[1], pl[2], pl[3]);
#pragma unroll
    for (int half = 0; half < 2; ++half) {  // dims 8 m + 4 half + e
      uint32_t p[2][4], r[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u)
        widen_across<kCode>(half ? vc[u][0].y : vc[u][0].x, half ? vc[u][1].y : vc[u][1].x,
                            half ? vc[u][2].y : vc[u][2].x, half ? vc[u][3].y : vc[u][3].x, p[u], r[u]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const h8v a = as_h8(p[0][e], r[0][e], p[1][e], r[1][e]);
        const int n = 4 * half + e;
        o[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, bh, o[n], 0, 0, 0);
        o[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, bl, o[n], 0, 0, 0);
      }
    }
    if (more) {
      load_v(0, b0);
      load_v(1, b1);
    }
  }
  }

  // ---- the block's four waves combined (m in log2 units): each brings its sums to the block's
  // maximum before it writes them; the odd row pitch of sO keeps the layout's writes and the
  // reads along d free of bank conflicts
  // (the addresses are formed here: kept across the loop they spill registers)
  int t_here = tid;
  asm volatile("" : "+v"(t_here));
  const int c_here = t_here & 15, r_here = (t_here >> 4) & 3;
  l = rows_sum(l);
  if (r_here == 0) sM[wave][c_here] = m;
  __syncthreads();
  {
    const float mx = fmaxf(fmaxf(sM[0][c_here], sM[1][c_here]), fmaxf(sM[2][c_here], sM[3][c_here]));
    const float wt = __builtin_amdgcn_exp2f(m - fmaxf(mx, -3.0e38f));
    const float down = ldexpf(wt * kUnit<kCode>, ve - 15);
    if (r_here == 0) sL[wave][c_here] = l * wt;
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) sO[wave][32 * r_here + 8 * j + n][c_here] = o[n][j] * down;
  }
  __syncthreads();
  for (int g = t_here >> 7, c = t_here & (kDim - 1); g < G; g += 2) {
    const float acc = (sO[0][c][g] + sO[1][c][g]) + (sO[2][c][g] + sO[3][c][g]);
    const float ls = (sL[0][g] + sL[1][g]) + (sL[2][g] + sL[3][g]);
    const float mx = fmaxf(fmaxf(sM[0][g], sM[1][g]), fmaxf(sM[2][g], sM[3][g]));
    const long row = (long)s * H_q + h * G + g;
    if (complete) {
      out[row * kDim + c] = ls == 0.0f ? 0.0f : acc / ls;
      if (c == 0 && out_lse) out_lse[row] = ls == 0.0f ? -INFINITY : mx * kLn2 + logf(ls);
    } else {
      float* pr = partial + ((blockIdx.x + (long)s * H_kv + h) * G + g) * (kDim + 2);
      pr[c] = acc;
      if (c < 2) pr[kDim + c] = c ? ls : mx;
    }
  }
  // ---- the next list with units
  left -= taken;
  if (left <= 0) return;
  at = 0;
  if (++h == H_kv) {
    h = 0;
    do ++s;
    while (order.list_units(s) == 0);
  }
  __syncthreads();
  }
}

// Combines a row's partials (max in log2 units), of the blocks that hold a piece of its list; a
// list within one block has its output already.  kWaves waves a row, 16 partials in flight each;
// lane c holds dims 2 c and 2 c + 1.
template <int kWaves>
__global__ __launch_bounds__(kWaves == 1 ? 256 : 64 * kWaves) void q8_merge_kernel(
    int S, int H_q, int H_kv, Cut cut, const int32_t* __restrict__ seq_lens,
    const float* __restrict__ partial, float* __restrict__ out, float* __restrict__ out_lse) {
  __shared__ float sO[kWaves][kDim], sM[kWaves], sL[kWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const long row = kWaves == 1 ? (long)blockIdx.x * 4 + wave : blockIdx.x;
  if (kWaves == 1 && row >= (long)S * H_q) return;
  const int G = H_q / H_kv, s = (int)(row / H_q), h = (int)(row % H_q) / G, g = (int)(row % G);
  const Order order(cut, seq_lens, S, H_kv);
  const int mine = order.list_units(s);
  const unsigned share = order.share, u0 = (unsigned)order.before(s) * H_kv + h * mine;
  const unsigned b0 = u0 / share;
  const int n_parts = mine > 0 ? (int)((u0 + mine - 1) / share - b0 + 1) : 0;
  if (n_parts == 1) return;
  const float* p = partial + ((b0 + (long)s * H_kv + h) * G + g) * (kDim + 2);
  const long pitch = (long)G * (kDim + 2);
  constexpr int kFly = 16, kStep = 4;  // partials in flight, requested four at a time
  float m = -INFINITY, l = 0.0f, o0 = 0.0f, o1 = 0.0f;
  for (int t0 = (kWaves == 1 ? 0 : wave) * kFly; t0 < n_parts; t0 += kWaves * kFly) {
    float mt[kFly], lt[kFly];
    float2 ot[kFly];
#pragma unroll
    for (int u0 = 0; u0 < kFly; u0 += kStep) {
      const bool any = t0 + u0 < n_parts;
#pragma unroll
      for (int u = u0; u < u0 + kStep; ++u) {
        ot[u] = make_float2(0.0f, 0.0f);
        mt[u] = -INFINITY;
        lt[u] = 0.0f;
      }
      if (any) {
#pragma unroll
        for (int u = u0; u < u0 + kStep; ++u) {
          const float* pt = p + min(t0 + u, n_parts - 1) * pitch;
          ot[u] = reinterpret_cast<const float2*>(pt)[lane];
          const float2 ml = reinterpret_cast<const float2*>(pt)[kDim / 2];
          mt[u] = t0 + u < n_parts ? ml.x : -INFINITY;
          lt[u] = ml.y;
        }
      }
    }
    float mm = m;
#pragma unroll
    for (int u = 0; u < kFly; ++u) mm = fmaxf(mm, mt[u]);
    const float at = fmaxf(mm, -3.0e38f);
    const float sc = __builtin_amdgcn_exp2f(m - at);
    m = mm;
    l *= sc;
    o0 *= sc;
    o1 *= sc;
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      const float w = __builtin_amdgcn_exp2f(mt[u] - at);
      l = fmaf(lt[u], w, l);
      o0 = fmaf(ot[u].x, w, o0);
      o1 = fmaf(ot[u].y, w, o1);
    }
  }
  if constexpr (kWaves == 1) {
    reinterpret_cast<float2*>(out + row * kDim)[lane] =
        l == 0.0f ? make_float2(0.0f, 0.0f) : make_float2(o0 / l, o1 / l);
    if (out_lse && lane == 0) out_lse[row] = l == 0.0f ? -INFINITY : m * kLn2 + logf(l);
  } else {
    *reinterpret_cast<float2*>(&sO[wave][2 * lane]) = make_float2(o0, o1);
    if (lane == 0) { sM[wave] = m; sL[wave] = l; }
    __syncthreads();
    if (threadIdx.x >= kDim) return;
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, sM[w]);
    const float at = fmaxf(mx, -3.0e38f);
    float ls = 0.0f, acc = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float wt = __builtin_amdgcn_exp2f(sM[w] - at);
      ls = fmaf(sL[w], wt, ls);
      acc = fmaf(sO[w][threadIdx.x], wt, acc);
    }
    out[row * kDim + threadIdx.x] = ls == 0.0f ? 0.0f : acc / ls;
    if (out_lse && threadIdx.x == 0) out_lse[row] = ls == 0.0f ? -INFINITY : mx * kLn2 + logf(ls);
  }
}

}  // namespace

hipError_t launch_q8_attend(const locks_cfg_t& c, const void* q, const locks_q8_t& cache,
                            const int32_t* page_table, const int32_t* seq_lens,
                            const int32_t* page_ids, const Q8Plan& plan, float* partial, float* out,
                            float* out_lse, hipStream_t st) {
  const Cut cut{page_ids ? page_budget(c) << sub_page_log2(c) : 0, plan.blocks, plan.few};
  const int lists = c.num_seqs * c.num_kv_heads;
  const dim3 grid(plan.grid);
#define LOCKS_Q8_ATTEND_S(QT, C, ST)                                                            \
  hipLaunchKernelGGL((q8_attend_kernel<QT, C, ST>), grid, dim3(256), 0, st, c.num_seqs,          \
                     c.num_q_heads, c.num_kv_heads, c.max_pages_per_seq, page_budget(c),        \
                     c.page_size, sub_page_log2(c), static_cast<const QT*>(q),                  \
                     static_cast<const uint8_t*>(cache.k), static_cast<const uint8_t*>(cache.v), \
                     cache.k_scale, cache.v_scale, page_table, seq_lens, page_ids, cut, partial, \
                     out, out_lse)
#define LOCKS_Q8_ATTEND(QT, C)                            \
  if (page_ids) LOCKS_Q8_ATTEND_S(QT, C, false);          \
  else LOCKS_Q8_ATTEND_S(QT, C, true)
  if (c.q_dtype == LOCKS_BF16) {
    if (cache.code == LOCKS_Q8_INT8) {
      LOCKS_Q8_ATTEND(uint16_t, LOCKS_Q8_INT8);
    } else {
      LOCKS_Q8_ATTEND(uint16_t, LOCKS_Q8_E4M3);
    }
  } else if (cache.code == LOCKS_Q8_INT8) {
    LOCKS_Q8_ATTEND(float, LOCKS_Q8_INT8);
  } else {
    LOCKS_Q8_ATTEND(float, LOCKS_Q8_E4M3);
  }
#undef LOCKS_Q8_ATTEND
#undef LOCKS_Q8_ATTEND_S
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !plan.blocks) return e;
  const int rows = c.num_seqs * c.num_q_heads;
#define LOCKS_Q8_MERGE(W, GRID, BLOCK)                                                          \
  hipLaunchKernelGGL(q8_merge_kernel<W>, dim3(GRID), dim3(BLOCK), 0, st, c.num_seqs, c.num_q_heads, \
                     c.num_kv_heads, cut, seq_lens, partial, out, out_lse)
  // waves a row by the partials of an average list
  if (plan.few <= 2 * lists) LOCKS_Q8_MERGE(1, (rows + 3) / 4, 256);
  else if (plan.few <= 64 * lists) LOCKS_Q8_MERGE(4, rows, 256);
  else LOCKS_Q8_MERGE(16, rows, 1024);
#undef LOCKS_Q8_MERGE
  return hipGetLastError();
}

}  // namespace locks
