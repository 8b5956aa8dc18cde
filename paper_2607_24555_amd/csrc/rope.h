// Device pieces shared by the appends: which sequence a row belongs to, the rotation of a
// row spread over 16 lanes, and the rotated copy of a token's rows.
//
// Every operation of the rotation is one fp32 rounding (no fused multiply-add), so that a
// row's result does not depend on how a kernel arranges it.
#pragma once

#include "cache_internal.h"

#pragma clang fp contract(off)

namespace locks {
namespace {

typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
typedef float f2v __attribute__((ext_vector_type(2)));
typedef float f4v __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));

// Two floats to bf16 bits, round to nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2v{a, b}, bf2v));
}

// A lane's eight elements of a row: chunks of four from a and from b, as stored, as floats,
// and back.
// kStream: past the cache levels' replacement.
template <bool kStream, typename V, typename T>
__device__ __forceinline__ V load_as(const T* p) {
  if constexpr (kStream) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  else return *reinterpret_cast<const V*>(p);
}
template <bool kStream, typename V, typename T>
__device__ __forceinline__ void store_as(V v, T* p) {
  if constexpr (kStream) __builtin_nontemporal_store(v, reinterpret_cast<V*>(p));
  else *reinterpret_cast<V*>(p) = v;
}

template <typename T>
struct Row8;
template <>
struct Row8<uint16_t> {
  u2v lo, hi;
  template <bool kStream = false>
  __device__ __forceinline__ void load(const uint16_t* p, int a, int b) {
    lo = load_as<kStream, u2v>(p + a);
    hi = load_as<kStream, u2v>(p + b);
  }
  template <bool kStream>
  __device__ __forceinline__ void store(uint16_t* p, int a, int b) const {
    store_as<kStream>(lo, p + a);
    store_as<kStream>(hi, p + b);
  }
  __device__ __forceinline__ void to(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      x[2 * e] = __uint_as_float(lo[e] << 16);
      x[2 * e + 1] = __uint_as_float(lo[e] & 0xffff0000u);
      x[4 + 2 * e] = __uint_as_float(hi[e] << 16);
      x[5 + 2 * e] = __uint_as_float(hi[e] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void from(const float (&x)[8]) {
    lo = u2v{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    hi = u2v{pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
  }
};
template <>
struct Row8<float> {
  f4v lo, hi;
  template <bool kStream = false>
  __device__ __forceinline__ void load(const float* p, int a, int b) {
    lo = load_as<kStream, f4v>(p + a);
    hi = load_as<kStream, f4v>(p + b);
  }
  template <bool kStream>
  __device__ __forceinline__ void store(float* p, int a, int b) const {
    store_as<kStream>(lo, p + a);
    store_as<kStream>(hi, p + b);
  }
  __device__ __forceinline__ void to(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = lo[e];
      x[4 + e] = hi[e];
    }
  }
  __device__ __forceinline__ void from(const float (&x)[8]) {
    lo = f4v{x[0], x[1], x[2], x[3]};
    hi = f4v{x[4], x[5], x[6], x[7]};
  }
};

// Largest s in [0, S) whose key(s) <= at, or -1 (key ascending; the same for the whole
// wave): 64 keys a round, so one round trip up to 64 sequences and two up to 4,096.
template <typename Key>
__device__ __forceinline__ int wave_search(int S, long at, Key key) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = S;
  while (true) {
    const int step = (hi - lo + 63) / 64;
    const int i = lo + lane * step;
    const int n = __popcll(__ballot(i < hi && key(i) <= at));
    if (n == 0) return -1;
    lo += (n - 1) * step;
    if (step == 1) return lo;
    hi = min(hi, lo + step);
  }
}

// The new tokens of sequence s: rows [row0, row0 + n) of the input are tokens
// [tok0, tok0 + n) of the sequence.
struct NewTokens {
  int s, row0, n, tok0;
};
// ... of the sequence with the largest key(cu[s], s) <= at (s = -1: none).  Up to 64 sequences
// every lane holds one's entries, so that nothing is loaded once the sequence is known.
template <typename Key>
__device__ __forceinline__ NewTokens find_tokens(const RowArgs& a, const int32_t* seq_lens, int S, long at, Key key) {
  const int32_t* cu = a.cu;
  int s, r0, r1, L;
  if (S <= 64) {
    const int lane = threadIdx.x & 63, i = min(lane, S - 1);
    const int c = cu[i], len = seq_lens[i];
    const int end = cu[S];
    s = __popcll(__ballot(lane < S && key(c, i) <= at)) - 1;
    if (s < 0) return NewTokens{-1, 0, 0, 0};
    r0 = __builtin_amdgcn_readlane(c, s);
    r1 = s + 1 < S ? __builtin_amdgcn_readlane(c, min(s + 1, 63)) : end;
    L = __builtin_amdgcn_readlane(len, s);
  } else {
    s = wave_search(S, at, [cu, key](int i) { return key(cu[i], i); });
    if (s < 0) return NewTokens{-1, 0, 0, 0};
    s = __builtin_amdgcn_readfirstlane(s);
    r0 = cu[s];
    r1 = cu[s + 1];
    L = seq_lens[s];
  }
  r1 = min(r1, a.n_tokens);
  const int n = r0 >= 0 && r1 > r0 ? r1 - r0 : 0;
  return NewTokens{s, r0, n, L - n};
}
// One new token a sequence, row s.
__device__ __forceinline__ NewTokens one_token(const int32_t* seq_lens, int s) {
  const int L = seq_lens[s];
  return NewTokens{s, s, L > 0 ? 1 : 0, L - 1};
}
// ... of the sequence that input row `row` belongs to.
__device__ __forceinline__ NewTokens tokens_of_row(const RowArgs& a, const int32_t* seq_lens, int S, int row) {
  if (!a.cu) return one_token(seq_lens, row);
  return find_tokens(a, seq_lens, S, row, [](int c, int) { return (long)c; });
}

// Which elements of a row lane cg of 16 holds: both of each of its four pairs, so that a
// rotation stays in the lane and a lane needs four angles.  Half-split pairs: chunk a in the
// first half and chunk b in the second; interleaved or not rotated: eight in a row.
struct Lane {
  int a, b, pair0;
  bool turn;
};
__device__ __forceinline__ Lane lane_of(const RopeArgs& r, int cg) {
  const int n = r.interleaved ? 0 : r.half >> 2;  // lanes of half-split pairs
  if (cg < n) return Lane{4 * cg, r.half + 4 * cg, 4 * cg, true};
  // (the rest of a half-split row starts at 2 half = 8 n)
  return Lane{8 * cg, 8 * cg + 4, 4 * cg, r.interleaved && 4 * cg < r.half};
}

struct Angles {
  float c[4], s[4];
};
// The table rows of a token's axes, or false where one lies outside the table (the same for
// all lanes of the token).
struct Positions {
  int p0, p1, p2;
};
__device__ __forceinline__ bool positions_of(const RopeArgs& r, int row, int tok, Positions& p) {
  p = Positions{tok, tok, tok};
  if (r.half == 0) return true;
  if (r.positions) {
    p.p0 = p.p1 = p.p2 = r.positions[row];
    if (r.n_axes > 1) p.p1 = p.p2 = r.positions[(long)r.n_tokens + row];
    if (r.n_axes > 2) p.p2 = r.positions[2 * (long)r.n_tokens + row];
  }
  const unsigned n = r.n_pos;
  return (unsigned)p.p0 < n && (unsigned)p.p1 < n && (unsigned)p.p2 < n;
}
// The lane's angles at a token's positions.  (Values, not members, are selected: a select of
// members is one of addresses, which puts the struct into LDS and makes the kernel read its
// dispatch packet from host memory: 64 tokens 3.1 us without, 13 with.)
__device__ __forceinline__ void load_angles(const RopeArgs& r, const Lane& ln, const Positions& p, Angles& A) {
  if (!ln.turn) return;
  const int p0 = p.p0, p1 = p.p1, p2 = p.p2;
  if (r.n_axes == 1) {
    const float* t = r.table + (long)p0 * (2 * r.half) + ln.pair0;  // 16-byte aligned
    const float4 c = *reinterpret_cast<const float4*>(t), s = *reinterpret_cast<const float4*>(t + r.half);
    A.c[0] = c.x; A.c[1] = c.y; A.c[2] = c.z; A.c[3] = c.w;
    A.s[0] = s.x; A.s[1] = s.y; A.s[2] = s.z; A.s[3] = s.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = ln.pair0 + e;
      const int at = i < r.axis1 ? p0 : (i < r.axis2 ? p1 : p2);
      const float* t = r.table + (long)at * (2 * r.half) + i;
      A.c[e] = t[0];
      A.s[e] = t[r.half];
    }
  }
}

// The lane's eight elements, rotated in place.
__device__ __forceinline__ void rotate(const RopeArgs& r, const Lane& ln, const Angles& A, float (&x)[8]) {
  if (!ln.turn) return;
  if (r.interleaved) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float a = x[2 * e], b = x[2 * e + 1];
      x[2 * e] = a * A.c[e] - b * A.s[e];
      x[2 * e + 1] = b * A.c[e] + a * A.s[e];
    }
    asm volatile("");  // (else the two orders are merged into one that indexes x in memory)
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float a = x[e], b = x[4 + e];
      x[e] = a * A.c[e] - b * A.s[e];
      x[4 + e] = b * A.c[e] + a * A.s[e];
    }
  }
}

// Rows [r0, r1) of one token, four at a time with 16 lanes each, kRows in flight per lane:
// those below n_turned are rotated.  begin() requests the first ones, which may come before
// the token's place and angles are known.
template <typename T, int kRows, bool kStream>
struct Mover {
  Row8<T> w[kRows];
  template <typename Src>
  __device__ __forceinline__ void begin(const Lane& ln, int r, int r1, Src src) {
#pragma unroll
    for (int u = 0; u < kRows; ++u) w[u].template load<kStream>(src(min(r + 4 * u, r1 - 1)), ln.a, ln.b);
  }
  template <typename Src, typename Dst>
  __device__ __forceinline__ void move(const RopeArgs& rope, const Lane& ln, const Angles& A, int tg, int r0,
                                       int r1, int n_turned, Src src, Dst dst) {
    for (int r = r0;; r += 4 * kRows) {
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int ru = r + tg + 4 * u;
        Row8<T> y = w[u];
        if (ru < n_turned && ln.turn) {
          float x[8];
          y.to(x);
          rotate(rope, ln, A, x);
          y.from(x);
        }
        if (ru < r1) y.template store<kStream>(dst(ru), ln.a, ln.b);
      }
      if (r + 4 * kRows >= r1) return;
      begin(ln, r + tg + 4 * kRows, r1, src);
    }
  }
};

}  // namespace
}  // namespace locks
