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
template <typename T>
struct Row8;
template <>
struct Row8<uint16_t> {
  u2v lo, hi;
  __device__ __forceinline__ void load(const uint16_t* p, int a, int b) {
    lo = *reinterpret_cast<const u2v*>(p + a);
    hi = *reinterpret_cast<const u2v*>(p + b);
  }
  __device__ __forceinline__ void store(uint16_t* p, int a, int b) const {
    *reinterpret_cast<u2v*>(p + a) = lo;
    *reinterpret_cast<u2v*>(p + b) = hi;
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
  __device__ __forceinline__ void load(const float* p, int a, int b) {
    lo = *reinterpret_cast<const f4v*>(p + a);
    hi = *reinterpret_cast<const f4v*>(p + b);
  }
  __device__ __forceinline__ void store(float* p, int a, int b) const {
    *reinterpret_cast<f4v*>(p + a) = lo;
    *reinterpret_cast<f4v*>(p + b) = hi;
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
  int row0, n, tok0;
};
__device__ __forceinline__ NewTokens new_tokens(const RowArgs& a, const int32_t* seq_lens, int s) {
  const int L = seq_lens[s];
  if (!a.cu) return NewTokens{s, L > 0 ? 1 : 0, L - 1};
  const int r0 = a.cu[s], r1 = min(a.cu[s + 1], a.n_tokens);
  const int n = r0 >= 0 && r1 > r0 ? r1 - r0 : 0;
  return NewTokens{r0, n, L - n};
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
// The lane's angles for the token of a row.  Returns false where a position lies outside the
// table (the same for all lanes of the token).
__device__ __forceinline__ bool load_angles(const RopeArgs& r, const Lane& ln, int row, int tok, Angles& A) {
  if (r.half == 0) return true;
  int p0 = tok, p1 = tok, p2 = tok;
  if (r.positions) {
    p0 = p1 = p2 = r.positions[row];
    if (r.n_axes > 1) p1 = p2 = r.positions[(long)r.n_tokens + row];
    if (r.n_axes > 2) p2 = r.positions[2 * (long)r.n_tokens + row];
  }
  if ((unsigned)p0 >= (unsigned)r.n_pos || (unsigned)p1 >= (unsigned)r.n_pos || (unsigned)p2 >= (unsigned)r.n_pos)
    return false;
  if (!ln.turn) return true;
  if (r.n_axes == 1) {
    const float* t = r.table + (long)p0 * (2 * r.half) + ln.pair0;  // 16-byte aligned
    const float4 c = *reinterpret_cast<const float4*>(t), s = *reinterpret_cast<const float4*>(t + r.half);
    A.c[0] = c.x; A.c[1] = c.y; A.c[2] = c.z; A.c[3] = c.w;
    A.s[0] = s.x; A.s[1] = s.y; A.s[2] = s.z; A.s[3] = s.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = ln.pair0 + e;
      const float* t = r.table + (long)(i < r.axis1 ? p0 : (i < r.axis2 ? p1 : p2)) * (2 * r.half) + i;
      A.c[e] = t[0];
      A.s[e] = t[r.half];
    }
  }
  return true;
}

// The lane's eight elements, rotated in place.  (Elements are picked by value: with the two
// orders as branches the compiler merges them into one that indexes x from memory.)
__device__ __forceinline__ void rotate(const RopeArgs& r, const Lane& ln, const Angles& A, float (&x)[8]) {
  if (!ln.turn) return;
  const bool il = r.interleaved;
  const float x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3], x4 = x[4], x5 = x[5], x6 = x[6], x7 = x[7];
  const float a[4] = {x0, il ? x2 : x1, il ? x4 : x2, il ? x6 : x3};
  const float b[4] = {il ? x1 : x4, il ? x3 : x5, il ? x5 : x6, x7};
  float u[4], w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    u[e] = a[e] * A.c[e] - b[e] * A.s[e];
    w[e] = b[e] * A.c[e] + a[e] * A.s[e];
  }
  x[0] = u[0];
  x[1] = il ? w[0] : u[1];
  x[2] = il ? u[1] : u[2];
  x[3] = il ? w[1] : u[3];
  x[4] = il ? u[2] : w[0];
  x[5] = il ? w[2] : w[1];
  x[6] = il ? u[3] : w[2];
  x[7] = w[3];
}

// Rows [r0, r1) of one token, four at a time with 16 lanes each, kRows in flight per lane:
// those below n_turned are rotated.  begin() requests the first ones, which may come before
// the token's place and angles are known.
template <typename T, int kRows>
struct Mover {
  Row8<T> w[kRows];
  template <typename Src>
  __device__ __forceinline__ void begin(const Lane& ln, int r, int r1, Src src) {
#pragma unroll
    for (int u = 0; u < kRows; ++u) w[u].load(src(min(r + 4 * u, r1 - 1)), ln.a, ln.b);
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
        if (ru < r1) y.store(dst(ru), ln.a, ln.b);
      }
      if (r + 4 * kRows >= r1) return;
      begin(ln, r + tg + 4 * kRows, r1, src);
    }
  }
};

}  // namespace
}  // namespace locks
