// Device pieces shared by the appends: which sequence a row belongs to, the rotation of a
// row spread over 16 lanes, and the rotated copy of query (and key, value) rows.
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

// Two floats to bf16 bits, round to nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2v{a, b}, bf2v));
}

// Eight consecutive elements of a row: as stored, as floats, and back.
template <typename T>
struct Row8;
template <>
struct Row8<uint16_t> {
  uint4 w;
  __device__ __forceinline__ void load(const uint16_t* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<uint4*>(p) = w; }
  __device__ __forceinline__ void to(float (&x)[8]) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(u[e] << 16);
      x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void from(const float (&x)[8]) {
    w = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]),
                   pack_bf16(x[6], x[7]));
  }
  __device__ __forceinline__ Row8 at_lane(int l) const {
    Row8 r;
    r.w = make_uint4(__shfl(w.x, l, 64), __shfl(w.y, l, 64), __shfl(w.z, l, 64), __shfl(w.w, l, 64));
    return r;
  }
};
template <>
struct Row8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<float4*>(p)[0] = a;
    reinterpret_cast<float4*>(p)[1] = b;
  }
  __device__ __forceinline__ void to(float (&x)[8]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  __device__ __forceinline__ void from(const float (&x)[8]) {
    a = make_float4(x[0], x[1], x[2], x[3]);
    b = make_float4(x[4], x[5], x[6], x[7]);
  }
  __device__ __forceinline__ Row8 at_lane(int l) const {
    Row8 r;
    r.a = make_float4(__shfl(a.x, l, 64), __shfl(a.y, l, 64), __shfl(a.z, l, 64), __shfl(a.w, l, 64));
    r.b = make_float4(__shfl(b.x, l, 64), __shfl(b.y, l, 64), __shfl(b.z, l, 64), __shfl(b.w, l, 64));
    return r;
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

// Angles of the eight elements that a lane holds of one token's rows.
// Element e becomes x[e] * c[e] + partner[e] * s[e], the partner's sign in s.
struct Angles {
  float c[8], s[8];
};
// Lane cg of 16 holds elements 8 cg .. 8 cg + 7.  Returns false where a position lies
// outside the table (the same for the 16 lanes).
__device__ __forceinline__ bool load_angles(const RopeArgs& r, int row, int tok, int cg, Angles& A) {
  if (r.half == 0) return true;
  int p0 = tok, p1 = tok, p2 = tok;
  if (r.positions) {
    p0 = p1 = p2 = r.positions[row];
    if (r.n_axes > 1) p1 = p2 = r.positions[(long)r.n_tokens + row];
    if (r.n_axes > 2) p2 = r.positions[2 * (long)r.n_tokens + row];
  }
  if ((unsigned)p0 >= (unsigned)r.n_pos || (unsigned)p1 >= (unsigned)r.n_pos || (unsigned)p2 >= (unsigned)r.n_pos)
    return false;
  if (8 * cg >= 2 * r.half) return true;
  auto at = [&](int i) {  // row of the table that pair i reads
    return r.table + (long)(i < r.axis1 ? p0 : (i < r.axis2 ? p1 : p2)) * (2 * r.half) + i;
  };
  if (r.interleaved) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float* t = at(4 * cg + e);
      A.c[2 * e] = A.c[2 * e + 1] = t[0];
      const float s = t[r.half];
      A.s[2 * e] = -s;
      A.s[2 * e + 1] = s;
    }
  } else {
    const bool first = 8 * cg < r.half;
    const int i0 = 8 * cg - (first ? 0 : r.half);
    if (r.n_axes == 1) {  // 32-byte aligned: half is a multiple of 8
      const float4* t = reinterpret_cast<const float4*>(at(i0));
      const float4* u = reinterpret_cast<const float4*>(at(i0) + r.half);
      const float4 c0 = t[0], c1 = t[1], s0 = u[0], s1 = u[1];
      const float cs[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
      const float ss[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        A.c[e] = cs[e];
        A.s[e] = first ? -ss[e] : ss[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float* t = at(i0 + e);
        A.c[e] = t[0];
        const float s = t[r.half];
        A.s[e] = first ? -s : s;
      }
    }
  }
  return true;
}

// The lane's eight elements of a row, rotated, as floats.  All 64 lanes take part.
template <typename T>
__device__ __forceinline__ void rotated(const RopeArgs& r, const Angles& A, const Row8<T>& w, int lane,
                                        float (&x)[8]) {
  const int cg = lane & 15, h8 = r.half >> 3;
  const bool turn = 8 * cg < 2 * r.half;
  w.to(x);
  if (r.interleaved) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float a = x[e], b = x[e + 1];
      if (turn) {
        x[e] = a * A.c[e] + b * A.s[e];
        x[e + 1] = b * A.c[e + 1] + a * A.s[e + 1];
      }
    }
  } else {
    const int other = turn ? (cg < h8 ? lane + h8 : lane - h8) : lane;
    float y[8];
    w.at_lane(other).to(y);
    if (turn) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = x[e] * A.c[e] + y[e] * A.s[e];
    }
  }
}

}  // namespace
}  // namespace locks
