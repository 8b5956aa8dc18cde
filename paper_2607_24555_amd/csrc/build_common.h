// Pieces shared by the summary builds: key conversion, quantisers, the zero-mode floor.
#pragma once

#include "locks_internal.h"

namespace locks {
namespace {

constexpr float kZeroRel = 1e-6f;
constexpr float kZeroAbs = 1e-10f;

// Elements of a 16-byte chunk of bf16 or fp32 keys as floats.
template <typename KT>
__device__ __forceinline__ void chunk_to_f(const uint4& w, float* out);
template <>
__device__ __forceinline__ void chunk_to_f<uint16_t>(const uint4& w, float* out) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    out[2 * e] = __uint_as_float(u[e] << 16);
    out[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
  }
}
template <>
__device__ __forceinline__ void chunk_to_f<float>(const uint4& w, float* out) {
  out[0] = __uint_as_float(w.x); out[1] = __uint_as_float(w.y);
  out[2] = __uint_as_float(w.z); out[3] = __uint_as_float(w.w);
}

// Where a build's keys come from: a cache of bf16 or fp32, or 8-bit codes of a page with its
// scale, which count as the fp32 keys code * scale.
struct Int8Codes { uint8_t bits; };
struct E4m3Codes { uint8_t bits; };
// The keys of a word of codes.  The product is rounded, whatever is done with it: no
// contraction.
template <typename ST>
__device__ __forceinline__ void codes_to_f(uint32_t w, float scale, float* out) {
#pragma clang fp contract(off)
  float x[4];
  if constexpr (__is_same(ST, Int8Codes)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (float)(int8_t)(w >> (8 * e));
  } else {
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
    x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
    x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = x[e] * scale;
}
// Elements of a chunk (16 bytes, of codes also 8) as floats; scale: of codes only.
template <typename ST, typename W>
__device__ __forceinline__ void keys_to_f(const W& w, float scale, float* out) {
  if constexpr (sizeof(ST) > 1) {
    chunk_to_f<ST>(w, out);
  } else {
    codes_to_f<ST>(w.x, scale, out);
    codes_to_f<ST>(w.y, scale, out + 4);
    if constexpr (sizeof(W) == 16) {
      codes_to_f<ST>(w.z, scale, out + 8);
      codes_to_f<ST>(w.w, scale, out + 12);
    }
  }
}
// Four fp32 keys from the codes at element `at` of the cache.
template <typename ST>
__device__ __forceinline__ uint4 load_codes(const ST* cache, long at, float scale) {
  float x[4];
  codes_to_f<ST>(*reinterpret_cast<const uint32_t*>(cache + at), scale, x);
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                    __float_as_uint(x[3]));
}

__device__ __forceinline__ float f16_scale(float amax, float qmax) {
  float s = fminf(amax / qmax, 65504.0f);
  return (float)(_Float16)s;
}

// 1 / s for a code scale s (0 when s is 0: every code is then 0)
__device__ __forceinline__ float inv_scale(float s) { return s > 0.0f ? 1.0f / s : 0.0f; }
// code of x at scale 1 / inv: nearest integer, clamped to +-qmax (x inv may differ
// from x / s in the last bit, which moves a code only at an exact half)
__device__ __forceinline__ int quant(float x, float inv, int qmax) {
  float c = rintf(x * inv);
  c = fminf(fmaxf(c, (float)-qmax), (float)qmax);
  return (int)c;
}

// code of x at scale s by a correctly rounded division
__device__ __forceinline__ int quant_div(float x, float s, int qmax) {
  if (!(s > 0.0f)) return 0;
  return (int)fminf(fmaxf(rintf(x / s), (float)-qmax), (float)qmax);
}

// Nearest bfloat16 (ties to even) of a finite float, as its 16-bit pattern.
__device__ __forceinline__ uint32_t bf16_rne_bits(float f) {
  const uint32_t u = __float_as_uint(f);
  return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

__device__ __forceinline__ uint16_t f16_bits(float s) {
  _Float16 h = (_Float16)s;
  return *reinterpret_cast<uint16_t*>(&h);
}

}  // namespace
}  // namespace locks
