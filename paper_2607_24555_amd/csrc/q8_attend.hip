// Decode attention over a paged cache held in 8 bits (locks_q8_dense_attend,
// locks_q8_sparse_attend): with ck, cv the codes and sk, sv the scales of token i's page,
//   o_g = sum_i softmax_i(sk q_g^T ck_i / sqrt d) sv cv_i
// over the listed pages' tokens (page_ids == nullptr: every page).
//
// Split-K as in the bf16 kernel: block (split, KV head, seq), four waves with consecutive
// units (16 tokens) of the list, one partial (o, max, sum) a block, merged afterwards.  A wave
// takes two units a step on the matrix cores and holds the next two units' codes in flight.
// Codes are exact in bf16 (int8: 7 bits and sign; e4m3: 4 bits), so the products with a bf16
// query are too; the key scale multiplies the logits, the value scale the weights, which enter
// as bf16 hi + lo.  fp32 queries enter as three bf16 terms (24 bits).
#include "cache_internal.h"

namespace locks {
namespace {

typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
typedef float f2v __attribute__((ext_vector_type(2)));
typedef float f4v __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2v{a, b}, bf2v));
}
__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ bf8v as_bf8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf8v, make_uint4(a, b, c, d));
}

// Four codes (one word) as two words of bf16 pairs, in order.
template <int kCode>
__device__ __forceinline__ void widen(uint32_t w, uint32_t& a, uint32_t& b) {
  if constexpr (kCode == LOCKS_Q8_INT8) {
    // small integers: the upper halves of their floats are their bf16 values
    const uint32_t f0 = __float_as_uint((float)(int8_t)w), f1 = __float_as_uint((float)(int8_t)(w >> 8));
    const uint32_t f2 = __float_as_uint((float)(int8_t)(w >> 16)), f3 = __float_as_uint((float)((int32_t)w >> 24));
    a = __builtin_amdgcn_perm(f1, f0, 0x07060302u);
    b = __builtin_amdgcn_perm(f3, f2, 0x07060302u);
  } else {
    a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
    b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
  }
}

// Codes of four tokens (words t0 .. t3 hold four elements each) as, per element e, the
// bf16 pairs (t0, t1) in p[e] and (t2, t3) in q[e].
template <int kCode>
__device__ __forceinline__ void widen_across(uint32_t t0, uint32_t t1, uint32_t t2, uint32_t t3,
                                             uint32_t (&p)[4], uint32_t (&q)[4]) {
  if constexpr (kCode == LOCKS_Q8_INT8) {
    const uint32_t t[4] = {t0, t1, t2, t3};
    uint32_t f[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) f[j][e] = __float_as_uint((float)(int8_t)(t[j] >> (8 * e)));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      p[e] = __builtin_amdgcn_perm(f[1][e], f[0][e], 0x07060302u);
      q[e] = __builtin_amdgcn_perm(f[3][e], f[2][e], 0x07060302u);
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

// Codes of two units.  Lane (c = l % 16, r = l / 16):
//   k[u][a]: token c, dims 64 a + 16 r .. + 15      v[u][j]: token 4 r + j, dims 8 c .. + 7
struct Codes {
  uint4 k[2][2];
  uint2 v[2][4];
};

// Lane layout (l = 16 r + c):
//   S^T = K Q^T  (mfma 16x16x32, M = token, N = head; step 2 a + b holds dims
//                 64 a + 16 r + 8 b + e): lane holds S^T[4 r + j][c] of each unit
//   O^T += V^T P (mfma 16x16x32, M = dim, N = head, K = (r, 4 u + j) = token 4 r + j of
//                 unit u; tile n covers dims 8 m + n): P is the B operand exactly as S^T
//                 left it, and lane holds O^T for head c, dims 32 r + 8 j + n.
template <typename QT, int kCode>
__global__ __launch_bounds__(256) void q8_attend_kernel(
    int H_q, int H_kv, int max_pages, int k_list, int pgsz, int lg_sub, const QT* __restrict__ q,
    const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ v_codes,
    const float* __restrict__ k_scale, const float* __restrict__ v_scale,
    const int32_t* __restrict__ page_table, const int32_t* __restrict__ seq_lens,
    const int32_t* __restrict__ page_ids, int units_per_split, int n_splits,
    float* __restrict__ partial, float* __restrict__ out, float* __restrict__ out_lse) {
  constexpr int kTerms = sizeof(QT) == 2 ? 1 : 3;
  __shared__ float sO[4][kDim][kMaxGroup + 1];
  __shared__ float sM[4][kMaxGroup], sL[4][kMaxGroup];
  const int split = blockIdx.x, h = blockIdx.y, s = blockIdx.z;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int c16 = lane & 15, r4 = lane >> 4;
  const int G = H_q / H_kv;
  const int L = seq_lens[s];
  const int n = (L + pgsz - 1) / pgsz;
  const int upw = units_per_split / 4;  // units per wave, at most 64
  const int t_begin = split * units_per_split + wave * upw;

  // ---- lane j: the wave's unit j (first token, or -1: nothing to attend), its codes and scales
  int my_tok = -1, my_blk = 0;
  float my_ks = 0.0f, my_vs = 0.0f;
  if (lane < upw) {
    const int t = t_begin + lane, entry = t >> lg_sub;
    int id = entry;
    if (page_ids) id = entry < k_list ? page_ids[((long)s * H_kv + h) * k_list + entry] : -1;
    if (id >= 0 && id < n) {
      const int tok0 = id * pgsz + (t & ((1 << lg_sub) - 1)) * kPage;
      if (tok0 < L) {
        my_tok = tok0;
        my_blk = page_table[(long)s * max_pages + id];
        my_ks = k_scale[(long)my_blk * H_kv + h] * (kLog2e / 11.313708498984761f);  // / sqrt(128)
        my_vs = v_scale[(long)my_blk * H_kv + h];
      }
    }
  }
  const unsigned long long live = __ballot(my_tok >= 0);
  const int cnt = live ? 64 - __clzll(live) : 0;  // units up to the last one with tokens
  // an empty unit's loads read another unit of the wave
  const int spare = live ? __ffsll((unsigned long long)live) - 1 : 0;

  // ---- queries: B operand of step 2 a + b, in kTerms bf16 terms
  uint4 qb[kTerms][4];
  {
    const QT* row = q + ((long)s * H_q + h * G + min(c16, G - 1)) * kDim + 16 * r4;
#pragma unroll
    for (int st = 0; st < 4; ++st) {
      const QT* p = row + 64 * (st >> 1) + 8 * (st & 1);
      if constexpr (kTerms == 1) {
        qb[0][st] = *reinterpret_cast<const uint4*>(p);
      } else {
        const float4 x0 = reinterpret_cast<const float4*>(p)[0], x1 = reinterpret_cast<const float4*>(p)[1];
        float x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
#pragma unroll
        for (int m = 0; m < kTerms; ++m) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            w[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
            x[2 * e] -= lo_f(w[e]);
            x[2 * e + 1] -= hi_f(w[e]);
          }
          qb[m][st] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
    }
  }

  const long page_bytes = (long)pgsz * kDim;
  const int k_off = c16 * kDim + 16 * r4, v_off = 4 * r4 * kDim + 8 * c16;
  auto load_pair = [&](Codes& C, int j) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int i = j + u < cnt && ((live >> (j + u)) & 1) ? j + u : spare;
      const long blk = __builtin_amdgcn_readlane(my_blk, i);
      const int tok0 = __builtin_amdgcn_readlane(my_tok, i);
      const long base = (blk * H_kv + h) * page_bytes + (long)(tok0 & (pgsz - 1)) * kDim;
      const uint8_t* kp = k_codes + base + k_off;
      const uint8_t* vp = v_codes + base + v_off;
#pragma unroll
      for (int a = 0; a < 2; ++a) C.k[u][a] = *reinterpret_cast<const uint4*>(kp + 64 * a);
#pragma unroll
      for (int t = 0; t < 4; ++t) C.v[u][t] = *reinterpret_cast<const uint2*>(vp + t * kDim);
    }
  };

  float m = -INFINITY, l = 0.0f;  // l: this lane's tokens only
  f4v o[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) o[t] = f4v{0.0f, 0.0f, 0.0f, 0.0f};

  auto use_pair = [&](Codes& C, int j) {
    float z[2][4], vs[2];
    int valid[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int i = min(j + u, 63);
      const int tok0 = __builtin_amdgcn_readlane(my_tok, i);
      valid[u] = j + u < cnt && tok0 >= 0 ? min(kPage, L - tok0) : 0;
      const float ks = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_ks), i));
      vs[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_vs), i));
      f4v st = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const uint32_t w[4] = {C.k[u][a].x, C.k[u][a].y, C.k[u][a].z, C.k[u][a].w};
        uint32_t b[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) widen<kCode>(w[e], b[2 * e], b[2 * e + 1]);
#pragma unroll
        for (int mt = kTerms - 1; mt >= 0; --mt) {
          st = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf8(b[0], b[1], b[2], b[3]),
                                                       __builtin_bit_cast(bf8v, qb[mt][2 * a]), st, 0, 0, 0);
          st = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf8(b[4], b[5], b[6], b[7]),
                                                       __builtin_bit_cast(bf8v, qb[mt][2 * a + 1]), st, 0, 0, 0);
        }
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) z[u][t] = st[t] * ks;
      if (valid[u] < kPage) {  // uniform: an empty or partial unit; its codes may be anything
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (4 * r4 + t >= valid[u]) {
            z[u][t] = -INFINITY;
            C.v[u][t] = make_uint2(0u, 0u);
          }
        if (valid[u] == 0) vs[u] = 0.0f;
      }
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
      for (int t = 0; t < 2; ++t) {
        const float p0 = __builtin_amdgcn_exp2f(z[u][2 * t] - at), p1 = __builtin_amdgcn_exp2f(z[u][2 * t + 1] - at);
        ps += p0 + p1;
        const float w0 = p0 * vs[u], w1 = p1 * vs[u];
        ph[2 * u + t] = pack_bf16(w0, w1);
        pl[2 * u + t] = pack_bf16(w0 - lo_f(ph[2 * u + t]), w1 - hi_f(ph[2 * u + t]));
      }
    l = fmaf(l, sc, ps);
    if (__any(sc != 1.0f)) {
#pragma unroll
      for (int t = 0; t < 8; ++t) o[t] *= sc;
    }
    const bf8v bh = as_bf8(ph[0], ph[1], ph[2], ph[3]), bl = as_bf8(pl[0], pl[1], pl[2], pl[3]);
#pragma unroll
    for (int half = 0; half < 2; ++half) {  // dims 8 m + 4 half + e
      uint32_t p[2][4], r[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u)
        widen_across<kCode>(half ? C.v[u][0].y : C.v[u][0].x, half ? C.v[u][1].y : C.v[u][1].x,
                            half ? C.v[u][2].y : C.v[u][2].x, half ? C.v[u][3].y : C.v[u][3].x, p[u], r[u]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bf8v a = as_bf8(p[0][e], r[0][e], p[1][e], r[1][e]);
        const int t = 4 * half + e;
        o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, bh, o[t], 0, 0, 0);
        o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, bl, o[t], 0, 0, 0);
      }
    }
  };

  if (cnt > 0) {
    Codes A, B;
    load_pair(A, 0);
    for (int j = 0; j < cnt; j += 4) {
      load_pair(B, j + 2);
      use_pair(A, j);
      load_pair(A, j + 4);
      if (j + 2 < cnt) use_pair(B, j + 2);
    }
  }

  // ---- the block's four waves combined (m in log2 units until here); the odd row pitch of
  // sO keeps the layout's writes and the reads along d free of bank conflicts
  l = rows_sum(l);
  if (r4 == 0) { sM[wave][c16] = m; sL[wave][c16] = l; }
#pragma unroll
  for (int t = 0; t < 8; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) sO[wave][32 * r4 + 8 * j + t][c16] = o[t][j];
  __syncthreads();
  for (int e = tid; e < G * (kDim + 2); e += 256) {
    const int g = e / (kDim + 2), c = e % (kDim + 2);
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sM[w][g]);
    float acc = 0.0f, ls = 0.0f;
    if (mx > -INFINITY) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float wt = __builtin_amdgcn_exp2f(sM[w][g] - mx);
        ls += sL[w][g] * wt;
        if (c < kDim) acc += sO[w][c][g] * wt;
      }
    }
    const float mn = mx == -INFINITY ? mx : mx * kLn2;
    const long row = (long)s * H_q + h * G + g;
    if (n_splits == 1) {
      if (c < kDim) out[row * kDim + c] = ls > 0.0f ? acc / ls : 0.0f;
      else if (c == kDim && out_lse) out_lse[row] = ls > 0.0f ? mn + logf(ls) : -INFINITY;
    } else {
      partial[(row * n_splits + split) * (kDim + 2) + c] = c < kDim ? acc : (c == kDim ? mn : ls);
    }
  }
}

}  // namespace

hipError_t launch_q8_attend(const locks_cfg_t& c, const void* q, const locks_q8_t& cache,
                            const int32_t* page_table, const int32_t* seq_lens,
                            const int32_t* page_ids, int units_per_split, int n_splits,
                            float* partial, float* out, float* out_lse, hipStream_t st) {
  const dim3 grid(n_splits, c.num_kv_heads, c.num_seqs);
#define LOCKS_Q8_ATTEND(QT, C)                                                                  \
  hipLaunchKernelGGL((q8_attend_kernel<QT, C>), grid, dim3(256), 0, st, c.num_q_heads,           \
                     c.num_kv_heads, c.max_pages_per_seq, page_budget(c), c.page_size,          \
                     sub_page_log2(c), static_cast<const QT*>(q),                               \
                     static_cast<const uint8_t*>(cache.k), static_cast<const uint8_t*>(cache.v), \
                     cache.k_scale, cache.v_scale, page_table, seq_lens, page_ids,              \
                     units_per_split, n_splits, partial, out, out_lse)
  if (c.q_dtype == LOCKS_BF16) {
    if (cache.code == LOCKS_Q8_INT8) LOCKS_Q8_ATTEND(uint16_t, LOCKS_Q8_INT8);
    else LOCKS_Q8_ATTEND(uint16_t, LOCKS_Q8_E4M3);
  } else {
    if (cache.code == LOCKS_Q8_INT8) LOCKS_Q8_ATTEND(float, LOCKS_Q8_INT8);
    else LOCKS_Q8_ATTEND(float, LOCKS_Q8_E4M3);
  }
#undef LOCKS_Q8_ATTEND
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || n_splits == 1) return e;
  return launch_merge(c, n_splits, partial, out, out_lse, st);
}

}  // namespace locks
