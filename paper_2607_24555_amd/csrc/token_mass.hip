// The attention weight that every cached token gets from the new ones, added to what it had:
//   mass_t = decay mass_t + sum_{i sees t, g} exp(q_ig . k_t / sqrt d - lse_ig).
//
// A wave keeps the keys of 32 kGroups tokens in registers and goes through the rows
// r = i G + g in chunks of 32, whose queries the block's four waves read from LDS:
//   S = Q K^T   (M = row, N = token), whose result has a token per lane column, so that a
//               token's sum needs no lane until the last swap.
// Every key is read once whatever the number of rows, all of a wave's keys are requested
// before the first is used, and the order of a sum is that of the rows.  The units
// (128 kGroups tokens of a sequence and KV head) of up to kSeqs sequences are counted on the
// device, so that a wide table of short sequences costs what its tokens cost.
#include <type_traits>

#include "tokens_internal.h"

namespace locks {
namespace {

constexpr int kSeqs = 512;          // sequences whose units are counted on the device
constexpr int kMassBlocks = 2048;

// kF32: products in fp32 (32x32x2 MFMA), else bf16 (32x32x16).
template <bool kF32, typename TQ, typename TK>
__global__ __launch_bounds__(256, 2) void mass_kernel(DraftArgs a, const float* __restrict__ lse,
                                                      const TK* __restrict__ k_cache, float decay,
                                                      float* __restrict__ mass, int bound_units) {
  constexpr int kGroups = kF32 ? 2 : 4, kUnit = 128 * kGroups;
  constexpr int kRow = kF32 ? 132 * 4 : 256;   // bytes of a query in LDS
  __shared__ __align__(16) unsigned char s_q[2][32 * kRow];
  __shared__ float s_nl[2][32];                // -lse log2 e; -inf: adds nothing
  __shared__ int s_i[2][32];                   // the row's token
  __shared__ long s_units[kSeqs + 1], s_sum[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;
  const float zs = kLog2e / sqrtf((float)kDim);
  const int lgP = a.pgsz == 64 ? 6 : a.pgsz == 32 ? 5 : 4;

  // ---- the units of sequence s: none without new tokens
  auto units_of = [&](int s) {
    const int2 rows = draft_rows(a, s);
    return rows.y > rows.x ? (draft_len(a, s) + kUnit - 1) / kUnit : 0;
  };
  long total = (long)bound_units * a.H * a.S;
  const bool counted = a.S <= kSeqs;
  if (counted) {
    constexpr int kPer = kSeqs / 256;
    long before[kPer], v = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      before[e] = v;
      if (tid * kPer + e < a.S) v += units_of(tid * kPer + e);
    }
    const long at = scan256(v, s_sum, total);
#pragma unroll
    for (int e = 0; e < kPer; ++e) s_units[tid * kPer + e] = at + before[e];
    if (tid == 0) s_units[kSeqs] = total;
    __syncthreads();
    total *= a.H;
  }

  for (long x = blockIdx.x; x < total; x += gridDim.x) {
    int s, h, u;
    if (counted) {
      int lo = 0, hi = a.S;
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (s_units[mid] * a.H <= x) lo = mid;
        else hi = mid;
      }
      const int per = (int)(s_units[lo + 1] - s_units[lo]);
      const long in = x - s_units[lo] * a.H;
      s = lo, h = (int)(in / per), u = (int)(in % per);
    } else {
      s = (int)(x / ((long)bound_units * a.H)), h = (int)(x / bound_units % a.H), u = (int)(x % bound_units);
      if (u >= units_of(s)) continue;
    }
    s = __builtin_amdgcn_readfirstlane(s), h = __builtin_amdgcn_readfirstlane(h);
    u = __builtin_amdgcn_readfirstlane(u);
    const int2 rows = draft_rows(a, s);
    const int n = rows.y - rows.x, L = draft_len(a, s), first = L - n, count = n * a.G;

    // ---- this wave's keys: lane (col, half) has token t0 + 32 g + col, dimensions
    // 16 ks + 8 half + 0 .. 7 (or 8 u + 4 half + 0 .. 3)
    const int t0 = u * kUnit + wave * 32 * kGroups;
    int blk[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
      blk[g] = a.page_table[(long)s * a.max_pages + (min(t0 + 32 * g + col, L - 1) >> lgP)];
    using Raw = typename std::conditional<kF32 && sizeof(TK) == 2, u2, u4>::type;
    constexpr int kLoads = kF32 ? 16 : 8;
    Raw kr[kGroups][kLoads];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int t = min(t0 + 32 * g + col, L - 1);
      const long b = (unsigned)blk[g] < (unsigned)a.num_blocks ? blk[g] : 0;
      const TK* p = k_cache + ((b * a.H + h) * a.pgsz + (t & (a.pgsz - 1))) * kDim + (kF32 ? 4 : 8) * half;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) kr[g][j] = *reinterpret_cast<const Raw*>(p + (kF32 ? 8 : 16) * j);
    }
    float* const m = mass + ((long)s * a.H + h) * a.max_pages * a.pgsz;
    float old[kGroups], sum[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int t = t0 + 32 * g + col;
      old[g] = t < first ? m[t] : 0.0f;
      sum[g] = 0.0f;
    }

    // ---- rows in chunks of 32; eight threads stage a row
    const int rr = tid >> 3, seg = tid & 7;
    u4 qr[kF32 && sizeof(TQ) == 4 ? 4 : 2];
    float nl_next = 0.0f;
    int i_next = 0;
    auto request = [&](int c) {
      const int r = 32 * c + rr;
      const bool there = r < count;
      const int i = there ? r / a.G : 0, hq = h * a.G + (there ? r % a.G : 0);
      const TQ* q = static_cast<const TQ*>(a.q) + (long)(rows.x + i) * a.q_stride + hq * kDim;
      const u4 none = {};
#pragma unroll
      for (int e = 0; e < (int)(sizeof(qr) / 16); ++e) {
        // pieces of 16 bytes, seg + 8 e
        const u4 w = *reinterpret_cast<const u4*>(q + (16 / sizeof(TQ)) * (seg + 8 * e));
        qr[e] = there ? w : none;
      }
      const float l = lse[(long)(rows.x + i) * a.H * a.G + hq];
      nl_next = !there || l == -INFINITY ? -INFINITY : -l * kLog2e;
      i_next = i;
    };
    auto put = [&](int buf) {
      unsigned char* q = s_q[buf] + rr * kRow;
#pragma unroll
      for (int e = 0; e < (int)(sizeof(qr) / 16); ++e) {
        const int pc = seg + 8 * e;
        if constexpr (!kF32) {
          *reinterpret_cast<u4*>(q + 16 * (pc ^ piece_xor(rr))) = qr[e];
        } else if constexpr (sizeof(TQ) == 4) {
          *reinterpret_cast<u4*>(q + 16 * pc) = qr[e];
        } else {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const u4 w = {qr[e][2 * k] << 16, qr[e][2 * k] & 0xffff0000u, qr[e][2 * k + 1] << 16,
                          qr[e][2 * k + 1] & 0xffff0000u};
            *reinterpret_cast<u4*>(q + 32 * pc + 16 * k) = w;
          }
        }
      }
      if (seg == 0) {
        s_nl[buf][rr] = nl_next;
        s_i[buf][rr] = i_next;
      }
    };
    // (a run: rows before the unit's first token do not see it)
    const int c0 = a.mask ? 0 : max(0, u * kUnit - first) * a.G / 32, c1 = (count + 31) / 32;
    if (c0 < c1) {
      request(c0);
      __syncthreads();  // (the last unit's readers)
      put(c0 & 1);
    }
    for (int c = c0; c < c1; ++c) {
      const int buf = c & 1;
      if (c + 1 < c1) request(c + 1);
      __syncthreads();
      const int live = min(32, count - 32 * c);
      // element e of a product: row 8 (e / 4) + 4 half + e % 4 of the chunk
      float nl[16];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const float4 v = *reinterpret_cast<const float4*>(&s_nl[buf][8 * b + 4 * half]);
        nl[4 * b] = v.x, nl[4 * b + 1] = v.y, nl[4 * b + 2] = v.z, nl[4 * b + 3] = v.w;
      }
      auto weigh = [&](int g, const f16v& z) {
        const int t = t0 + 32 * g + col;
        const bool tail = t0 + 32 * g + 31 >= first;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          if (8 * b >= live) break;
#pragma unroll
          for (int e = 4 * b; e < 4 * b + 4; ++e) {
            const float w = __builtin_amdgcn_exp2f(fmaf(z[e], zs, nl[e]));
            bool sees = nl[e] != -INFINITY;
            if (tail) {
              const int i = s_i[buf][8 * b + 4 * half + e % 4];
              sees = sees && t < L && draft_sees(a, rows.x + i, i, t, first);
            }
            sum[g] += sees ? w : 0.0f;
          }
        }
      };
      f16v zero;
#pragma unroll
      for (int e = 0; e < 16; ++e) zero[e] = 0.0f;
      if constexpr (kF32) {
        f16v z[kGroups];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) z[g] = zero;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float4 q = *reinterpret_cast<const float4*>(s_q[buf] + col * kRow + 32 * j + 16 * half);
          const float qv[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
              float k;
              if constexpr (sizeof(TK) == 2)
                k = __uint_as_float(e & 1 ? kr[g][j][e / 2] & 0xffff0000u : kr[g][j][e / 2] << 16);
              else
                k = __uint_as_float(kr[g][j][e]);
              z[g] = __builtin_amdgcn_mfma_f32_32x32x2f32(qv[e], k, z[g], 0, 0, 0);
            }
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g) weigh(g, z[g]);
      } else {
        const int px = piece_xor(col) ^ half;
        u4 q[8];
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
          q[ks] = *reinterpret_cast<const u4*>(s_q[buf] + col * kRow + 16 * (px ^ (2 * ks)));
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          f16v z = zero;
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, q[ks]),
                                                        __builtin_bit_cast(bf8, kr[g][ks]), z, 0, 0, 0);
          weigh(g, z);
        }
      }
      if (c + 1 < c1) put(buf ^ 1);
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int t = t0 + 32 * g + col;
      auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum[g]), __float_as_uint(sum[g]), false, false);
      const float both = __uint_as_float(p[0]) + __uint_as_float(p[1]);
      if (half == 0 && t < L && (unsigned)blk[g] < (unsigned)a.num_blocks)
        m[t] = (t < first ? decay * old[g] : 0.0f) + both;
    }
  }
}

}  // namespace

hipError_t launch_token_mass(const locks_cfg_t& c, const DraftArgs& a, const float* lse,
                             const void* k_cache, float decay, float* mass, hipStream_t st) {
  const bool f32 = c.q_dtype != LOCKS_BF16 || c.kv_dtype != LOCKS_BF16;
  const int unit = f32 ? 256 : 512;
  const int units = (int)(((long)a.max_pages * a.pgsz + unit - 1) / unit);
  const long all = (long)units * a.H * a.S;
  const dim3 grid((unsigned)(all < kMassBlocks ? all : kMassBlocks)), block(256);
#define MASS(F32, TQ, TK)                                                                  \
  hipLaunchKernelGGL((mass_kernel<F32, TQ, TK>), grid, block, 0, st, a, lse,               \
                     static_cast<const TK*>(k_cache), decay, mass, units)
  if (!f32) MASS(false, uint16_t, uint16_t);
  else if (c.q_dtype == LOCKS_BF16) MASS(true, uint16_t, float);
  else if (c.kv_dtype == LOCKS_BF16) MASS(true, float, uint16_t);
  else MASS(true, float, float);
#undef MASS
  return hipGetLastError();
}

}  // namespace locks
