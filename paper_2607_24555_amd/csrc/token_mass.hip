// The attention weight that every cached token gets from the new ones, added to what it had:
//   mass_t = decay mass_t + sum_{i sees t, g} exp(q_ig . k_t / sqrt d - lse_ig).
//
// A wave keeps the keys of 32 tokens in registers and goes through the rows r = i G + g in
// chunks of 32, whose queries the block's four waves read from LDS:
//   S = Q K^T   (M = row, N = token), whose result has a token per lane column, so that a
//               token's sum needs no lane until the last swap.
// Every key is read once whatever the number of rows, two units ahead of its use, and the
// order of a sum is that of the rows.  The units (128 tokens of a sequence and KV head) of up
// to kSeqs sequences are counted on the device and cut into equal runs, one a block, so that a
// wide table of short sequences costs what its tokens cost; a run mostly stays with one KV
// head, whose queries then stay in LDS.  Of more sequences a block takes whole lists.
//
// Bound by HBM: 64 sequences of 1.5K to 8K tokens, 8 heads, a new token each: 128 us, 4.9 TB/s
// (a copy here 5.1).  Keys read in the product's order, 32 bytes of each of 32 rows a load, took
// 154.  With 128 rows (the last 32 tokens of prompts of 20K to 32K) 117 us, 3.7 TB/s: the vector
// work (16 powers a lane and 32 x 32 logits) is half of that and the products a fifth, but a wave
// does the three in turn, and two waves a SIMD do not hide all of it.  Among the new tokens a lane first has
// what its row sees of the 32 tokens, one window of the mask, and the tokens' lanes take their bits
// from it (15 trees of 34 to 104 tokens, eight heads a group, over up to 232: 44 us; with a mask
// load for each row and token 116).
#include <type_traits>

#include "tokens_internal.h"

namespace locks {
namespace {

constexpr int kSeqs = 512;          // sequences whose units are counted on the device
constexpr int kMassBlocks = 512;    // two per compute unit
constexpr int kManyRows = 128;      // of a sequence and KV head

// kF32: products in fp32 (32x32x2 MFMA), else bf16 (32x32x16).
template <bool kF32, typename TQ, typename TK>
__global__ __launch_bounds__(256, kF32 ? 1 : 2) void mass_kernel(DraftArgs a, const float* __restrict__ lse,
                                                      const TK* __restrict__ k_cache, float decay,
                                                      float* __restrict__ mass) {
  constexpr int kUnit = 128;
  constexpr int kSet = kF32 ? 64 : 128;        // rows in LDS at once
  constexpr int kRow = kF32 ? 132 * 4 : 256;   // bytes of a query in LDS
  __shared__ __align__(16) unsigned char s_q[kSet * kRow];
  __shared__ __align__(16) unsigned char s_k[kF32 ? 16 : 4 * 32 * 256];
  __shared__ __align__(16) float s_nl[kSet];   // -lse log2 e; -inf: adds nothing
  __shared__ int s_i[kSet];                    // the row's token
  __shared__ long s_units[kSeqs + 1], s_sum[4];
  __shared__ int s_row0[kSeqs], s_rows[kSeqs], s_len[kSeqs];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const float zs = kLog2e / sqrtf((float)kDim);
  const int lgP = a.pgsz == 64 ? 6 : a.pgsz == 32 ? 5 : 4;
  const bool counted = a.S <= kSeqs;

  // ---- a unit, and the one after it in this block's run
  struct Unit {
    int s, h, u, per;          // unit u of the list's `per`
    int row0, n, L;
  };
  auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  auto list_of = [&](Unit& w) {
    if (counted) {
      w.row0 = uniform(s_row0[w.s]), w.n = uniform(s_rows[w.s]), w.L = uniform(s_len[w.s]);
    } else {
      const int2 rows = draft_rows(a, w.s);
      w.row0 = uniform(rows.x), w.n = uniform(rows.y - rows.x), w.L = uniform(draft_len(a, w.s));
    }
    w.per = w.n > 0 ? (w.L + kUnit - 1) / kUnit : 0;  // none without new tokens
  };
  Unit cur{};
  long left = 0;  // units of the run (not counted: of the block's lists, unknown)
  long list = blockIdx.x;
  const long lists = (long)a.S * a.H;
  auto next_list = [&](Unit& w) {  // not counted: the first list from `list` on that has units
    for (; list < lists; list += gridDim.x) {
      Unit y;
      y.s = (int)(list / a.H), y.h = (int)(list % a.H), y.u = 0;
      list_of(y);
      if (y.per) {
        list += gridDim.x;
        w = y;
        return true;
      }
    }
    return false;
  };
  if (counted) {
    constexpr int kPer = kSeqs / 256;
    long before[kPer], v = 0, total;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int s = tid * kPer + e;
      before[e] = v;
      if (s < a.S) {
        const int2 rows = draft_rows(a, s);
        const int L = draft_len(a, s);
        s_row0[s] = rows.x, s_rows[s] = rows.y - rows.x, s_len[s] = L;
        v += rows.y > rows.x ? (L + kUnit - 1) / kUnit : 0;
      }
    }
    const long at = scan_block<4>(v, s_sum, total);
#pragma unroll
    for (int e = 0; e < kPer; ++e) s_units[tid * kPer + e] = at + before[e];
    if (tid == 0) s_units[kSeqs] = total;
    __syncthreads();
    total *= a.H;
    const long share = (total + gridDim.x - 1) / gridDim.x, x = blockIdx.x * share;
    left = min(total, x + share) - x;
    if (left <= 0) return;
    int lo = 0, hi = a.S;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (s_units[mid] * a.H <= x) lo = mid;
      else hi = mid;
    }
    cur.s = uniform(lo);
    list_of(cur);
    const unsigned in = (unsigned)(x - s_units[lo] * a.H);
    cur.h = uniform((int)(in / (unsigned)cur.per)), cur.u = uniform((int)(in % (unsigned)cur.per));
  } else if (!next_list(cur)) {
    return;
  }
  // the unit after w; false at the run's end (w is then left as it is, to be requested again)
  auto advance = [&](Unit& w) {
    if (counted && --left <= 0) return false;
    if (w.u + 1 < w.per) {
      ++w.u;
      return true;
    }
    if (!counted) return next_list(w);
    w.u = 0;
    if (++w.h == a.H) {
      w.h = 0;
      do ++w.s;
      while (s_rows[w.s] == 0 || s_len[w.s] == 0);  // (a unit is left)
      w.s = uniform(w.s);
      list_of(w);
    }
    return true;
  };

  // ---- its keys: lane (col, half) gets token t0 + col, dimensions 16 ks + 8 half + 0 .. 7
  // (or 8 u + 4 half + 0 .. 3)
  using Raw = typename std::conditional<kF32 && sizeof(TK) == 2, u2, u4>::type;
  constexpr int kLoads = kF32 ? 16 : 8;
  auto block_of = [&](const Unit& w) {  // of this lane's token
    return a.page_table[(long)w.s * a.max_pages + (min(w.u * kUnit + wave * 32 + col, w.L - 1) >> lgP)];
  };
  auto request = [&](const Unit& w, int blk, Raw (&raw)[kLoads]) {
    const int t0 = w.u * kUnit + wave * 32;
    if constexpr (kF32) {
      const int t = min(t0 + col, w.L - 1);
      const long b = (unsigned)blk < (unsigned)a.num_blocks ? blk : 0;
      const TK* p = k_cache + ((b * a.H + w.h) * a.pgsz + (t & (a.pgsz - 1))) * kDim + 4 * half;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) raw[j] = *reinterpret_cast<const Raw*>(p + 8 * j);
    } else {
      // whole rows, four at a time, turned in LDS (in the product's order a load takes 32 bytes
      // of each of 32 rows)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int y = __builtin_amdgcn_readlane(blk, 16 * b);
        const TK* page = k_cache + ((long)((unsigned)y < (unsigned)a.num_blocks ? y : 0) * a.H + w.h) * a.pgsz * kDim;
#pragma unroll
        for (int j = 4 * b; j < 4 * b + 4; ++j) {
          const int t = min(t0 + 4 * j + (lane >> 4), w.L - 1);
          raw[j] = *reinterpret_cast<const u4*>(page + (unsigned)((t & (a.pgsz - 1)) * kDim + 8 * (lane & 15)));
        }
      }
    }
  };

  // ---- rows [32 c0, ..) of a KV head into LDS, kSet of them
  constexpr int kPieces = 16 * (int)sizeof(TQ) / 2, kMine = kSet * kPieces / 256;
  auto fill = [&](const Unit& w, int set) {
    u4 q[kMine];
#pragma unroll
    for (int e = 0; e < kMine; ++e) {
      const int rr = (tid + 256 * e) / kPieces, pc = (tid + 256 * e) % kPieces, r = set * kSet + rr;
      const bool there = r < w.n * a.G;
      const int i = there ? r / a.G : 0, hq = w.h * a.G + (there ? r % a.G : 0);
      const u4 none = {};
      const u4 v = *reinterpret_cast<const u4*>(static_cast<const TQ*>(a.q) + (long)(w.row0 + i) * a.q_stride +
                                                hq * kDim + (16 / sizeof(TQ)) * pc);
      q[e] = there ? v : none;
    }
    if (tid < kSet) {
      const int r = set * kSet + tid;
      const bool there = r < w.n * a.G;
      const int i = there ? r / a.G : 0, hq = w.h * a.G + (there ? r % a.G : 0);
      const float l = lse[(long)(w.row0 + i) * a.H * a.G + hq];
      s_nl[tid] = !there || l == -INFINITY ? -INFINITY : -l * kLog2e;
      s_i[tid] = i;
    }
#pragma unroll
    for (int e = 0; e < kMine; ++e) {
      const int rr = (tid + 256 * e) / kPieces, pc = (tid + 256 * e) % kPieces;
      unsigned char* to = s_q + rr * kRow;
      if constexpr (!kF32) {
        *reinterpret_cast<u4*>(to + 16 * (pc ^ piece_xor(rr))) = q[e];
      } else if constexpr (sizeof(TQ) == 4) {
        *reinterpret_cast<u4*>(to + 16 * pc) = q[e];
      } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const u4 v = {q[e][2 * k] << 16, q[e][2 * k] & 0xffff0000u, q[e][2 * k + 1] << 16,
                        q[e][2 * k + 1] & 0xffff0000u};
          *reinterpret_cast<u4*>(to + 32 * pc + 16 * k) = v;
        }
      }
    }
  };

  int in_s = -1, in_h = -1, in_set = -1;  // whose rows are in LDS

  // one unit, its keys in `raw`, which then takes those of the unit two after it
  auto step = [&](const Unit& w, int blk, Raw (&raw)[kLoads], const Unit& later, int later_blk) {
    const int first = w.L - w.n, count = w.n * a.G, t = w.u * kUnit + wave * 32 + col;
    Raw kr[kLoads];
    if constexpr (kF32) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) kr[j] = raw[j];
    } else {
      unsigned char* k = s_k + wave * 32 * 256;
      const int px = piece_xor(col) ^ half;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (the wave's own, in order)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int r = 4 * j + (lane >> 4);
        *reinterpret_cast<u4*>(k + r * 256 + 16 * ((lane & 15) ^ piece_xor(r))) = raw[j];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) kr[ks] = *reinterpret_cast<const u4*>(k + col * 256 + 16 * (px ^ (2 * ks)));
    }
    float* const m = mass + ((long)w.s * a.H + w.h) * a.max_pages * a.pgsz;
    const float old = t < first ? m[t] : 0.0f;
    float sum = 0.0f;
    // (a run: rows before the unit's first token do not see it)
    const int r0 = a.mask ? 0 : max(0, w.u * kUnit - first) * a.G;
    auto have = [&](int set) {
      if (set == in_set && w.s == in_s && w.h == in_h) return;
      __syncthreads();  // (the set's last readers)
      fill(w, set);
      __syncthreads();
      in_set = set, in_s = w.s, in_h = w.h;
    };
    have(r0 / kSet);
    request(later, later_blk, raw);
#pragma unroll 1
    for (int set = r0 / kSet; set * kSet < count; ++set) {
      have(set);
#pragma unroll 1
      for (int c = max(0, r0 - set * kSet) / 32; c < kSet / 32 && set * kSet + 32 * c < count; ++c) {
        const int live = min(32, count - set * kSet - 32 * c);
        f16v z;
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = 0.0f;
        const unsigned char* qp = s_q + (32 * c + col) * kRow;
        // among the new tokens: which of the wave's 32 tokens row 32 c + col sees
        const int tb = w.u * kUnit + wave * 32;
        const bool tail = tb + 31 >= first;
        uint32_t seen = ~0u;
        if (tail) {
          const int i = s_i[32 * c + col];
          seen = draft_window(a, w.row0 + i, i, tb - first, w.L - tb);
        }
        if constexpr (kF32) {
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float4 q = *reinterpret_cast<const float4*>(qp + 32 * j + 16 * half);
            const float qv[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float k;
              if constexpr (sizeof(TK) == 2) k = __uint_as_float(e & 1 ? kr[j][e / 2] & 0xffff0000u : kr[j][e / 2] << 16);
              else k = __uint_as_float(kr[j][e]);
              z = __builtin_amdgcn_mfma_f32_32x32x2f32(qv[e], k, z, 0, 0, 0);
            }
          }
        } else {
          const int px = piece_xor(col) ^ half;
          u4 q[8];
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) q[ks] = *reinterpret_cast<const u4*>(qp + 16 * (px ^ (2 * ks)));
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
            z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, q[ks]), __builtin_bit_cast(bf8, kr[ks]),
                                                        z, 0, 0, 0);
        }
        // element e of the product: row 8 (e / 4) + 4 half + e % 4 of the chunk
        float nl[16];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const float4 v = *reinterpret_cast<const float4*>(&s_nl[32 * c + 8 * b + 4 * half]);
          nl[4 * b] = v.x, nl[4 * b + 1] = v.y, nl[4 * b + 2] = v.z, nl[4 * b + 3] = v.w;
        }
        uint32_t on = 0;  // of this lane's 16 rows, those that count
#pragma unroll
        for (int e = 0; e < 16; ++e) on |= nl[e] != -INFINITY ? 1u << e : 0u;
        if (tail) {  // a bit of each of this lane's rows, from the lane that has the row
#pragma unroll 1
          for (int e0 = 0; e0 < 16; e0 += 4)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t y = __shfl(seen, 2 * e0 + 4 * half + e, 64);
              on &= ~((~y >> col & 1u) << (e0 + e));
            }
        }
        if (__all(on == 0xffffu)) {
#pragma unroll
          for (int e = 0; e < 16; ++e) sum += __builtin_amdgcn_exp2f(fmaf(z[e], zs, nl[e]));
        } else {
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            if (8 * b >= live) break;
#pragma unroll
            for (int e = 4 * b; e < 4 * b + 4; ++e) {
              const float y = __builtin_amdgcn_exp2f(fmaf(z[e], zs, nl[e]));
              sum += on >> e & 1u ? y : 0.0f;
            }
          }
        }
      }
    }
    auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
    const float both = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    if (half == 0 && t < w.L && (unsigned)blk < (unsigned)a.num_blocks)
      m[t] = (t < first ? decay * old : 0.0f) + both;
  };

  // Units w0 (being computed), w1, w2, w3; the keys of two and the blocks of three are on their
  // way.  A unit's blocks are requested before the keys of the one before it, so that they never
  // wait for more than what is needed first.
  Raw raw0[kLoads], raw1[kLoads];
  Unit w1 = cur;
  bool more1 = advance(w1);
  Unit w2 = w1;
  bool more2 = more1 && advance(w2);
  int b0 = block_of(cur), b1 = block_of(w1), b2 = block_of(w2);
  request(cur, b0, raw0);
  request(w1, b1, raw1);
  auto turn = [&](Raw (&raw)[kLoads]) {
    Unit w3 = w2;
    const bool more3 = more2 && advance(w3);
    const int b3 = block_of(w3);
    step(cur, b0, raw, w2, b2);
    const bool more = more1;
    cur = w1, w1 = w2, w2 = w3;
    b0 = b1, b1 = b2, b2 = b3;
    more1 = more2, more2 = more3;
    return more;
  };
  while (turn(raw0) && turn(raw1)) {
  }
}

// Many rows over few tokens: a block takes 32 tokens of a list and its eight waves every eighth
// chunk of rows, whose queries they read as the product takes them; their sums are added in
// order.  Above, a wave goes through all rows alone: 7 prompts of 159 to 477 tokens over up to
// 577, 16 heads a group, fp32 147 us instead of 745; 15 trees of 34 to 104, eight heads a group,
// bf16 12.6 instead of 43.6.
constexpr int kRowWaves = 8;
template <bool kF32, typename TQ, typename TK>
__global__ __launch_bounds__(64 * kRowWaves) void mass_rows_kernel(DraftArgs a, const float* __restrict__ lse,
                                                                   const TK* __restrict__ k_cache, float decay,
                                                                   float* __restrict__ mass) {
  __shared__ float s_sum[kRowWaves][32];
  const int h = blockIdx.y, s = blockIdx.z, t0 = blockIdx.x * 32;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const float zs = kLog2e / sqrtf((float)kDim);
  const DraftSeq w = draft_seq(a, s);
  if (w.n == 0 || t0 >= w.L) return;
  const int first = w.L - w.n, count = w.n * a.G, j0 = t0 - first, t = min(t0 + col, w.L - 1);
  const bool tail = j0 > -32;
  const int lgP = a.pgsz == 64 ? 6 : a.pgsz == 32 ? 5 : 4;
  const int blk = a.page_table[(long)s * a.max_pages + (t >> lgP)];
  const bool live = (unsigned)blk < (unsigned)a.num_blocks;

  using RawK = typename std::conditional<kF32 && sizeof(TK) == 2, u2, u4>::type;
  using RawQ = typename std::conditional<kF32 && sizeof(TQ) == 2, u2, u4>::type;
  constexpr int kLoads = kF32 ? 16 : 8, kElems = kF32 ? 4 : 8;
  RawK kr[kLoads];
  const TK* k = k_cache + (((long)(live ? blk : 0) * a.H + h) * a.pgsz + (t & (a.pgsz - 1))) * kDim + kElems * half;
#pragma unroll
  for (int j = 0; j < kLoads; ++j) kr[j] = *reinterpret_cast<const RawK*>(k + 2 * kElems * j);

  float sum = 0.0f;
  const int r0 = a.mask ? 0 : max(0, j0) * a.G;  // (a run: earlier rows do not see these tokens)
  for (int c = r0 / 32 + wave; 32 * c < count; c += kRowWaves) {
    const int r = 32 * c + col, i = min(r, count - 1) / a.G, hq = h * a.G + min(r, count - 1) % a.G;
    const TQ* qp = static_cast<const TQ*>(a.q) + (long)(w.row0 + i) * a.q_stride + (long)hq * kDim + kElems * half;
    RawQ qr[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) qr[j] = *reinterpret_cast<const RawQ*>(qp + 2 * kElems * j);
    const float l = lse[(long)(w.row0 + i) * a.H * a.G + hq];
    const float nl = -l * kLog2e;
    uint32_t seen = tail ? draft_window(a, w.row0 + i, i, j0, w.L - t0) : ~0u;
    if (r >= count || fabsf(l) == INFINITY) seen = 0u;
    f16v z;
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = 0.0f;
    if constexpr (kF32) {
      auto at = [](const auto& x, int e) {
        if constexpr (sizeof(x) == 8) return __uint_as_float(e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16);
        else return __uint_as_float(x[e]);
      };
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) z = __builtin_amdgcn_mfma_f32_32x32x2f32(at(qr[j], e), at(kr[j], e), z, 0, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, qr[j]), __builtin_bit_cast(bf8, kr[j]), z,
                                                    0, 0, 0);
    }
    // element e: row 8 (e / 4) + 4 half + e % 4 of the chunk, whose lane has its sum and window
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int from = 8 * (e / 4) + 4 * half + e % 4;
      const float y = __builtin_amdgcn_exp2f(fmaf(z[e], zs, __shfl(nl, from, 64)));
      sum += __shfl(seen, from, 64) >> col & 1u ? y : 0.0f;
    }
  }
  auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
  if (half == 0) s_sum[wave][col] = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  __syncthreads();
  if (tid < 32 && t0 + tid < w.L && live) {
    float all = 0.0f;
#pragma unroll
    for (int e = 0; e < kRowWaves; ++e) all += s_sum[e][tid];
    float* const m = mass + ((long)s * a.H + h) * a.max_pages * a.pgsz + t0 + tid;
    *m = (t0 + tid < first ? decay * *m : 0.0f) + all;
  }
}

}  // namespace

hipError_t launch_token_mass(const locks_cfg_t& c, const DraftArgs& a, const float* lse,
                             const void* k_cache, float decay, float* mass, hipStream_t st) {
  const bool f32 = c.q_dtype != LOCKS_BF16 || c.kv_dtype != LOCKS_BF16;
  const long width = (long)a.max_pages * a.pgsz, all = (width + 127) / 128 * a.H * a.S;
  // by the average sequence's rows, and the most units there can be (4 trees of up to 45 tokens over
  // 3.7K, 8 heads of 5 queries, some thousand units: by rows 25 us, else 17.5).  The lengths are not
  // known here, so short sequences in wide tables take the other way: 7 fp32 prompts as above in
  // tables of 128K tokens 778 us instead of 157, 15 runs of 34 to 104 40 instead of 11.
  const bool by_rows = (long)a.n_tokens * a.G / a.S >= kManyRows && all <= kMassBlocks;
  const dim3 grid = by_rows ? dim3((unsigned)((width + 31) / 32), a.H, a.S) : dim3((unsigned)(all < kMassBlocks ? all : kMassBlocks));
#define MASS(F32, TQ, TK)                                                                            \
  if (by_rows)                                                                                       \
    hipLaunchKernelGGL((mass_rows_kernel<F32, TQ, TK>), grid, dim3(64 * kRowWaves), 0, st, a, lse,   \
                       static_cast<const TK*>(k_cache), decay, mass);                                \
  else                                                                                               \
    hipLaunchKernelGGL((mass_kernel<F32, TQ, TK>), grid, dim3(256), 0, st, a, lse,                   \
                       static_cast<const TK*>(k_cache), decay, mass)
  if (!f32) {
    MASS(false, uint16_t, uint16_t);
  } else if (c.q_dtype == LOCKS_BF16) {
    MASS(true, uint16_t, float);
  } else if (c.kv_dtype == LOCKS_BF16) {
    MASS(true, float, uint16_t);
  } else {
    MASS(true, float, float);
  }
#undef MASS
  return hipGetLastError();
}

}  // namespace locks
