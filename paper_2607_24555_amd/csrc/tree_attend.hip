// Attention of several new tokens of a sequence over the paged cache:
//   o_i = sum_{t seen by i} softmax_t(q_i . k_t / sqrt d) v_t.
//
// The new tokens' query heads of one KV head are the rows of a matrix product (row
// r = i G + g), in tiles of 32 RW rows; a block goes through units of 32 NB TW tokens, its
// waves RW by rows and TW by tokens.  Per 32 rows and 32 tokens a wave computes
//   S^T = K Q^T   (M = token, N = row), whose result has a row per lane column, so that the
//                 online softmax (running maximum and sum, fp32) needs one lane swap,
//   O^T += V^T P  (M = dimension, N = row, K = token), with P exactly as S^T left it.
// Rows lie in LDS with their 16-byte pieces permuted by the token, so that neither the key
// reads nor the transposed value reads meet on a bank.
//
// Tiles, by the average sequence's rows (bf16; 8 heads of 4 queries unless said):
//   up to 32   four waves with tokens of their own and no barrier: keys in registers as the
//              product takes them, values through LDS.  Bound by HBM from some thousand tokens
//              (8 sequences of 32K, 8 new: 210 us, 5.1 TB/s), below by latency: 5 new tokens
//              over 4K take 19.3 us, 12 of it here (plan 2.0, rows to sums 2.8, joins and
//              partials 2.5 of a block's 7.4) and 6.5 in the merge's launch.
//   up to 64   two waves by rows, two by tokens (16 new: 216 us, 5.0 TB/s).
//   up to 128  four waves by rows, two blocks a compute unit.
//   more       eight waves by rows, with three units of copies to LDS on their way.  Against the
//              128-row tile: ragged trees of 140 to 248 rows 394 us (449), 16 tokens of 16 heads
//              over 1M 501 (536), pieces of prompts 594 (637).  Its products and the weights'
//              vector work overlap by half: the matrix pipe is busy 54% of the time and the
//              vector one 53% (pieces of prompts, 700 TFLOP/s; 1,050 with the second term's).
// fp32 products (any other types) take 32 or 128 rows and run at 69 TFLOP/s of the 154 of a
// large product, the matrix pipe half busy: of a compute unit's two blocks the older one is
// served first, and the other ends alone (82 and 105 us).
//
// All (sequence, KV head, tile) items' units, in order, are cut into equal shares, one a
// block (every block derives the cut from the lengths), so ragged batches and long lists
// fill the chip; a unit counts by the 32s of rows that its tile has (see weight_of); an item
// within a share writes its output, others leave partials (o, max, sum), which
// tree_merge_kernel combines in order.  Where there are more tiles than kTiles, or the tables are
// short, an item is a block's and there is nothing to merge.
//
// What a row does not see is masked by one 32-bit window per row and 32 tokens, the
// ancestors' bits shifted to the tile; only units that hold tokens some row does not see look
// at it.
#include <type_traits>

#include "tokens_internal.h"

namespace locks {
namespace {

constexpr int kTiles = 512;        // row tiles of a launch whose items are cut into shares
constexpr int kTreeBlocks = 512;   // two per compute unit

constexpr int kMaskWords = 6;      // of a row's mask that lie in LDS (trees of up to 192 tokens)

struct TreeArgs {
  DraftArgs d;
  const void *k, *v;
  void* out;
  float* lse;
  float* po;       // [2 blocks][rows][128]
  float* pml;      // [2 blocks][rows][2]
  int32_t* rec;    // [blocks][8]: the item that begins in a block and ends in a later one
  int tiles;       // most row tiles there can be, of row ranges that ascend
  int split, out_bf16;
};

__device__ __forceinline__ float swap_max(float v) {
  auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float swap_sum(float v) {
  auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// kF32: products in fp32 (32x32x2 MFMA), else bf16 (32x32x16), the weights in NT terms.
template <bool kF32, typename TQ, typename TK, int NT, int RW, int TW, int NB>
struct Tree {
  static constexpr int kRows = 32 * RW, kGroup = 32 * NB, kUnit = kGroup * TW;
  static constexpr int kThreads = 64 * RW;                 // of a group of waves with the same tokens
  static constexpr int kPieces = kF32 ? 32 : 16;           // of a row: 4 floats, or 8 bf16
  static constexpr int kLoads = kGroup * kPieces / kThreads;
  static constexpr int kTokStep = kThreads / kPieces;      // tokens between a thread's loads
  static constexpr int kKRow = kF32 ? 132 * 4 : 256, kVRow = kF32 ? 512 : 256;  // bytes
  // a wave of its own reads its keys from memory as the product takes them
  static constexpr bool kDirect = !kF32 && RW == 1;
  static constexpr int kKeys = kDirect ? 4096 : kGroup * kKRow;  // (4 KB of scratch at least)
  static constexpr int kTile = kKeys + kGroup * kVRow;     // of one group's unit
  // bf16 rows that waves share go to LDS without passing registers: three units ahead where a
  // block has the compute unit for itself, else one
  static constexpr bool kDma = !kF32 && RW > 1;
  static constexpr int kBufs = RW == 8 ? 4 : RW > 1 ? 2 : 1;
  static constexpr int kLead = kBufs - 1;
  static constexpr int kDmaLoads = kDma ? kGroup / 4 / RW : 0;  // of a wave and tensor: 4 rows each
  static constexpr int kJoin = TW > 1 ? TW * kRows * 132 * 4 : 0;
  // (direct) the rows' queries lie behind the tiles, to leave the registers to the loads
  static constexpr int kUsed = kTile * TW * kBufs + (kDirect ? 32 * 256 : 0);
  static constexpr int kLds = kUsed > kJoin ? kUsed : kJoin;
};

// 16 bytes a lane from memory to LDS: lane l's to lds + 16 l.  Counted by vmcnt only; whoever
// reads them waits (wait_vm) and passes a barrier.
__device__ __forceinline__ void copy_to_lds(const char* base, uint32_t offset, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, %1"
      :
      : "v"(offset), "s"(base), "s"(lds)
      : "memory", "m0");
}
template <int kLeft>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kLeft) : "memory");
}

struct Segment {
  int s, h, tile;
  int u0, count, units;
  int row0, n, L;
};

template <bool kF32, typename TQ, typename TK, int NT, int RW, int TW, int NB, int kWaves>
__global__ __launch_bounds__(64 * RW * TW, kWaves) void tree_kernel(TreeArgs a) {
  using C = Tree<kF32, TQ, TK, NT, RW, TW, NB>;
  constexpr int kBlock = 64 * RW * TW;
  __shared__ __align__(16) unsigned char lds[C::kLds];
  __shared__ int s_units[kTiles + 1], s_first[kTiles + 1], s_sum[RW * TW];
  __shared__ int s_row0[kTiles], s_rows[kTiles], s_len[kTiles];
  __shared__ float s_m[TW][C::kRows], s_l[TW][C::kRows];
  __shared__ float2 s_all[TW > 1 ? C::kRows : 1];
  __shared__ uint32_t s_mask[C::kRows][kMaskWords + 1];
  const DraftArgs& d = a.d;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % RW, wt = wave / RW;
  const int col = lane & 31, half = lane >> 5;
  const int Hq = d.H * d.G;
  const float zs = kLog2e / sqrtf((float)kDim);

  auto tiles_of = [&](int n) { return (int)(((long)n * d.G + C::kRows - 1) / C::kRows); };
  // rows of a sequence's tiles, in whole 32s and as even as they go
  auto tile_rows = [&](int n) {
    const int tiles = tiles_of(n), b = (int)(((long)n * d.G + 31) / 32);
    return tiles > 1 ? 32 * ((b + tiles - 1) / tiles) : C::kRows;
  };
  // tokens that a tile's rows can see
  auto reach = [&](int n, int L, int tile) {
    if (d.mask) return L;
    const long last = min((long)n, ((long)(tile + 1) * tile_rows(n) - 1) / d.G + 1);
    return (int)min((long)L, L - n + last);
  };
  auto units_of = [&](int n, int L, int tile) { return max(1, (reach(n, L, tile) + C::kUnit - 1) / C::kUnit); };

  // What a unit of a tile costs.  In the 256-row tile the products of more rows show a little
  // (pieces of prompts 594 us; with 8 instead of 12: 596, 4: 625); in the others two blocks of a compute
  // unit hide that.
  constexpr int kMostWeight = RW == 8 ? 20 : 1;
  auto weight_of = [&](int n, int tile) {
    if (RW < 8) return 1;
    const int tr = tile_rows(n), rows = (int)min((long)n * d.G - (long)tile * tr, (long)tr);
    return 12 + (rows + 31) / 32;
  };

  // ---- one segment: units [u0, u0 + count) of an item, whose units lie in `parts` blocks
  auto process = [&](const Segment& g, int lb, int parts) {
    const int s = g.s, h = g.h, row0 = g.row0, n = g.n, L = g.L, first = L - n;
    const int tr = tile_rows(n), r0 = g.tile * tr, count_rows = min(n * d.G - r0, tr);
    const int r = r0 + wr * 32 + col;
    const bool live = wr * 32 + col < count_rows, busy = wr * 32 < count_rows;
    const int i = live ? r / d.G : 0, hg = h * d.G + (live ? r % d.G : 0);
    const long row = row0 + i;
    const uint32_t* mask = d.mask ? d.mask + row * d.words : nullptr;

    // this lane's query: dimensions 16 ks + 8 half + 0 .. 7, or 8 u + 4 half + 0 .. 3
    bf8 qb[kF32 || C::kDirect ? 1 : 8];
    float qf[kF32 ? 64 : 1];
    unsigned char* const q_lds = lds + C::kTile * TW * C::kBufs;
    if constexpr (C::kDirect) {
      __syncthreads();  // (the queries' last readers)
      const int rr = tid >> 3, rg = r0 + rr;  // 32 rows, two pieces a thread
      const bool there = rr < count_rows;
      const TQ* q = static_cast<const TQ*>(d.q) +
                    (long)(row0 + (there ? rg / d.G : 0)) * d.q_stride + (h * d.G + (there ? rg % d.G : 0)) * kDim;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int pc = (tid & 7) + 8 * e;
        const u4 w = *reinterpret_cast<const u4*>(q + 8 * pc), none = {};
        *reinterpret_cast<u4*>(q_lds + rr * 256 + 16 * (pc ^ piece_xor(rr))) = there ? w : none;
      }
    } else {
      const TQ* q = static_cast<const TQ*>(d.q) + row * d.q_stride + hg * kDim;
      if constexpr (kF32) {
#pragma unroll
        for (int u = 0; u < 16; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) qf[4 * u + j] = live ? load_elem(q, 8 * u + 4 * half + j) : 0.0f;
      } else {
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          const u4 w = *reinterpret_cast<const u4*>(q + 16 * ks + 8 * half), none = {};
          qb[ks] = __builtin_bit_cast(bf8, live ? w : none);
        }
      }
    }

    // ---- staging
    using Raw = typename std::conditional<kF32 && sizeof(TK) == 2, u2, u4>::type;
    Raw kr[C::kLoads], vr[C::kLoads];
    static_assert(!C::kDirect || C::kLoads == 8, "a lane's half of a key row");
    int blk[2 * NB];
    const int gt = wr * 64 + lane, piece = gt % C::kPieces, tok_in = gt / C::kPieces;
    const int32_t* table = d.page_table + (long)s * d.max_pages;
    const int lgP = d.pgsz == 64 ? 6 : d.pgsz == 32 ? 5 : 4;
    auto look_up = [&](int u) {
#pragma unroll
      for (int b = 0; b < 2 * NB; ++b) {
        const int t = min(u * C::kUnit + wt * C::kGroup + 16 * b, L - 1);
        blk[b] = table[t >> lgP];
      }
    };
    const uint32_t page_bytes = (uint32_t)d.pgsz * kDim * sizeof(TK), blk_bytes = page_bytes * d.H;
    const char* const k_head = static_cast<const char*>(a.k) + (size_t)h * page_bytes;
    const char* const v_head = static_cast<const char*>(a.v) + (size_t)h * page_bytes;
    size_t base[2 * NB];  // (the same in every lane)
    auto load = [&](int u) {
#pragma unroll
      for (int b = 0; b < 2 * NB; ++b) {
        const uint32_t x = (uint32_t)__builtin_amdgcn_readfirstlane(blk[b]);
        base[b] = (size_t)(x < (uint32_t)d.num_blocks ? x : 0u) * blk_bytes;
      }
#pragma unroll
      for (int j = 0; j < C::kLoads; ++j) {
        constexpr int kElems = kF32 ? 4 : 8;
        const int t = min(u * C::kUnit + wt * C::kGroup + j * C::kTokStep + tok_in, L - 1);
        const uint32_t at = ((t & (d.pgsz - 1)) * kDim + kElems * piece) * sizeof(TK);
        static_assert(C::kDma || C::kTokStep <= 16, "a step's tokens lie in one page");
        const size_t page = base[j * C::kTokStep / 16];
        if constexpr (!C::kDirect) kr[j] = *reinterpret_cast<const Raw*>(k_head + page + at);
        vr[j] = *reinterpret_cast<const Raw*>(v_head + page + at);
      }
    };
    // (direct) this lane's half of its token's key, of the unit whose values were loaded last
    auto load_keys = [&](int u) {
      if constexpr (C::kDirect) {
        const int t = min(u * C::kUnit + wt * C::kGroup + col, L - 1);
        const TK* p = reinterpret_cast<const TK*>(k_head + (col < 16 ? base[0] : base[1])) +
                      (t & (d.pgsz - 1)) * kDim + 8 * half;
#pragma unroll
        for (int j = 0; j < 8; ++j) kr[j] = *reinterpret_cast<const Raw*>(p + 16 * j);
      }
    };
    // (kDma) this wave's rows of unit u: they lie in one page, whose block was looked up before
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds;
    const __attribute__((address_space(4))) int32_t* const const_table =
        (const __attribute__((address_space(4))) int32_t*)table;
    constexpr int kMine = 4 * C::kDmaLoads;  // rows of a wave
    static_assert(!C::kDma || 16 % kMine == 0, "rows of one page");
    auto block_of = [&](int u) {
      const int t = min(u * C::kUnit + wt * C::kGroup + wr * kMine, L - 1);
      return const_table[t >> lgP];
    };
    auto issue = [&](int u, int blk) {
      const uint32_t x = (uint32_t)blk;
      const size_t page = (size_t)(x < (uint32_t)d.num_blocks ? x : 0u) * blk_bytes;
      const uint32_t to = lds_at + (wt * C::kBufs + (u & (C::kBufs - 1))) * C::kTile + wr * kMine * 256;
#pragma unroll
      for (int j = 0; j < C::kDmaLoads; ++j) {
        const int in = wr * kMine + 4 * j + (lane >> 4);  // the tile's token
        const int t = min(u * C::kUnit + wt * C::kGroup + in, L - 1);
        const uint32_t at = ((t & (d.pgsz - 1)) * kDim + 8 * ((lane & 15) ^ piece_xor(in))) * 2;
        copy_to_lds(k_head + page, at, to + 1024 * j);
        copy_to_lds(v_head + page, at, to + C::kKeys + 1024 * j);
      }
    };
    auto tile_at = [&](int u) { return lds + (wt * C::kBufs + (u & (C::kBufs - 1))) * C::kTile; };
    // writes the loaded unit; returns whether this thread's values are all finite (where asked)
    auto store = [&](int u, bool check) -> bool {
      unsigned char* kt = tile_at(u);
      unsigned char* vt = kt + C::kKeys;
      bool ok = true;
#pragma unroll
      for (int j = 0; j < C::kLoads; ++j) {
        const int tok = j * C::kTokStep + tok_in;
        if constexpr (kF32) {
          float4 kf, vf;
          if constexpr (sizeof(TK) == 2) {
            kf = make_float4(__uint_as_float(kr[j].x << 16), __uint_as_float(kr[j].x & 0xffff0000u),
                             __uint_as_float(kr[j].y << 16), __uint_as_float(kr[j].y & 0xffff0000u));
            vf = make_float4(__uint_as_float(vr[j].x << 16), __uint_as_float(vr[j].x & 0xffff0000u),
                             __uint_as_float(vr[j].y << 16), __uint_as_float(vr[j].y & 0xffff0000u));
          } else {
            kf = __builtin_bit_cast(float4, kr[j]);
            vf = __builtin_bit_cast(float4, vr[j]);
          }
          if (check) ok = ok && finite(vf.x) && finite(vf.y) && finite(vf.z) && finite(vf.w);
          *reinterpret_cast<float4*>(kt + tok * C::kKRow + 16 * piece) = kf;
          *reinterpret_cast<float4*>(vt + tok * C::kVRow + 16 * piece) = vf;
        } else {
          const int at = 16 * (piece ^ piece_xor(tok));
          if (check) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              ok = ok && (vr[j][e] & 0x7f80u) != 0x7f80u && (vr[j][e] & 0x7f800000u) != 0x7f800000u;
          }
          *reinterpret_cast<u4*>(vt + tok * C::kVRow + at) = vr[j];  // (keys stay in registers)
        }
      }
      return ok;
    };

    // ---- which of the 32 tokens from tb on this lane's row sees
    auto window = [&](int tb) -> uint32_t {
      const int e = L - tb, j0 = tb - first;
      if (e <= 0) return 0u;
      const uint32_t lim = e >= 32 ? ~0u : (1u << e) - 1u;
      if (j0 <= -32) return lim;
      uint32_t seen = j0 < 0 ? (1u << -j0) - 1u : 0u;
      if (mask) {
        const int w = j0 >> 5, sh = j0 & 31;
        uint32_t lo = 0u, hi = 0u;
        if (d.words <= kMaskWords) {
          if ((unsigned)w < (unsigned)d.words) lo = s_mask[wr * 32 + col][w];
          if ((unsigned)(w + 1) < (unsigned)d.words) hi = s_mask[wr * 32 + col][w + 1];
        } else {
          if ((unsigned)w < (unsigned)d.words) lo = mask[w];
          if ((unsigned)(w + 1) < (unsigned)d.words) hi = mask[w + 1];
        }
        seen |= sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
      } else {
        const int c = i - j0;
        if (c >= 0) seen |= c >= 31 ? ~0u : (2u << c) - 1u;
      }
      return seen & lim;
    };

    float m = -INFINITY, l = 0.0f;
    f16v o[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[dt][e] = 0.0f;

    if (L > 0) {
      // units that every row of the tile sees whole (of a run, up to its first row's token), then
      // the others
      const int all_see = d.mask ? first : first + r0 / d.G + 1;
      const int u_end = g.u0 + g.count, u_tail = min(u_end, max(g.u0, all_see > 0 ? all_see / C::kUnit : 0));
      // the rows' masks, for those others: read from memory there, they would wait for
      // the rows on their way too
      auto fill_masks = [&] {
        if (!mask || d.words > kMaskWords || u_tail == u_end) return;
        for (int e = tid; e < count_rows * d.words; e += kBlock) {
          const int rr = e / d.words, w = e % d.words;
          s_mask[rr][w] = d.mask[(long)(row0 + (r0 + rr) / d.G) * d.words + w];
        }
      };
      int next_blk = 0;  // (kDma) of the unit kLead after the one at hand
      if constexpr (C::kDma) {
        __syncthreads();  // (the tiles' last readers: the segment before)
        fill_masks();
#pragma unroll
        for (int e = 0; e < C::kLead; ++e)
          if (e < g.count) issue(g.u0 + e, block_of(g.u0 + e));
        if (C::kLead < g.count) next_blk = block_of(g.u0 + C::kLead);
      } else {
        look_up(g.u0);
        load(g.u0);
        load_keys(g.u0);
        __syncthreads();
        fill_masks();
        if constexpr (RW == 1) __syncthreads();
        if (g.count > 1) look_up(g.u0 + 1);
      }
      auto step = [&](int u, auto tail_unit) {
        constexpr bool tail = decltype(tail_unit)::value;
        const int t0 = u * C::kUnit + wt * C::kGroup;
        bool bad;
        if constexpr (C::kDma) {
          // this unit's copies are here; those of the units behind it may be on their way
          constexpr int kUnitLoads = 2 * C::kDmaLoads;
          if (C::kLead > 2 && u + 2 < u_end) wait_vm<2 * kUnitLoads>();
          else if (C::kLead > 1 && u + 1 < u_end) wait_vm<kUnitLoads>();
          else wait_vm<0>();
          __syncthreads();
          if (u + C::kLead < u_end) {
            issue(u + C::kLead, next_blk);
            if (u + C::kLead + 1 < u_end) next_blk = block_of(u + C::kLead + 1);
          }
          bad = false;
          if constexpr (tail) {
            const unsigned char* v = tile_at(u) + C::kKeys;
#pragma unroll
            for (int j = 0; j < C::kGroup * 16 / C::kThreads; ++j) {
              const u4 x = *reinterpret_cast<const u4*>(v + 16 * (gt + j * C::kThreads));
#pragma unroll
              for (int e = 0; e < 4; ++e)
                bad = bad || (x[e] & 0x7f80u) == 0x7f80u || (x[e] & 0x7f800000u) == 0x7f800000u;
            }
            bad = __syncthreads_or(bad);
          }
        } else {
          // (a wave that owns its tile needs no barrier, its LDS accesses being in order; the
          // fences keep the compiler's order)
          if constexpr (RW == 1) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          bad = !store(u, tail);
          if constexpr (RW == 1) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          if (u + 1 < u_end) {
            load(u + 1);
            if (u + 2 < u_end) look_up(u + 2);
          }
          if constexpr (RW == 1) bad = tail && __any(bad);
          else if constexpr (tail) bad = __syncthreads_or(bad);
          else __syncthreads();
        }
        if (!busy && !(tail && bad)) return;  // (no rows: the wave only loads)
        unsigned char* kt = tile_at(u);
        unsigned char* vt = kt + C::kKeys;

        // ---- logits
        f16v z[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) z[b][e] = 0.0f;
        const unsigned char* kp = kt + col * C::kKRow;
        if constexpr (kF32) {
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int u8 = 0; u8 < 16; ++u8) {
              const float4 x = *reinterpret_cast<const float4*>(kp + 32 * b * C::kKRow + 32 * u8 + 16 * half);
              z[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.x, qf[4 * u8], z[b], 0, 0, 0);
              z[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.y, qf[4 * u8 + 1], z[b], 0, 0, 0);
              z[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.z, qf[4 * u8 + 2], z[b], 0, 0, 0);
              z[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(x.w, qf[4 * u8 + 3], z[b], 0, 0, 0);
            }
        } else if constexpr (C::kDirect) {
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {
            const u4 y = *reinterpret_cast<const u4*>(q_lds + col * 256 + 16 * (piece_xor(col) ^ half ^ (2 * ks)));
            z[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, kr[ks]), __builtin_bit_cast(bf8, y),
                                                           z[0], 0, 0, 0);
          }
          if (u + 1 < u_end) load_keys(u + 1);
        } else {
          const int px = piece_xor(col) ^ half;
          u4 x[8][NB];
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
#pragma unroll
            for (int b = 0; b < NB; ++b)
              x[ks][b] = *reinterpret_cast<const u4*>(kp + 32 * b * C::kKRow + 16 * (px ^ (2 * ks)));
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
#pragma unroll
            for (int b = 0; b < NB; ++b)
              z[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, x[ks][b]), qb[ks], z[b], 0, 0, 0);
        }
        if constexpr (!kF32 && !C::kDirect) {
          // four key pieces ahead of the products
          __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
          for (int e = 0; e < 8 * NB - 4; ++e) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          }
          __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        }
        // ---- masks (element e of a lane: token 8 (e / 4) + 4 half + e % 4)
        if constexpr (tail) {
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            const uint32_t seen = window(t0 + 32 * b) >> (4 * half);
            if (!__all(seen == (~0u >> (4 * half)))) {
#pragma unroll
              for (int e = 0; e < 16; ++e)
                z[b][e] = seen >> (8 * (e / 4) + e % 4) & 1u ? z[b][e] : -INFINITY;
            }
          }
        }
        // ---- online softmax; the maximum follows only where a row grows by more than 2^8
        float big = -INFINITY;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) big = fmaxf(big, z[b][e]);
        big = swap_max(big) * zs;
        if (__any(big > m + 8.0f)) {
          const float mn = big > m + 8.0f ? big : m;  // (by the row: no row's bits depend on another's)
          const float sc = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - mn);
          m = mn;
          l *= sc;
#pragma unroll
          for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[dt][e] *= sc;
        }
        const float ms = m == -INFINITY ? 0.0f : m;
        auto weigh = [&](int b, int e0, int e1) {
#pragma unroll
          for (int e = e0; e < e1; ++e) {
            z[b][e] = __builtin_amdgcn_exp2f(fmaf(z[b][e], zs, -ms));
            l += z[b][e];
          }
        };
        if constexpr (kF32 || tail) {
#pragma unroll
          for (int b = 0; b < NB; ++b) weigh(b, 0, 16);
        }

        // ---- values that are not finite, among the new tokens: 0 times them would reach rows
        // that do not see them, so they are added by hand and leave the tile
        auto value = [&](int tok, int dim) -> float {
          if constexpr (kF32) return *reinterpret_cast<const float*>(vt + tok * C::kVRow + 4 * dim);
          else
            return bf16_bits_to_f32(*reinterpret_cast<const uint16_t*>(
                vt + tok * C::kVRow + 16 * ((dim >> 3) ^ piece_xor(tok)) + 2 * (dim & 7)));
        };
        auto row_bad = [&](int tok) { return __any(!finite(value(tok, 2 * lane)) || !finite(value(tok, 2 * lane + 1))); };
        if (tail && bad) {
          if constexpr (RW > 1) __syncthreads();  // (the keys' last readers)
          // the weights of 16 tokens at a time, 2 KB a wave in the keys' place
          float* w = reinterpret_cast<float*>(kt) + wr * 512;
#pragma unroll
          for (int c = 0; c < 2 * NB; ++c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[(8 * (e / 4) + 4 * half + e % 4) * 32 + col] = z[c / 2][8 * (c & 1) + e];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            for (int t = 0; t < 16; ++t) {
              if (!row_bad(16 * c + t)) continue;
              const float p = w[t * 32 + col];
#pragma unroll
              for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  const float x = value(16 * c + t, 32 * dt + 8 * (e / 4) + 4 * half + e % 4);
                  o[dt][e] += p != 0.0f ? p * x : 0.0f;
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          }
          if constexpr (RW > 1) __syncthreads();
          for (int t = wr; t < C::kGroup; t += RW)
            if (row_bad(t)) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int dim = 2 * lane + e;
                if constexpr (kF32) *reinterpret_cast<float*>(vt + t * C::kVRow + 4 * dim) = 0.0f;
                else
                  *reinterpret_cast<uint16_t*>(vt + t * C::kVRow + 16 * ((dim >> 3) ^ piece_xor(t)) + 2 * (dim & 7)) = 0;
              }
            }
          if constexpr (RW > 1) __syncthreads();
          else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }

        // ---- values
        if constexpr (kF32) {
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const unsigned char* vp = vt + (32 * b + 8 * (e / 4) + 4 * half + e % 4) * C::kVRow + 4 * col;
#pragma unroll
              for (int dt = 0; dt < 4; ++dt)
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(vp + 128 * dt),
                                                             z[b][e], o[dt], 0, 0, 0);
            }
        } else {
          // 16 lanes read 4 tokens x 16 dimensions transposed: lane c gets dimension c of each
          const int c = lane & 15, tv = 4 * half + (c >> 2);
          const int p0 = (2 * ((lane >> 4) & 1) + ((c & 3) >> 1)) ^ piece_xor(tv);
          const unsigned char* vp = vt + tv * C::kVRow + 8 * (c & 1);
          // In pieces of 16 tokens: between the products of one, the next one's values are
          // fetched and its weights formed.
          using LdsS4 = __attribute__((address_space(3))) s4;
          bf8 x[2][4], p[2][NT];
          auto fetch = [&](int c) {
            const unsigned char* vb = vp + 16 * c * C::kVRow;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {
              const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsS4*)(vb + 16 * (p0 ^ (4 * dt))));
              const s4 hi =
                  __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsS4*)(vb + 8 * C::kVRow + 16 * (p0 ^ (4 * dt) ^ 8)));
              x[c & 1][dt] = __builtin_bit_cast(bf8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
          };
          auto form = [&](int c) {
            if constexpr (!tail) weigh(c / 2, 8 * (c & 1), 8 * (c & 1) + 8);
            float rest[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) rest[e] = z[c / 2][8 * (c & 1) + e];
#pragma unroll
            for (int k = 0; k < NT; ++k)
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                p[c & 1][k][e] = (__bf16)rest[e];
                rest[e] -= (float)p[c & 1][k][e];
              }
          };
          constexpr bool kAhead = !C::kDirect;  // (there is no room for it beside the loads)
          if constexpr (kAhead) {
            fetch(0);
            form(0);
            __builtin_amdgcn_sched_barrier(0);
          }
#pragma unroll
          for (int c = 0; c < 2 * NB; ++c) {
            if constexpr (!kAhead) {
              fetch(c);
              form(c);
            }
            if (kAhead && c + 1 < 2 * NB) fetch(c + 1);
#pragma unroll
            for (int k = 0; k < NT; ++k)
#pragma unroll
              for (int dt = 0; dt < 4; ++dt)
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[c & 1][dt], p[c & 1][k], o[dt], 0, 0, 0);
            if (kAhead && c + 1 < 2 * NB) {
              form(c + 1);
              __builtin_amdgcn_sched_group_barrier(0x100, 8, 1);
#pragma unroll
              for (int e = 0; e < 4 * NT; ++e) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
                __builtin_amdgcn_sched_group_barrier(0x402, 6, 1);
              }
            }
            if constexpr (kAhead) __builtin_amdgcn_sched_barrier(0);
          }
        }
      };
      for (int u = g.u0; u < u_tail; ++u) step(u, std::false_type{});
      for (int u = u_tail; u < u_end; ++u) step(u, std::true_type{});
    }

    // ---- the item's output, or a partial
    l = swap_sum(l);
    const bool whole = g.count == g.units;
    const long slot = g.u0 > 0 ? 2L * lb : 2L * lb + 1;
    auto emit = [&](int rr, int dim, float x0, float x1, float x2, float x3, float mm, float ll, bool stats) {
      // four dimensions of row rr of the tile
      const int rg = r0 + rr;
      if (rr >= count_rows) return;
      if (whole) {
        const long to = (long)(row0 + rg / d.G) * Hq + h * d.G + rg % d.G;
        const float inv = ll > 0.0f || ll != ll ? 1.0f / ll : 0.0f;
        if (a.out_bf16) {
          typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
          const bf4 y = {(__bf16)(x0 * inv), (__bf16)(x1 * inv), (__bf16)(x2 * inv), (__bf16)(x3 * inv)};
          *reinterpret_cast<bf4*>(static_cast<__bf16*>(a.out) + to * kDim + dim) = y;
        } else {
          *reinterpret_cast<float4*>(static_cast<float*>(a.out) + to * kDim + dim) =
              make_float4(x0 * inv, x1 * inv, x2 * inv, x3 * inv);
        }
        if (stats && a.lse) a.lse[to] = ll == 0.0f ? -INFINITY : kLn2 * mm + logf(ll);
      } else {
        *reinterpret_cast<float4*>(a.po + (slot * C::kRows + rr) * kDim + dim) = make_float4(x0, x1, x2, x3);
        if (stats) *reinterpret_cast<float2*>(a.pml + (slot * C::kRows + rr) * 2) = make_float2(mm, ll);
      }
    };
    if constexpr (TW == 1) {
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          emit(wr * 32 + col, 32 * dt + 2 * e + 4 * half, o[dt][e], o[dt][e + 1], o[dt][e + 2], o[dt][e + 3], m, l,
               dt == 0 && e == 0 && half == 0);
    } else {
      if (half == 0) {
        s_m[wt][wr * 32 + col] = m;
        s_l[wt][wr * 32 + col] = l;
      }
      __syncthreads();
      // all waves' parts of a row at its largest maximum, and their sum
      float mx = -INFINITY, ls = 0.0f;
#pragma unroll
      for (int w = 0; w < TW; ++w) mx = fmaxf(mx, s_m[w][wr * 32 + col]);
#pragma unroll
      for (int w = 0; w < TW; ++w) {
        const float mw = s_m[w][wr * 32 + col];
        // (a product also where the wave has no maximum: of NaN logits the sum is NaN, the maximum -inf)
        ls += s_l[w][wr * 32 + col] * (mw == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mw - mx));
      }
      const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - mx);
      float* to = reinterpret_cast<float*>(lds) + (wt * C::kRows + wr * 32 + col) * 132;
      if (wr * 32 + col < count_rows) {
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<float4*>(to + 32 * dt + 2 * e + 4 * half) =
                make_float4(o[dt][e] * f, o[dt][e + 1] * f, o[dt][e + 2] * f, o[dt][e + 3] * f);
      }
      if (wt == 0 && half == 0) s_all[wr * 32 + col] = make_float2(mx, ls);
      __syncthreads();
      for (int e = tid; e < count_rows * 32; e += kBlock) {
        const int rr = e >> 5, dim = 4 * (e & 31);
        float4 x = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < TW; ++w) {
          const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<float*>(lds) + (w * C::kRows + rr) * 132 + dim);
          x.x += y.x, x.y += y.y, x.z += y.z, x.w += y.w;
        }
        const float2 st = s_all[rr];
        emit(rr, dim, x.x, x.y, x.z, x.w, st.x, st.y, dim == 0);
      }
      __syncthreads();
    }
    if (!whole && g.u0 == 0 && tid == 0) {
      int32_t* rec = a.rec + 8 * lb;
      rec[0] = count_rows;
      rec[1] = parts;
      rec[2] = row0;
      rec[3] = r0;
      rec[4] = h;
    }
  };

  // ---- what this block computes
  auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  int x = 0, end = 1, lb = 0, share = 1, parts = 1;
  Segment g{};
  if (!a.split) {
    // an item a block: tile slots, s + cu[s] G / rows on for sequence s, some of them empty
    const int slot = blockIdx.x / d.H, h = blockIdx.x % d.H;
    auto base = [&](int s) { return s + (int)((long)draft_rows(d, s).x * d.G / C::kRows); };
    int lo = 0, hi = d.S;  // the last sequence whose slots begin at `slot` or before
    while (hi - lo > 1) {
      const int step = (hi - lo + 63) / 64, s = lo + lane * step;
      const unsigned long long ok = __ballot(s < hi && base(s) <= slot);
      const int k = max(0, (int)__popcll(ok) - 1);
      lo += k * step;
      hi = min(hi, lo + step);
    }
    const DraftSeq q = draft_seq(d, lo);
    const int tile = slot - base(lo);
    if (tile < 0 || tile >= tiles_of(q.n)) return;
    const int units = units_of(q.n, q.L, tile);
    g = Segment{uniform(lo), h, uniform(tile), 0, uniform(units), uniform(units), uniform(q.row0), uniform(q.n), uniform(q.L)};
  } else {
    // the cut: tiles before each sequence, units before each tile
    auto fill_seq = [&](int q) {
      const DraftSeq v = draft_seq(d, q);
      s_row0[q] = v.row0, s_rows[q] = v.n, s_len[q] = v.L;
      return tiles_of(v.n);
    };
    auto cost_of = [&](int q, int tile) { return units_of(s_rows[q], s_len[q], tile) * weight_of(s_rows[q], tile); };
    auto seq_of = [&](int t) {  // the last sequence whose tiles begin at t or before
      int lo = 0, hi = d.S;
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (s_first[mid] <= t) lo = mid;
        else hi = mid;
      }
      return lo;
    };
    // few sequences and tiles: every wave for itself, in lanes, all writing the same (without the
    // barriers of the other way a run of 5 tokens over 4K is planned in 1.3 us instead of 2.7)
    // (tiles beyond a.tiles, of row ranges that do not ascend, are left out: all sums below are then
    // within what tree_plan allows)
    const int few = min(64, a.tiles);
    int total = kTiles + 1;
    if (d.S <= 64) {
      int v = lane < d.S ? fill_seq(lane) : 0;
      const int own = v;
      for (int o = 1; o < d.S; o <<= 1) {
        const int y = __shfl_up(v, o, 64);
        if (lane >= o) v += y;
      }
      if (lane < d.S) s_first[lane] = v - own;
      total = __builtin_amdgcn_readlane(v, d.S - 1);
      s_first[d.S] = total;
      if (total <= few) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        int c = 0;
        if (lane < total) {
          const int q = seq_of(lane);
          c = cost_of(q, lane - s_first[q]);
        }
        int sum = c;
        for (int o = 1; o < total; o <<= 1) {
          const int y = __shfl_up(sum, o, 64);
          if (lane >= o) sum += y;
        }
        const int all = total > 0 ? __builtin_amdgcn_readlane(sum, total - 1) : 0;
        s_units[lane] = lane < total ? sum - c : all;
        s_units[64] = s_units[kTiles] = all;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
    }
    if (total > few) {
      __syncthreads();
      constexpr int kPer = kTiles / kBlock;
      int before[kPer], sum = 0, v = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const int q = tid * kPer + e;
        before[e] = v;
        if (q < d.S) v += fill_seq(q);
      }
      const int at = scan_block<RW * TW>(v, s_sum, total);
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const int q = tid * kPer + e;
        if (q < d.S) s_first[q] = min(at + before[e], a.tiles);
      }
      if (tid == 0) s_first[d.S] = min(total, a.tiles);
      __syncthreads();
      const int T = min(total, a.tiles);
      v = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const int t = tid * kPer + e;
        before[e] = v;
        if (t < T) {
          const int q = seq_of(t);
          v += cost_of(q, t - s_first[q]);
        }
      }
      const int ut = scan_block<RW * TW>(v, s_sum, sum);
#pragma unroll
      for (int e = 0; e < kPer; ++e) s_units[tid * kPer + e] = ut + before[e];
      if (tid == 0) s_units[kTiles] = sum;
      __syncthreads();
    }
    const int all = s_units[kTiles] * d.H;  // (below 2^31: see tree_plan)
    // (at least a unit, so that a block between an item's first and last has some of it)
    share = max((all + (int)gridDim.x - 1) / (int)gridDim.x, kMostWeight);
    // (blocks that share an item or its keys run on one XCD)
    lb = (gridDim.x & 7) ? blockIdx.x : (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    x = lb * share;
    end = min(all, x + share);
    if (tid == 0) a.rec[8 * lb] = 0;
  }
  while (x < end) {
    if (a.split) {
      int lo = 0, hi = d.S;
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (s_units[s_first[mid]] * d.H <= x) lo = mid;
        else hi = mid;
      }
      lo = uniform(lo);
      const int t0 = s_first[lo], t1 = s_first[lo + 1];
      const int first = s_units[t0], per = s_units[t1] - first, in = x - first * d.H;
      const int h = (int)((unsigned)in / (unsigned)per), rest = in - h * per + first;
      int tl = t0, th = t1;
      while (th - tl > 1) {
        const int mid = (tl + th) / 2;
        if (s_units[mid] <= rest) tl = mid;
        else th = mid;
      }
      // the item's units that begin in [x, end)
      const int n = s_rows[lo], w = weight_of(n, tl - t0), at = x - (rest - s_units[tl]);
      const int units = (s_units[tl + 1] - s_units[tl]) / w;
      const int u0 = (x - at + w - 1) / w, u1 = min(units, (end - at + w - 1) / w);
      parts = (at + (units - 1) * w) / share - lb + 1;
      x = min(end, at + units * w);
      if (u0 >= u1) continue;
      g = Segment{lo, uniform(h), uniform(tl - t0), uniform(u0), uniform(u1 - u0), uniform(units),
                  uniform(s_row0[lo]), uniform(n), uniform(s_len[lo])};
    }
    process(g, lb, parts);
    if (!a.split) break;
  }
}

// The items that end in a later block than they begin in (rec: rows, parts, first row of the
// input, first row of the sequence's, KV head).  All their rows, in order, are cut into equal
// runs, one a block; 32 lanes have a row's 128 dimensions, and where a block has fewer than 16
// rows several such groups share a row's parts.  Block lb's own part is in slot 2 lb + 1, the
// later ones' in 2 (lb + 1), ...  (A wave a row, its loads behind its weights: 10 us instead of
// 5 for 8 items of 20 rows in 33 parts, 51 instead of 20 for 512 items of 128 rows in two.)
constexpr int kMergeBlocks = 1024;
__global__ __launch_bounds__(512) void tree_merge_kernel(const int32_t* __restrict__ recs, int blocks,
                                                         const float* __restrict__ po,
                                                         const float* __restrict__ pml, int tile_rows, int G,
                                                         int Hq, void* __restrict__ out, int out_bf16,
                                                         float* __restrict__ out_lse) {
  __shared__ int s_end[kTreeBlocks], s_rec[kTreeBlocks][4], s_wave[8];
  __shared__ __align__(16) float s_o[16][132];
  __shared__ float s_m[16], s_l[16];
  const int tid = threadIdx.x, lane = tid & 63, l32 = tid & 31, grp = tid >> 5;
  // rows up to each block's item
  int4 r = make_int4(0, 0, 0, 0);
  if (tid < blocks) {
    r = *reinterpret_cast<const int4*>(recs + 8 * tid);
    s_rec[tid][3] = recs[8 * tid + 4];
  }
  s_rec[tid][0] = r.y, s_rec[tid][1] = r.z, s_rec[tid][2] = r.w;
  int v = r.x;
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(v, o, 64);
    if (lane >= o) v += y;
  }
  if (lane == 63) s_wave[tid >> 6] = v;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    if (w < (tid >> 6)) v += s_wave[w];
    total += s_wave[w];
  }
  s_end[tid] = v;
  __syncthreads();
  int per = (total + gridDim.x - 1) / gridDim.x;
  if (per < 16) per = per <= 1 ? 1 : 1 << (32 - __clz(per - 1));
  const int groups = per < 16 ? 16 / per : 1, part0 = grp % groups;
  const int row_end = min(total, (int)(blockIdx.x + 1) * per);
  for (int row = blockIdx.x * per + grp / groups; row - grp / groups < row_end; row += 16 / groups) {
    const bool live = row < row_end;
    float4 acc = make_float4(0, 0, 0, 0);
    float mx = -INFINITY, l = 0.0f;
    long to = 0;
    if (live) {
      int lo = 0, hi = blocks - 1;  // the first block whose rows end behind `row`
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (s_end[mid] > row) hi = mid;
        else lo = mid + 1;
      }
      const int parts = s_rec[lo][0], rr = row - (lo ? s_end[lo - 1] : 0), rg = s_rec[lo][2] + rr;
      to = (long)(s_rec[lo][1] + rg / G) * Hq + s_rec[lo][3] * G + rg % G;
      auto slot = [&](int p) { return p ? 2L * (lo + p) : 2L * lo + 1; };
      const int mine = (parts - part0 + groups - 1) / groups;  // parts part0, part0 + groups, ..
      auto add = [&](auto batch) {
        constexpr int kBatch = decltype(batch)::value;
        for (int k = 0; k < mine; k += kBatch) {
          float4 x[kBatch];
          float2 st[kBatch];
#pragma unroll
          for (int e = 0; e < kBatch; ++e) {
            const long at = slot(part0 + min(k + e, mine - 1) * groups) * tile_rows + rr;
            st[e] = *reinterpret_cast<const float2*>(pml + at * 2);
            x[e] = *reinterpret_cast<const float4*>(po + at * kDim + 4 * l32);
          }
          float mn = mx;
#pragma unroll
          for (int e = 0; e < kBatch; ++e) mn = fmaxf(mn, st[e].x);
          const float f = mx == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mx - mn);
          mx = mn;
          l *= f;
          acc.x *= f, acc.y *= f, acc.z *= f, acc.w *= f;
#pragma unroll
          for (int e = 0; e < kBatch; ++e) {
            if (k + e >= mine) break;
            const float w = st[e].x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(st[e].x - mn);
            l = fmaf(w, st[e].y, l);
            acc.x = fmaf(w, x[e].x, acc.x);
            acc.y = fmaf(w, x[e].y, acc.y);
            acc.z = fmaf(w, x[e].z, acc.z);
            acc.w = fmaf(w, x[e].w, acc.w);
          }
        }
      };
      if (mine <= 2) add(std::integral_constant<int, 2>{});
      else add(std::integral_constant<int, 8>{});
    }
    if (groups > 1) {
      *reinterpret_cast<float4*>(&s_o[grp][4 * l32]) = acc;
      if (l32 == 0) s_l[grp] = l, s_m[grp] = mx;
      __syncthreads();
      if (part0 == 0) {
        for (int g = 1; g < groups; ++g) mx = fmaxf(mx, s_m[grp + g]);
        acc = make_float4(0, 0, 0, 0);
        l = 0.0f;
        for (int g = 0; g < groups; ++g) {
          const float4 x = *reinterpret_cast<const float4*>(&s_o[grp + g][4 * l32]);
          const float w = s_m[grp + g] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(s_m[grp + g] - mx);
          l = fmaf(w, s_l[grp + g], l);
          acc.x = fmaf(w, x.x, acc.x);
          acc.y = fmaf(w, x.y, acc.y);
          acc.z = fmaf(w, x.z, acc.z);
          acc.w = fmaf(w, x.w, acc.w);
        }
      }
    }
    if (live && part0 == 0) {
      const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
      if (out_bf16) {
        typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
        const bf4 y = {(__bf16)(acc.x * inv), (__bf16)(acc.y * inv), (__bf16)(acc.z * inv), (__bf16)(acc.w * inv)};
        *reinterpret_cast<bf4*>(static_cast<__bf16*>(out) + to * kDim + 4 * l32) = y;
      } else {
        *reinterpret_cast<float4*>(static_cast<float*>(out) + to * kDim + 4 * l32) =
            make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
      }
      if (out_lse && l32 == 0) out_lse[to] = l == 0.0f ? -INFINITY : kLn2 * mx + logf(l);
    }
  }
}

struct Plan {
  int rows, unit;      // of a tile, of a unit
  int blocks, split;
  long tiles;
  size_t po, pml;
};

// Rows of a tile by the average sequence's rows.
Plan tree_plan(const locks_cfg_t& c, int n_tokens) {
  const int G = c.num_q_heads / c.num_kv_heads, S = c.num_seqs > 0 ? c.num_seqs : 1;
  const bool f32 = c.q_dtype != LOCKS_BF16 || c.kv_dtype != LOCKS_BF16;
  const long rows = ((long)n_tokens * G + S - 1) / S;
  Plan p{};
  p.rows = rows <= 32 ? 32 : f32 ? 128 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256;
  p.unit = p.rows == 32 ? 128 : f32 ? 32 : 64;
  p.tiles = S + (long)n_tokens * G / p.rows;
  const long width = (long)c.max_pages_per_seq * c.page_size, units = (width + p.unit - 1) / p.unit;
  const long most = p.tiles * units * c.num_kv_heads;
  // short tables: a block goes through an item's tokens sooner than a second launch joins its
  // parts (5 new tokens, 8 heads, tables of 512: 12.8 us, cut 14.2; of 1,024 17.6 and 14.5;
  // 16 sequences 16.4 and 24.2; fp32 trees of 30, tables of 128: 30.1 and 30.6, of 256 46.9 and
  // 43.0; where the sequences are short all of these are 3 to 8 us less without the cut)
  const long alone = !f32 ? 512 : p.rows == 32 ? 256 : 128;
  p.split = width > alone && p.tiles <= kTiles && most <= 0x7fffffffL / 32;  // (a unit weighs up to 20)
  if (p.split) {
    const long fill = p.rows == 256 ? kTreeBlocks / 2 : kTreeBlocks;
    p.blocks = (int)(most < fill ? (most + 7) / 8 * 8 : fill);
    p.po = (size_t)2 * p.blocks * p.rows * kDim * sizeof(float);
    p.pml = (size_t)2 * p.blocks * p.rows * 2 * sizeof(float);
  }
  return p;
}

template <bool kF32, typename TQ, typename TK, int NT, int RW, int TW, int NB, int kWaves>
void launch_one(const TreeArgs& a, const Plan& p, hipStream_t st) {
  const unsigned grid = p.split ? (unsigned)p.blocks : (unsigned)(p.tiles * a.d.H);
  hipLaunchKernelGGL((tree_kernel<kF32, TQ, TK, NT, RW, TW, NB, kWaves>), dim3(grid), dim3(64 * RW * TW), 0, st, a);
}

template <typename TQ, typename TK>
void launch_f32(const TreeArgs& a, const Plan& p, hipStream_t st) {
  if (p.rows == 32) launch_one<true, TQ, TK, 1, 1, 4, 1, 1>(a, p, st);
  else launch_one<true, TQ, TK, 1, 4, 1, 1, 2>(a, p, st);
}
template <int NT>
void launch_terms(const TreeArgs& a, const Plan& p, hipStream_t st) {
  if (p.rows == 32) launch_one<false, uint16_t, uint16_t, NT, 1, 4, 1, 2>(a, p, st);
  else if (p.rows == 64) launch_one<false, uint16_t, uint16_t, NT, 2, 2, 1, 2>(a, p, st);
  else if (p.rows == 128) launch_one<false, uint16_t, uint16_t, NT, 4, 1, 2, 2>(a, p, st);
  else launch_one<false, uint16_t, uint16_t, NT, 8, 1, 2, 2>(a, p, st);
}
// Terms of a weight, by the output's type alone: three for fp32 (2^-24 of it), two for bf16 (2^-16, a
// 256th of the output's own rounding).  One term (2^-8) puts a bf16 output as far off again as its own
// rounding does, 2.3e-3 of its norm instead of 1.7e-3 (ragged trees 304 us in one term, 394 in two, 492 in
// three; pieces of prompts 447, 594 and 751).
void launch_bf16(const TreeArgs& a, const Plan& p, hipStream_t st) {
  if (a.out_bf16) launch_terms<2>(a, p, st);
  else launch_terms<3>(a, p, st);
}

// Of tiles of so many rows (256: half the blocks, so as much as 128).
size_t scratch_of(int rows) {
  return (size_t)kTreeBlocks * (2 * (size_t)(rows < 128 ? rows : 128) * (kDim + 2) * sizeof(float) + 8 * sizeof(int32_t));
}

}  // namespace

size_t tree_scratch_bytes(const locks_cfg_t& c, int n_tokens) { return scratch_of(tree_plan(c, n_tokens).rows); }

// What no launch of as many sequences and tokens or fewer needs more than: fewer sequences have
// larger tiles, and one with all the tokens has the largest.
size_t tree_scratch_most(const locks_cfg_t& c, int n_tokens) {
  locks_cfg_t one = c;
  if (one.num_seqs > 1) one.num_seqs = 1;
  return tree_scratch_bytes(one, n_tokens);
}

hipError_t launch_tree_attend(const locks_cfg_t& c, const DraftArgs& d, const void* k_cache,
                              const void* v_cache, void* out, bool out_bf16, float* out_lse,
                              void* scratch, hipStream_t st) {
  const Plan p = tree_plan(c, d.n_tokens);
  char* w = static_cast<char*>(scratch);
  const TreeArgs a{d, k_cache, v_cache, out, out_lse, reinterpret_cast<float*>(w),
                   reinterpret_cast<float*>(w + p.po), reinterpret_cast<int32_t*>(w + p.po + p.pml),
                   (int)p.tiles, p.split, out_bf16 ? 1 : 0};
  if (c.q_dtype == LOCKS_BF16 && c.kv_dtype == LOCKS_BF16) {
    launch_bf16(a, p, st);
  } else if (c.q_dtype == LOCKS_BF16) {
    launch_f32<uint16_t, float>(a, p, st);
  } else if (c.kv_dtype == LOCKS_BF16) {
    launch_f32<float, uint16_t>(a, p, st);
  } else {
    launch_f32<float, float>(a, p, st);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.split) return e;
  const long rows = (long)p.blocks * p.rows;  // at most
  hipLaunchKernelGGL(tree_merge_kernel, dim3((unsigned)(rows < kMergeBlocks ? rows : kMergeBlocks)), dim3(512), 0, st,
                     a.rec, p.blocks, a.po, a.pml, p.rows, d.G, d.H * d.G, out, a.out_bf16, out_lse);
  return hipGetLastError();
}

}  // namespace locks
