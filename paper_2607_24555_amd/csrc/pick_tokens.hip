// The tokens of a list (sequence, KV head) to keep: the first n_sink, the last n_recent and
// the others of largest mass, in order.
//
// With the masses as unsigned keys of the same order, the key T of the last token kept is found
// in three digits (11, 11 and 10 bits): a histogram of the digit over the tokens whose higher
// digits are T's, and the bin where the count from above passes the number to keep.  Then the
// tokens above T, and the first ones equal to it, are written at their ranks.  A block holds up
// to 32 K tokens of a list in registers, a wave 64 kKeys of them in a row, so that ranks within
// a wave are counts of ballots.  Lists of up to that many tokens take one launch; longer ones
// are cut into chunks of 8 K to 32 K, each with a block that writes its chunk's histogram, and four
// launches: a launch's blocks each sum the chunks' histograms of the digit before (which also
// tells how many tokens kept lie before their chunk).
//
// Bound by latency, of barriers and launches: 8 lists of 4K tokens 10.4 us; 64 lists of 128K (33
// MB, 6.5 us of HBM) with ties 54 us, without 51, in launches of 10, 12, 13 and 18; two of 1M
// 38 us.  The number of launches goes by the tables' width: 64 lists of 4K in tables of 128K take
// 43 us, in their own 12.
#include <type_traits>

#include "tokens_internal.h"

namespace locks {
namespace {

constexpr int kPickBlock = 1024, kWaves = kPickBlock / 64;
constexpr int kBins = 2048;
constexpr int kOneLaunch = 32768;  // tokens of a list that one block takes
constexpr int kPickChunk = 32768;
constexpr uint32_t kZeroKey = 0x80000000u;

// Unsigned key of a mass: order as the values', -0 as 0, NaN below everything.
__device__ __forceinline__ uint32_t mass_key(float x) {
  if (x != x) return 0;
  return f32_order_key(x + 0.0f);
}

struct PickArgs {
  const float* mass;
  const int32_t* seq_lens;
  int32_t* out;
  uint16_t* hist;   // [3][lists][chunks][kBins]
  int32_t* state;   // [lists][chunks][4]: T's digits, left to keep from the bin, kept before the
                    // chunk, whether the whole bin is kept
  int H, width, n_keep, n_sink, n_recent, chunks;
  long lists;
};

// kPhase -1: the whole of it.  0, 1, 2: the histogram of that digit; 3: the output.
template <int kKeys, int kPhase>
__global__ __launch_bounds__(kPickBlock) void pick_kernel(PickArgs a) {
  // copies of the first digit's bins, by lane: masses of a list share few exponents, so that a
  // wave's additions would meet (64 lists of 128K with ties 53.6 us instead of 55.2; without ties,
  // where few meet, 51.4 instead of 50.3)
  constexpr int kCopies = kPhase == 0 ? 8 : 1;
  __shared__ int s_hist[kBins * kCopies], s_wave[kWaves], s_bin, s_left, s_all;
  const long list = blockIdx.x / a.chunks;
  const int chunk = blockIdx.x % a.chunks, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int L = min(max(a.seq_lens[list / a.H], 0), a.width);
  int32_t* out = a.out + list * a.n_keep;
  if (L <= a.n_keep) {
    if ((kPhase == -1 || kPhase == 3) && chunk == 0)
      for (unsigned i = tid; i < (unsigned)a.n_keep; i += kPickBlock) out[i] = i < (unsigned)L ? (int)i : -1;
    return;
  }
  constexpr int kChunk = kPickBlock * kKeys;
  const int i0 = chunk * kChunk + wave * 64 * kKeys + lane;  // this thread's tokens: i0 + 64 e
  if (chunk * kChunk >= L && kPhase != -1) {
    if (kPhase < 3) {  // an empty chunk's histogram
      uint16_t* to = a.hist + ((kPhase * a.lists + list) * a.chunks + chunk) * kBins;
      reinterpret_cast<uint32_t*>(to)[tid] = 0;
    }
    return;
  }
  const int lo = a.n_sink, hi = L - a.n_recent;  // the candidates (lo < hi as L > n_keep)
  const float* x = a.mass + list * a.width;
  // bit e: token i0 + 64 e is a candidate (a register a lane; as masks of lanes they spill)
  uint32_t in_range = 0;
#pragma unroll
  for (int e = 0; e < kKeys; ++e) in_range |= i0 + 64 * e >= lo && i0 + 64 * e < hi ? 1u << e : 0u;
  asm volatile("" : "+v"(in_range));
  auto open = [&](int e) { return (in_range >> e & 1u) != 0; };

  uint32_t prefix = 0;                              // T's digits so far
  int left = a.n_keep - a.n_sink - a.n_recent;      // to keep of the tokens that have them
  int above = 0;                                    // of earlier chunks, tokens above T's digits
  bool all = false;                                 // every token that has them is kept
  if (kPhase > 1) {
    const int32_t* st = a.state + (list * a.chunks + chunk) * 4;
    prefix = (uint32_t)st[0], left = st[1], above = st[2], all = st[3] != 0;
  }
  const bool none = a.n_keep == a.n_sink + a.n_recent;
  // the chunks' histograms of the digit before (this thread's two bins over all chunks, and over
  // the earlier ones), requested before the masses, so that the bin is found while those are on
  // their way; where every token is kept already they hold anything, and are not used
  int h0 = 0, h1 = 0, p0 = 0, p1 = 0;
  if (kPhase > 0) {
    const uint32_t* hist = reinterpret_cast<const uint32_t*>(a.hist + ((kPhase - 1) * a.lists + list) * a.chunks * kBins) +
                           (kPickBlock - 1 - tid);
    auto few = [&](auto most) {  // all together (64 lists of 128K, four chunks: 53.6 us, in turn 55.8)
      constexpr int kMost = decltype(most)::value;
      uint32_t v[kMost];
#pragma unroll
      for (int e = 0; e < kMost; ++e) v[e] = hist[min(e, a.chunks - 1) * (kBins / 2)];
#pragma unroll
      for (int e = 0; e < kMost; ++e) {
        if (e < a.chunks) h0 += v[e] >> 16, h1 += v[e] & 0xffffu;
        if (e < chunk) p0 += v[e] >> 16, p1 += v[e] & 0xffffu;
      }
    };
    if (a.chunks <= 4) {
      few(std::integral_constant<int, 4>{});
    } else if (a.chunks <= 8) {
      few(std::integral_constant<int, 8>{});
    } else {
#pragma unroll 16
      for (int c = 0; c < a.chunks; ++c) {
        const uint32_t v = hist[(long)c * (kBins / 2)];
        h0 += v >> 16, h1 += v & 0xffffu;
        if (c < chunk) p0 += v >> 16, p1 += v & 0xffffu;
      }
    }
  }
  uint32_t key[kKeys];
#pragma unroll
  for (int e = 0; e < kKeys; ++e) key[e] = __float_as_uint(x[min(i0 + 64 * e, L - 1)]);
  auto arrived = [&] {
#pragma unroll
    for (int e = 0; e < kKeys; ++e) key[e] = mass_key(__uint_as_float(key[e]));
  };
  if (kPhase <= 0) arrived();

  auto shift_of = [](int d) { return d == 0 ? 21 : d == 1 ? 10 : 0; };
  // counts digit d of the tokens whose higher digits are T's
  auto count = [&](int d) {
#pragma unroll
    for (int e = 0; e < kCopies * kBins / kPickBlock; ++e) s_hist[tid + e * kPickBlock] = 0;
    __syncthreads();
    const int shift = shift_of(d), mask = d == 2 ? 1023 : 2047;
    int zeros = 0;  // counted by ballots: as one bin's additions they would queue
#pragma unroll
    for (int e = 0; e < kKeys; ++e) {
      const bool in = open(e) && (d == 0 || key[e] >> (d == 1 ? 21 : 10) == prefix >> (d == 1 ? 21 : 10));
      const bool zero = key[e] == kZeroKey;
      zeros += (int)__popcll(__ballot(in && zero));
      if (in && !zero) atomicAdd(&s_hist[(key[e] >> shift & mask) * kCopies + lane % kCopies], 1);
    }
    if (lane == 0 && zeros) atomicAdd(&s_hist[(kZeroKey >> shift & mask) * kCopies], zeros);
    __syncthreads();
  };
  // the bin of digit d in which the count from above passes `left`; h: this thread's two bins,
  // kBins - 1 - 2 tid and the one below, over all chunks; p: over the earlier ones
  auto choose = [&](int d, int h0, int h1, int p0, int p1) {
    int sum;
    const int from = scan_block<kWaves>(h0 + h1, s_wave, sum);
    const int b = kBins - 1 - 2 * tid;
    if (from < left && from + h0 >= left) s_bin = b, s_left = left - from, s_all = from + h0 == left;
    else if (from + h0 < left && from + h0 + h1 >= left)
      s_bin = b - 1, s_left = left - from - h0, s_all = from + h0 + h1 == left;
    __syncthreads();
    const int bin = s_bin;
    prefix |= (uint32_t)bin << shift_of(d);
    left = s_left;
    all = s_all != 0;
    if (kPhase != -1) {
      const int from_bin = all ? bin : bin + 1;  // (those of a bin kept whole count as above)
      scan_block<kWaves>((b >= from_bin ? p0 : 0) + (b - 1 >= from_bin ? p1 : 0), s_wave, sum);
      above += sum;
    }
  };
  int ties = 0;  // tokens equal to T in earlier chunks
  if (kPhase == -1 && !none) {
    for (int d = 0; d < 3 && !all; ++d) {
      count(d);
      choose(d, s_hist[kBins - 1 - 2 * tid], s_hist[kBins - 2 - 2 * tid], 0, 0);
      __syncthreads();
    }
  }
  if (kPhase > 0 && !none && !all) {
    const int d = kPhase - 1;
    choose(d, h0, h1, p0, p1);
    if (kPhase == 3) {
      int sum;
      const int b = kBins - 1 - 2 * tid, bin = s_bin;
      scan_block<kWaves>((b == bin ? p0 : 0) + (b - 1 == bin ? p1 : 0), s_wave, sum);
      ties = all ? 0 : sum;
    } else if (tid == 0) {
      int32_t* st = a.state + (list * a.chunks + chunk) * 4;
      st[0] = (int32_t)prefix, st[1] = left, st[2] = above, st[3] = all;
    }
  }
  if (kPhase > 0) arrived();
  if (kPhase >= 0 && kPhase < 3) {
    if (none || all) return;
    count(kPhase);
    uint16_t* to = a.hist + ((kPhase * a.lists + list) * a.chunks + chunk) * kBins;
    uint32_t n0 = 0, n1 = 0;
#pragma unroll
    for (int e = 0; e < kCopies; ++e)
      n0 += s_hist[2 * tid * kCopies + e], n1 += s_hist[(2 * tid + 1) * kCopies + e];
    reinterpret_cast<uint32_t*>(to)[tid] = n0 | n1 << 16;
    return;
  }

  // ---- the first n_sink and the last n_recent
  if (chunk == 0) {
    // (unsigned, as above: the last step may pass 2^31)
    for (unsigned i = tid; i < (unsigned)lo; i += kPickBlock) out[i] = (int)i;
    for (unsigned i = tid; i < (unsigned)a.n_recent; i += kPickBlock) out[a.n_keep - a.n_recent + i] = hi + (int)i;
  }
  // ---- ranks.  Lane g takes the 64 tokens of the wave's group g: which are above T, and which
  // equal to it.
  unsigned long long over = 0, tie = 0;
#pragma unroll
  for (int e = 0; e < kKeys; ++e) {
    const bool cand = !none && open(e);
    const unsigned long long o = __ballot(cand && (key[e] > prefix || (all && key[e] == prefix)));
    const unsigned long long t = __ballot(cand && !all && key[e] == prefix);
    over = lane == e ? o : over;
    tie = lane == e ? t : tie;
  }
  int n_over = (int)__popcll(over), n_tie = (int)__popcll(tie);
  for (int o = 1; o < 64; o <<= 1) {  // inclusive over the lanes
    const int p = __shfl_up(n_over, o, 64), q = __shfl_up(n_tie, o, 64);
    if (lane >= o) n_over += p, n_tie += q;
  }
  __syncthreads();
  if (lane == 63) s_wave[wave] = n_over, s_hist[wave] = n_tie;
  __syncthreads();
  for (int w = 0; w < wave; ++w) above += s_wave[w], ties += s_hist[w];
  above += n_over - (int)__popcll(over);
  ties += n_tie - (int)__popcll(tie);
  const int g0 = chunk * kChunk + wave * 64 * kKeys + 64 * lane;  // the group's first token
  if (lane < kKeys && g0 < L) {
    unsigned long long take = over;
    int at = lo + above + min(ties, left);
    for (int room = left - ties; tie && room > 0; --room) {  // the first ones equal to T
      take |= tie & -tie;
      tie &= tie - 1;
    }
    for (; take; take &= take - 1) out[at++] = g0 + __ffsll(take) - 1;
  }
}

// Tokens of a chunk: as few as leave each block a compute unit, and at most 64 histograms to
// sum where there is a choice (16 lists of 128K in chunks of 8 K: 28 us, of 32 K 44; 64 of 128K in
// chunks of 32 K 51, of 16 K 57, of 8 K 64; 2 of 1M in chunks of 16 K 36, of 32 K 42, of 8 K 46; 64 of
// 40K in chunks of 16 K 31.5, of 32 K 45; 2 of 256K in chunks of 8 K 24, of 16 K 27).
int pick_chunk(const locks_cfg_t& c) {
  const long width = (long)c.max_pages_per_seq * c.page_size, lists = (long)c.num_seqs * c.num_kv_heads;
  if (width <= kOneLaunch) return kOneLaunch;
  int chunk = kPickBlock * 8;
  while (chunk < kPickChunk && ((width + chunk - 1) / chunk > 64 || lists * ((width + chunk - 1) / chunk) > 256)) chunk *= 2;
  return chunk;
}
int pick_chunks(const locks_cfg_t& c) {
  const long width = (long)c.max_pages_per_seq * c.page_size, chunk = pick_chunk(c);
  return (int)((width + chunk - 1) / chunk);
}

}  // namespace

size_t pick_scratch_bytes(const locks_cfg_t& c) {
  const size_t chunks = pick_chunks(c), lists = (size_t)c.num_seqs * c.num_kv_heads;
  return 256 + (chunks > 1 ? lists * chunks * (3 * kBins * sizeof(uint16_t) + 4 * sizeof(int32_t)) : 0);
}

// What no launch of as many sequences or fewer needs more than: fewer lists can be cut into more
// chunks in all, where chunks are below the largest, so of up to 256 lists.
size_t pick_scratch_most(const locks_cfg_t& c) {
  size_t most = pick_scratch_bytes(c);
  locks_cfg_t fewer = c;
  for (fewer.num_seqs = 1; fewer.num_seqs < c.num_seqs && fewer.num_seqs <= 256; ++fewer.num_seqs) {
    const size_t n = pick_scratch_bytes(fewer);
    if (n > most) most = n;
  }
  return most;
}

hipError_t launch_pick_tokens(const locks_cfg_t& c, const float* mass, const int32_t* seq_lens,
                              int n_keep, int n_sink, int n_recent, int32_t* out_ids, void* scratch,
                              hipStream_t st) {
  const long lists = (long)c.num_seqs * c.num_kv_heads;
  const int width = c.max_pages_per_seq * c.page_size, chunks = pick_chunks(c);
  uint16_t* hist = static_cast<uint16_t*>(scratch);
  const PickArgs a{mass,   seq_lens, out_ids, hist,     reinterpret_cast<int32_t*>(hist + 3 * lists * chunks * kBins),
                   c.num_kv_heads, width, n_keep, n_sink, n_recent, chunks, lists};
  const dim3 grid((unsigned)(lists * chunks)), block(kPickBlock);
#define PICK(KEYS, PHASE) hipLaunchKernelGGL((pick_kernel<KEYS, PHASE>), grid, block, 0, st, a)
  if (chunks == 1) {
    if (width <= 4 * kPickBlock) PICK(4, -1);
    else if (width <= 8 * kPickBlock) PICK(8, -1);
    else if (width <= 16 * kPickBlock) PICK(16, -1);
    else PICK(32, -1);
  } else {
#define PICK4(KEYS) PICK(KEYS, 0); PICK(KEYS, 1); PICK(KEYS, 2); PICK(KEYS, 3)
    switch (pick_chunk(c) / kPickBlock) {
      case 8: PICK4(8); break;
      case 16: PICK4(16); break;
      default: PICK4(32);
    }
#undef PICK4
  }
#undef PICK
  return hipGetLastError();
}

}  // namespace locks
