// Draws from the softmax of rows of scores, by temperature, top-k, top-p and
// min-p, with given uniform numbers (the definition stands in ml2.h).
//
// All three limits keep a prefix of the order (score descending, index
// ascending).  Every entry has a unique 64-bit key, larger is better,
//   (ord(score) << 32) | (0xFFFFFFFF - index),
// so a limit is a key: the cut.  Weights are whole numbers, so their sums are
// exact in any order and every comparison of sums has one answer, whatever
// the split of the work and the order of the atomics.
//
// A cut is found in two steps.  Entries are counted and weighed in bins of
// equal width in z (of those that can be drawn: z above kLowest); the bin in
// which the wanted count or weight is reached holds the cut.  Inside that bin
// the interval of keys is split into kSub parts again and again until the
// wanted amount ends with a part or 64 entries are left, which one wave compares
// with one another (1 x 16.8M: two steps a cut instead of three, 111 -> 108 us).
//
// Rows of at most kRowMost entries: row_kernel, one workgroup and one launch,
// scores and weights in LDS.  Longer rows are cut into chunks:
//   range_kernel    a chunk's best and worst score (and clears the counts)
//   count_kernel    counts and weights by bin, in LDS, then added up
//   settle_kernel   a workgroup a row: the bins that hold the cuts, and the
//                   scores at their ends
//   collect_kernel  lists the entries whose place the bins do not settle, and
//                   weighs those kept for sure by tile of the row
//   finish_kernel   a workgroup a row: the cuts from the list, the tiles'
//                   running weights, and few draws
//   draw_kernel     many draws: a wave a draw
// top-k with a small k needs no weights before its cut is known: count_kernel
// then only counts, and collect_kernel lists every entry down to the cut's bin.
// Long rows of 16-bit scores with one draw are counted by score instead (below).
#include <algorithm>
#include <type_traits>

#include "draw.h"

namespace ml2 {
namespace {

constexpr int kBins = 2048;         // bins of a long row
constexpr int kSub = 512;           // bins of a short row, parts of an interval of keys
constexpr int kMaxTiles = 4096;     // tiles of a row
constexpr int kTile = 512;          // smallest tile: 8 entries a lane
constexpr int kSpan = 16 * kTile;   // smallest part of count_kernel: 16 waves
constexpr int kPacked = 32768;      // entries that a packed LDS bin holds
constexpr int kFew = 256;           // k of top-k that lists everything it keeps
constexpr int kList = 4096;         // list entries held in LDS
constexpr int kSegments = 32;       // of a row's list, at most
constexpr int kOpen = 1024;         // list entries that collect_kernel gathers before it adds them
constexpr int kFewDraws = 32;       // draws a row that finish_kernel makes itself
constexpr int kRowMost = 14336;     // entries of a row in one workgroup's LDS, 9 bytes each
constexpr int kRanked = 128;        // list entries that are ranked against one another
constexpr int kRowList = 512;       // open entries of a short row held apart
constexpr int kBatch = 1024;        // long rows of one set of launches
constexpr float kLowest = -22.25f;  // exp(z) * 2^31 rounds to 0 below -22.181
constexpr float kOne = 2147483648.0f;

__device__ __forceinline__ uint32_t ordered(float x) {  // x is not NaN
  const uint32_t b = __float_as_uint(x + 0.0f);  // -0.0 is +0.0
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

__device__ __forceinline__ u64 key_of(float x, int64_t i) {
  return ((u64)ordered(x) << 32) | (u64)(0xFFFFFFFFu - (uint32_t)i);
}

__device__ __forceinline__ float key_score(u64 key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float((o & 0x80000000u) ? o & 0x7FFFFFFFu : ~o);
}

__device__ __forceinline__ int64_t key_index(u64 key) {
  return (int64_t)(0xFFFFFFFFu - (uint32_t)key);
}

// What all entries of a row share.
struct RowLimits {
  float m, r;       // best included score (-inf: none), 1 / T
  float range;      // z of interest reaches down to -range
  float min_z;      // log(min_p), or -inf
  int64_t k;        // entries top-k keeps (n: all)
  float p;          // top_p, or 2 where it keeps all
};

// A row's own settings, read ahead of its scores.
struct RowSettings {
  float temperature, p, min_p;
  int32_t k;
};

__device__ __forceinline__ RowSettings row_settings(const SampleArgs &a, int64_t row) {
  return {a.s.temperature ? a.s.temperature[row] : 1.0f, a.top_p ? a.top_p[row] : 1.0f,
          a.min_p ? a.min_p[row] : 0.0f, a.top_k ? a.top_k[row] : 0};
}

// hi, lo: the row's best and worst included scores.
__device__ __forceinline__ RowLimits row_limits(const RowSettings &s, int64_t n, float hi,
                                                float lo) {
  RowLimits l;
  const bool greedy = !(s.temperature > 0.0f);
  l.m = hi;
  l.r = greedy ? 1.0f : 1.0f / s.temperature;
  const float low = lo == hi ? 0.0f : (lo - hi) * l.r;
  l.range = fminf(-kLowest, fmaxf(-low, 1e-20f));
  const int32_t k = greedy ? 1 : s.k;
  l.k = k > 0 && k < n ? k : n;
  l.p = s.p < 1.0f ? s.p : 2.0f;
  l.min_z = s.min_p > 0.0f ? logf(fminf(s.min_p, 1.0f)) : -__builtin_inff();
  return l;
}

__device__ __forceinline__ float exponent(float x, const RowLimits &l) {
  return x == l.m ? 0.0f : (x - l.m) * l.r;
}

// 0 for an entry that is not included (x = -inf or NaN, so z is) too: the
// instruction takes a NaN to 0, where C++ leaves the conversion undefined.
__device__ __forceinline__ uint32_t weight(float z) {
  uint32_t q;
  asm("v_cvt_u32_f32 %0, %1" : "=v"(q) : "v"(rintf(expf(z) * kOne)));
  return q;
}

// Eight consecutive entries of a row as they come from memory, so that the
// next ones can be on their way while these are worked on.
template <typename T>
struct Eight {
  typedef T V __attribute__((ext_vector_type(8), aligned(sizeof(T))));
  typedef u64 Mask __attribute__((aligned(1)));
  V v;
  u64 mask;

  // Entries i .. i+7 of a row that ends at n.
  __device__ __forceinline__ void load(const T *scores, const uint8_t *valid, int64_t i,
                                       int64_t n) {
    if (i + 8 <= n) {
      v = *reinterpret_cast<const V *>(scores + i);
      if (valid) mask = *reinterpret_cast<const Mask *>(valid + i);
    } else {
      mask = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = i + j < n ? scores[i + j] : (T)-__builtin_inff();
        if (valid && i + j < n) mask |= (u64)valid[i + j] << (8 * j);
      }
    }
  }

  // The scores, -inf where the mask excludes an entry; a NaN stays.
  __device__ __forceinline__ void get(bool masked, float (&x)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = widen<T>(v[j]);
    if (masked) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (((mask >> (8 * j)) & 0xFF) == 0) x[j] = -__builtin_inff();
    }
  }
};

// Bin of an entry with z > kLowest, best first; scale = bins / range.
template <int BINS>
__device__ __forceinline__ int bin_of(float z, float scale) {
  return min(BINS - 1, (int)(-z * scale));
}

// Weight that top-p wants of `total`.
__device__ __forceinline__ u64 share_of(float p, u64 total) {
  const double share = ceil((double)p * (double)total);
  return share >= 1.0 ? (u64)share : 1ull;
}

// Exclusive sum over the threads of a workgroup of at most 16 waves; *all: the
// whole sum.  Ends without a barrier: `lds` may be written after the next one.
__device__ __forceinline__ u64 block_prefix(u64 v, u64 *lds, u64 *all) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const u64 incl = wave_prefix(v);
  if (lane == 63) lds[wave] = incl;
  __syncthreads();
  u64 w = lane < (int)(blockDim.x >> 6) ? lds[lane] : 0;
  w += lane_move<0x111, 0xF>(w, 0);
  w += lane_move<0x112, 0xF>(w, 0);
  w += lane_move<0x114, 0xF>(w, 0);
  w += lane_move<0x118, 0xF>(w, 0);
  *all = from_lane(w, 15);
  return incl - v + (wave > 0 ? from_lane(w, wave - 1) : 0);
}

// State of a search for a cut, in LDS.
struct Search {
  u64 amount[kSub];  // count or weight of a part
  u64 lo, hi;    // the smallest and largest key of the part that holds the cut
  u64 wave_sum[16];
  int bin;       // of block_find: the bin found, or -1
  u64 above;     // the amount of better ones
  uint32_t few;  // keys of a part, the first 64 of them with their amounts
  u64 few_key[64];
  uint32_t few_amount[64];
};

// Looks through `bins` bins, best first, for the one in which the running sum
// of amount(b) on top of `base` reaches need(sum of all, with base).  s.bin and
// s.above say which and what lies above it; the result is the sum of all.
// Every thread of the workgroup calls it, after a barrier that completes the
// bins; it ends with one.
template <typename F, typename N>
__device__ __forceinline__ u64 block_find(Search &s, int bins, N need_of, u64 base, F amount) {
  const int per = (bins + blockDim.x - 1) / blockDim.x;
  const int b0 = min(bins, (int)threadIdx.x * per), b1 = min(bins, b0 + per);
  u64 sum = 0;
  for (int b = b0; b < b1; ++b) sum += amount(b);
  if (threadIdx.x == 0) s.bin = -1;
  u64 all;
  u64 run = base + block_prefix(sum, s.wave_sum, &all);
  const u64 need = need_of(base + all);
  if (run < need && run + sum >= need) {  // one thread at most
    for (int b = b0; b < b1; ++b) {
      const u64 next = run + amount(b);
      if (next >= need) {
        s.bin = b;
        s.above = run;
        break;
      }
      run = next;
    }
  }
  __syncthreads();
  return base + all;
}

// Adds v (1, or an entry's weight) to amount[b] for every active lane.  Lanes of
// one part whose v is the same, as entries of equal scores are, are one
// addition: those of one address wait for one another.
__device__ __forceinline__ void add_amount(u64 *amount, int b, uint32_t v) {
  const int lane = threadIdx.x & 63;
  for (u64 rest = __ballot(true); rest;) {
    const int leader = __ffsll(rest) - 1;
    const u64 same = __ballot(b == __builtin_amdgcn_readlane(b, leader) &&
                              v == (uint32_t)__builtin_amdgcn_readlane((int)v, leader));
    const int lanes = __popcll(same & rest);
    if (lanes < 8) {
      if ((rest >> lane) & 1) atomicAdd(&amount[b], (u64)v);
      return;
    }
    if (lane == leader) atomicAdd(&amount[b], (u64)v * (uint32_t)lanes);
    rest &= ~same;
  }
}

// The least of at most 64 keys before which less than `need` lies, with `above`
// before all of them.  Every wave works it out for itself.
__device__ __forceinline__ u64 few_cut(const Search &s, u64 above, u64 need) {
  const int lane = threadIdx.x & 63, few = (int)s.few;
  const u64 key = lane < few ? s.few_key[lane] : 0;
  const uint32_t amount = lane < few ? s.few_amount[lane] : 0;
  u64 before = above;
#pragma unroll 1
  for (int j = 0; j < few; ++j) before += from_lane(key, j) > key ? from_lane(amount, j) : 0u;
  const u64 least = wave_fold(lane < few && before < need ? key : ~0ull, ~0ull,
                              [](u64 a, u64 b) { return min(a, b); });
  return from_lane(least, 63);
}

// The cut among the keys that each(f) hands to f(key, weight(), bin()) and that
// are at least `from` and inside(bin), in which the count (by_count) or weight
// on top of `above` reaches `need`: entries with key >= the result are kept.
// Keys between two that are inside are inside too.  Every thread of the
// workgroup calls it, with the same `above` and `need`, and there is such a key.
template <typename Each, typename In>
__device__ __forceinline__ u64 find_cut(Search &s, bool by_count, u64 above, u64 need, u64 from,
                                        Each each, In inside) {
  u64 to = ~0ull;
  bool known = false;  // that keys from .. to are inside
  bool done = false;
  if (threadIdx.x == 0) {
    s.lo = ~0ull;
    s.hi = 0;
    s.few = 0;
  }
  for (;;) {
    for (int b = threadIdx.x; b < kSub; b += blockDim.x) s.amount[b] = 0;
    // the smallest and largest key left
    u64 first = ~0ull, last = 0;
    each([&](u64 key, auto weight, auto bin) {
      if (key < from || key > to || !(known || inside(bin))) return;
      first = min(first, key);
      last = max(last, key);
      if (!known) return;
      const uint32_t at = atomicAdd(&s.few, 1u);
      if (at < 64) {
        s.few_key[at] = key;
        s.few_amount[at] = by_count ? 1u : weight();
      }
    });
    first = wave_fold(first, ~0ull, [](u64 a, u64 b) { return min(a, b); });
    last = wave_fold(last, 0ull, [](u64 a, u64 b) { return max(a, b); });
    __syncthreads();
    if ((threadIdx.x & 63) == 63 && last) atomicMin(&s.lo, first), atomicMax(&s.hi, last);
    __syncthreads();
    const u64 lo = s.lo, hi = s.hi;
    if (done || lo >= hi) return lo;  // all of the part is kept, or one entry
    if (known && s.few <= 64) return few_cut(s, above, need);
    const int width = 64 - __clzll(hi - lo);
    const int shift = max(0, width - 9);
    each([&](u64 key, auto weight, auto) {
      if (key < lo || key > hi) return;
      // best first
      add_amount(s.amount, kSub - 1 - (int)((key - lo) >> shift), by_count ? 1u : weight());
    });
    __syncthreads();
    if (threadIdx.x == 0) {
      s.lo = ~0ull;
      s.hi = 0;
      s.few = 0;
    }
    block_find(s, kSub, [&](u64) { return need; }, above, [&](int b) { return s.amount[b]; });
    const int b = s.bin < 0 ? kSub - 1 : s.bin;  // the amount is always reached
    above = s.above;
    done = above + s.amount[b] == need;
    known = true;
    from = lo + ((u64)(kSub - 1 - b) << shift);
    to = from + min((1ull << shift) - 1, ~from);
    __syncthreads();
  }
}

// What the bins settle: entries of bins better than `sure` are kept, those of
// bins [sure, last] and of bin `k_bin` are listed, the others dropped.
struct Bins {
  int k_bin;       // holds top-k's cut (the number of bins: none)
  u64 k_above, k_mass;  // better bins' count and weight
  u64 all;         // all bins' weight
  int sure, last;
  u64 sure_mass;   // weight of bins better than `sure`
};

__device__ __forceinline__ bool limited(const RowLimits &l, int64_t n) {
  return l.k < n || l.p < 2.0f;
}

// Whether rank_cuts settles a list.
__device__ __forceinline__ bool ranked(const RowLimits &l, int64_t n, uint32_t listed) {
  return l.k < n && l.p < 2.0f && listed <= (uint32_t)min(kRanked, (int)blockDim.x);
}

// counted(b), weighed(b): what lies in a bin.  everything: there are no weights
// by bin, and all entries down to top-k's bin are listed.
template <typename C, typename W>
__device__ __forceinline__ Bins settle(Search &s, const RowLimits &l, int64_t n, int bins,
                                       bool everything, C counted, W weighed) {
  Bins b = {bins, 0, 0, 0, bins, -1, 0};
  if (l.k < n) {
    const u64 entries = block_find(s, bins, [&](u64) { return (u64)l.k; }, 0, counted);
    if ((u64)l.k < entries) {
      b.k_bin = s.bin;
      b.k_above = s.above;
      b.sure = b.last = b.k_bin;
    }
    __syncthreads();
  }
  const auto share = [&](u64 all) { return share_of(l.p, all); };
  if (everything) {
    // all down to the bin (to the last one where k keeps all)
    if (b.k_bin == bins) b.last = bins - 1;
    b.sure = 0;
  } else if (l.p < 2.0f) {
    if (b.k_bin < bins) {
      // between the weight of better bins and that with the cut's own
      b.k_mass = b.sure_mass = block_find(s, b.k_bin, share, 0, weighed);
      if (s.bin >= 0) {  // (no weight above the cut's bin: that one is the first)
        b.sure = s.bin;
        b.sure_mass = s.above;
      }
      __syncthreads();
      block_find(s, b.k_bin + 1, share, 0, weighed);
    } else {
      b.all = block_find(s, bins, share, 0, weighed);
      b.sure = s.bin;
      b.sure_mass = s.above;
    }
    b.last = min(s.bin, b.k_bin < bins ? b.k_bin : bins - 1);
    __syncthreads();
  }
  return b;
}

// The cut of both limits.  each(f) calls f(key, weight, bin) for the listed
// entries, where weight() and bin() are only worked out where they are needed.
template <typename W, typename Each>
__device__ __forceinline__ u64 find_cuts(Search &s, const RowLimits &l, const Bins &b, int bins,
                                         bool everything, W weighed, Each each) {
  u64 cut = 0;
  if (b.k_bin < bins)
    cut = find_cut(s, true, b.k_above, (u64)l.k, 0, each,
                   [&](auto bin) { return bin() == b.k_bin; });
  if (!(l.p < 2.0f)) return cut;
  __syncthreads();
  // the weight that top-k keeps: better bins' and the listed entries'
  u64 total = b.all;
  if (everything || b.k_bin < bins) {
    u64 part = 0;
    each([&](u64 key, auto q, auto bin) {
      if (key >= cut && (everything || bin() == b.k_bin)) part += q();
    });
    block_prefix(part, s.wave_sum, &total);
    total += everything ? 0 : b.k_mass;
    __syncthreads();
  }
  const u64 share = share_of(l.p, total);
  int p_bin = -1;  // all bins
  u64 above = 0;
  if (!everything) {
    block_find(s, bins, [&](u64) { return share; }, 0, weighed);
    p_bin = s.bin;
    above = s.above;
    __syncthreads();
  }
  return find_cut(s, false, above, share, cut, each,
                  [&](auto bin) { return p_bin < 0 || bin() == p_bin; });
}

// The same for a list of at most 64 entries in LDS: one wave, an entry a lane,
// without a barrier but the last (1 x 4,096 with 26 such entries: 12.3 us, 14.2
// in the way below, which all waves go).
__device__ __forceinline__ u64 wave_cuts(Search &s, const RowLimits &l, const Bins &b, int bins,
                                         bool everything, int open, const u64 *keys,
                                         const uint32_t *qs, const uint16_t *bin_of_entry) {
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    const u64 key = lane < open ? keys[lane] : 0;  // 0: below every key
    const int bin = lane < open ? bin_of_entry[lane] : bins;
    const uint32_t q = lane < open ? qs[lane] : 0;
    const u64 in_bin = __ballot(lane < open && bin == b.k_bin);
    u64 before = b.k_above, mass = b.sure_mass;
#pragma unroll 4
    for (int j = 0; j < open; ++j) {
      const bool better = from_lane(key, j) > key;
      mass += better ? from_lane(q, j) : 0u;
      before += better ? (uint32_t)(in_bin >> j) & 1u : 0u;
    }
    bool kept = lane < open &&
                (b.k_bin == bins || bin < b.k_bin || (bin == b.k_bin && before < (u64)l.k));
    if (l.p < 2.0f) {
      u64 total = b.all;
      if (everything || b.k_bin < bins) {
        const u64 part = kept && (everything || bin == b.k_bin) ? q : 0u;
        total = from_lane(wave_prefix(part), 63) + (everything ? 0 : b.k_mass);
      }
      kept = kept && q != 0 && bin >= b.sure && bin <= b.last && mass < share_of(l.p, total);
    }
    // None of the list kept: all that is kept lies in better bins, whose keys are larger.
    const u64 least = wave_fold(kept ? key : ~0ull, ~0ull, [](u64 a, u64 b) { return min(a, b); });
    const u64 most = wave_fold(key, 0ull, [](u64 a, u64 b) { return max(a, b); });
    if (lane == 63) s.lo = least != ~0ull ? least : most + 1;
  }
  __syncthreads();
  return s.lo;
}

// The same for a list of at most kRanked entries in LDS, one a thread: every
// entry adds up those before it, which come from the wave's own registers, 64
// at a time.  Both cuts come of one pass, where find_cuts, at seven barriers a
// step, searches for one after the other; for a single cut find_cuts is the
// quicker one (96 entries, first this way, then find_cuts: 1 x 100,000 with both
// limits 33 us against 35, with one 33 against 29; 1 x 4,096 18 against 17, 16
// against 12).
__device__ __forceinline__ u64 rank_cuts(Search &s, const RowLimits &l, const Bins &b, int bins,
                                         bool everything, int open, const u64 *keys,
                                         const uint32_t *qs, const uint16_t *bin_of_entry) {
  const int e = threadIdx.x;
  const u64 key = e < open ? keys[e] : 0;
  const int bin = e < open ? bin_of_entry[e] : bins;
  const uint32_t q = e < open ? qs[e] : 0;
  u64 before = b.k_above, mass = b.sure_mass;
  const int lane = threadIdx.x & 63;
  if (e - lane < open) {
    for (int j0 = 0; j0 < open; j0 += 64) {
      const int mine = j0 + lane;
      const u64 theirs = mine < open ? keys[mine] : 0;  // below every key
      const uint32_t weight_of = mine < open ? qs[mine] : 0;
      const u64 in_bin = __ballot(mine < open && bin_of_entry[mine] == b.k_bin);
#pragma unroll 8
      for (int j = 0; j < 64; ++j) {
        const bool better = from_lane(theirs, j) > key;
        mass += better ? from_lane(weight_of, j) : 0u;
        if ((in_bin >> j) & 1) before += better ? 1u : 0u;
      }
    }
  }
  // kept by top-k
  bool kept = e < open && (b.k_bin == bins || bin < b.k_bin || (bin == b.k_bin && before < (u64)l.k));
  if (threadIdx.x == 0) s.lo = ~0ull;
  if (l.p < 2.0f) {
    u64 total = b.all;
    if (everything || b.k_bin < bins) {
      block_prefix(kept && (everything || bin == b.k_bin) ? q : 0u, s.wave_sum, &total);
      total += everything ? 0 : b.k_mass;
    }
    kept = kept && q != 0 && bin >= b.sure && bin <= b.last && mass < share_of(l.p, total);
  }
  __syncthreads();
  const u64 least = wave_fold(kept ? key : ~0ull, ~0ull, [](u64 a, u64 b) { return min(a, b); });
  if ((threadIdx.x & 63) == 63 && least != ~0ull) atomicMin(&s.lo, least);
  __syncthreads();
  // None of the list kept: all that is kept lies in better bins, whose keys are larger.
  const u64 cut = s.lo;
  if (cut != ~0ull) return cut;
  const u64 most = wave_fold(e < open ? key : 0, 0ull, [](u64 a, u64 b) { return max(a, b); });
  __syncthreads();
  if (threadIdx.x == 0) s.hi = 0;
  __syncthreads();
  if ((threadIdx.x & 63) == 63) atomicMax(&s.hi, most);
  __syncthreads();
  return s.hi + 1;
}

// floor(u * total), kept inside [0, total).
__device__ __forceinline__ u64 wanted(float u, u64 total) {
  const double at = floor((double)u * (double)total);
  return at >= 0.0 ? min(at < 9.0e18 ? (u64)at : total, total - 1) : 0;
}

__device__ __forceinline__ void no_entry(const SampleArgs &a, int64_t row) {
  for (int j = threadIdx.x; j < a.draws; j += blockDim.x) {
    a.idx[row * a.draws + j] = -1;
    a.logprob[row * a.draws + j] = -__builtin_inff();
  }
}

__device__ __forceinline__ float log_total(u64 total) { return logf((float)total / kOne); }

// Best and worst over the workgroup, in every thread.
__device__ __forceinline__ float2 block_range(float hi, float lo, float2 *lds) {
  const auto most = [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  };
  const auto least = [](uint32_t a, uint32_t b) {
    return __float_as_uint(fminf(__uint_as_float(a), __uint_as_float(b)));
  };
  const uint32_t inf = __float_as_uint(__builtin_inff());
  hi = __uint_as_float(wave_fold(__float_as_uint(hi), inf | 0x80000000u, most));
  lo = __uint_as_float(wave_fold(__float_as_uint(lo), inf, least));
  if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = make_float2(hi, lo);
  __syncthreads();
  hi = -__builtin_inff();
  lo = __builtin_inff();
  for (int w = 0; w < (int)blockDim.x >> 6; ++w) {
    hi = fmaxf(hi, lds[w].x);
    lo = fminf(lo, lds[w].y);
  }
  __syncthreads();
  return make_float2(hi, lo);
}

// ---- short rows: one workgroup -------------------------------------------------

// The row's scores and weights in LDS: every entry is read from memory and
// exponentiated once.  A thread's own entries are groups of 8.
template <typename T>
__global__ __launch_bounds__(1024) void row_kernel(SampleArgs a) {
  __shared__ Search s;
  __shared__ float2 range[16];
  __shared__ uint32_t count[kSub], list_q[kRowList], listed;
  __shared__ u64 mass[kSub], list_key[kRowList];
  __shared__ uint16_t list_bin[kRowList];
  extern __shared__ __attribute__((aligned(16))) char raw[];
  const int64_t row = blockIdx.x;
  const int n = (int)a.s.n, groups = (n + 7) / 8;
  float4 *xs = reinterpret_cast<float4 *>(raw);
  uint4 *qs = reinterpret_cast<uint4 *>(xs + groups * 2);
  u64 *group_end = reinterpret_cast<u64 *>(qs + groups * 2);  // running weight after 8 entries
  const T *scores = static_cast<const T *>(a.s.scores) + row * a.s.ld;
  const uint8_t *valid = a.s.valid ? a.s.valid + row * a.s.valid_ld : nullptr;
  const int threads = blockDim.x, t = threadIdx.x;
  const float ninf = -__builtin_inff();
  const RowSettings set = row_settings(a, row);
  const float u0 = t < a.draws ? a.u[row * a.draws + t] : 0.0f;

  for (int b = t; b < kSub; b += threads) count[b] = 0, mass[b] = 0;
  float hi = ninf, lo = __builtin_inff();
  for (int g = t; g < groups; g += threads) {
    float x[8];
    load8(scores, valid, (int64_t)g * 8, n, x);
    xs[g * 2] = make_float4(x[0], x[1], x[2], x[3]);
    xs[g * 2 + 1] = make_float4(x[4], x[5], x[6], x[7]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      hi = fmaxf(hi, x[j]);
      lo = fminf(lo, x[j] == ninf ? __builtin_inff() : x[j]);
    }
  }
  const float2 ends = block_range(hi, lo, range);
  if (ends.x == ninf) return no_entry(a, row);
  const RowLimits l = row_limits(set, n, ends.x, ends.y);
  const bool limits = limited(l, n);
  const float scale = (float)kSub / l.range;
  for (int h = t; h < groups * 2; h += threads) {
    const float4 x = xs[h];
    const float xv[4] = {x.x, x.y, x.z, x.w};
    uint32_t q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float z = exponent(xv[j], l);
      q[j] = weight(z);
      if (limits && q[j]) {
        const int b = bin_of<kSub>(z, scale);
        atomicAdd(&count[b], 1u);
        atomicAdd(&mass[b], (u64)q[j]);
      }
    }
    qs[h] = make_uint4(q[0], q[1], q[2], q[3]);
  }
  __syncthreads();

  u64 cut = 0;  // entries with a smaller key are not kept
  if (limits) {
    auto weighed = [&](int j) { return mass[j]; };
    const Bins b = settle(s, l, n, kSub, false, [&](int j) { return (u64)count[j]; }, weighed);
    // f(index, score, weight, bin) for the entries that the bins do not settle
    auto each_open = [&](auto f) {
#pragma unroll 1
      for (int h = t; h < groups * 2; h += threads) {
        const float4 x = xs[h];
        const uint4 q = qs[h];
        const float xv[4] = {x.x, x.y, x.z, x.w};
        const uint32_t qv[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (qv[j] == 0) continue;
          const int bin = bin_of<kSub>(exponent(xv[j], l), scale);
          if ((bin >= b.sure && bin <= b.last) || bin == b.k_bin)
            f(key_of(xv[j], h * 4 + j), [&] { return qv[j]; }, [&] { return bin; });
        }
      }
    };
    if (t == 0) listed = 0;
    __syncthreads();
    each_open([&](u64 key, auto q, auto bin) {
      const uint32_t at = atomicAdd(&listed, 1u);
      if (at < kRowList) {
        list_key[at] = key;
        list_q[at] = q();
        list_bin[at] = (uint16_t)bin();
      }
    });
    __syncthreads();
    const int open = (int)listed;
    if (open <= 64)
      cut = wave_cuts(s, l, b, kSub, false, open, list_key, list_q, list_bin);
    else if (ranked(l, n, listed))
      cut = rank_cuts(s, l, b, kSub, false, open, list_key, list_q, list_bin);
    else
      cut = find_cuts(s, l, b, kSub, false, weighed, [&](auto f) {
        if (open > kRowList) return each_open(f);
#pragma unroll 1
        for (int e = t; e < open; e += threads)
          f(list_key[e], [&] { return list_q[e]; }, [&] { return (int)list_bin[e]; });
      });
    __syncthreads();
  }

  // running weights of the kept entries, a round of `threads` groups at a time
  u64 total = 0;
  for (int g0 = 0; g0 < groups; g0 += threads) {
    const int g = g0 + t;
    u64 sum = 0;
    if (g < groups) {
      uint32_t q[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 x = xs[g * 2 + h];
        const uint4 w = qs[g * 2 + h];
        const float xv[4] = {x.x, x.y, x.z, x.w};
        const uint32_t wv[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          q[h * 4 + j] = exponent(xv[j], l) >= l.min_z && key_of(xv[j], g * 8 + h * 4 + j) >= cut
                             ? wv[j] : 0u;
          sum += q[h * 4 + j];
        }
      }
      qs[g * 2] = make_uint4(q[0], q[1], q[2], q[3]);
      qs[g * 2 + 1] = make_uint4(q[4], q[5], q[6], q[7]);
    }
    u64 all;
    const u64 before = block_prefix(sum, s.wave_sum, &all);
    if (g < groups) group_end[g] = total + before + sum;
    total += all;
    __syncthreads();
  }
  const float lt = log_total(total);
  const uint32_t *q1 = reinterpret_cast<const uint32_t *>(qs);
  for (int j = t; j < a.draws; j += threads) {
    const u64 want = wanted(j == t ? u0 : a.u[row * a.draws + j], total);
    int first = 0, last = groups - 1;  // the group whose end passes `want`
    while (first < last) {
      const int mid = (first + last) / 2;
      if (group_end[mid] > want) last = mid; else first = mid + 1;
    }
    u64 now = first > 0 ? group_end[first - 1] : 0;
    int e = first * 8;
    for (; e < first * 8 + 7; ++e) {
      now += q1[e];
      if (now > want) break;
    }
    a.idx[row * a.draws + j] = e;
    a.logprob[row * a.draws + j] = exponent(reinterpret_cast<const float *>(xs)[e], l) - lt;
  }
}

// ---- long rows -------------------------------------------------------------------

// A row as settle_kernel leaves it, the same as scores: x_keep: kept for sure;
// x_sure, x_last: the least of bins < sure, <= last; x_k, x_k_end: of bins
// <= k_bin, < k_bin where that lies apart (NaN: no score).
struct RowState {
  RowLimits l;
  Bins b;
  float x_keep, x_sure, x_last, x_k, x_k_end;
  u64 cut, total;  // of finish_kernel
};

struct Long {
  SampleArgs a;
  int64_t row0;              // first row of the batch
  int64_t chunk, chunks;     // entries of a chunk, chunks of a row
  int64_t span, spans;       // the same of count_kernel's parts
  int64_t tile, tiles;       // the same of tiles; a chunk is a number of tiles
  uint32_t segments, segment_most;  // of a row's list: parts with a counter each
  float2 *range;             // [rows][chunks]: best, worst
  u64 *mass;                 // [rows][kBins]
  uint32_t *count;           // [rows][kBins]
  u64 *tile_mass;            // [rows][tiles], running sums after finish_kernel
  u64 *list;                 // [rows][segments][segment_most] keys
  uint32_t *listed;          // [rows][kSegments]
  RowState *state;           // [rows]
};

template <typename T>
__device__ __forceinline__ const T *row_scores(const Long &k, int64_t r) {
  return static_cast<const T *>(k.a.s.scores) + (k.row0 + r) * k.a.s.ld;
}

__device__ __forceinline__ const uint8_t *row_mask(const Long &k, int64_t r) {
  return k.a.s.valid ? k.a.s.valid + (k.row0 + r) * k.a.s.valid_ld : nullptr;
}

__device__ __forceinline__ RowLimits chunk_limits(const Long &k, int64_t r, float2 *lds) {
  const RowSettings set = row_settings(k.a, k.row0 + r);
  float hi = -__builtin_inff(), lo = __builtin_inff();
  for (int64_t c = threadIdx.x; c < k.chunks; c += blockDim.x) {
    const float2 v = k.range[r * k.chunks + c];
    hi = fmaxf(hi, v.x);
    lo = fminf(lo, v.y);
  }
  const float2 v = block_range(hi, lo, lds);
  return row_limits(set, k.a.s.n, v.x, v.y);
}

template <typename T>
__global__ __launch_bounds__(256) void range_kernel(Long k) {
  __shared__ float2 lds[4];
  const int64_t r = blockIdx.x / k.chunks, c = blockIdx.x % k.chunks;
  for (int64_t b = c * 256 + threadIdx.x; b < kBins; b += k.chunks * 256) {
    k.mass[r * kBins + b] = 0;
    k.count[r * kBins + b] = 0;
  }
  if (c == 0 && threadIdx.x < kSegments) k.listed[r * kSegments + threadIdx.x] = 0;
  const T *scores = row_scores<T>(k, r);
  const uint8_t *valid = row_mask(k, r);
  const int64_t end = min(k.a.s.n, (c + 1) * k.chunk);
  const float ninf = -__builtin_inff();
  float hi = ninf, lo = __builtin_inff();
  for (int64_t i = c * k.chunk + threadIdx.x * 8; i < end; i += 256 * 16) {
    Eight<T> e[2];
    e[0].load(scores, valid, i, end);
    e[1].load(scores, valid, i + 256 * 8, end);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float x[8];
      e[h].get(valid != nullptr, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        hi = fmaxf(hi, x[j]);  // a NaN is neither
        lo = fminf(lo, x[j] == ninf ? __builtin_inff() : x[j]);
      }
    }
  }
  const float2 v = block_range(hi, lo, lds);
  if (threadIdx.x == 0) k.range[blockIdx.x] = v;
}

// A row whose top-k needs no weights by bin: everything it keeps is listed.
__device__ __forceinline__ bool lists_all(const RowLimits &l) { return l.k <= kFew; }

// A row whose entries need no care: z is (s - m) * R as it stands.
__device__ __forceinline__ bool ordinary(const RowLimits &l) {
  return l.m < __builtin_inff() && l.r < __builtin_inff();
}

// Entries base .. stop-1 into the bins.
template <typename T, bool WEIGH, bool ORDINARY>
__device__ __forceinline__ void count_entries(const T *scores, const uint8_t *valid, int64_t base,
                                              int64_t stop, const RowLimits &l, u64 *bins) {
  const float scale = (float)kBins / l.range;
  int64_t i = base + threadIdx.x * 8;
  Eight<T> next;
  next.load(scores, valid, i, stop);
  for (; i < stop; i += 1024 * 8) {
    const Eight<T> now = next;
    next.load(scores, valid, i + 1024 * 8, stop);
    float x[8];
    now.get(valid != nullptr, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float z = ORDINARY ? (x[j] - l.m) * l.r : exponent(x[j], l);
      if constexpr (WEIGH) {
        const uint32_t q = weight(z);
        if (q) atomicAdd(&bins[bin_of<kBins>(z, scale)], ((u64)q << 17) | 1ull);
      } else if (z > kLowest) {
        atomicAdd(reinterpret_cast<uint32_t *>(&bins[bin_of<kBins>(z, scale)]), 1u);
      }
    }
  }
}

// Adding a part's bins to the row's costs as much as some ten thousand
// entries, so the parts are as long as still fill the device: sixteen waves
// share the bins.  Counts serve top-k alone, weights top-p alone.
template <typename T>
__global__ __launch_bounds__(1024) void count_kernel(Long k) {
  __shared__ float2 lds[16];
  __shared__ u64 bins[kBins];  // (weight << 17) | count: up to kPacked entries
  const int64_t r = blockIdx.x / k.spans, c = blockIdx.x % k.spans;
  for (int b = threadIdx.x; b < kBins; b += 1024) bins[b] = 0;
  const RowLimits l = chunk_limits(k, r, lds);
  if (l.m == -__builtin_inff() || !limited(l, k.a.s.n)) return;
  const bool weigh = !lists_all(l) && l.p < 2.0f, counts = l.k < k.a.s.n;
  const T *scores = row_scores<T>(k, r);
  const uint8_t *valid = row_mask(k, r);
  const int64_t end = min(k.a.s.n, (c + 1) * k.span);
  for (int64_t base = c * k.span; base < end; base += kPacked) {
    const int64_t stop = min(end, base + kPacked);
    if (!ordinary(l))
      weigh ? count_entries<T, true, false>(scores, valid, base, stop, l, bins)
            : count_entries<T, false, false>(scores, valid, base, stop, l, bins);
    else
      weigh ? count_entries<T, true, true>(scores, valid, base, stop, l, bins)
            : count_entries<T, false, true>(scores, valid, base, stop, l, bins);
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += 1024) {
      const u64 v = bins[b];
      if (!v) continue;
      bins[b] = 0;
      if (counts) atomicAdd(&k.count[r * kBins + b], (uint32_t)(v & 0x1FFFF));
      if (weigh) atomicAdd(&k.mass[r * kBins + b], v >> 17);
    }
    __syncthreads();
  }
}

// The least score for which holds(score) is true, given that it is for the
// row's best score and stays true as scores rise.  Sixteen lanes of a row of
// lanes look for one score together, each row of lanes for its own.
template <typename F>
__device__ __forceinline__ float least_score(const RowLimits &l, F holds) {
  const int lane = threadIdx.x & 63, row0 = lane & ~15;
  uint32_t lo = ordered(-__builtin_inff()), hi = ordered(l.m);  // holds(hi)
  while (__any(lo < hi)) {
    // 16 probes in [lo, hi): the first that holds and the one before it
    const uint32_t step = (hi - lo) / 17 + 1, at = lo + step * (uint32_t)(lane & 15);
    const bool yes = at >= hi || holds(key_score((u64)at << 32));
    const uint32_t rows = (uint32_t)(__ballot(yes) >> row0) & 0xFFFFu;
    const int first = rows ? __ffs((int)rows) - 1 : 16;
    if (lo < hi) {
      const uint32_t low = first > 0 ? lo + step * (uint32_t)(first - 1) + 1 : lo;
      if (first < 16) hi = min(hi, lo + step * (uint32_t)first);
      lo = min(hi, low);
    }
  }
  return key_score((u64)hi << 32);
}

// What the bins say of every entry, as scores to compare with: bins fall as
// scores rise.  A workgroup a row.
__global__ __launch_bounds__(512) void settle_kernel(Long k) {
  __shared__ Search s;
  __shared__ float2 lds[8];
  __shared__ uint32_t count[kBins];
  __shared__ u64 mass[kBins];
  __shared__ float edges[5];
  const int64_t r = blockIdx.x;
  if (k.a.top_k || k.a.top_p || k.a.s.temperature) {
    for (int j = threadIdx.x; j < kBins; j += 512) {
      count[j] = k.count[r * kBins + j];
      mass[j] = k.mass[r * kBins + j];
    }
  }
  const RowLimits l = chunk_limits(k, r, lds);  // ends with a barrier
  if (l.m == -__builtin_inff()) {
    if (threadIdx.x == 0) k.state[r].l = l;
    return;
  }
  Bins b = {kBins, 0, 0, 0, kBins, -1, 0};
  if (limited(l, k.a.s.n))
    b = settle(s, l, k.a.s.n, kBins, lists_all(l), [&](int j) { return (u64)count[j]; },
               [&](int j) { return mass[j]; });
  // the edges: a row of 16 lanes each
  const float scale = (float)kBins / l.range;
  const int which = (int)threadIdx.x >> 4;
  const bool apart = b.k_bin < kBins && (b.k_bin < b.sure || b.k_bin > b.last);
  if (threadIdx.x < 128) {
    const int of = which == 0 ? b.sure - 1 : which == 1 ? b.last
                 : !apart ? -1 : which == 2 ? b.k_bin : b.k_bin - 1;
    float edge;
    if (threadIdx.x < 64)
      edge = least_score(l, [&](float x) {
        const float z = exponent(x, l);
        return z > kLowest && bin_of<kBins>(z, scale) <= max(of, 0);
      });
    else
      edge = least_score(l, [&](float x) { return exponent(x, l) >= l.min_z; });
    if (which < 4 && of < 0) edge = __builtin_nanf("");
    if ((threadIdx.x & 15) == 0 && which < 5) edges[which] = edge;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    RowState &st = k.state[r];
    st.l = l;
    st.b = b;
    st.x_sure = edges[0];
    st.x_last = edges[1];
    st.x_k = edges[2];
    st.x_k_end = edges[3];
    st.x_keep = edges[0] == edges[0] ? fmaxf(edges[0], edges[4]) : edges[0];
  }
}

// Where few of the entries are kept for sure, their scores go through a queue
// in LDS, so that the exponentials run on full waves.  Listed entries are
// gathered in LDS and added to one of the row's segments: additions to one
// counter wait for one another, some 20 ns each.
template <typename T>
__global__ __launch_bounds__(256) void collect_kernel(Long k) {
  __shared__ float queues[4][kTile / 2 + 64];
  __shared__ u64 open[kOpen];
  __shared__ uint32_t opened, open_at;
  if (threadIdx.x == 0) opened = 0;
  __syncthreads();
  const int64_t r = blockIdx.x / k.chunks, c = blockIdx.x % k.chunks;
  const RowState &st = k.state[r];
  const RowLimits l = st.l;
  if (l.m == -__builtin_inff()) return;
  const float x_keep = st.x_keep, x_sure = st.x_sure, x_last = st.x_last, x_k = st.x_k,
              x_k_end = st.x_k_end;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T *scores = row_scores<T>(k, r);
  const uint8_t *valid = row_mask(k, r);
  const uint32_t part = (uint32_t)c % k.segments;
  u64 *list = k.list + ((size_t)r * k.segments + part) * k.segment_most;
  uint32_t *listed = &k.listed[r * kSegments + part];
  const int64_t end = min(k.a.s.n, (c + 1) * k.chunk);
  const bool plain = ordinary(l), apart = x_k == x_k;
  float *queue = queues[wave];
  int queued = 0;
  const int steps = (int)(k.tile / kTile);
  const int64_t t0 = c * k.chunk + wave * k.tile;
  Eight<T> next;
  if (t0 < end) next.load(scores, valid, t0 + lane * 8, end);
  for (int64_t t = t0; t < end; t += 4 * k.tile) {
    u64 sum = 0;
    for (int step = 0; step < steps; ++step) {
      const int64_t i = t + step * kTile + lane * 8;
      const Eight<T> now = next;
      next.load(scores, valid, step + 1 < steps ? i + kTile : t + 4 * k.tile + lane * 8, end);
      float x[8];
      now.get(valid != nullptr, x);
      // no short-circuits: comparisons go to scalar masks, without branches
      u64 keep[8];
      bool waits = false;
      int kept = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        keep[j] = __ballot(x[j] >= x_keep);
        kept += __popcll(keep[j]);
        waits = waits | ((x[j] >= x_last) & !(x[j] >= x_sure));
      }
      if (apart) {
#pragma unroll
        for (int j = 0; j < 8; ++j) waits = waits | ((x[j] >= x_k) & !(x[j] >= x_k_end));
      }
      if (kept > kTile / 2) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          sum += x[j] >= x_keep ? weight(plain ? (x[j] - l.m) * l.r : exponent(x[j], l)) : 0u;
      } else if (kept) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (x[j] >= x_keep)
            queue[queued + __builtin_amdgcn_mbcnt_hi((uint32_t)(keep[j] >> 32),
                                                     __builtin_amdgcn_mbcnt_lo((uint32_t)keep[j], 0))] =
                x[j];
          queued += __popcll(keep[j]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        while (queued >= 64) {
          queued -= 64;
          sum += weight(exponent(queue[queued + lane], l));
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
      if (__any(waits)) {
        uint32_t wait = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          wait |= (((x[j] >= x_last) & !(x[j] >= x_sure)) | ((x[j] >= x_k) & !(x[j] >= x_k_end)))
                      ? 1u << j : 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (!((wait >> j) & 1u)) continue;
          const u64 key = key_of(x[j], i + j);
          const uint32_t at = atomicAdd(&opened, 1u);
          if (at < kOpen) {
            open[at] = key;
          } else {
            const uint32_t to = atomicAdd(listed, 1u);
            if (to < k.segment_most) list[to] = key;
          }
        }
      }
    }
    if (lane < queued) sum += weight(exponent(queue[lane], l));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    queued = 0;
    sum = wave_prefix(sum);
    if (lane == 63) k.tile_mass[r * k.tiles + t / k.tile] = sum;
  }
  __syncthreads();
  const uint32_t count = min(opened, (uint32_t)kOpen);
  if (count == 0) return;
  if (threadIdx.x == 0) open_at = atomicAdd(listed, count);
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < count; e += 256)
    if (open_at + e < k.segment_most) list[open_at + e] = open[e];
}

// One draw by one wave: the tile whose running weight passes `want`, then the
// entry inside it.
template <typename T>
__device__ __forceinline__ void draw_one(const Long &k, int64_t r, int j, float u,
                                         const RowLimits &l, u64 cut, u64 total,
                                         const u64 *tile_end) {
  const int lane = threadIdx.x & 63;
  const int64_t at = (k.row0 + r) * k.a.draws + j;
  const u64 want = wanted(u, total);
  // the first tile whose end passes `want`: 64 candidates at a time
  int first = 0;
  for (int width = 4096; width > 1; width >>= 6) {
    const int part = width >> 6, last = first + lane * part + part - 1;
    const u64 passed =
        __ballot(last >= (int)k.tiles - 1 || tile_end[min(last, (int)k.tiles - 1)] > want);
    first += part * (__ffsll(passed) - 1);
  }
  u64 run = first > 0 ? tile_end[first - 1] : 0;
  const T *scores = row_scores<T>(k, r);
  const uint8_t *valid = row_mask(k, r);
  const int64_t end = min(k.a.s.n, (first + 1) * k.tile);
  Eight<T> next[2];
  next[0].load(scores, valid, first * k.tile + lane * 8, end);
  next[1].load(scores, valid, first * k.tile + kTile + lane * 8, end);
  for (int64_t base = first * k.tile; base < end; base += kTile) {
    const int64_t i = base + lane * 8;
    const Eight<T> now = next[0];
    next[0] = next[1];
    next[1].load(scores, valid, i + 2 * kTile, end);
    float x[8];
    now.get(valid != nullptr, x);
    uint32_t q[8];
    u64 sum = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float z = exponent(x[e], l);
      q[e] = z >= l.min_z && key_of(x[e], i + e) >= cut ? weight(z) : 0u;
      sum += q[e];
    }
    const u64 incl = wave_prefix(sum);
    const u64 found = __ballot(run + incl > want);
    if (found) {
      if (lane == __ffsll(found) - 1) {
        u64 now_at = run + incl - sum;
        float z = 0.0f;
        int e = -1;
#pragma unroll
        for (int f = 0; f < 8; ++f) {
          now_at += q[f];
          if (e < 0 && now_at > want) {
            e = f;
            z = exponent(x[f], l);
          }
        }
        k.a.idx[at] = (int32_t)(i + e);
        k.a.logprob[at] = z - log_total(total);
      }
      return;
    }
    run += from_lane(incl, 63);
  }
}

struct Finish {
  Search s;
  u64 mass[kBins];
  u64 keys[kList];
  uint32_t q[kList];
  uint16_t bin[kList];
  u64 tile[kMaxTiles];
  u64 wave_sum[16];
  uint32_t segment_end[kSegments];
};

template <typename T>
__global__ __launch_bounds__(1024) void finish_kernel(Long k) {
  extern __shared__ __attribute__((aligned(16))) char raw[];
  Finish &sh = *reinterpret_cast<Finish *>(raw);
  const int64_t r = blockIdx.x, row = k.row0 + r, n = k.a.s.n;
  const int wave = threadIdx.x >> 6, threads = blockDim.x, waves = threads >> 6;
  const RowState &settled = k.state[r];
  const T *scores = row_scores<T>(k, r);
  const uint8_t *valid = row_mask(k, r);
  const u64 *list = k.list + (size_t)r * k.segments * k.segment_most;
  const int lane = threadIdx.x & 63;
  uint32_t part = lane < kSegments ? k.listed[r * kSegments + lane] : 0;
  const bool fits = !__any(part > k.segment_most);
  part = wave_prefix(part);
  const uint32_t listed = from_lane(part, 63);
  if (threadIdx.x < kSegments) sh.segment_end[threadIdx.x] = part;
  const bool held = fits && listed <= (uint32_t)kList;
  // entry e of the list: its segment by the segments' ends
  auto entry = [&](uint32_t e) {
    uint32_t at = 0;
#pragma unroll
    for (uint32_t step = kSegments / 2; step; step >>= 1)
      if (sh.segment_end[at + step - 1] <= e) at += step;
    return list[(size_t)at * k.segment_most + (e - (at ? sh.segment_end[at - 1] : 0))];
  };
  __syncthreads();
  const float u0 = wave < k.a.draws ? k.a.u[row * k.a.draws + wave] : 0.0f;
  for (int t = threadIdx.x; t < k.tiles; t += threads) sh.tile[t] = k.tile_mass[r * k.tiles + t];
  if (held)
    for (uint32_t e = threadIdx.x; e < listed; e += threads) sh.keys[e] = entry(e);
  const RowLimits l = settled.l;
  if (l.m == -__builtin_inff()) return no_entry(k.a, row);
  const Bins b = settled.b;
  const float scale = (float)kBins / l.range;
  if (held)
    for (uint32_t e = threadIdx.x; e < listed; e += threads) {
      const float z = exponent(key_score(sh.keys[e]), l);
      sh.q[e] = weight(z);
      sh.bin[e] = (uint16_t)bin_of<kBins>(z, scale);
    }

  u64 cut = 0;
  if (limited(l, n)) {
    const bool everything = lists_all(l);
    if (!everything && l.p < 2.0f) {
      for (int j = threadIdx.x; j < kBins; j += threads) sh.mass[j] = k.mass[r * kBins + j];
    }
    __syncthreads();
    // f(key, weight, bin) for every listed entry.  A list longer than LDS holds
    // stays in memory, its segments shared among the waves; one that did not
    // fit there is read from the row again, by this one workgroup and once a
    // step: where more entries than the list holds have nearly the score of a
    // cut.  Equal scores are the worst of it: 1 x 65,536 of them 0.2 ms, 1 x
    // 1,048,576 2 ms, 1 x 16,777,216 40 ms.
    auto each = [&](auto f) {
      auto one = [&](u64 key) {
        const float z = exponent(key_score(key), l);
        f(key, [&] { return weight(z); }, [&] { return bin_of<kBins>(z, scale); });
      };
      if (held) {
#pragma unroll 1
        for (uint32_t e = threadIdx.x; e < listed; e += threads)
          f(sh.keys[e], [&] { return sh.q[e]; }, [&] { return (int)sh.bin[e]; });
      } else if (fits) {
        const int segments = (int)k.segments;
#pragma unroll 1
        for (int g = wave % segments; g < segments; g += waves) {
          // the waves that share this segment, and which of them this one is
          const int sharing = waves > segments ? (waves - g + segments - 1) / segments : 1;
          const uint32_t from = g ? sh.segment_end[g - 1] : 0, count = sh.segment_end[g] - from;
          const u64 *keys = list + (size_t)g * k.segment_most;
#pragma unroll 1
          for (uint32_t e = (uint32_t)(wave / segments * 64 + lane); e < count; e += sharing * 512) {
            u64 key[8];  // on their way at once
#pragma unroll
            for (int j = 0; j < 8; ++j)
              key[j] = e + j * sharing * 64 < count ? keys[e + j * sharing * 64] : 0;
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (key[j]) one(key[j]);
          }
        }
      } else {
#pragma unroll 1
        for (int64_t i = (int64_t)threadIdx.x * 8; i < n; i += (int64_t)threads * 8) {
          float x[8];
          load8(scores, valid, i, n, x);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float z = exponent(x[j], l);
            if (!(z > kLowest)) continue;
            const int bin = bin_of<kBins>(z, scale);
            if ((bin >= b.sure && bin <= b.last) || bin == b.k_bin) one(key_of(x[j], i + j));
          }
        }
      }
    };
    if (fits && listed <= 64)
      cut = wave_cuts(sh.s, l, b, kBins, everything, (int)listed, sh.keys, sh.q, sh.bin);
    else if (fits && ranked(l, n, listed))
      cut = rank_cuts(sh.s, l, b, kBins, everything, (int)listed, sh.keys, sh.q, sh.bin);
    else
      cut = find_cuts(sh.s, l, b, kBins, everything, [&](int j) { return sh.mass[j]; }, each);
    __syncthreads();
    // the listed entries that are kept join their tiles
    each([&](u64 key, auto q, auto bin) {
      if (key >= cut && bin() >= b.sure && exponent(key_score(key), l) >= l.min_z)
        atomicAdd(&sh.tile[key_index(key) / k.tile], (u64)q());
    });
  }
  __syncthreads();
  // running weights of the tiles, each thread a few in a row
  const int per = ((int)k.tiles + threads - 1) / threads;
  const int first = min((int)k.tiles, (int)threadIdx.x * per), last = min((int)k.tiles, first + per);
  u64 sum = 0;
  for (int t = first; t < last; ++t) sum += sh.tile[t];
  u64 total;
  u64 run = block_prefix(sum, sh.wave_sum, &total);
  for (int t = first; t < last; ++t) sh.tile[t] = run += sh.tile[t];
  __syncthreads();
  if (k.a.draws <= kFewDraws) {
    for (int j = wave; j < k.a.draws; j += waves)
      draw_one<T>(k, r, j, j == wave ? u0 : k.a.u[row * k.a.draws + j], l, cut, total, sh.tile);
    return;
  }
  for (int t = threadIdx.x; t < k.tiles; t += threads) k.tile_mass[r * k.tiles + t] = sh.tile[t];
  if (threadIdx.x == 0) {
    k.state[r].cut = cut;
    k.state[r].total = total;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void draw_kernel(Long k, int blocks) {
  const int64_t r = blockIdx.x / blocks;
  const int j = (int)(blockIdx.x % blocks) * 4 + (threadIdx.x >> 6);
  const RowState &st = k.state[r];
  const RowLimits l = st.l;
  if (j >= k.a.draws || l.m == -__builtin_inff()) return;
  draw_one<T>(k, r, j, k.a.u[(k.row0 + r) * k.a.draws + j], l, st.cut, st.total,
              k.tile_mass + r * k.tiles);
}

// ---- long rows of 16-bit scores, one draw ----------------------------------------

// Such a row has at most 65,536 different scores, and far fewer in practice: a
// weight is worked out once for each of them and not for each entry.
//   value_kernel  counts a part's entries by their bit pattern, in LDS, and
//                 lists the (score, count) pairs
//   pick_kernel   a workgroup a row: the cuts from the pairs, as a score and how
//                 many of the entries that have it are kept; the parts' weights;
//                 and a walk over the part that holds the draw
// The row is read once, and one of its parts once more.  The chunked path reads
// it three times and takes two exponentials an entry, but a workgroup a row goes
// through all its pairs here, of which 16-bit floats of 10 bits an octave have
// more.  The settings are the device's, so length and type decide.  Times in us,
// here / there, of normal scores of deviation 2.5 at top-k 50 and top-p 0.9, at
// top-p 0.95, and with no limit:
//                     4 rows                64 rows               256 rows
//   fp16   65,536   25/31 41/37 34/25     26/42 44/50 37/32     39/53 59/72 51/46
//   fp16   98,304   26/30 47/36 35/23     27/41 52/51 40/32     42/64 66/87 58/56
//   bf16  131,072   25/32 32/34 27/25     27/45 34/54 29/37     49/77 56/106 51/68
//   bf16  262,144   24/33 42/37 33/25     36/53 49/70 43/45     95/116 118/166 107/107
//   bf16  524,288   26/36 45/43 34/27     47/74 70/105 61/66
// fp16 ends where a row of top-p alone no longer gains in any number of rows but
// the largest, bf16 where a few such rows have lost as much.  More draws walk more
// parts: four of 16 x 50,000 rows 40 us against 32.
constexpr int kPartVecs = 7;                      // vectors of 8 entries of a thread
constexpr int kPartMost = kPartVecs * 1024 * 8;   // below 65,536: 16-bit counters
// Smallest part: 64 rows of 50,021 at top-p 0.95 with 16,384, this, 32,768: fp16
// 43.9, 41.4, 42.0 us, bf16 28.4, 29.1, 34.2; of 32,768 fp16 36.4, 35.5, 35.4, bf16
// 26.7, 28.4, 28.2.
constexpr int kPartLeast = 24576;
constexpr int kParts = 16;                        // of a row, at most
constexpr int64_t kValueMostBf16 = 1 << 18, kValueMostF16 = 1 << 16;
static_assert(kValueMostBf16 <= (int64_t)kParts * kPartMost);
constexpr int64_t kValueBatch = (int64_t)1 << 25; // entries of one set of launches
constexpr int kHeld = 28672;   // pairs of a row held in LDS
constexpr int kWords = 32768;  // word i counts patterns i (low half) and i | 0x8000

struct Values {
  SampleArgs a;
  int64_t row0;      // first row of the batch
  int64_t part;      // entries of a part, a number of tiles
  int parts;         // of a row
  uint32_t *list;    // [rows][parts][part] (order << 16) | count
  uint32_t *listed;  // [rows][parts]
  uint32_t *best;    // [rows][parts] largest order listed, 0: none
};

// The place of a 16-bit pattern in the order of scores (-0.0 is +0.0), and back.
__device__ __forceinline__ uint32_t order_of(uint32_t pattern) {
  if (pattern == 0x8000u) pattern = 0;
  return pattern & 0x8000u ? pattern ^ 0xFFFFu : pattern | 0x8000u;
}

template <typename T>
__device__ __forceinline__ float score_of(uint32_t order) {
  const uint16_t pattern = (uint16_t)(order & 0x8000u ? order ^ 0x8000u : order ^ 0xFFFFu);
  return (float)__builtin_bit_cast(T, pattern);
}

template <typename T>
__global__ __launch_bounds__(1024) void value_kernel(Values k) {
  constexpr int kInfinity = std::is_same<T, _Float16>::value ? 0x7C00 : 0x7F80;
  __shared__ uint32_t listed, best, least;
  __shared__ uint32_t block_count[kWords / 512];  // of 512 words: both halves' sums
  extern __shared__ __attribute__((aligned(16))) char raw[];
  uint32_t *count = reinterpret_cast<uint32_t *>(raw);
  const int64_t r = blockIdx.x / k.parts, c = blockIdx.x % k.parts, row = k.row0 + r;
  const T *scores = static_cast<const T *>(k.a.s.scores) + row * k.a.s.ld;
  const uint8_t *valid = k.a.s.valid ? k.a.s.valid + row * k.a.s.valid_ld : nullptr;
  const int64_t lo = c * k.part, end = min(k.a.s.n, lo + k.part);
  const int t = threadIdx.x, lane = t & 63;
  const RowSettings set = row_settings(k.a, row);
  const int32_t top_k = set.temperature > 0.0f ? set.k : 1;
  // the whole part is on its way while the counters are cleared
  Eight<T> e[kPartVecs];
#pragma unroll
  for (int v = 0; v < kPartVecs; ++v)
    e[v].load(scores, valid, lo + (int64_t)(v * 1024 + t) * 8, end);
  uint4 *clear = reinterpret_cast<uint4 *>(raw);
  for (int w = t; w < kWords / 4; w += 1024) clear[w] = make_uint4(0, 0, 0, 0);
  if (t == 0) listed = best = least = 0;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < kPartVecs; ++v) {
    const int64_t i = lo + (int64_t)(v * 1024 + t) * 8;
    if (i >= end) break;
    const uint4 w4 = __builtin_bit_cast(uint4, e[v].v);
    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
    const u64 mask = valid ? e[v].mask : ~0ull;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // beyond the row's end there are entries of -inf, which are not listed
      if (!valid || (mask >> (16 * j)) & 0xFF)
        atomicAdd(&count[w[j] & 0x7FFFu], 1u << ((w[j] >> 11) & 16u));
      if (!valid || (mask >> (16 * j + 8)) & 0xFF)
        atomicAdd(&count[(w[j] >> 16) & 0x7FFFu], 1u << ((w[j] >> 27) & 16u));
    }
  }
  __syncthreads();
  // This lane's eight of 512 words from w0 on, without what is not included.
  auto words = [&](int w0, uint32_t (&w)[8]) {
    const uint4 x = clear[w0 / 4 + lane * 2], y = clear[w0 / 4 + lane * 2 + 1];
    w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
    w[4] = y.x, w[5] = y.y, w[6] = y.z, w[7] = y.w;
    if (w0 + 512 <= kInfinity) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = w0 + lane * 8 + j;
      if (i > kInfinity) w[j] = 0;          // NaN
      if (i == kInfinity) w[j] &= 0xFFFFu;  // -inf
    }
  };
  auto sum_of = [](const uint32_t (&w)[8]) {
    return w[0] + w[1] + w[2] + w[3] + w[4] + w[5] + w[6] + w[7];
  };
  // The row's best k entries are among the parts' best k: nothing worse than
  // eight scores around a part's k-th is listed.
  if (top_k > 0 && top_k < end - lo) {
    for (int b = t >> 6; b * 512 <= kInfinity; b += 16) {
      uint32_t w[8];
      words(b * 512, w);
      const uint32_t sum = wave_prefix(sum_of(w));
      if (lane == 63) block_count[b] = sum;
    }
    __syncthreads();
    if (t < 64) {
      // best first: the positive halves from the last block down, then the
      // negative ones up
      const uint32_t own = lane * 512 <= kInfinity ? block_count[lane] : 0;
      const uint32_t low = own & 0xFFFFu, up = own >> 16;
      const uint32_t low_upto = wave_prefix(low), lows = from_lane(low_upto, 63);
      const uint32_t before_low = lows - low_upto, upto_up = lows + wave_prefix(up);
      const u64 in_low = __ballot(before_low < (uint32_t)top_k && before_low + low >= (uint32_t)top_k);
      const u64 in_up = __ballot(upto_up - up < (uint32_t)top_k && upto_up >= (uint32_t)top_k);
      if (in_low | in_up) {
        const bool negative = in_low == 0;
        const int b = __ffsll(negative ? in_up : in_low) - 1;
        const uint32_t before = negative ? from_lane(upto_up - up, b) : from_lane(before_low, b);
        uint32_t w[8];
        words(b * 512, w);
        const uint32_t both = sum_of(w);
        const uint32_t here = negative ? both >> 16 : both & 0xFFFFu;
        const uint32_t upto = wave_prefix(here), all = from_lane(upto, 63);
        const uint32_t reached = before + (negative ? upto : all - upto + here);
        const u64 yes = __ballot(reached >= (uint32_t)top_k);
        const int at = negative ? __ffsll(yes) - 1 : 63 - __clzll(yes);
        const uint32_t i = (uint32_t)(b * 512 + at * 8);
        if (lane == 0) least = negative ? order_of((i + 7) | 0x8000u) : order_of(i);
      }
    }
    __syncthreads();
  }
  const uint32_t drop = least;
  // Patterns that follow one another are listed eight apart, as pick_kernel
  // adds neighbours of the list to different bins.
  uint32_t *list = k.list + (size_t)blockIdx.x * k.part;
  uint32_t most = 0;
  for (int w0 = (t >> 6) * 512; w0 <= kInfinity; w0 += 16 * 512) {
    uint32_t w[8];
    words(w0, w);
    if (!__any((w[0] | w[1] | w[2] | w[3] | w[4] | w[5] | w[6] | w[7]) != 0)) continue;
    u64 on[16];
    int total = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = w0 + lane * 8 + j;
      if (order_of((uint32_t)i) < drop) w[j] &= 0xFFFF0000u;
      if (order_of((uint32_t)i | 0x8000u) < drop) w[j] &= 0xFFFFu;
      on[2 * j] = __ballot((w[j] & 0xFFFFu) != 0);
      on[2 * j + 1] = __ballot((w[j] >> 16) != 0);
      total += __popcll(on[2 * j]) + __popcll(on[2 * j + 1]);
    }
    if (total == 0) continue;
    uint32_t at = 0;
    if (lane == 0) at = atomicAdd(&listed, (uint32_t)total);
    at = (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      if (!on[j]) continue;
      const uint32_t i = (uint32_t)(w0 + lane * 8 + j / 2);
      const uint32_t here = j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xFFFFu;
      if (here) {
        const uint32_t order = order_of(j & 1 ? i | 0x8000u : i);
        most = max(most, order);
        list[at + __builtin_amdgcn_mbcnt_hi((uint32_t)(on[j] >> 32),
                                            __builtin_amdgcn_mbcnt_lo((uint32_t)on[j], 0))] =
            (order << 16) | here;
      }
      at += (uint32_t)__popcll(on[j]);
    }
  }
  most = wave_fold(most, 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
  if (lane == 63 && most) atomicMax(&best, most);
  __syncthreads();
  if (t == 0) {
    k.listed[blockIdx.x] = listed;
    k.best[blockIdx.x] = best;
  }
}

template <typename T>
__global__ __launch_bounds__(1024) void pick_kernel(Values k) {
  constexpr int kFine = 32;               // scores of a bin
  constexpr int kCoarse = 65536 / kFine;  // bins, best first
  __shared__ Search s;
  __shared__ uint32_t count[kCoarse];
  __shared__ u64 mass[kCoarse], fine[kFine];
  __shared__ u64 part_mass[kParts], tile_mass[128];
  __shared__ uint32_t part_ties[kParts], tile_ties[128];
  extern __shared__ __attribute__((aligned(16))) char raw[];
  const int64_t r = blockIdx.x, row = k.row0 + r, n = k.a.s.n;
  const int t = threadIdx.x, lane = t & 63, parts = k.parts;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const T *scores = static_cast<const T *>(k.a.s.scores) + row * k.a.s.ld;
  const uint8_t *valid = k.a.s.valid ? k.a.s.valid + row * k.a.s.valid_ld : nullptr;
  const RowSettings set = row_settings(k.a, row);
  // a part's list is shared by `sharing` waves
  const int sharing = 16 / parts, mine = wave / sharing;
  const uint32_t each_listed = lane < parts ? k.listed[r * parts + lane] : 0;
  const uint32_t *list = k.list + (size_t)(r * parts + min(mine, parts - 1)) * k.part;
  uint32_t order = lane < parts ? k.best[r * parts + lane] : 0;
  const float u = k.a.u[row];
  for (int b = t; b < kCoarse; b += 1024) count[b] = 0, mass[b] = 0;
  if (t < kParts) part_mass[t] = 0, part_ties[t] = 0;
  order = from_lane(wave_fold(order, 0u, [](uint32_t a, uint32_t b) { return max(a, b); }), 63);
  if (order == 0) return no_entry(k.a, row);
  const RowLimits l = row_limits(set, n, score_of<T>(order), -__builtin_inff());

  // A thread's pairs are e0, e0 + step, ...: those it brings to LDS itself,
  // unless all of the row's are too many.
  const uint32_t listed_upto = wave_prefix(each_listed);
  const uint32_t pairs = mine < parts ? from_lane(each_listed, min(mine, parts - 1)) : 0;
  const bool held = from_lane(listed_upto, 63) <= (uint32_t)kHeld;
  const uint32_t step = (uint32_t)sharing * 64, e0 = (uint32_t)(wave % sharing) * 64 + lane;
  uint32_t *pair =
      reinterpret_cast<uint32_t *>(raw) + from_lane(listed_upto - each_listed, min(mine, parts - 1));
  if (held) {
    for (uint32_t e = e0; e < pairs; e += 8 * step) {
      uint32_t v[8];  // on their way at once
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = e + j * step < pairs ? list[e + j * step] : 0;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (v[j]) pair[e + j * step] = v[j];
    }
  }
  __syncthreads();
  // f(order, count) for the pairs of this thread
  auto each = [&](auto f) {
    auto walk = [&](const auto *from) {
#pragma unroll 1
      for (uint32_t e = e0; e < pairs; e += 4 * step) {
        uint32_t v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = e + j * step < pairs ? from[e + j * step] : 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (v[j]) f(v[j] >> 16, v[j] & 0xFFFFu);
      }
    };
    if (held) walk(pair);
    else walk(list);
  };
  auto weight_at = [&](uint32_t o) { return weight(exponent(score_of<T>(o), l)); };
  auto bin = [&](uint32_t o) { return kCoarse - 1 - (int)(o / kFine); };

  // Inside bin `b`, with `above` in better ones: the score at which the count or
  // weight reaches `need`.  What better scores amount to goes back to `above`.
  auto score_in = [&](int b, bool by_count, u64 need, u64 *above) {
    if (t < kFine) fine[t] = 0;
    __syncthreads();
    each([&](uint32_t o, uint32_t c) {
      if (bin(o) == b)
        atomicAdd(&fine[kFine - 1 - (int)(o & (kFine - 1))], by_count ? c : (u64)c * weight_at(o));
    });
    __syncthreads();
    const u64 v = lane < kFine ? fine[lane] : 0, upto = wave_prefix(v);
    const int f = __ffsll(__ballot(lane < kFine && *above + upto >= need)) - 1;
    *above += from_lane(upto - v, f);
    return (uint32_t)((kCoarse - 1 - b) * kFine + kFine - 1 - f);
  };

  // The cut: entries of better scores than `edge` are kept, and the first
  // `edge_kept` of those that have it.  top-k's needs no weights, and top-p's
  // only those of what top-k keeps.
  uint32_t at = 0;  // the edge's place in the order, 0: below all
  u64 edge_kept = 0;
  if (l.k < n) {
    each([&](uint32_t o, uint32_t c) { atomicAdd(&count[bin(o)], c); });
    __syncthreads();
    block_find(s, kCoarse, [&](u64) { return (u64)l.k; }, 0,
               [&](int b) { return (u64)count[b]; });
    if (s.bin >= 0) {  // the row has k entries
      u64 above = s.above;
      at = score_in(s.bin, true, (u64)l.k, &above);
      edge_kept = (u64)l.k - above;
    }
    __syncthreads();
  }
  if (l.p < 2.0f) {
    each([&](uint32_t o, uint32_t c) {
      if (o <= at) return;
      const u64 q = (u64)c * weight_at(o);
      if (q) atomicAdd(&mass[bin(o)], q);
    });
    if (t == 0 && at) atomicAdd(&mass[bin(at)], edge_kept * weight_at(at));
    __syncthreads();
    u64 need = 0;
    block_find(s, kCoarse, [&](u64 all) { return need = share_of(l.p, all); }, 0,
               [&](int b) { return mass[b]; });
    u64 above = s.above;
    at = score_in(s.bin, false, need, &above);
    const uint32_t q = weight_at(at);
    edge_kept = (need - above + q - 1) / q;
  }
  float edge = -__builtin_inff();
  uint32_t edge_weight = 0;
  if (at) {
    edge = score_of<T>(at);
    const float z = exponent(edge, l);
    edge_weight = weight(z);
    if (!(z >= l.min_z)) edge_kept = 0;
  }
  auto kept = [&](float x, float z) { return x > edge && z >= l.min_z; };

  // what each part keeps: the weight of better scores, entries at the edge
  u64 sum = 0;
  uint32_t ties = 0;
  each([&](uint32_t o, uint32_t c) {
    if (o < at) return;
    const float x = score_of<T>(o), z = exponent(x, l);
    if (kept(x, z)) sum += (u64)c * weight(z);
    if (x == edge) ties += c;
  });
  sum = wave_prefix(sum);
  ties = wave_prefix(ties);
  if (lane == 63 && mine < parts) {
    atomicAdd(&part_mass[mine], sum);
    atomicAdd(&part_ties[mine], ties);
  }
  __syncthreads();
  // of `have` entries at the edge, `before` of them in earlier places
  auto kept_ties = [](u64 have, u64 before, u64 most) {
    return before >= most ? 0ull : min(have, most - before);
  };
  const u64 have = lane < parts ? part_ties[lane] : 0;
  const u64 part_kept = kept_ties(have, wave_prefix(have) - have, edge_kept);
  const u64 part_upto =
      wave_prefix(lane < parts ? part_mass[lane] + part_kept * edge_weight : 0);
  const u64 total = from_lane(part_upto, 63);

  // The part that holds the draw, by tile.
  u64 want = wanted(u, total);
  const int p = __ffsll(__ballot(part_upto > want)) - 1;
  if (p > 0) want -= from_lane(part_upto, p - 1);
  const u64 keeps = from_lane(part_kept, p);  // entries at the edge
  const int64_t lo = p * k.part, end = min(n, lo + k.part);
  const int tiles = (int)((end - lo + kTile - 1) / kTile);
  Eight<T> all[kPartVecs];
#pragma unroll
  for (int v = 0; v < kPartVecs; ++v)
    all[v].load(scores, valid, lo + (v * 16 + wave) * kTile + lane * 8, end);
#pragma unroll
  for (int v = 0; v < kPartVecs; ++v) {
    const int tile = v * 16 + wave;
    if (tile >= tiles) break;
    float x[8];
    all[v].get(valid != nullptr, x);
    u64 q = 0;
    uint32_t at_edge = 0;
    bool some = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) some = some | (x[i] >= edge);
    if (__any(some)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float z = exponent(x[i], l);
        q += kept(x[i], z) ? weight(z) : 0u;
        at_edge += x[i] == edge ? 1u : 0u;
      }
      q = wave_prefix(q);
      at_edge = wave_prefix(at_edge);
    }
    if (lane == 63) tile_mass[tile] = q, tile_ties[tile] = at_edge;
  }
  __syncthreads();
  if (wave != 0) return;
  // the tile, two a lane, and the entry inside it
  const int t0 = lane * 2;
  const u64 tie0 = t0 < tiles ? tile_ties[t0] : 0, tie1 = t0 + 1 < tiles ? tile_ties[t0 + 1] : 0;
  const u64 before = wave_prefix(tie0 + tie1) - tie0 - tie1;
  const u64 m0 = (t0 < tiles ? tile_mass[t0] : 0) + kept_ties(tie0, before, keeps) * edge_weight;
  const u64 m1 = (t0 + 1 < tiles ? tile_mass[t0 + 1] : 0) +
                 kept_ties(tie1, before + tie0, keeps) * edge_weight;
  const u64 upto = wave_prefix(m0 + m1);
  // (always found; with scores that another stream rewrites meanwhile it may be
  // the last lane, which reads nothing)
  const int in = __ffsll(__ballot(upto > want) | (1ull << 63)) - 1;
  const u64 ahead = from_lane(upto - m0 - m1, in), first = from_lane(m0, in);
  const bool second = ahead + first <= want;
  want -= ahead + (second ? first : 0);
  const u64 ties_before = from_lane(before + (second ? tie0 : 0), in);
  const int64_t i = lo + (int64_t)(in * 2 + (second ? 1 : 0)) * kTile + lane * 8;
  Eight<T> e;
  e.load(scores, valid, i, end);
  float x[8];
  e.get(valid != nullptr, x);
  uint32_t own = 0;
#pragma unroll
  for (int f = 0; f < 8; ++f) own += x[f] == edge ? 1u : 0u;
  u64 tie = ties_before + wave_prefix(own) - own;
  uint32_t q[8];
  u64 weights = 0;
#pragma unroll
  for (int f = 0; f < 8; ++f) {
    const float z = exponent(x[f], l);
    q[f] = kept(x[f], z) ? weight(z) : 0u;
    if (x[f] == edge) q[f] = tie++ < keeps ? edge_weight : 0u;
    weights += q[f];
  }
  const u64 incl = wave_prefix(weights);
  if (lane == __ffsll(__ballot(incl > want)) - 1) {
    u64 now = incl - weights;
    int f = 0;
    float score = x[0];
#pragma unroll
    for (int g = 0; g < 8; ++g) {
      now += q[g];
      if (now <= want) f = g + 1;
    }
#pragma unroll
    for (int g = 1; g < 8; ++g) score = g == f ? x[g] : score;
    k.a.idx[row] = (int32_t)(i + f);
    k.a.logprob[row] = exponent(score, l) - log_total(total);
  }
}

// ---- plans -------------------------------------------------------------------

struct LongPlan {
  int64_t batch, tile, tiles, most_chunks;
  uint32_t list_most;  // entries of a row's list
  size_t range, mass, count, tile_mass, list, listed, state, bytes;
};

LongPlan long_plan(int64_t n, int64_t rows) {
  LongPlan p{};
  p.batch = std::min<int64_t>(rows, kBatch);
  // A tile's sum costs a wave as much as a hundred of its entries a lane would:
  // long tiles where there are waves enough.
  const int64_t least = p.batch * n >= (int64_t)kTile * 4 * 4096 ? kTile * 4 : kTile;
  p.tile = std::max<int64_t>(least, ((n + kMaxTiles - 1) / kMaxTiles + kTile - 1) / kTile * kTile);
  p.tiles = (n + p.tile - 1) / p.tile;
  // as many chunks as workgroups may be wanted: 4,096 in all, one a row at least
  p.most_chunks = std::max<int64_t>(1, 4096 / std::max<int64_t>(1, p.batch));
  p.list_most = (uint32_t)(2 * kList + n / 32);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) & ~(size_t)255;
    return here;
  };
  const size_t b = (size_t)p.batch;
  p.range = take(b * p.most_chunks * sizeof(float2));
  p.mass = take(b * kBins * 8);
  p.count = take(b * kBins * 4);
  p.tile_mass = take(b * p.tiles * 8);
  p.list = take(b * p.list_most * 8);
  p.listed = take(b * kSegments * 4);
  p.state = take(b * sizeof(RowState));
  p.bytes = at;
  return p;
}

template <typename T>
hipError_t launch_long(const SampleArgs &a, void *ws, int cu_count, hipStream_t s) {
  const LongPlan p = long_plan(a.s.n, a.s.rows);
  char *base = static_cast<char *>(ws);
  Long k{};
  k.a = a;
  k.tile = p.tile;
  k.tiles = p.tiles;
  k.range = reinterpret_cast<float2 *>(base + p.range);
  k.mass = reinterpret_cast<u64 *>(base + p.mass);
  k.count = reinterpret_cast<uint32_t *>(base + p.count);
  k.tile_mass = reinterpret_cast<u64 *>(base + p.tile_mass);
  k.list = reinterpret_cast<u64 *>(base + p.list);
  k.listed = reinterpret_cast<uint32_t *>(base + p.listed);
  k.state = reinterpret_cast<RowState *>(base + p.state);
  hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(finish_kernel<T>), sizeof(Finish));
  if (e != hipSuccess) return e;
  for (k.row0 = 0; k.row0 < a.s.rows; k.row0 += p.batch) {
    const int64_t rows = std::min(p.batch, a.s.rows - k.row0);
    // about eight workgroups a CU, none over less than four tiles; chunks
    // are whole tiles, a wave's at a time
    const int64_t want = std::min(p.most_chunks, std::max<int64_t>(1, (int64_t)cu_count * 8 / rows));
    const int64_t unit = 4 * p.tile;
    k.chunk = std::max<int64_t>(1, (a.s.n + want * unit - 1) / (want * unit)) * unit;
    k.chunks = (a.s.n + k.chunk - 1) / k.chunk;
    k.segments = (uint32_t)std::min<int64_t>(kSegments, k.chunks);
    k.segment_most = p.list_most / k.segments;
    // the bins' parts: two workgroups a CU, of sixteen waves
    const int64_t parts = std::max<int64_t>(1, (int64_t)cu_count * 2 / rows);
    k.span = std::max<int64_t>(1, (a.s.n + parts * kSpan - 1) / (parts * kSpan)) * kSpan;
    k.spans = (a.s.n + k.span - 1) / k.span;
    const uint32_t grid = (uint32_t)(rows * k.chunks);
    range_kernel<T><<<grid, 256, 0, s>>>(k);
    if (a.top_k || a.top_p || a.s.temperature)
      count_kernel<T><<<(uint32_t)(rows * k.spans), 1024, 0, s>>>(k);
    settle_kernel<<<(uint32_t)rows, 512, 0, s>>>(k);
    collect_kernel<T><<<grid, 256, 0, s>>>(k);
    finish_kernel<T><<<(uint32_t)rows, 1024, sizeof(Finish), s>>>(k);
    if (a.draws > kFewDraws) {
      const int blocks = (a.draws + 3) / 4;
      draw_kernel<T><<<(uint32_t)(rows * blocks), 256, 0, s>>>(k, blocks);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

struct ValuePlan {
  int64_t batch, part;
  int parts;
  size_t list, listed, best, bytes;
};

bool by_values(int64_t n, int32_t draws, int64_t most) {
  return n > kRowMost && n <= most && draws == 1;
}

// `cus` workgroups fill the device; 0: the plan of the most parts, for the workspace.
ValuePlan value_plan(int64_t n, int64_t rows, int cus) {
  ValuePlan p{};
  p.batch = std::max<int64_t>(1, std::min(rows, kValueBatch / n));
  const int64_t least = (n + kPartMost - 1) / kPartMost, most = std::max<int64_t>(1, n / kPartLeast);
  const int64_t want = cus ? (cus + p.batch - 1) / p.batch : kParts;
  p.parts = (int)std::max(least, std::min({want, most, (int64_t)kParts}));
  p.part = ((n + p.parts - 1) / p.parts + kTile - 1) / kTile * kTile;
  p.parts = (int)((n + p.part - 1) / p.part);
  const size_t b = (size_t)p.batch;
  auto aligned = [](size_t bytes) { return (bytes + 255) & ~(size_t)255; };
  p.listed = aligned(b * (size_t)(n + kParts * kTile) * 4);
  p.best = p.listed + aligned(b * kParts * 4);
  p.bytes = p.best + aligned(b * kParts * 4);
  return p;
}

template <typename T>
hipError_t launch_values(const SampleArgs &a, void *ws, int cu_count, hipStream_t s) {
  const ValuePlan p = value_plan(a.s.n, a.s.rows, cu_count);
  char *base = static_cast<char *>(ws);
  Values k{};
  k.a = a;
  k.part = p.part;
  k.parts = p.parts;
  k.list = reinterpret_cast<uint32_t *>(base + p.list);
  k.listed = reinterpret_cast<uint32_t *>(base + p.listed);
  k.best = reinterpret_cast<uint32_t *>(base + p.best);
  const size_t lds = kWords * sizeof(uint32_t);
  hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(value_kernel<T>), lds);
  const size_t held = kHeld * sizeof(uint32_t);
  if (e == hipSuccess) e = ensure_dynamic_lds(reinterpret_cast<const void *>(pick_kernel<T>), held);
  for (k.row0 = 0; k.row0 < a.s.rows && e == hipSuccess; k.row0 += p.batch) {
    const uint32_t rows = (uint32_t)std::min(p.batch, a.s.rows - k.row0);
    value_kernel<T><<<rows * (uint32_t)k.parts, 1024, lds, s>>>(k);
    pick_kernel<T><<<rows, 1024, held, s>>>(k);
    e = hipGetLastError();
  }
  return e;
}

template <typename T>
hipError_t launch_row(const SampleArgs &a, hipStream_t s) {
  const int groups = (int)((a.s.n + 7) / 8);
  const int threads = std::min(1024, std::max(64, (groups + 63) / 64 * 64));
  const size_t lds = (size_t)groups * (8 * 8 + 8);
  const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(row_kernel<T>), lds);
  if (e != hipSuccess) return e;
  row_kernel<T><<<(uint32_t)a.s.rows, threads, lds, s>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch(const SampleArgs &a, void *ws, int cu_count, hipStream_t s) {
  if (a.s.n <= kRowMost) return launch_row<T>(a, s);
  if constexpr (sizeof(T) == 2) {
    const int64_t most = std::is_same<T, _Float16>::value ? kValueMostF16 : kValueMostBf16;
    if (by_values(a.s.n, a.draws, most)) return launch_values<T>(a, ws, cu_count, s);
  }
  return launch_long<T>(a, ws, cu_count, s);
}

}  // namespace

size_t sample_workspace_bytes(int64_t n, int64_t rows, int32_t draws) {
  if (n <= kRowMost || rows <= 0) return 256;
  const size_t bytes = long_plan(n, rows).bytes;  // the type is not known here
  return by_values(n, draws, kValueMostBf16) ? std::max(bytes, value_plan(n, rows, 0).bytes) : bytes;
}

hipError_t launch_sample(int dtype, const SampleArgs &a, void *ws, int cu_count, hipStream_t s) {
  if (a.s.rows == 0 || a.draws == 0) return hipSuccess;
  switch (dtype) {
    case ML2_F32: return launch<float>(a, ws, cu_count, s);
    case ML2_BF16: return launch<__bf16>(a, ws, cu_count, s);
    default: return launch<_Float16>(a, ws, cu_count, s);
  }
}

}  // namespace ml2
