// Draws from the softmax of rows of scores, by temperature, top-k, top-p and
// min-p, with given uniform numbers (the definition stands in ml2.h).
//
// All three limits keep a prefix of the order (score descending, index
// ascending).  Every entry has a unique 64-bit key, larger is better,
//   (ord(score) << 32) | (0xFFFFFFFF - index),
// so a limit is a key: the cut.  Weights are whole numbers, so their sums are
// exact in any order and every comparison of sums has one answer.
//
// A cut is found in two steps.  Entries are counted and weighed in kBins bins
// of equal width in z (of those that can be drawn: z above kLowest); the bin
// in which the wanted count or weight is reached holds the cut.  Inside that
// bin the interval of keys is split into kSub parts again and again until one
// entry is left or the wanted amount ends with a part.
#include <algorithm>

#include "draw.h"

namespace ml2 {
namespace {

constexpr int kThreads = 1024;
constexpr int kBins = 2048;
constexpr int kSub = 512;           // parts of an interval of keys
constexpr int kTiles = 1024;        // parts of a row whose kept weights are held
constexpr float kLowest = -22.25f;  // exp(z) * 2^31 rounds to 0 below -22.181
constexpr float kOne = 2147483648.0f;

typedef unsigned long long u64;

__device__ __forceinline__ uint32_t ordered(float x) {  // x is not NaN, not -0.0
  const uint32_t b = __float_as_uint(x);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

__device__ __forceinline__ u64 key_of(float x, int64_t i) {
  return ((u64)ordered(x) << 32) | (u64)(0xFFFFFFFFu - (uint32_t)i);
}

// What all entries of a row share.
struct RowLimits {
  float m, r;      // best included score, 1 / T
  float bin_scale; // bins per unit of z
  float min_z;     // log(min_p), or -inf
  int64_t k;       // entries top-k keeps (n: all)
  double p;        // top_p, or 2 where it keeps all
};

__device__ __forceinline__ float exponent(float x, const RowLimits &l) {
  return x == l.m ? 0.0f : (x - l.m) * l.r;
}

__device__ __forceinline__ uint32_t weight(float z) {
  return z > kLowest ? (uint32_t)rintf(expf(z) * kOne) : 0u;
}

__device__ __forceinline__ int bin_of(float z, const RowLimits &l) {
  return min(kBins - 1, (int)(-z * l.bin_scale));
}

struct Amount {
  u64 count, mass;
};

// Wave 0 looks through `bins` bins (a multiple of 64), best first, for the one
// in which the running amount reaches `need`: count where by_count, else mass.
// *before: the amounts of better bins, on top of `base`.  The last bin where
// `need` is never reached.
template <int BINS>
__device__ __forceinline__ int find_bin(const uint32_t *count, const u64 *mass, bool by_count,
                                        u64 need, Amount base, Amount *before) {
  constexpr int kPer = BINS / 64;
  const int lane = threadIdx.x & 63;
  Amount sum = {0, 0};
  for (int j = 0; j < kPer; ++j) {
    sum.count += count[lane * kPer + j];
    sum.mass += mass[lane * kPer + j];
  }
  Amount incl = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const u64 c = __shfl_up(incl.count, d), q = __shfl_up(incl.mass, d);
    if (lane >= d) incl.count += c, incl.mass += q;
  }
  Amount run = {base.count + incl.count - sum.count, base.mass + incl.mass - sum.mass};
  const u64 reached = by_count ? base.count + incl.count : base.mass + incl.mass;
  const u64 ballot = __ballot(reached >= need);
  const int at = ballot ? __ffsll(ballot) - 1 : 63;
  int bin = BINS - 1;
  if (lane == at) {
    for (int j = 0; j < kPer; ++j) {
      const Amount next = {run.count + count[lane * kPer + j], run.mass + mass[lane * kPer + j]};
      bin = lane * kPer + j;
      if ((by_count ? next.count : next.mass) >= need || j == kPer - 1) break;
      run = next;
    }
  }
  bin = __shfl(bin, at);
  before->count = __shfl(run.count, at);
  before->mass = __shfl(run.mass, at);
  return bin;
}

struct Shared {
  uint32_t count[kBins];
  u64 mass[kBins];
  uint32_t sub_count[kSub];
  u64 sub_mass[kSub];
  u64 tile[kTiles + 1];
  float fmax[16], fmin[16];
  u64 lo, hi;       // interval of keys that holds the cut
  u64 need;
  Amount above;     // amounts better than the interval
  int bin, done;
};

// The cut in the interval [sh.lo, sh.hi] of the keys that each(f) hands to
// f(key, weight), given the smallest and the largest of those keys: afterwards
// the entries with key >= sh.lo are kept (no entry of a worse bin has such a
// key), and sh.above holds the amounts with them.
template <typename Each>
__device__ __forceinline__ void refine(Shared &sh, bool by_count, Each each) {
  for (;;) {
    __syncthreads();
    const u64 lo = sh.lo, hi = sh.hi;
    if (sh.done) return;
    const int width = 64 - __clzll((hi - lo) | 1ull);
    const int shift = max(0, width - 9);
    for (int b = threadIdx.x; b < kSub; b += kThreads) sh.sub_count[b] = 0, sh.sub_mass[b] = 0;
    __syncthreads();
    each([&](u64 key, uint32_t q) {
      if (key < lo || key > hi) return;
      const int b = kSub - 1 - (int)((key - lo) >> shift);  // best first
      atomicAdd(&sh.sub_count[b], 1u);
      atomicAdd(&sh.sub_mass[b], (u64)q);
    });
    __syncthreads();
    if (threadIdx.x < 64) {
      Amount before;
      const int b = find_bin<kSub>(sh.sub_count, sh.sub_mass, by_count, sh.need, sh.above, &before);
      if (threadIdx.x == 0) {
        const u64 part = (u64)(kSub - 1 - b);
        const Amount with = {before.count + sh.sub_count[b], before.mass + sh.sub_mass[b]};
        sh.lo = lo + (part << shift);
        sh.hi = min(hi, sh.lo + ((1ull << shift) - 1));
        // one entry, or all of the part is kept
        sh.done = shift == 0 || sh.sub_count[b] <= 1 ||
                  (by_count ? with.count : with.mass) == sh.need;
        sh.above = sh.done ? with : before;
      }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void row_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int64_t row = blockIdx.x, n = a.s.n;
  const T *scores = static_cast<const T *>(a.s.scores) + row * a.s.ld;
  const uint8_t *valid = a.s.valid ? a.s.valid + row * a.s.valid_ld : nullptr;
  const float ninf = -__builtin_inff();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto load = [&](int64_t i) { return included((float)scores[i], !valid || valid[i] != 0); };

  // the row's best and worst included scores
  float hi = ninf, lo = __builtin_inff();
  for (int64_t i = threadIdx.x; i < n; i += kThreads) {
    const float x = load(i);
    hi = fmaxf(hi, x);
    if (x != ninf) lo = fminf(lo, x);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    hi = fmaxf(hi, __shfl_xor(hi, d));
    lo = fminf(lo, __shfl_xor(lo, d));
  }
  if (lane == 0) sh.fmax[wave] = hi, sh.fmin[wave] = lo;
  __syncthreads();
  for (int w = 0; w < kThreads / 64; ++w) {
    hi = fmaxf(hi, sh.fmax[w]);
    lo = fminf(lo, sh.fmin[w]);
  }
  if (hi == ninf) {
    for (int j = threadIdx.x; j < a.draws; j += kThreads) {
      a.idx[row * a.draws + j] = -1;
      a.logprob[row * a.draws + j] = ninf;
    }
    return;
  }
  RowLimits l;
  bool greedy;
  l.m = hi;
  l.r = inverse_temperature(a.s.temperature, row, &greedy);
  const float range = fminf(-kLowest, fmaxf(-exponent(lo, l), 1e-20f));
  l.bin_scale = (float)kBins / range;
  const int32_t k = greedy ? 1 : a.top_k ? a.top_k[row] : 0;
  l.k = k > 0 && k < n ? k : n;
  const float p = a.top_p ? a.top_p[row] : 1.0f;
  l.p = p < 1.0f ? (double)p : 2.0;
  const float mp = a.min_p ? a.min_p[row] : 0.0f;
  l.min_z = mp > 0.0f ? logf(fminf(mp, 1.0f)) : ninf;

  u64 cut = 0;  // entries with a smaller key are not kept
  if (l.k < n || l.p < 2.0) {
    for (int b = threadIdx.x; b < kBins; b += kThreads) sh.count[b] = 0, sh.mass[b] = 0;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < n; i += kThreads) {
      const float x = load(i);
      const float z = exponent(x, l);
      const uint32_t q = weight(z);
      if (x == ninf || q == 0) continue;
      atomicAdd(&sh.count[bin_of(z, l)], 1u);
      atomicAdd(&sh.mass[bin_of(z, l)], (u64)q);
    }
    __syncthreads();
    // The cut among the entries of bin sh.bin with key >= cut.
    auto search = [&](bool by_count, u64 need) {
      if (wave == 0) {
        Amount before;
        const int b = find_bin<kBins>(sh.count, sh.mass, by_count, need, Amount{0, 0}, &before);
        if (lane == 0) {
          sh.bin = b;
          sh.need = need;
          sh.above = before;
          sh.lo = ~0ull;
          sh.hi = 0;
          sh.done = 0;
        }
      }
      __syncthreads();
      const int bin = sh.bin;
      auto each = [&](auto f) {
        for (int64_t i = threadIdx.x; i < n; i += kThreads) {
          const float x = load(i);
          if (x == ninf) continue;
          const float z = exponent(x, l);
          const uint32_t q = weight(z);
          const u64 key = key_of(x, i);
          if (q != 0 && bin_of(z, l) == bin && key >= cut) f(key, q);
        }
      };
      u64 first = ~0ull, last = 0;
      each([&](u64 key, uint32_t) {
        first = min(first, key);
        last = max(last, key);
      });
      if (last) atomicMin(&sh.lo, first), atomicMax(&sh.hi, last);
      refine(sh, by_count, each);
      cut = sh.lo;
    };
    u64 total = 0;
    if (wave == 0) {
      Amount all;
      find_bin<kBins>(sh.count, sh.mass, true, ~0ull, Amount{0, 0}, &all);
      if (lane == 0) {
        sh.above.count = all.count + sh.count[kBins - 1];
        sh.above.mass = all.mass + sh.mass[kBins - 1];
      }
    }
    __syncthreads();
    const Amount all = sh.above;
    __syncthreads();
    total = all.mass;
    if ((u64)l.k < all.count) {
      search(true, (u64)l.k);
      total = sh.above.mass;
      __syncthreads();
    }
    if (l.p < 2.0) {
      const double share = ceil(l.p * (double)total);
      search(false, share >= 1.0 ? (u64)share : 1ull);
      __syncthreads();
    }
  }
  auto kept = [&](float x, int64_t i, float *z) {
    *z = exponent(x, l);
    return x != ninf && key_of(x, i) >= cut && *z >= l.min_z ? weight(*z) : 0u;
  };

  // weights of the tiles, one wave a tile
  const int64_t tile = ((n + kTiles - 1) / kTiles + 63) / 64 * 64;
  const int tiles = (int)((n + tile - 1) / tile);
  for (int t = wave; t < tiles; t += kThreads / 64) {
    u64 sum = 0;
    for (int64_t i = t * tile + lane; i < min(n, (t + 1) * tile); i += 64) {
      float z;
      sum += kept(load(i), i, &z);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) sh.tile[t + 1] = sum;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    sh.tile[0] = 0;
    for (int t = 0; t < tiles; ++t) sh.tile[t + 1] += sh.tile[t];
  }
  __syncthreads();
  const u64 total = sh.tile[tiles];
  const float log_total = logf((float)total / kOne);
  for (int j = wave; j < a.draws; j += kThreads / 64) {
    const double at = floor((double)a.u[row * a.draws + j] * (double)total);
    const u64 want = at >= 0.0 ? min(at < 9.0e18 ? (u64)at : total, total - 1) : 0;
    int lo_t = 0, hi_t = tiles - 1;  // the tile whose end passes `want`
    while (lo_t < hi_t) {
      const int mid = (lo_t + hi_t) / 2;
      if (sh.tile[mid + 1] > want) hi_t = mid; else lo_t = mid + 1;
    }
    u64 run = sh.tile[lo_t];
    for (int64_t base = lo_t * tile; base < n; base += 64) {
      const int64_t i = base + lane;
      float z = 0.0f;
      u64 incl = i < n ? kept(load(i), i, &z) : 0u;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const u64 o = __shfl_up(incl, d);
        if (lane >= d) incl += o;
      }
      const u64 found = __ballot(run + incl > want);
      if (found) {
        if (lane == __ffsll(found) - 1) {
          a.idx[row * a.draws + j] = (int32_t)i;
          a.logprob[row * a.draws + j] = z - log_total;
        }
        break;
      }
      run += __shfl(incl, 63);
    }
  }
}

template <typename T>
hipError_t launch(const SampleArgs &a, hipStream_t s) {
  row_kernel<T><<<(uint32_t)a.s.rows, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t sample_workspace_bytes(int64_t n, int64_t rows, int32_t draws) {
  (void)n, (void)rows, (void)draws;
  return 256;
}

hipError_t launch_sample(int dtype, const SampleArgs &a, void *ws, int cu_count, hipStream_t s) {
  (void)ws, (void)cu_count;
  if (a.s.rows == 0 || a.draws == 0) return hipSuccess;
  switch (dtype) {
    case ML2_F32: return launch<float>(a, s);
    case ML2_BF16: return launch<__bf16>(a, s);
    default: return launch<_Float16>(a, s);
  }
}

}  // namespace ml2
