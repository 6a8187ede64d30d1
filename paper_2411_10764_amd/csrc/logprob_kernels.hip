// Log-probabilities of given entries of rows of scores under the masked
// softmax, and the gradient of their weighted sum.
//
//   z_i = (s_i - m) * R,  l = sum_i exp(z_i)
//   logprob_j = z_{t_j} - log l
//   grad_i = R * (sum_{j: t_j = i} w_j - exp(z_i) / l * sum_j w_j)
//
// Bytes bound it: a row is read once, its gradient written once.
//
// Rows that fit a workgroup's registers (row_kernel): one launch, the row's
// scores stay as they came, in registers, between the maximum, the sum and
// the gradient; two exponentials an entry cost less than the registers that
// would hold the first ones in float32 (and with them the second workgroup
// of a CU, whose loads run beside this one's arithmetic).
//
// Other rows are cut into chunks.  stats_kernel reads a chunk once and keeps
// a running maximum and sum (of exp of differences to that maximum);
// finish_kernel and grad_kernel join the chunks' pairs in chunk order, so
// every workgroup of a row arrives at the same m and l.  Weights are joined
// in the order of j inside a chunk, then in chunk order.
//
// Weights below 2^-126 of the best entry's are 0, as the exp2 instruction flushes
// them: the sum, which is at least 1, does not show it, and such an entry's own
// gradient is 0.
//
// Measured: 4,096 x 50,021 bf16 gradient 191 us (820 MB, 4.3 TB/s of a copy's
// 4.65; rows padded to 50,024 entries, 231 where they follow one another); 1 x
// 4,194,304 float32 with 512 targets 12 us; 1 x 262,144 gradient with 128 targets
// 15 us, two launches of dependent loads.  What a second read of the scores costs:
// 4,096 rows of 65,536 bf16 211 us, of 65,537 384; of 32,768 float32 191, of
// 32,769 357.
#include <algorithm>

#include "draw.h"

namespace ml2 {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 2048;      // smallest chunk
constexpr int kPairs = 128;       // targets of a workgroup compared pair by pair
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kPlainMost = 4294967296.0f;  // 2^32: what row_kernel's fast sum stays below

struct Stat {
  float m, l;  // maximum of the included scores, sum of exp((s - m) * R)
};

struct Part {
  Stat s;
  float w;     // weights of the included targets
};

__device__ __forceinline__ float ninf() { return -__builtin_inff(); }

// exp(z) of a score against the maximum.  Where both are infinite their
// difference is NaN and the entry counts as the maximum.  R is multiplied before
// log2(e): their product passes float32 where R alone, at temperatures below
// 4.3e-39, does not.
__device__ __forceinline__ float weight_of(float x, float m, float r) {
  return fminf(__builtin_amdgcn_exp2f((x - m) * r * kLog2e), 1.0f);
}

// A part of the gradient times R = 1 / T, which comes last: what is 0 (an entry
// without probability, a target that holds all of it) stays 0 where R, or R times
// the weights, passes float32.
__device__ __forceinline__ float times_r(float part, float r) {
  return part == 0.0f ? 0.0f : part * r;
}

// Maximum and sum over the workgroup, in every thread; sums in the order of
// the lanes and then of the waves.  They begin with the barrier that frees lds.
__device__ __forceinline__ float block_max(float v, float *lds) {
  const uint32_t none = __float_as_uint(ninf());
  v = __uint_as_float(wave_fold(__float_as_uint(v), none, [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
  __syncthreads();
  if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
  for (int w = 1; w < (int)blockDim.x >> 6; ++w) v = fmaxf(v, lds[w]);
  return v;
}

__device__ __forceinline__ float block_sum(float v, float *lds) {
  v = __uint_as_float(wave_fold(__float_as_uint(v), 0u, [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
  __syncthreads();
  if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
  for (int w = 1; w < (int)blockDim.x >> 6; ++w) v += lds[w];
  return v;
}

// The threads' pairs as one: their maximum, and their sums brought to it.
__device__ __forceinline__ Stat block_join(Stat s, float r, float *lds) {
  const float m = block_max(s.m, lds);
  return {m, block_sum(s.m == ninf() ? 0.0f : s.l * weight_of(s.m, m, r), lds)};
}

struct Rows {
  LogprobArgs a;
  Part *part;      // [rows][chunks]
  int64_t chunk;   // entries of a chunk
  int64_t chunks;
};

enum Mode { kForward, kGradient, kGradientPastCache };

// A gradient of more bytes than this (half of the last cache) is written past
// the caches; a smaller one stays there for whoever reads it next.  50,021 bf16
// entries a row, past the caches and not: 700 rows (67 MiB) 36 and 38 us, 1,300
// (124 MiB) 67 and 71, 1,400 (134 MiB) 66 and 80, 2,680 (256 MiB) 124 and 161,
// 4,096 (391 MiB) 231 and 240.
constexpr int64_t kPastCache = (int64_t)128 << 20;

template <typename T>
__device__ __forceinline__ const T *row_scores(const Rows &k, int64_t row) {
  return static_cast<const T *>(k.a.s.scores) + row * k.a.s.ld;
}

__device__ __forceinline__ const uint8_t *row_mask(const Rows &k, int64_t row) {
  return k.a.s.valid ? k.a.s.valid + row * k.a.s.valid_ld : nullptr;
}

template <typename T>
__device__ __forceinline__ float load_score(const Rows &k, int64_t row, int64_t i) {
  const uint8_t *valid = row_mask(k, row);
  return included((float)row_scores<T>(k, row)[i], !valid || valid[i] != 0);
}

// log-probability of an included score
__device__ __forceinline__ float logprob_of(float x, Stat st, float r) {
  return x == ninf() ? x : (x == st.m ? 0.0f : (x - st.m) * r) - logf(st.l);
}

// ---- targets of a range of entries ----------------------------------------------

// Handles the targets in [lo, hi): afterwards list[0..count) holds them as
// (entry << 32) | j in the order of j.  Every thread of the workgroup calls it.
__device__ __forceinline__ int list_targets(const int32_t *targets, int per_row, int64_t lo,
                                            int64_t hi, unsigned long long *list, int *waves_at) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  int count = 0;
  for (int j0 = 0; j0 < per_row; j0 += blockDim.x) {
    const int j = j0 + threadIdx.x;
    const int64_t t = j < per_row ? targets[j] : -1;
    const bool mine = t >= lo && t < hi;
    const unsigned long long on = __ballot(mine);
    __syncthreads();
    if (lane == 0) waves_at[wave] = __popcll(on);
    __syncthreads();
    int at = count;
    for (int w = 0; w < waves; ++w) {
      if (w == wave && mine)
        list[at + __popcll(on & ((1ull << lane) - 1))] =
            ((unsigned long long)t << 32) | (unsigned)j;
      at += waves_at[w];
    }
    count = at;
  }
  __syncthreads();
  return count;
}

// Calls f(entry, sum of weights) once for every entry the list names; weights
// of one entry are added in the order of j.  Few targets are compared pair by
// pair, many are sorted first (list has room for the next power of two).  Every
// thread of the workgroup calls it.
template <typename F>
__device__ __forceinline__ void each_entry(unsigned long long *list, int count,
                                           const float *weight, F f) {
  const int threads = blockDim.x;
  if (count <= kPairs) {
    // a repeated target's weights come from LDS, not one after the other from memory
    __shared__ float weights[kPairs];
    for (int a = threadIdx.x; a < count; a += threads) weights[a] = weight[(uint32_t)list[a]];
    __syncthreads();
    for (int a = threadIdx.x; a < count; a += threads) {
      const uint32_t t = (uint32_t)(list[a] >> 32);
      bool first = true;
      for (int b = 0; b < a && first; ++b) first = (uint32_t)(list[b] >> 32) != t;
      if (!first) continue;
      float sum = weights[a];
#pragma unroll 4
      for (int b = a + 1; b < count; ++b)
        if ((uint32_t)(list[b] >> 32) == t) sum += weights[b];
      f((int64_t)t, sum);
    }
    return;
  }
  int size = 256;
  while (size < count) size <<= 1;
  for (int a = count + threadIdx.x; a < size; a += threads) list[a] = ~0ull;
  for (int k = 2; k <= size; k <<= 1) {
    for (int d = k >> 1; d > 0; d >>= 1) {
      __syncthreads();
      for (int a = threadIdx.x; a < size / 2; a += threads) {
        const int i = (a / d) * 2 * d + a % d, j = i + d;
        const unsigned long long x = list[i], y = list[j];
        if ((x > y) == ((i & k) == 0)) list[i] = y, list[j] = x;
      }
    }
  }
  __syncthreads();
  // in order now: weights take the places of the j
  for (int a = threadIdx.x; a < count; a += threads)
    list[a] = (list[a] & ~0xFFFFFFFFull) | __float_as_uint(weight[(uint32_t)list[a]]);
  __syncthreads();
  for (int a = threadIdx.x; a < count; a += threads) {
    const uint32_t t = (uint32_t)(list[a] >> 32);
    if (a > 0 && (uint32_t)(list[a - 1] >> 32) == t) continue;
    float sum = 0.0f;
    bool same = true;
    for (int b = a; same; b += 8) {
      unsigned long long x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = list[min(b + j, count - 1)];  // on their way at once
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        same = same & (b + j < count) & ((uint32_t)(x[j] >> 32) == t);
        sum += same ? __uint_as_float((uint32_t)x[j]) : 0.0f;
      }
    }
    f((int64_t)t, sum);
  }
}

// Weights of the listed targets that are included, added in an order that
// depends on the list alone.
template <typename T>
__device__ __forceinline__ float listed_weight(const Rows &k, int64_t row, const float *weight,
                                               const unsigned long long *list, int count,
                                               float *lds) {
  float w = 0.0f;
  for (int a = threadIdx.x; a < count; a += blockDim.x)
    if (load_score<T>(k, row, (int64_t)(list[a] >> 32)) != ninf())
      w += weight[(uint32_t)list[a]];
  return count > 0 ? block_sum(w, lds) : 0.0f;
}

// Log-probabilities of targets that lie outside the row.
__device__ __forceinline__ void outside(const Rows &k, int64_t row) {
  for (int j = threadIdx.x; j < k.a.per_row; j += blockDim.x) {
    const int64_t t = k.a.targets[row * k.a.per_row + j];
    if (t < 0 || t >= k.a.s.n) k.a.logprob[row * k.a.per_row + j] = 0.0f;
  }
}

// The listed targets' log-probabilities and the gradient at their entries;
// share = (sum of weights) / l.
template <typename T>
__device__ __forceinline__ void at_targets(const Rows &k, int64_t row, unsigned long long *list,
                                           int count, Stat st, float r, float share) {
  const float *weight = k.a.weight + row * k.a.per_row;
  if (k.a.logprob) {
    for (int a = threadIdx.x; a < count; a += blockDim.x) {
      const float x = load_score<T>(k, row, (int64_t)(list[a] >> 32));
      k.a.logprob[row * k.a.per_row + (uint32_t)list[a]] = logprob_of(x, st, r);
    }
  }
  if (count > kPairs) __syncthreads();  // the list is sorted in place
  T *grad = static_cast<T *>(k.a.grad) + row * k.a.grad_ld;
  each_entry(list, count, weight, [&](int64_t t, float sum) {
    const float x = load_score<T>(k, row, t);
    if (x != ninf())
      grad[t] = narrow<T>(times_r(sum - weight_of(x, st.m, r) * share, r));
  });
}

// ---- rows in registers -----------------------------------------------------------

// VECS vectors of 16 bytes a thread, as they came (64 registers a lane in all:
// eight waves on a SIMD).  hold() keeps the compiler from carrying a pass's
// float32 values over to the next one.
template <typename T, int VECS, Mode MODE>
__global__ __launch_bounds__(1024, 8) void row_kernel(Rows k) {
  using V = typename Vec<T>::type;
  typedef uint32_t Raw __attribute__((ext_vector_type(4)));
  constexpr bool GRAD = MODE != kForward;
  constexpr int kLen = Vec<T>::kLen;
  Raw raw[VECS];
  auto get = [&](int g) { return __builtin_bit_cast(V, raw[g]); };
  auto hold = [&] {
#pragma unroll
    for (int g = 0; g < VECS; ++g) asm volatile("" : "+v"(raw[g]));
  };
  __shared__ float red[16];
  __shared__ int waves_at[16];
  extern __shared__ unsigned long long list[];
  const int64_t row = blockIdx.x;
  const int n = (int)k.a.s.n;
  const T *scores = row_scores<T>(k, row);
  const uint8_t *valid = row_mask(k, row);
  const int threads = blockDim.x;
  bool greedy;
  const float r = inverse_temperature(k.a.s.temperature, row, &greedy), c = r * kLog2e;

  // the targets first: nothing else is held in registers yet
  const int32_t *targets = k.a.targets + row * k.a.per_row;
  int count = 0;
  float w = 0.0f;
  if constexpr (GRAD) {
    count = list_targets(targets, k.a.per_row, 0, n, list, waves_at);
    w = listed_weight<T>(k, row, k.a.weight + row * k.a.per_row, list, count, red);
    if (k.a.logprob && count < k.a.per_row) outside(k, row);
    __syncthreads();
  }

  float m = ninf();
#pragma unroll
  for (int g = 0; g < VECS; ++g) {
    const int i = (g * threads + (int)threadIdx.x) * kLen;
    V v;
    if (i + kLen <= n) {
      v = *reinterpret_cast<const V *>(scores + i);
    } else {
#pragma unroll
      for (int j = 0; j < kLen; ++j) v[j] = i + j < n ? scores[i + j] : (T)ninf();
    }
    raw[g] = __builtin_bit_cast(Raw, v);
  }
  if (valid) {
#pragma unroll
    for (int g = 0; g < VECS; ++g) {
      const int i = (g * threads + (int)threadIdx.x) * kLen;
      V v = get(g);
#pragma unroll
      for (int j = 0; j < kLen; ++j)
        if (i + j < n && valid[i + j] == 0) v[j] = (T)ninf();
      raw[g] = __builtin_bit_cast(Raw, v);
    }
  }
#pragma unroll
  for (int g = 0; g < VECS; ++g) {
    const V v = get(g);
#pragma unroll
    for (int j = 0; j < kLen; ++j) m = fmaxf(m, widen<T>(v[j]));  // a NaN never is the larger
  }
  hold();
  m = block_max(m, red);

  // exp2(s * c - b) with b = m * c rounded: one fused operation an entry.
  // What b is off by is put right in l.  Where m / T passes 2^24 that can be
  // many powers of two, in either direction; NaN scores, infinite maxima and
  // temperatures that overflow c leave a NaN or nothing.  So the sum has to be
  // from 1/2 to 2^32: with the at most 2^16 entries of a row here the best one
  // then counts 2^-17 to 2^32, and factors that mend that are far from the ends
  // of float32.  Any other row is summed again, entry by entry, as differences to
  // the maximum.
  const float b = m * c;
  float l = 0.0f;
#pragma unroll
  for (int g = 0; g < VECS; ++g) {
    const V v = get(g);
#pragma unroll
    for (int j = 0; j < kLen; ++j)
      l += __builtin_amdgcn_exp2f(__builtin_fmaf((float)v[j], c, -b));
  }
  hold();
  l = block_sum(l, red);
  const float fast = l;
  const bool plain = fast >= 0.5f && fast < kPlainMost;
  if (plain) {
    l *= __builtin_amdgcn_exp2f(-__builtin_fmaf(m, c, -b));
  } else {
    l = 0.0f;
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += threads) {
      const float x = load_score<T>(k, row, i);
      if (x != ninf()) l += weight_of(x, m, r);
    }
    l = block_sum(l, red);
  }
  const Stat st = {m, l};
  if constexpr (!GRAD) {
    for (int j = threadIdx.x; j < k.a.per_row; j += threads) {
      const int64_t t = targets[j];
      k.a.logprob[row * k.a.per_row + j] =
          t < 0 || t >= n ? 0.0f : logprob_of(load_score<T>(k, row, t), st, r);
    }
    return;
  }
  const float share = w / l;
  T *grad = static_cast<T *>(k.a.grad) + row * k.a.grad_ld;
  // what the fast weights are off by, the fast sum is too.  A factor that passes
  // float32 would make a NaN of a weight of 0: the way entry by entry, then.
  const float fit = -w / fast * r;
  if (plain && __builtin_fabsf(fit) < __builtin_inff()) {
#pragma unroll
    for (int g = 0; g < VECS; ++g) {
      const int i = (g * threads + (int)threadIdx.x) * kLen;
      const V v = get(g);
      V o;
#pragma unroll
      for (int j = 0; j < kLen; ++j)
        o[j] = narrow<T>(__builtin_amdgcn_exp2f(__builtin_fmaf((float)v[j], c, -b)) * fit);
      if (i + kLen <= n) {
        if constexpr (MODE == kGradientPastCache)
          __builtin_nontemporal_store(o, reinterpret_cast<V *>(grad + i));
        else
          *reinterpret_cast<V *>(grad + i) = o;
      } else {
#pragma unroll
        for (int j = 0; j < kLen; ++j)
          if (i + j < n) grad[i + j] = o[j];
      }
    }
  } else {
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += threads) {
      const float x = load_score<T>(k, row, i);
      grad[i] = narrow<T>(x == ninf() ? 0.0f : times_r(weight_of(x, m, r) * -share, r));
    }
  }
  __syncthreads();
  at_targets<T>(k, row, list, count, st, r, share);
}

// ---- rows in chunks ----------------------------------------------------------------

template <typename T, bool GRAD>
__global__ __launch_bounds__(kThreads) void stats_kernel(Rows k) {
  __shared__ float red[kThreads / 64];
  __shared__ int waves_at[kThreads / 64];
  extern __shared__ unsigned long long list[];
  const int64_t row = blockIdx.x / k.chunks, chunk = blockIdx.x % k.chunks;
  const int64_t lo = chunk * k.chunk, hi = min(k.a.s.n, lo + k.chunk);
  const T *scores = row_scores<T>(k, row);
  const uint8_t *valid = row_mask(k, row);
  bool greedy;
  const float r = inverse_temperature(k.a.s.temperature, row, &greedy);
  Stat s = {ninf(), 0.0f};
  float next[8];
  load8(scores, valid, lo + threadIdx.x * 8, hi, next);
  float w = 0.0f;
  if constexpr (GRAD) {
    const int count = list_targets(k.a.targets + row * k.a.per_row, k.a.per_row, lo, hi, list,
                                   waves_at);
    w = listed_weight<T>(k, row, k.a.weight + row * k.a.per_row, list, count, red);
  }
  for (int64_t i = lo + threadIdx.x * 8; i < hi; i += kThreads * 8) {
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = next[j];
    load8(scores, valid, i + kThreads * 8, hi, next);
    float m = s.m;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, x[j]);
    if (m == ninf()) continue;
    float l = s.m == ninf() ? 0.0f : s.l * weight_of(s.m, m, r);
#pragma unroll
    for (int j = 0; j < 8; ++j) l += x[j] == ninf() ? 0.0f : weight_of(x[j], m, r);
    s = {m, l};
  }
  s = block_join(s, r, red);
  if (threadIdx.x == 0) k.part[blockIdx.x] = {s, w};
}

// The row's maximum, sum and weights, in every thread.
__device__ __forceinline__ Part row_part(const Rows &k, int64_t row, float r, float *red) {
  Part p = {{ninf(), 0.0f}, 0.0f};
  for (int64_t i = threadIdx.x; i < k.chunks; i += blockDim.x) {
    const Part o = k.part[row * k.chunks + i];
    if (o.s.m != ninf()) {
      const float m = fmaxf(p.s.m, o.s.m);
      const float l = p.s.m == ninf() ? 0.0f : p.s.l * weight_of(p.s.m, m, r);
      p.s = {m, l + o.s.l * weight_of(o.s.m, m, r)};
    }
    p.w += o.w;
  }
  p.s = block_join(p.s, r, red);
  if (k.a.grad) p.w = block_sum(p.w, red);
  return p;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void finish_kernel(Rows k) {
  __shared__ float red[kThreads / 64];
  const int64_t row = blockIdx.x;
  bool greedy;
  const float r = inverse_temperature(k.a.s.temperature, row, &greedy);
  const Part p = row_part(k, row, r, red);
  for (int j = threadIdx.x; j < k.a.per_row; j += kThreads) {
    const int64_t t = k.a.targets[row * k.a.per_row + j];
    k.a.logprob[row * k.a.per_row + j] =
        t < 0 || t >= k.a.s.n ? 0.0f : logprob_of(load_score<T>(k, row, t), p.s, r);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void grad_kernel(Rows k) {
  typedef T V __attribute__((ext_vector_type(8), aligned(sizeof(T))));
  __shared__ float red[kThreads / 64];
  __shared__ int waves_at[kThreads / 64];
  extern __shared__ unsigned long long list[];
  const int64_t row = blockIdx.x / k.chunks, chunk = blockIdx.x % k.chunks;
  const int64_t lo = chunk * k.chunk, hi = min(k.a.s.n, lo + k.chunk);
  const T *scores = row_scores<T>(k, row);
  const uint8_t *valid = row_mask(k, row);
  bool greedy;
  const float r = inverse_temperature(k.a.s.temperature, row, &greedy);
  const int32_t *targets = k.a.targets + row * k.a.per_row;
  // what does not wait for the row's sum first: its first scores, its targets
  float x[8];
  load8(scores, valid, lo + threadIdx.x * 8, hi, x);
  const int count = list_targets(targets, k.a.per_row, lo, hi, list, waves_at);
  const Part p = row_part(k, row, r, red);
  if (chunk == 0 && k.a.logprob) outside(k, row);
  const float share = p.w / p.s.l;
  T *grad = static_cast<T *>(k.a.grad) + row * k.a.grad_ld;
  for (int64_t i = lo + threadIdx.x * 8; i < hi; i += kThreads * 8) {
    V o;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      o[j] = narrow<T>(x[j] == ninf() ? 0.0f : times_r(weight_of(x[j], p.s.m, r) * -share, r));
    if (i + 8 <= hi) {
      *reinterpret_cast<V *>(grad + i) = o;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (i + j < hi) grad[i + j] = o[j];
    }
    load8(scores, valid, i + kThreads * 8, hi, x);
  }
  __syncthreads();
  at_targets<T>(k, row, list, count, p.s, r, share);
}

// ---- plans -------------------------------------------------------------------

// Chunks of a row: about four workgroups a CU where rows are few, none of them
// over fewer than kChunk entries.
void cut(int64_t n, int64_t rows, int cu_count, int64_t *chunk, int64_t *chunks) {
  const int64_t want = std::max<int64_t>(1, (int64_t)cu_count * 4 / std::max<int64_t>(1, rows));
  const int64_t most = std::max<int64_t>(1, (n + kChunk - 1) / kChunk);
  const int64_t c = std::min(want, most);
  *chunk = std::max<int64_t>(1, ((n + c - 1) / c + 63) / 64 * 64);
  *chunks = std::max<int64_t>(1, (n + *chunk - 1) / *chunk);
}

// LDS of a list of targets: its own length, or the power of two it is sorted in.
size_t list_bytes(int32_t per_row) {
  size_t size = (size_t)per_row;
  if (per_row > kPairs)
    for (size = 256; size < (size_t)per_row;) size <<= 1;
  return size * sizeof(unsigned long long);
}

template <typename T, int VECS>
hipError_t launch_row(const Rows &k, hipStream_t s) {
  const int64_t vecs = (k.a.s.n + Vec<T>::kLen - 1) / Vec<T>::kLen;
  const int threads = (int)std::max<int64_t>(64, ((vecs + VECS - 1) / VECS + 63) / 64 * 64);
  if (!k.a.grad) {
    row_kernel<T, VECS, kForward><<<(uint32_t)k.a.s.rows, threads, 0, s>>>(k);
    return hipGetLastError();
  }
  auto *kernel = k.a.s.rows * k.a.s.n * (int64_t)sizeof(T) > kPastCache
                     ? row_kernel<T, VECS, kGradientPastCache> : row_kernel<T, VECS, kGradient>;
  const size_t lds = list_bytes(k.a.per_row);
  const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(kernel), lds);
  if (e != hipSuccess) return e;
  kernel<<<(uint32_t)k.a.s.rows, threads, lds, s>>>(k);
  return hipGetLastError();
}

template <typename T>
hipError_t launch(const LogprobArgs &a, void *ws, int cu_count, hipStream_t s) {
  Rows k{};
  k.a = a;
  // A row in one workgroup's registers, unless its length would keep few
  // workgroups busy for long.
  const int64_t vecs = (a.s.n + Vec<T>::kLen - 1) / Vec<T>::kLen;
  if (vecs <= 8 * 1024 && (vecs <= 1024 || a.s.rows * 4 >= cu_count)) {
    if (vecs <= 1024) return launch_row<T, 1>(k, s);
    if (vecs <= 2 * 1024) return launch_row<T, 2>(k, s);
    if (vecs <= 4 * 1024) return launch_row<T, 4>(k, s);
    return launch_row<T, 8>(k, s);
  }
  k.part = static_cast<Part *>(ws);
  cut(a.s.n, a.s.rows, cu_count, &k.chunk, &k.chunks);
  const uint32_t grid = (uint32_t)(a.s.rows * k.chunks);
  if (!a.grad) {
    stats_kernel<T, false><<<grid, kThreads, 0, s>>>(k);
    finish_kernel<T><<<(uint32_t)a.s.rows, kThreads, 0, s>>>(k);
    return hipGetLastError();
  }
  const size_t lds = list_bytes(a.per_row);
  hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(stats_kernel<T, true>), lds);
  if (e == hipSuccess) e = ensure_dynamic_lds(reinterpret_cast<const void *>(grad_kernel<T>), lds);
  if (e != hipSuccess) return e;
  stats_kernel<T, true><<<grid, kThreads, lds, s>>>(k);
  grad_kernel<T><<<grid, kThreads, lds, s>>>(k);
  return hipGetLastError();
}

}  // namespace

size_t logprob_workspace_bytes(int64_t n, int64_t rows, int32_t per_row) {
  (void)per_row;
  (void)n;
  // chunks: at most 4 workgroups a CU (of at most 1,024 CUs), or one a row
  const int64_t chunks = std::max<int64_t>(1, 4096 / std::max<int64_t>(1, rows));
  return std::max<size_t>(256, (size_t)rows * chunks * sizeof(Part));
}

hipError_t launch_logprob(int dtype, const LogprobArgs &a, void *ws, int cu_count, hipStream_t s) {
  if (a.s.rows == 0) return hipSuccess;
  cu_count = std::min(cu_count, 1024);
  switch (dtype) {
    case ML2_F32: return launch<float>(a, ws, cu_count, s);
    case ML2_BF16: return launch<__bf16>(a, ws, cu_count, s);
    default: return launch<_Float16>(a, ws, cu_count, s);
  }
}

}  // namespace ml2
