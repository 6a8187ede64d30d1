// Rows of a learned table, scaled, and the gradient of that table.
//
//   lookup    out_i = scale * table[ids_i]
//   gradient  grad_v = scale * sum over the i with ids_i = v of dout_i
//
// Both move data and little else.  The gradient adds in a fixed order: the
// (id, position) pairs are sorted stably by id (least-significant-digit radix
// sort), the sorted list is cut into pieces of equal length, and a group of
// lanes adds the rows of one piece one after the other in registers.  A run
// of one id that lies inside a piece is finished there; the parts of a run
// that crosses pieces go to the workspace and are joined by join_kernel.  No
// floating-point atomics, so results are the same in every run.
#include <algorithm>

#include "draw.h"

namespace ml2 {
namespace {

constexpr int kThreads = 256;
constexpr int kWaveKeys = 512;   // keys of one wave in a sort pass
constexpr int kMaxBits = 9;      // digit of a sort pass
constexpr int kMaxBins = 1 << kMaxBits;

// ---- lookup -------------------------------------------------------------------

// Lanes of a group share a token's row; 256 / G tokens per workgroup and step.
template <typename T>
__global__ __launch_bounds__(kThreads) void lookup_kernel(EmbedArgs a, int log_g) {
  using V = typename Vec<T>::type;
  constexpr int kLen = Vec<T>::kLen;
  const int lane = threadIdx.x & ((1 << log_g) - 1);
  const int64_t per = kThreads >> log_g;
  for (int64_t i = (int64_t)blockIdx.x * per + (threadIdx.x >> log_g); i < a.n;
       i += (int64_t)gridDim.x * per) {
    const int64_t id = a.ids[i];
    const bool ok = id >= 0 && id < a.table_rows;
    const T *src = static_cast<const T *>(a.table) + (ok ? id : 0) * a.ld;
    T *dst = static_cast<T *>(a.out) + i * a.out_ld;
    for (int64_t c = (int64_t)lane * kLen; c < a.width; c += (int64_t)kLen << log_g) {
      if (c + kLen <= a.width) {
        V v = {};
        if (ok) {
          v = *reinterpret_cast<const V *>(src + c);
#pragma unroll
          for (int j = 0; j < kLen; ++j) v[j] = narrow<T>((float)v[j] * a.scale);
        }
        *reinterpret_cast<V *>(dst + c) = v;
      } else {
        for (int64_t j = c; j < a.width; ++j)
          dst[j] = ok ? narrow<T>((float)src[j] * a.scale) : (T)0.0f;
      }
    }
  }
}

// ---- stable sort of (id, position) by id ----------------------------------------

// The key of position i: its id, or table_rows (sorted last) outside the table.
__device__ __forceinline__ uint32_t token_key(const int32_t *ids, int64_t i, uint32_t rows) {
  const uint32_t id = (uint32_t)ids[i];
  return id < rows ? id : rows;
}

struct SortPass {
  const int32_t *ids;          // first pass: the tokens themselves
  const uint32_t *key, *pos;   // later passes: the last one's output
  uint32_t *key_out, *pos_out;
  uint32_t *hist;              // [bins][tiles]
  uint32_t n, rows, tiles;
  int shift, bits;
};

__device__ __forceinline__ uint32_t pass_key(const SortPass &p, uint32_t i) {
  return p.ids ? token_key(p.ids, i, p.rows) : p.key[i];
}

template <int WAVES>
__global__ __launch_bounds__(WAVES * 64) void sort_count(SortPass p) {
  __shared__ uint32_t h[kMaxBins];
  const uint32_t bins = 1u << p.bits;
  for (uint32_t b = threadIdx.x; b < bins; b += WAVES * 64) h[b] = 0;
  __syncthreads();
  const uint32_t base = blockIdx.x * (uint32_t)(WAVES * kWaveKeys);
#pragma unroll
  for (int r = 0; r < kWaveKeys / 64; ++r) {
    const uint64_t i = (uint64_t)base + (uint32_t)(r * WAVES * 64) + threadIdx.x;
    if (i < p.n) atomicAdd(&h[(pass_key(p, (uint32_t)i) >> p.shift) & (bins - 1)], 1u);
  }
  __syncthreads();
  for (uint32_t b = threadIdx.x; b < bins; b += WAVES * 64)
    p.hist[(size_t)b * p.tiles + blockIdx.x] = h[b];
}

// Exclusive prefix sum of h[0..total) in place: one workgroup.
__global__ __launch_bounds__(1024) void sort_scan(uint32_t *h, uint32_t total) {
  __shared__ uint32_t wave_sum[16];
  const uint32_t per = (total + 1023) / 1024;
  const uint32_t lo = min(total, threadIdx.x * per), hi = min(total, lo + per);
  uint32_t sum = 0;
  for (uint32_t i = lo; i < hi; ++i) sum += h[i];
  uint32_t incl = sum;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 63) wave_sum[wave] = incl;
  __syncthreads();
  uint32_t run = incl - sum;
  for (int w = 0; w < wave; ++w) run += wave_sum[w];
  for (uint32_t i = lo; i < hi; ++i) {
    const uint32_t v = h[i];
    h[i] = run;
    run += v;
  }
}

// The lanes of this wave that hold the same digit.
__device__ __forceinline__ unsigned long long same_digit(uint32_t digit, int bits, bool active) {
  unsigned long long peers = __ballot(active);
  for (int b = 0; b < bits; ++b) {
    const unsigned long long ones = __ballot(active && ((digit >> b) & 1u));
    peers &= ((digit >> b) & 1u) ? ones : ~ones;
  }
  return peers;
}

template <int WAVES>
__global__ __launch_bounds__(WAVES * 64) void sort_scatter(SortPass p) {
  __shared__ uint32_t at[WAVES][kMaxBins];
  const uint32_t bins = 1u << p.bits;
  for (uint32_t b = threadIdx.x; b < WAVES * (uint32_t)kMaxBins; b += WAVES * 64)
    (&at[0][0])[b] = 0;
  __syncthreads();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t base = (uint64_t)blockIdx.x * (WAVES * kWaveKeys) + (uint32_t)(wave * kWaveKeys);
  uint32_t key[kWaveKeys / 64], pos[kWaveKeys / 64], rank[kWaveKeys / 64];
#pragma unroll
  for (int r = 0; r < kWaveKeys / 64; ++r) {
    const uint64_t i = base + (uint32_t)(r * 64 + lane);
    const bool in = i < p.n;
    key[r] = in ? pass_key(p, (uint32_t)i) : 0u;
    pos[r] = !in ? 0u : p.ids ? (uint32_t)i : p.pos[i];
  }
#pragma unroll
  for (int r = 0; r < kWaveKeys / 64; ++r) {
    const bool in = base + (uint32_t)(r * 64 + lane) < p.n;
    const uint32_t digit = (key[r] >> p.shift) & (bins - 1);
    const unsigned long long peers = same_digit(digit, p.bits, in);
    const unsigned long long below = peers & ((1ull << lane) - 1);
    const int leader = __ffsll(peers | (1ull << 63)) - 1;  // a lane even where none is active
    uint32_t old = 0;
    if (in && below == 0) old = atomicAdd(&at[wave][digit], (uint32_t)__popcll(peers));
    rank[r] = __shfl(old, leader) + (uint32_t)__popcll(below);
  }
  __syncthreads();
  for (uint32_t b = threadIdx.x; b < bins; b += WAVES * 64) {
    uint32_t run = p.hist[(size_t)b * p.tiles + blockIdx.x];
    for (int w = 0; w < WAVES; ++w) {
      const uint32_t c = at[w][b];
      at[w][b] = run;
      run += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kWaveKeys / 64; ++r) {
    if (base + (uint32_t)(r * 64 + lane) >= p.n) continue;
    const uint32_t to = at[wave][(key[r] >> p.shift) & (bins - 1)] + rank[r];
    p.key_out[to] = key[r];
    p.pos_out[to] = pos[r];
  }
}

// ---- sums over the sorted list ---------------------------------------------------

struct SumArgs {
  EmbedGradArgs a;
  const uint32_t *key, *pos;  // sorted
  float *part;                // [pieces][2][width]: the run that entered a piece, the run that leaves it
  uint32_t n, rows, piece, pieces;
  int log_g;                  // lanes that share a row
};

template <typename T, typename O>
__device__ __forceinline__ void store_row(const SumArgs &s, uint32_t id, int64_t c,
                                          const float (&acc)[Vec<T>::kLen]) {
  constexpr int kLen = Vec<T>::kLen;
  typedef O OV __attribute__((ext_vector_type(kLen), aligned(sizeof(O))));
  O *dst = static_cast<O *>(s.a.grad) + (int64_t)id * s.a.grad_ld + c;
  if (c + kLen <= s.a.width) {
    OV v;
#pragma unroll
    for (int j = 0; j < kLen; ++j) v[j] = narrow<O>(acc[j] * s.a.scale);
    *reinterpret_cast<OV *>(dst) = v;
  } else {
#pragma unroll
    for (int j = 0; j < kLen; ++j)
      if (c + j < s.a.width) dst[j] = narrow<O>(acc[j] * s.a.scale);
  }
}

template <int LEN>
__device__ __forceinline__ void store_part(float *dst, int64_t c, int64_t width,
                                           const float (&acc)[LEN]) {
#pragma unroll
  for (int j = 0; j < LEN; ++j)
    if (c + j < width) dst[c + j] = acc[j];
}

template <typename T>
__device__ __forceinline__ void load_row(const T *src, int64_t c, int64_t width,
                                         typename Vec<T>::type &v) {
  using V = typename Vec<T>::type;
  if (c + Vec<T>::kLen <= width) {
    v = *reinterpret_cast<const V *>(src + c);
  } else {
#pragma unroll
    for (int j = 0; j < Vec<T>::kLen; ++j) v[j] = c + j < width ? src[c + j] : (T)0.0f;
  }
}

template <typename T, typename O>
__global__ __launch_bounds__(kThreads) void sum_kernel(SumArgs s) {
  using V = typename Vec<T>::type;
  constexpr int kLen = Vec<T>::kLen;
  constexpr int kAhead = 4;
  const int64_t c = ((int64_t)blockIdx.y << s.log_g) * kLen +
                    (int64_t)(threadIdx.x & ((1 << s.log_g) - 1)) * kLen;
  const uint32_t p = blockIdx.x * (uint32_t)(kThreads >> s.log_g) + (threadIdx.x >> s.log_g);
  if (p >= s.pieces || c >= s.a.width) return;
  const uint32_t lo = p * s.piece, hi = min(s.n, lo + s.piece);
  const uint32_t before = lo > 0 ? s.key[lo - 1] : 0xFFFFFFFFu;
  const uint32_t after = hi < s.n ? s.key[hi] : 0xFFFFFFFFu;
  const T *dout = static_cast<const T *>(s.a.dout);
  float acc[kLen] = {};
  uint32_t cur = s.key[lo];
  bool entered = cur == before;  // the current run began in an earlier piece
  for (uint32_t e = lo; e < hi; e += kAhead) {
    uint32_t key[kAhead];
    V v[kAhead] = {};
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      key[j] = s.rows;
      if (e + j < hi) {
        key[j] = s.key[e + j];
        if (key[j] < s.rows)
          load_row<T>(dout + (int64_t)s.pos[e + j] * s.a.dout_ld, c, s.a.width, v[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (e + j >= hi) break;
      if (key[j] != cur) {
        if (entered)
          store_part(s.part + (size_t)p * 2 * s.a.width, c, s.a.width, acc);
        else
          store_row<T, O>(s, cur, c, acc);
        cur = key[j];
        entered = false;
#pragma unroll
        for (int q = 0; q < kLen; ++q) acc[q] = 0.0f;
      }
#pragma unroll
      for (int q = 0; q < kLen; ++q) acc[q] += (float)v[j][q];
    }
  }
  if (cur >= s.rows) return;
  if (entered)
    store_part(s.part + (size_t)p * 2 * s.a.width, c, s.a.width, acc);
  else if (cur == after)
    store_part(s.part + ((size_t)p * 2 + 1) * s.a.width, c, s.a.width, acc);
  else
    store_row<T, O>(s, cur, c, acc);
}

// Joins the runs that cross pieces: a workgroup looks at 64 pieces and adds,
// for each run that leaves one of them and did not enter it, the parts of the
// pieces it reaches.  Groups of lanes take every 256/G-th part in order; their
// sums are added in group order.
template <typename T, typename O>
__global__ __launch_bounds__(kThreads) void join_kernel(SumArgs s) {
  constexpr int kLen = Vec<T>::kLen;
  __shared__ float sums[kThreads][kLen];
  const int lane = threadIdx.x & 63;
  const uint32_t p0 = blockIdx.x * 64u;
  bool starts = false;
  {
    const uint32_t p = p0 + lane;
    if (p + 1 < s.pieces) {
      const uint32_t lo = p * s.piece, hi = lo + s.piece, id = s.key[hi - 1];
      starts = id < s.rows && s.key[hi] == id &&
               (s.key[lo] != id || lo == 0 || s.key[lo - 1] != id);
    }
  }
  unsigned long long todo = __ballot(starts);  // the same in every wave
  const int g = 1 << s.log_g, groups = kThreads >> s.log_g;
  const int group = threadIdx.x >> s.log_g;
  const int64_t c = (int64_t)blockIdx.y * g * kLen + (int64_t)(threadIdx.x & (g - 1)) * kLen;
  const bool live = c < s.a.width;
  while (todo) {
    const uint32_t p = p0 + (uint32_t)(__ffsll(todo) - 1);
    todo &= todo - 1;
    const uint32_t id = s.key[(p + 1) * s.piece - 1];
    uint32_t lo = (p + 1) * s.piece, hi = s.n;  // first entry past the run
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo) / 2;
      if (s.key[mid] == id) lo = mid + 1; else hi = mid;
    }
    const uint32_t last = (lo - 1) / s.piece;
    float acc[kLen] = {};
    if (live) {
      for (uint32_t q = p + group; q <= last; q += groups) {
        const float *src = s.part + ((size_t)q * 2 + (q == p ? 1 : 0)) * s.a.width;
#pragma unroll
        for (int j = 0; j < kLen; ++j)
          if (c + j < s.a.width) acc[j] += src[c + j];
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kLen; ++j) sums[threadIdx.x][j] = acc[j];
    __syncthreads();
    if (group == 0 && live) {
      for (int q = 1; q < groups; ++q)
#pragma unroll
        for (int j = 0; j < kLen; ++j) acc[j] += sums[(q << s.log_g) + threadIdx.x][j];
      store_row<T, O>(s, id, c, acc);
    }
  }
}

// Zeros for the table rows that no token names: a wave looks 64 rows up in
// the sorted list at once.
template <typename O>
__global__ __launch_bounds__(kThreads) void fill_kernel(SumArgs s) {
  typedef O OV __attribute__((ext_vector_type(16 / sizeof(O)), aligned(sizeof(O))));
  constexpr int kLen = 16 / sizeof(O);
  const int lane = threadIdx.x & 63;
  const int64_t r0 = ((int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)) * 64;
  if (r0 >= s.rows) return;
  const int64_t r = r0 + lane;
  uint32_t lo = 0, hi = s.n;
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if ((int64_t)s.key[mid] < r) lo = mid + 1; else hi = mid;
  }
  const bool none = r < s.rows && !(lo < s.n && (int64_t)s.key[lo] == r);
  O *grad = static_cast<O *>(s.a.grad);
  if (s.a.width <= 16) {
    if (none)
      for (int64_t c = 0; c < s.a.width; ++c) grad[r * s.a.grad_ld + c] = (O)0.0f;
    return;
  }
  for (unsigned long long todo = __ballot(none); todo; todo &= todo - 1) {
    O *dst = grad + (r0 + (__ffsll(todo) - 1)) * s.a.grad_ld;
    for (int64_t c = (int64_t)lane * kLen; c < s.a.width; c += 64 * kLen) {
      if (c + kLen <= s.a.width) {
        *reinterpret_cast<OV *>(dst + c) = OV{};
      } else {
        for (int64_t j = c; j < s.a.width; ++j) dst[j] = (O)0.0f;
      }
    }
  }
}

// ---- plans -------------------------------------------------------------------

// Lanes that share a row: enough 16-byte vectors for its width, at most `most`.
int log_group(int64_t width, int len, int most) {
  int g = 0;
  while (g < most && ((int64_t)len << g) < width) ++g;
  return g;
}

struct GradPlan {
  int bits, passes, waves;  // of a digit; sort passes; waves of a sort workgroup
  uint32_t tiles, piece, pieces;
  size_t keys, hist, part;  // byte offsets of the second key buffer, counts, parts
  size_t bytes;
};

GradPlan grad_plan(int64_t n, int64_t rows, int64_t width) {
  GradPlan p{};
  int bits = 1;
  while (((int64_t)1 << bits) <= rows) ++bits;  // keys 0 .. rows
  p.passes = (bits + kMaxBits - 1) / kMaxBits;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.waves = n > (1 << 18) ? 16 : 4;
  const int64_t tile = (int64_t)p.waves * kWaveKeys;
  p.tiles = (uint32_t)((n + tile - 1) / tile);
  p.piece = 32;
  p.pieces = (uint32_t)((n + p.piece - 1) / p.piece);
  auto align = [](size_t b) { return (b + 255) & ~(size_t)255; };
  const size_t list = align((size_t)n * 4);
  p.keys = 2 * list;
  p.hist = 4 * list;
  p.part = p.hist + align(((size_t)p.tiles << p.bits) * 4);
  p.bytes = p.part + align((size_t)p.pieces * 2 * (size_t)width * 4);
  return p;
}

template <typename T, typename O>
hipError_t launch_sums(const SumArgs &s, int64_t width, hipStream_t st) {
  const uint32_t slabs = (uint32_t)((width + ((int64_t)Vec<T>::kLen << s.log_g) - 1) /
                                    ((int64_t)Vec<T>::kLen << s.log_g));
  const uint32_t per = kThreads >> s.log_g;
  if (s.rows > 0)
    fill_kernel<O><<<(s.rows + 255u) / 256u, kThreads, 0, st>>>(s);
  if (s.n > 0) {
    sum_kernel<T, O><<<dim3((s.pieces + per - 1) / per, slabs), kThreads, 0, st>>>(s);
    if (s.pieces > 1)
      join_kernel<T, O><<<dim3((s.pieces + 63) / 64, slabs), kThreads, 0, st>>>(s);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_lookup(const EmbedArgs &a, int cu_count, hipStream_t s) {
  const int log_g = log_group(a.width, Vec<T>::kLen, 6);
  const int64_t per = kThreads >> log_g;
  const int64_t grid = std::min<int64_t>((a.n + per - 1) / per, (int64_t)cu_count * 32);
  lookup_kernel<T><<<(uint32_t)grid, kThreads, 0, s>>>(a, log_g);
  return hipGetLastError();
}

template <int WAVES>
void launch_pass(const SortPass &p, hipStream_t st) {
  sort_count<WAVES><<<p.tiles, WAVES * 64, 0, st>>>(p);
  sort_scan<<<1, 1024, 0, st>>>(p.hist, p.tiles << p.bits);
  sort_scatter<WAVES><<<p.tiles, WAVES * 64, 0, st>>>(p);
}

}  // namespace

hipError_t launch_embed(int dtype, const EmbedArgs &a, int cu_count, hipStream_t s) {
  if (a.n == 0 || a.width == 0) return hipSuccess;
  switch (dtype) {
    case ML2_F32: return launch_lookup<float>(a, cu_count, s);
    case ML2_BF16: return launch_lookup<__bf16>(a, cu_count, s);
    default: return launch_lookup<_Float16>(a, cu_count, s);
  }
}

size_t embed_grad_workspace_bytes(int64_t n, int64_t table_rows, int64_t width) {
  return std::max<size_t>(256, grad_plan(n, table_rows, width).bytes);
}

hipError_t launch_embed_grad(int dtype, int grad_dtype, const EmbedGradArgs &a, void *ws,
                             int cu_count, hipStream_t st) {
  (void)cu_count;
  if (a.table_rows == 0 || a.width == 0) return hipSuccess;
  const GradPlan g = grad_plan(a.n, a.table_rows, a.width);
  char *base = static_cast<char *>(ws);
  uint32_t *list[2] = {reinterpret_cast<uint32_t *>(base),
                       reinterpret_cast<uint32_t *>(base + g.keys)};
  const size_t half = g.keys / 2 / 4;  // positions follow the keys
  int at = 0;
  for (int pass = 0; pass < g.passes && a.n > 0; ++pass) {
    SortPass p{};
    if (pass == 0) {
      p.ids = a.ids;
    } else {
      p.key = list[at];
      p.pos = list[at] + half;
      at ^= 1;
    }
    p.key_out = list[at];
    p.pos_out = list[at] + half;
    p.hist = reinterpret_cast<uint32_t *>(base + g.hist);
    p.n = (uint32_t)a.n;
    p.rows = (uint32_t)a.table_rows;
    p.tiles = g.tiles;
    p.shift = pass * g.bits;
    p.bits = g.bits;
    if (g.waves == 16) launch_pass<16>(p, st); else launch_pass<4>(p, st);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  SumArgs s{};
  s.a = a;
  s.key = list[at];
  s.pos = list[at] + half;
  s.part = reinterpret_cast<float *>(base + g.part);
  s.n = (uint32_t)a.n;
  s.rows = (uint32_t)a.table_rows;
  s.piece = g.piece;
  s.pieces = g.pieces;
  s.log_g = log_group(a.width, dtype == ML2_F32 ? 4 : 8, 6);
  const bool wide = grad_dtype == ML2_F32;
  switch (dtype) {
    case ML2_F32: return launch_sums<float, float>(s, a.width, st);
    case ML2_BF16:
      return wide ? launch_sums<__bf16, float>(s, a.width, st)
                  : launch_sums<__bf16, __bf16>(s, a.width, st);
    default:
      return wide ? launch_sums<_Float16, float>(s, a.width, st)
                  : launch_sums<_Float16, _Float16>(s, a.width, st);
  }
}

}  // namespace ml2
