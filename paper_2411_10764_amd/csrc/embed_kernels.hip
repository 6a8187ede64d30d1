// Rows of a learned table, scaled, and the gradient of that table.
//
//   lookup    out_i = scale * table[ids_i]
//   gradient  grad_v = scale * sum over the i with ids_i = v of dout_i
//
// Both move data and little else.  The gradient adds in a fixed order: the
// (id, position) pairs are sorted stably by id (least-significant-digit radix
// sort, in one workgroup up to kOneSort tokens), the sorted list is cut into
// pieces of equal length, and a group of lanes adds the rows of one piece one
// after the other in registers.  A run of one id that lies inside a piece is
// finished there; the parts of a run that crosses pieces go to the workspace
// and are joined by join_kernel.  No floating-point atomics, so results are
// the same in every run.  The rows that no token names are cleared by further
// workgroups of all those launches.
//
// A table of few numbers (rows * width at most kFewCells, width at most
// kFewWidth) needs no sort: every lane of a wave holds a table of its own in
// LDS (few_kernel), and the lanes' and waves' tables are added up in order.
// More numbers do not fit the LDS of a compute unit: 4,194,304 tokens into 512
// float32 numbers 52 us, into 513, sorted, 160.
//
// Measured: lookup of 32,768 x 1,024 bf16 22 us; its gradient into 131,072
// float32 rows 149 us (604 MB, 4.1 TB/s, most of it the clearing); 4,194,304
// tokens into 81 numbers 18 us.
#include <algorithm>

#include "draw.h"

namespace ml2 {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxBits = 9;      // digit of a sort pass
constexpr int kMaxBins = 1 << kMaxBits;
constexpr int kMaxTiles = 256;   // workgroups of a sort pass
constexpr int kFewCells = 512;
constexpr int kFewWidth = 4;

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

// ---- clearing beside the sort ------------------------------------------------------

// The sort keeps few compute units busy.  Further workgroups of its launches
// clear the table's first rows meanwhile, named by a token or not.
struct Clear {
  uint16_t *grad;          // in halves of 4 bytes: every type is a number of them
  int64_t row0, row1;      // rows of this launch
  int64_t width, ld;       // of a row, in halves
  uint32_t first, blocks;  // workgroups first .. first + blocks - 1 clear
};

typedef uint16_t Halves __attribute__((ext_vector_type(8), aligned(2)));

__device__ __forceinline__ void clear_part(const Clear &f) {
  // rows that follow one another are one long row
  const bool flat = f.ld == f.width;
  const int64_t rows = flat ? 1 : f.row1 - f.row0;
  const int64_t width = flat ? (f.row1 - f.row0) * f.width : f.width;
  // vector v of a row, then of the next: narrow rows keep all threads at work
  const int64_t vecs = (width + 7) / 8, step = (int64_t)f.blocks * blockDim.x;
  const int64_t first = (int64_t)(blockIdx.x - f.first) * blockDim.x + threadIdx.x;
  int64_t r = first / vecs, v = first % vecs;
  const int64_t down = step / vecs, along = step % vecs;
  while (r < rows) {
    uint16_t *row = f.grad + (f.row0 + r) * f.ld;
    const int64_t c = v * 8;
    if (c + 8 <= width) {
      __builtin_nontemporal_store(Halves{}, reinterpret_cast<Halves *>(row + c));
    } else {
      for (int64_t j = c; j < width; ++j) row[j] = 0;
    }
    r += down;
    v += along;
    if (v >= vecs) v -= vecs, ++r;
  }
}

// ---- stable sort of (id, position) by id ----------------------------------------

// The key of position i: its id, or table_rows (sorted last) outside the table.
__device__ __forceinline__ uint32_t token_key(const int32_t *ids, int64_t i, uint32_t rows) {
  const uint32_t id = (uint32_t)ids[i];
  return id < rows ? id : rows;
}

// A pass sorts by one digit.  A workgroup takes a tile: `subs` times WAVES *
// ROUNDS * 64 keys in a row.
struct SortPass {
  const int32_t *ids;          // first pass: the tokens themselves
  const uint32_t *key, *pos;   // later passes: the last one's output
  uint32_t *key_out, *pos_out;
  uint32_t *hist;              // [tiles][bins]
  uint32_t n, rows, tiles, subs;
  int shift, bits;
};

__device__ __forceinline__ uint32_t pass_key(const SortPass &p, uint32_t i) {
  return p.ids ? token_key(p.ids, i, p.rows) : p.key[i];
}

template <int WAVES, int ROUNDS>
__global__ __launch_bounds__(WAVES * 64) void sort_count(SortPass p, Clear f) {
  __shared__ uint32_t h[kMaxBins];
  if (blockIdx.x >= f.first) return clear_part(f);
  const uint32_t bins = 1u << p.bits;
  for (uint32_t b = threadIdx.x; b < bins; b += WAVES * 64) h[b] = 0;
  __syncthreads();
  for (uint32_t sub = 0; sub < p.subs; ++sub) {
    const uint64_t base = ((uint64_t)blockIdx.x * p.subs + sub) * (WAVES * ROUNDS * 64);
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const uint64_t i = base + (uint32_t)(r * WAVES * 64) + threadIdx.x;
      if (i < p.n) atomicAdd(&h[(pass_key(p, (uint32_t)i) >> p.shift) & (bins - 1)], 1u);
    }
  }
  __syncthreads();
  for (uint32_t b = threadIdx.x; b < bins; b += WAVES * 64) p.hist[blockIdx.x * bins + b] = h[b];
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

template <int WAVES, int ROUNDS>
__global__ __launch_bounds__(WAVES * 64) void sort_scatter(SortPass p, Clear f) {
  constexpr uint32_t kBlock = WAVES * 64;
  __shared__ uint32_t at[WAVES][kMaxBins];
  __shared__ uint32_t base[kMaxBins], total[kMaxBins];
  if (blockIdx.x >= f.first) return clear_part(f);
  const uint32_t bins = 1u << p.bits;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // Where this tile's keys of a digit go: all keys of smaller digits, and the
  // earlier tiles' keys of the same.  Slices of threads share the tiles.
  for (uint32_t b = threadIdx.x; b < bins; b += kBlock) base[b] = total[b] = 0;
  __syncthreads();
  const uint32_t slices = max(1u, kBlock >> p.bits);
  const uint32_t per = (p.tiles + slices - 1) / slices;
  for (uint32_t e = threadIdx.x; e < slices * bins; e += kBlock) {
    const uint32_t b = e & (bins - 1), t0 = (e >> p.bits) * per, t1 = min(p.tiles, t0 + per);
    uint32_t before = 0, all = 0;
#pragma unroll 8
    for (uint32_t t = t0; t < t1; ++t) {
      const uint32_t c = p.hist[t * bins + b];
      all += c;
      before += t < blockIdx.x ? c : 0u;
    }
    atomicAdd(&total[b], all);
    atomicAdd(&base[b], before);
  }
  __syncthreads();
  if (wave == 0) {
    uint32_t carry = 0;
    for (uint32_t b0 = 0; b0 < bins; b0 += 64) {
      const uint32_t b = b0 + lane, own = b < bins ? total[b] : 0u;
      uint32_t incl = own;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(incl, d);
        if (lane >= d) incl += o;
      }
      if (b < bins) base[b] += carry + incl - own;
      carry += __shfl(incl, 63);
    }
  }
  for (uint32_t sub = 0; sub < p.subs; ++sub) {
    const uint64_t first = ((uint64_t)blockIdx.x * p.subs + sub) * (kBlock * ROUNDS);
    if (first >= p.n) return;
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < WAVES * (uint32_t)kMaxBins; b += kBlock) (&at[0][0])[b] = 0;
    __syncthreads();
    const uint64_t own = first + (uint32_t)(wave * ROUNDS * 64);
    uint32_t key[ROUNDS], pos[ROUNDS], rank[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const uint64_t i = own + (uint32_t)(r * 64 + lane);
      const bool in = i < p.n;
      key[r] = in ? pass_key(p, (uint32_t)i) : 0u;
      pos[r] = !in ? 0u : p.ids ? (uint32_t)i : p.pos[i];
    }
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const bool in = own + (uint32_t)(r * 64 + lane) < p.n;
      const uint32_t digit = (key[r] >> p.shift) & (bins - 1);
      const unsigned long long peers = same_digit(digit, p.bits, in);
      const unsigned long long below = peers & ((1ull << lane) - 1);
      const int leader = __ffsll(peers | (1ull << 63)) - 1;  // a lane even where none is active
      uint32_t old = 0;
      if (in && below == 0) old = atomicAdd(&at[wave][digit], (uint32_t)__popcll(peers));
      rank[r] = __shfl(old, leader) + (uint32_t)__popcll(below);
    }
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < bins; b += kBlock) {
      uint32_t run = base[b];
      for (int w = 0; w < WAVES; ++w) {
        const uint32_t c = at[w][b];
        at[w][b] = run;
        run += c;
      }
      base[b] = run;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      if (own + (uint32_t)(r * 64 + lane) >= p.n) continue;
      const uint32_t to = at[wave][(key[r] >> p.shift) & (bins - 1)] + rank[r];
      p.key_out[to] = key[r];
      p.pos_out[to] = pos[r];
    }
  }
}

// All passes over at most kOneSort tokens in one workgroup: keys and positions
// stay in registers, LDS carries them from one order to the next.  PACKED: both
// in one word, where the table's rows leave the bits.
constexpr int kOneRounds = 8;
constexpr int kOneSort = 1024 * kOneRounds;
constexpr int kOneBits = 13;  // of a position

struct OneSort {
  const int32_t *ids;
  uint32_t *key_out, *pos_out;
  uint32_t n, rows;
  int passes, bits;
};

template <bool PACKED>
__global__ __launch_bounds__(1024) void sort_one(OneSort p, Clear f) {
  __shared__ uint32_t at[16][kMaxBins], base[kMaxBins];
  if (blockIdx.x >= f.first) return clear_part(f);
  extern __shared__ uint32_t exchange[];  // [n rounded up to 1024]
  const uint32_t bins = 1u << p.bits;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rounds = (int)((p.n + 1023) / 1024);
  const uint32_t own = (uint32_t)(wave * rounds * 64 + lane);  // a wave's keys are consecutive
  uint32_t key[kOneRounds], pos[kOneRounds], to[kOneRounds];
#pragma unroll
  for (int r = 0; r < kOneRounds; ++r) {
    const uint32_t i = own + (uint32_t)(r * 64);
    key[r] = r < rounds && i < p.n ? token_key(p.ids, i, p.rows) : 0u;
    pos[r] = i;
    if (PACKED) key[r] = key[r] << kOneBits | i;
  }
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * p.bits + (PACKED ? kOneBits : 0);
    for (uint32_t b = threadIdx.x; b < 16u * kMaxBins; b += 1024) (&at[0][0])[b] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kOneRounds; ++r) {
      if (r >= rounds) break;
      const bool in = own + (uint32_t)(r * 64) < p.n;
      const uint32_t digit = (key[r] >> shift) & (bins - 1);
      const unsigned long long peers = same_digit(digit, p.bits, in);
      const unsigned long long below = peers & ((1ull << lane) - 1);
      const int leader = __ffsll(peers | (1ull << 63)) - 1;
      uint32_t old = 0;
      if (in && below == 0) old = atomicAdd(&at[wave][digit], (uint32_t)__popcll(peers));
      to[r] = __shfl(old, leader) + (uint32_t)__popcll(below);
    }
    __syncthreads();
    if (threadIdx.x < bins) {
      uint32_t run = 0;
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        const uint32_t c = at[w][threadIdx.x];
        at[w][threadIdx.x] = run;
        run += c;
      }
      base[threadIdx.x] = run;
    }
    __syncthreads();
    if (wave == 0) {
      uint32_t carry = 0;
      for (uint32_t b0 = 0; b0 < bins; b0 += 64) {
        const uint32_t b = b0 + lane, own_count = b < bins ? base[b] : 0u;
        uint32_t incl = own_count;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const uint32_t o = __shfl_up(incl, d);
          if (lane >= d) incl += o;
        }
        if (b < bins) base[b] = carry + incl - own_count;
        carry += __shfl(incl, 63);
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kOneRounds; ++r) {
      const uint32_t digit = (key[r] >> shift) & (bins - 1);
      if (r < rounds && own + (uint32_t)(r * 64) < p.n) {
        to[r] += base[digit] + at[wave][digit];
        exchange[to[r]] = key[r];
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kOneRounds; ++r)
      if (r < rounds && own + (uint32_t)(r * 64) < p.n) key[r] = exchange[own + (uint32_t)(r * 64)];
    __syncthreads();
    if (PACKED) continue;
#pragma unroll
    for (int r = 0; r < kOneRounds; ++r)
      if (r < rounds && own + (uint32_t)(r * 64) < p.n) exchange[to[r]] = pos[r];
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kOneRounds; ++r)
      if (r < rounds && own + (uint32_t)(r * 64) < p.n) pos[r] = exchange[own + (uint32_t)(r * 64)];
    __syncthreads();
  }
#pragma unroll
  for (int r = 0; r < kOneRounds; ++r) {
    const uint32_t i = own + (uint32_t)(r * 64);
    if (r < rounds && i < p.n) {
      p.key_out[i] = PACKED ? key[r] >> kOneBits : key[r];
      p.pos_out[i] = PACKED ? key[r] & ((1u << kOneBits) - 1) : pos[r];
    }
  }
}

// ---- sums over the sorted list ---------------------------------------------------

struct SumArgs {
  EmbedGradArgs a;
  const uint32_t *key, *pos;  // sorted
  float *part;                // [pieces][2][width]: the run that entered a piece, the run that leaves it
  uint32_t n, rows, piece, pieces;
  int log_g;                  // lanes that share a row
  uint32_t slabs;             // of a row
  uint32_t sum_blocks, join_blocks;  // workgroups that add or join, the others clear
  uint32_t cleared, split;    // rows below `cleared` are; those below `split` are beside the sums,
                              // the others beside the joins
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

// Zeros for the rows that no token names: a wave looks 64 rows up in the
// sorted list at once.
template <typename O>
__device__ __forceinline__ void clear_rows(const SumArgs &s, uint32_t block, uint32_t row0,
                                           uint32_t row1) {
  constexpr int kLen = 16 / (int)sizeof(O);
  typedef O OV __attribute__((ext_vector_type(kLen), aligned(sizeof(O))));
  const int lane = threadIdx.x & 63;
  const int64_t r0 = row0 + ((int64_t)block * (blockDim.x / 64) + (threadIdx.x >> 6)) * 64;
  if (r0 >= row1) return;
  const int64_t r = r0 + lane;
  uint32_t lo = 0, hi = s.n;
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if ((int64_t)s.key[mid] < r) lo = mid + 1; else hi = mid;
  }
  const bool none = r < row1 && !(lo < s.n && (int64_t)s.key[lo] == r);
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
        __builtin_nontemporal_store(OV{}, reinterpret_cast<OV *>(dst + c));
      } else {
        for (int64_t j = c; j < s.a.width; ++j) dst[j] = (O)0.0f;
      }
    }
  }
}

// The keys and positions of a workgroup's pieces go through LDS (read once,
// in order); a row's load is then the only access to memory that an addition
// waits for, and kAhead of them are in flight.
template <typename T, typename O>
__global__ __launch_bounds__(kThreads) void sum_kernel(SumArgs s) {
  using V = typename Vec<T>::type;
  constexpr int kLen = Vec<T>::kLen;
  constexpr int kAhead = 8;
  extern __shared__ uint32_t staged[];  // [groups][piece + 1] keys, then positions
  if (blockIdx.x >= s.sum_blocks) return clear_rows<O>(s, blockIdx.x - s.sum_blocks, s.cleared, s.split);
  const uint32_t block = blockIdx.x / s.slabs, slab = blockIdx.x % s.slabs;
  const uint32_t groups = kThreads >> s.log_g, stride = s.piece + 1;
  uint32_t *keys = staged, *poss = staged + groups * stride;
  const uint32_t e0 = block * groups * s.piece;
  for (uint32_t e = threadIdx.x; e < groups * s.piece && e0 + e < s.n; e += kThreads) {
    const uint32_t at = e / s.piece * stride + e % s.piece;
    keys[at] = s.key[e0 + e];
    poss[at] = s.pos[e0 + e];
  }
  __syncthreads();
  const int64_t c = ((int64_t)slab << s.log_g) * kLen +
                    (int64_t)(threadIdx.x & ((1 << s.log_g) - 1)) * kLen;
  const uint32_t group = threadIdx.x >> s.log_g, p = block * groups + group;
  if (p >= s.pieces || c >= s.a.width) return;
  const uint32_t lo = p * s.piece, hi = min(s.n, lo + s.piece);
  const uint32_t before = lo > 0 ? s.key[lo - 1] : 0xFFFFFFFFu;
  const uint32_t after = hi < s.n ? s.key[hi] : 0xFFFFFFFFu;
  const T *dout = static_cast<const T *>(s.a.dout);
  const uint32_t *key = keys + group * stride, *pos = poss + group * stride;
  const int len = (int)(hi - lo);
  float acc[kLen] = {};
  uint32_t cur = key[0];
  bool entered = cur == before;  // the current run began in an earlier piece
  for (int e = 0; e < len; e += kAhead) {
    V v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      v[j] = V{};
      if (e + j < len && key[e + j] < s.rows)
        load_row<T>(dout + (int64_t)pos[e + j] * s.a.dout_ld, c, s.a.width, v[j]);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (e + j < len && key[e + j] != cur) {
        if (entered)
          store_part(s.part + (size_t)p * 2 * s.a.width, c, s.a.width, acc);
        else
          store_row<T, O>(s, cur, c, acc);
        cur = key[e + j];
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

// Joins the runs that cross pieces.  A group of lanes looks at one piece: a run
// that leaves it without having entered it is the group's to add up, part after
// part, where it reaches few pieces; a longer one is left to a wave, or to the
// whole workgroup, whose groups take every so-many-th part in order and fold
// their sums pairwise.
constexpr int kJoinThreads = 1024;
constexpr int kShortRun = 16;  // pieces that a group joins itself
constexpr int kWaveRun = 32;   // pieces of each of a wave's groups that a wave joins itself

template <typename T, typename O>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(SumArgs s) {
  constexpr int kLen = Vec<T>::kLen;
  typedef float Part __attribute__((ext_vector_type(kLen), aligned(4)));
  __shared__ float sums[kJoinThreads * kLen];
  // first pieces of longer runs, and the last ones of the longest
  __shared__ uint32_t long_run[kJoinThreads / kShortRun + 1];
  __shared__ uint32_t long_last[kJoinThreads / kShortRun + 1], longs;
  if (blockIdx.x >= s.join_blocks)
    return clear_rows<O>(s, blockIdx.x - s.join_blocks, s.split, s.rows);
  const int groups = kJoinThreads >> s.log_g, group = threadIdx.x >> s.log_g;
  const uint32_t block = blockIdx.x / s.slabs, slab = blockIdx.x % s.slabs;
  const int in = threadIdx.x & ((1 << s.log_g) - 1);
  const int64_t c = ((int64_t)slab << s.log_g) * kLen + (int64_t)in * kLen;
  const bool live = c < s.a.width, whole = c + kLen <= s.a.width;
  // adds the parts of pieces q, q + step, ... last
  auto add = [&](float (&acc)[kLen], uint32_t p, uint32_t q, uint32_t step, uint32_t last) {
#pragma unroll 8
    for (; q <= last; q += step) {
      const float *src = s.part + ((size_t)q * 2 + (q == p ? 1 : 0)) * s.a.width + c;
      if (whole) {
        const Part v = *reinterpret_cast<const Part *>(src);
#pragma unroll
        for (int j = 0; j < kLen; ++j) acc[j] += v[j];
      } else {
#pragma unroll
        for (int j = 0; j < kLen; ++j)
          if (c + j < s.a.width) acc[j] += src[j];
      }
    }
  };
  if (threadIdx.x == 0) longs = 0;
  __syncthreads();
  const uint32_t p = block * groups + group;
  if (p + 1 < s.pieces) {
    const uint32_t lo = p * s.piece, hi = lo + s.piece, id = s.key[hi - 1];
    if (id < s.rows && s.key[hi] == id && (s.key[lo] != id || lo == 0 || s.key[lo - 1] != id)) {
      uint32_t reach = 1;  // pieces that follow on and begin with the run's id
#pragma unroll
      for (uint32_t j = 2; j <= kShortRun; ++j)
        if (p + j < s.pieces && s.key[(p + j) * s.piece] == id) reach = j;
      if (reach < kShortRun) {
        float acc[kLen] = {};
        if (live) {
          add(acc, p, p, 1, p + reach);
          store_row<T, O>(s, id, c, acc);
        }
      } else if (in == 0) {
        long_run[atomicAdd(&longs, 1u)] = p;  // whose turn is first changes no sum
      }
    }
  }
  __syncthreads();
  // runs of more pieces, a wave each: its groups of lanes side by side
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, side = 64 >> s.log_g;
  for (uint32_t w = wave; w < longs; w += kJoinThreads / 64) {
    const uint32_t first = long_run[w], id = s.key[(first + 1) * s.piece - 1];
    // the last piece that begins with the run's id, between `last` and `end`: 64
    // places in between are looked at at once (60,526 tokens into 30 x 16: the
    // launch 15 us, 19 with 64 pieces after the other)
    uint32_t last = first + kShortRun, end = s.pieces;
    while (end - last > 1) {
      const uint32_t step = (end - last - 1 + 63) / 64, q = last + (lane + 1) * step;
      const uint32_t on = __popcll(__ballot(q < end && s.key[q * s.piece] == id));
      end = min(end, last + (on + 1) * step);
      last += on * step;
    }
    const bool wide = last - first >= (uint32_t)(kWaveRun * side);
    if (lane == 0) long_last[w] = wide ? last : 0;
    if (wide) continue;
    float acc[kLen] = {};
    if (live) add(acc, first, first + (lane >> s.log_g), side, last);
    for (int d = 1 << s.log_g; d < 64; d <<= 1) {
#pragma unroll
      for (int j = 0; j < kLen; ++j) acc[j] += __shfl_xor(acc[j], d);
    }
    if (lane >> s.log_g == 0 && live) store_row<T, O>(s, id, c, acc);
  }
  __syncthreads();
  // the longest, by the whole workgroup
  for (uint32_t w = 0; w < longs; ++w) {
    const uint32_t first = long_run[w], last = long_last[w];
    if (last == 0) continue;
    const uint32_t id = s.key[(first + 1) * s.piece - 1];
    float acc[kLen] = {};
    if (live) add(acc, first, first + group, groups, last);
    for (int half = groups / 2; half > 0; half >>= 1) {
      __syncthreads();
      if (group >= half && group < 2 * half) {
#pragma unroll
        for (int j = 0; j < kLen; ++j) sums[(threadIdx.x - (half << s.log_g)) * kLen + j] = acc[j];
      }
      __syncthreads();
      if (group < half) {
#pragma unroll
        for (int j = 0; j < kLen; ++j) acc[j] += sums[threadIdx.x * kLen + j];
      }
    }
    if (group == 0 && live) store_row<T, O>(s, id, c, acc);
  }
}

// ---- tables of few numbers -------------------------------------------------------

struct FewArgs {
  EmbedGradArgs a;
  float *part;       // [rows * width][waves]
  uint32_t cells, waves;
  int64_t per;       // tokens of a wave
};

// One wave a workgroup.  Number (v, d) of lane i's own table is
// mine[(v * width + d) * 64 + i]: no two lanes share a bank or a number.
// WIDTH: the row's width, or kFewWidth for all but the narrowest.
template <typename T, int WIDTH>
__global__ __launch_bounds__(64) void few_kernel(FewArgs f) {
  constexpr int kAhead = 16 / WIDTH;
  extern __shared__ float mine[];
  const int lane = threadIdx.x, width = WIDTH == 1 ? 1 : (int)f.a.width;
  const T *dout = static_cast<const T *>(f.a.dout);
  const int64_t lo = blockIdx.x * f.per, hi = min(f.a.n, lo + f.per);
  uint32_t id[kAhead];
  T v[kAhead][WIDTH];
  auto fetch = [&](int64_t i0) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int64_t i = i0 + j * 64;
      id[j] = i < hi ? (uint32_t)f.a.ids[i] : 0xFFFFFFFFu;
#pragma unroll
      for (int d = 0; d < WIDTH; ++d)
        v[j][d] = i < hi && d < width ? dout[i * f.a.dout_ld + d] : (T)0.0f;
    }
  };
  fetch(lo + lane);
  for (uint32_t c = lane; c < f.cells * 64; c += 64) mine[c] = 0.0f;
  for (int64_t i0 = lo + lane; i0 - lane < hi; i0 += 64 * kAhead) {
    uint32_t now[kAhead];
    T add[kAhead][WIDTH];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      now[j] = id[j];
#pragma unroll
      for (int d = 0; d < WIDTH; ++d) add[j][d] = v[j][d];
    }
    fetch(i0 + 64 * kAhead);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (now[j] >= (uint32_t)f.a.table_rows) continue;
      float *at = mine + (size_t)now[j] * width * 64 + lane;
#pragma unroll
      for (int d = 0; d < WIDTH; ++d)
        if (d < width) at[d * 64] += (float)add[j][d];
    }
  }
  __syncthreads();
  for (uint32_t c = lane; c < f.cells; c += 64) {
    float sum = 0.0f;
#pragma unroll 16
    for (int j = 0; j < 64; ++j) sum += mine[c * 64 + ((lane + j) & 63)];
    f.part[(size_t)c * f.waves + blockIdx.x] = sum;
  }
}

// The waves' sums of one number, added by a workgroup.
template <typename O>
__global__ __launch_bounds__(kThreads) void few_join(FewArgs f) {
  __shared__ float sums[kThreads];
  float sum = 0.0f;
  for (uint32_t w = threadIdx.x; w < f.waves; w += kThreads)
    sum += f.part[(size_t)blockIdx.x * f.waves + w];
  sums[threadIdx.x] = sum;
  __syncthreads();
  for (int d = kThreads / 2; d > 0; d >>= 1) {
    if ((int)threadIdx.x < d) sums[threadIdx.x] += sums[threadIdx.x + d];
    __syncthreads();
  }
  if (threadIdx.x == 0)
    static_cast<O *>(f.a.grad)[blockIdx.x / f.a.width * f.a.grad_ld + blockIdx.x % f.a.width] =
        narrow<O>(sums[0] * f.a.scale);
}

// ---- plans -------------------------------------------------------------------

// Lanes that share a row: enough 16-byte vectors for its width, at most `most`.
int log_group(int64_t width, int len, int most) {
  int g = 0;
  while (g < most && ((int64_t)len << g) < width) ++g;
  return g;
}

struct GradPlan {
  bool few;
  uint32_t waves;              // few: waves, one a workgroup
  int bits, passes, big;       // of a digit; sort passes; 8 keys a lane of a sort's step, else 2
  uint32_t tiles, subs, piece, pieces;
  size_t keys, hist, part;     // byte offsets of the second key buffer, counts, parts
  size_t bytes;
};

constexpr int kBigKeys = 16 * 8 * 64, kSmallKeys = 16 * 2 * 64;  // keys of a sort workgroup's step

GradPlan grad_plan(int64_t n, int64_t rows, int64_t width, int len) {
  GradPlan p{};
  auto align = [](size_t b) { return (b + 255) & ~(size_t)255; };
  p.few = n > 0 && width >= 1 && width <= kFewWidth && rows >= 1 && rows * width <= kFewCells;
  if (p.few) {
    // as many waves as 256 CUs' LDS holds tables, none for fewer than 512 tokens
    const int64_t per_cu = std::min<int64_t>(8, (160 * 1024) / (rows * width * 256));
    p.waves = (uint32_t)std::min<int64_t>(256 * per_cu, (n + 511) / 512);
    p.bytes = align((size_t)(rows * width) * p.waves * 4);
    return p;
  }
  int bits = 1;
  while (((int64_t)1 << bits) <= rows) ++bits;  // keys 0 .. rows
  p.passes = (bits + kMaxBits - 1) / kMaxBits;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.big = n > (int64_t)kMaxTiles * kSmallKeys;
  const int64_t step = p.big ? kBigKeys : kSmallKeys;
  p.subs = (uint32_t)std::max<int64_t>(1, (n + step * kMaxTiles - 1) / (step * kMaxTiles));
  p.tiles = (uint32_t)((n + step * p.subs - 1) / (step * p.subs));
  // Long pieces leave few parts, short ones more lanes at work: as long as
  // 32,768 lanes (two waves a CU) have one each.
  const int64_t vecs = (width + len - 1) / len;
  p.piece = (uint32_t)std::min<int64_t>(32, std::max<int64_t>(8, n * vecs / 32768 / 8 * 8));
  p.pieces = (uint32_t)((n + p.piece - 1) / p.piece);
  const size_t list = align((size_t)n * 4);
  p.keys = 2 * list;
  p.hist = 4 * list;
  p.part = p.hist + align(((size_t)p.tiles << p.bits) * 4);
  p.bytes = p.part + align((size_t)p.pieces * 2 * (size_t)width * 4);
  return p;
}

template <typename T, typename O>
hipError_t launch_few(const EmbedGradArgs &a, const GradPlan &g, void *ws, hipStream_t st) {
  FewArgs f{};
  f.a = a;
  f.part = static_cast<float *>(ws);
  f.cells = (uint32_t)(a.table_rows * a.width);
  f.waves = g.waves;
  f.per = ((a.n + g.waves - 1) / g.waves + 63) / 64 * 64;
  const size_t lds = (size_t)f.cells * 256;
  auto *kernel = a.width == 1 ? few_kernel<T, 1> : few_kernel<T, kFewWidth>;
  const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(kernel), lds);
  if (e != hipSuccess) return e;
  kernel<<<f.waves, 64, lds, st>>>(f);
  few_join<O><<<f.cells, kThreads, 0, st>>>(f);
  return hipGetLastError();
}

template <int WAVES, int ROUNDS>
void launch_pass(const SortPass &p, const Clear &count, const Clear &scatter, hipStream_t st) {
  sort_count<WAVES, ROUNDS><<<p.tiles + count.blocks, WAVES * 64, 0, st>>>(p, count);
  sort_scatter<WAVES, ROUNDS><<<p.tiles + scatter.blocks, WAVES * 64, 0, st>>>(p, scatter);
}

// Bytes that a sort launch clears beside its own work: at 6.5 TB/s about the
// time that the launch takes anyway.
constexpr int64_t kClearBytes = (int64_t)40 << 20;

template <typename T, typename O>
hipError_t launch_grad(const EmbedGradArgs &a, void *ws, hipStream_t st) {
  const GradPlan g = grad_plan(a.n, a.table_rows, a.width, Vec<T>::kLen);
  if (g.few) return launch_few<T, O>(a, g, ws, st);
  char *base = static_cast<char *>(ws);
  uint32_t *list[2] = {reinterpret_cast<uint32_t *>(base),
                       reinterpret_cast<uint32_t *>(base + g.keys)};
  const size_t half = g.keys / 2 / 4;  // positions follow the keys
  int at = 0;
  const int64_t row_bytes = a.width * (int64_t)sizeof(O);
  const int launches = a.n == 0 ? 0 : a.n <= kOneSort ? 1 : 2 * g.passes;
  const int64_t cleared = std::min(a.table_rows, launches * kClearBytes / row_bytes);
  // the part of launch i, after `own` workgroups of the sort
  auto clear = [&](int i, uint32_t own) {
    Clear f = {static_cast<uint16_t *>(a.grad), cleared * i / launches, cleared * (i + 1) / launches,
               row_bytes / 2, a.grad_ld * (int64_t)sizeof(O) / 2, own, 0};
    const int64_t vecs = (f.row1 - f.row0) * (f.width / 8 + 1);
    if (f.row1 > f.row0) f.blocks = (uint32_t)std::min<int64_t>((vecs + 1023) / 1024, 512);
    return f;
  };
  if (a.n > 0 && a.n <= kOneSort) {
    const OneSort p = {a.ids, list[0], list[0] + half, (uint32_t)a.n, (uint32_t)a.table_rows,
                       g.passes, g.bits};
    auto *kernel = a.table_rows < (1 << (32 - kOneBits)) ? sort_one<true> : sort_one<false>;
    const hipError_t e =
        ensure_dynamic_lds(reinterpret_cast<const void *>(kernel), kOneSort * sizeof(uint32_t));
    if (e != hipSuccess) return e;
    const Clear f = clear(0, 1);
    kernel<<<1 + f.blocks, 1024, (size_t)((a.n + 1023) / 1024) * 4096, st>>>(p, f);
  }
  for (int pass = 0; pass < g.passes && a.n > kOneSort; ++pass) {
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
    p.subs = g.subs;
    p.shift = pass * g.bits;
    p.bits = g.bits;
    const Clear f[2] = {clear(2 * pass, p.tiles), clear(2 * pass + 1, p.tiles)};
    if (g.big) launch_pass<16, 8>(p, f[0], f[1], st);
    else launch_pass<16, 2>(p, f[0], f[1], st);
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
  s.log_g = log_group(a.width, Vec<T>::kLen, 6);
  const int64_t slab = (int64_t)Vec<T>::kLen << s.log_g;
  s.slabs = (uint32_t)((a.width + slab - 1) / slab);
  const uint32_t per = kThreads >> s.log_g;
  s.sum_blocks = (s.pieces + per - 1) / per * s.slabs;
  // Half of the other rows wait for the joins: both launches then keep writing.
  s.cleared = (uint32_t)cleared;
  s.split = s.pieces > 1 ? s.cleared + (s.rows - s.cleared) / 2 : s.rows;
  const uint32_t clear1 = (s.split - s.cleared + kThreads - 1) / kThreads;
  const uint32_t clear2 = (s.rows - s.split + kJoinThreads - 1) / kJoinThreads;
  const size_t lds = (size_t)per * (g.piece + 1) * 8;
  const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(sum_kernel<T, O>), lds);
  if (e != hipSuccess) return e;
  if (s.sum_blocks + clear1 > 0)
    sum_kernel<T, O><<<s.sum_blocks + clear1, kThreads, lds, st>>>(s);
  if (s.pieces > 1) {
    const uint32_t join = kJoinThreads >> s.log_g;
    s.join_blocks = (s.pieces + join - 1) / join * s.slabs;
    join_kernel<T, O><<<s.join_blocks + clear2, kJoinThreads, 0, st>>>(s);
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
  // the type is not known here: vectors of 16-bit elements make the shorter pieces
  return std::max<size_t>(256, std::max(grad_plan(n, table_rows, width, 4).bytes,
                                        grad_plan(n, table_rows, width, 8).bytes));
}

hipError_t launch_embed_grad(int dtype, int grad_dtype, const EmbedGradArgs &a, void *ws,
                             hipStream_t st) {
  if (a.table_rows == 0 || a.width == 0) return hipSuccess;
  const bool wide = grad_dtype == ML2_F32;
  switch (dtype) {
    case ML2_F32: return launch_grad<float, float>(a, ws, st);
    case ML2_BF16:
      return wide ? launch_grad<__bf16, float>(a, ws, st)
                  : launch_grad<__bf16, __bf16>(a, ws, st);
    default:
      return wide ? launch_grad<_Float16, float>(a, ws, st)
                  : launch_grad<_Float16, _Float16>(a, ws, st);
  }
}

}  // namespace ml2
