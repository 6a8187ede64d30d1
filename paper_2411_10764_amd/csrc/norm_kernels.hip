// Layer norm of rows, and the gradients of the rows, the weight and the bias.
//
//   out_i = (x_i - m) rstd w_i + b_i,   rstd = 1 / sqrt(V + eps)
//   dx_i  = rstd (g_i - avg g - xhat_i avg(g xhat)),   g = dout w
//   dw_i  = sum over rows of dout_i xhat_i,   db_i = sum over rows of dout_i
//
// Bytes bound all of it: a row is read once, into registers, and what is
// computed of it is written once.
//
// Mean and variance: with a first mean m0 of the row, the sums of d = x - m0 and
// of d^2 are taken together; delta = avg d is what rounding took from m0, and
// V = avg d^2 - delta^2, m = m0 + delta (the corrected two-pass algorithm of Chan,
// Golub and LeVeque, 1983).  Rows far from 0, and rows of one value, keep all
// their digits that way.  The gradient takes the stored mean as m0 and finds
// delta beside its own two sums.
//
// Measured: 32,768 x 1,024 bf16 27 us (134 MB, 4.9 TB/s; a copy reaches 4.65 to
// 4.7), 8,192 x 4,096 float32 44 us (6.1 TB/s), 515 x 50,021 fp16 39 us; gradients of
// 32,768 x 1,024 bf16 41 to 44 us (201 MB), of 8,192 x 20,000 bf16 208 us (4.7 TB/s),
// of 260 x 50,021 float32 57 us, of 96 x 128 float32 7 us.
#include <algorithm>
#include <type_traits>

#include "train.h"

namespace ml2 {
namespace {

constexpr int kWaveBlock = 256;   // threads where a row has at most a wave
constexpr int kMaxBlock = 1024;

// A vector of a row, kLen columns from c on.  The one that the row ends in is
// loaded kLen columns before the end instead, so every load is a whole one; its
// first columns, and all of a vector behind the row, are another vector's and count
// for nothing (`skip` of them).
//
// Offsets are unsigned and in bytes, so that they are one register beside a row's
// address, which all lanes share.
template <typename A, typename T>
__device__ __forceinline__ A *at_column(T *row, int col) {
  typedef typename std::conditional<std::is_const<T>::value, const char, char>::type Byte;
  return reinterpret_cast<A *>(reinterpret_cast<Byte *>(row) + (uint32_t)col * (uint32_t)sizeof(T));
}

// What is known of a call's weight and bias where its kernel is chosen: that both
// are there, in float32 or in the rows' type.  Wide rows load them again for every
// row, and loads behind a branch would wait for one another.
enum Params { kAny, kFloat, kSame };

// How rows end: anywhere, before the first vector does (its columns are loaded one by
// one), or with the last lane's last vector.
enum Ends { kAnywhere, kShort, kWhole };

template <typename T, Ends ENDS>
struct Piece {
  static constexpr bool SHORT = ENDS == kShort;
  static constexpr int kLen = Vec<T>::kLen;
  int col, skip;
  __device__ __forceinline__ Piece(int c, int width) {
    col = SHORT ? 0 : ENDS == kWhole ? c : min(c, width - kLen);
    skip = SHORT ? (c == 0 ? 0 : kLen) : c - col;
  }
  __device__ __forceinline__ bool whole() const { return !SHORT && skip == 0; }
  __device__ __forceinline__ bool any() const { return skip < kLen; }
  __device__ __forceinline__ bool has(int j, int width) const {
    return SHORT ? skip == 0 && j < width : j >= skip;
  }
  __device__ __forceinline__ typename Vec<T>::type load(const T *row, int width) const {
    if (!SHORT) return *at_column<const typename Vec<T>::type>(row, col);
    typename Vec<T>::type v;
#pragma unroll
    for (int j = 0; j < kLen; ++j) v[j] = has(j, width) ? row[j] : (T)0.0f;
    return v;
  }
  __device__ __forceinline__ void store(T *row, int width, const float *x) const {
    if (whole()) {
      typename Vec<T>::type v;
#pragma unroll
      for (int j = 0; j < kLen; ++j) v[j] = narrow<T>(x[j]);
      *at_column<typename Vec<T>::type>(row, col) = v;
    } else if (any()) {
#pragma unroll
      for (int j = 0; j < kLen; ++j)
        if (has(j, width)) *at_column<T>(row, col + j) = narrow<T>(x[j]);
    }
  }
  // weight or bias, or `none` where there is none
  __device__ __forceinline__ void param(const void *p, int f32, float none, int width,
                                        float *x) const {
    typedef float F __attribute__((ext_vector_type(4), aligned(4)));
    if (!p || SHORT) {
#pragma unroll
      for (int j = 0; j < kLen; ++j)
        x[j] = !p || !has(j, width) ? none
               : f32                ? static_cast<const float *>(p)[j]
                                    : (float)static_cast<const T *>(p)[j];
    } else if (f32) {
#pragma unroll
      for (int j = 0; j < kLen; j += 4) {
        const F v = *at_column<const F>(static_cast<const float *>(p), col + j);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[j + i] = v[i];
      }
    } else {
      const auto v = *at_column<const typename Vec<T>::type>(static_cast<const T *>(p), col);
#pragma unroll
      for (int j = 0; j < kLen; ++j) x[j] = (float)v[j];
    }
  }
};

// A vector whose elements are widened again where they are used again: the
// compiler would keep them in float32, in twice the registers.
template <typename V>
__device__ __forceinline__ V anew(V v) {
  typedef int Bits __attribute__((ext_vector_type(4)));
  Bits b = __builtin_bit_cast(Bits, v);
  asm("" : "+v"(b));
  return __builtin_bit_cast(V, b);
}

// The same number, of which the compiler does not know it: where a vector lies and
// which of its columns count is worked out anew then.  Kept, all of that would fill
// the registers.
__device__ __forceinline__ int anew(int v) {
  asm volatile("" : "+s"(v));
  return v;
}

// N sums over the workgroup's waves, in every thread.
template <int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float (*lds)[N]) {
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  group_sums(v, 6);
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) lds[wave][i] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lds[0][i];
  for (int w = 1; w < waves; ++w) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += lds[w][i];
  }
}

// ---- forward --------------------------------------------------------------------

// E columns a lane, as they came, so that a wide row's fit the registers, and those
// of two rows where they are at most 128 bytes a lane (hence the bound of 8 waves a
// SIMD: a compute unit loads one row while it writes another; with 64 columns and
// parameters loaded ahead one to three registers do not fit and lie in scratch).  WAVE:
// 2^log_g lanes share a row, else the workgroup does.  Vector k of a lane lies at
// column (k * lanes + lane) * kLen.
template <typename T, int E, bool WAVE, Ends ENDS, Params HOW>
__global__ __launch_bounds__(WAVE ? kWaveBlock : kMaxBlock,
                             E >= 32 && E * sizeof(T) <= 128 ? 8 : 1) void norm_kernel(
    NormArgs a, int log_g, float over_width) {
  constexpr int kLen = Vec<T>::kLen, kVecs = E / kLen;
  constexpr bool kKeep = E <= 16;  // the parameters stay in registers
  typedef Piece<T, ENDS> Part;
  __shared__ float first[kMaxBlock / 64][1], second[kMaxBlock / 64][2];
  const int lanes = WAVE ? 1 << log_g : (int)blockDim.x, width = (int)a.width;
  const int lane = WAVE ? threadIdx.x & (lanes - 1) : threadIdx.x;
  const int64_t per = WAVE ? kWaveBlock >> log_g : 1;
  const int64_t group = WAVE ? threadIdx.x >> log_g : 0;
  float w[kKeep ? E : kLen], b[kKeep ? E : kLen], y[kLen];
  // The parameters of kStep columns at a time, in their type, the next ones loaded
  // before these are used.
  typedef typename std::conditional<HOW == kSame, T, float>::type Param;
  constexpr int kStep = HOW == kSame ? kLen : 4, kSteps = E / kStep;
  typedef Param ParamVec __attribute__((ext_vector_type(kStep), aligned(sizeof(Param))));
  ParamVec w1, b1;
  const auto fetch = [&](int q) {
    const Part at((q * kStep / kLen * lanes + lane) * kLen, anew(width));
    const int c = at.col + q * kStep % kLen;
    w1 = *at_column<const ParamVec>(static_cast<const Param *>(a.weight), c);
    b1 = *at_column<const ParamVec>(static_cast<const Param *>(a.bias), c);
  };
  if (kKeep) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const Part at((k * lanes + lane) * kLen, width);
      at.param(a.weight, a.param_f32, 1.0f, width, w + k * kLen);
      at.param(a.bias, a.param_f32, 0.0f, width, b + k * kLen);
    }
  }
  // A wave's next row is loaded while this one is worked on.  (Workgroups that share
  // a row do not: the registers would cost them more waves than it gains, 1,024 x
  // 16,384 fp16 17 and 23 us.)
  typename Vec<T>::type x1[kVecs];
  const auto load = [&](int64_t row) {
    const T *src = static_cast<const T *>(a.x) + min(row, a.rows - 1) * a.ld;
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
      x1[k] = Part((k * lanes + lane) * kLen, anew(width)).load(src, width);
  };
  const int64_t step = (int64_t)gridDim.x * per;
  if (WAVE) load((int64_t)blockIdx.x * per + group);
  for (int64_t row0 = (int64_t)blockIdx.x * per; row0 < a.rows; row0 += step) {
    const int64_t row = row0 + group;
    if (!WAVE) load(row);
    typename Vec<T>::type x[kVecs];
#pragma unroll
    for (int k = 0; k < kVecs; ++k) x[k] = x1[k];
    if (WAVE && row0 + step < a.rows) load(row + step);
    float s[1] = {0.0f};
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const Part at((k * lanes + lane) * kLen, anew(width));
      if (at.whole()) {
#pragma unroll
        for (int j = 0; j < kLen; ++j) s[0] += (float)x[k][j];
      } else if (!kKeep || at.any()) {
#pragma unroll
        for (int j = 0; j < kLen; ++j) s[0] += at.has(j, width) ? (float)x[k][j] : 0.0f;
      }
    }
    if (WAVE)
      group_sums(s, E > 8 ? 6 : log_g);  // more than 8 columns a lane: whole waves
    else
      block_sums(s, first);
    const float m0 = s[0] * over_width;
    float t[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      x[k] = anew(x[k]);
      const Part at((k * lanes + lane) * kLen, anew(width));
      if (at.whole()) {
#pragma unroll
        for (int j = 0; j < kLen; ++j) {
          const float d = (float)x[k][j] - m0;
          t[0] += d;
          t[1] = fmaf(d, d, t[1]);
        }
      } else if (!kKeep || at.any()) {
#pragma unroll
        for (int j = 0; j < kLen; ++j) {
          const float d = at.has(j, width) ? (float)x[k][j] - m0 : 0.0f;
          t[0] += d;
          t[1] = fmaf(d, d, t[1]);
        }
      }
    }
    if (HOW != kAny) fetch(0);
    if (WAVE)
      group_sums(t, E > 8 ? 6 : log_g);
    else
      block_sums(t, second);
    const float delta = t[0] * over_width;
    const float raw = fmaf(t[1], over_width, -delta * delta);
    const float var = raw < 0.0f ? 0.0f : raw;  // a NaN stays one
    const float rstd = 1.0f / sqrtf(var + a.eps), shift = -delta * rstd;
    if (row >= a.rows) continue;
    if (lane == 0) {
      if (a.mean) a.mean[row] = m0 + delta;
      if (a.rstd) a.rstd[row] = rstd;
    }
    T *dst = static_cast<T *>(a.out) + row * a.out_ld;
    if constexpr (HOW != kAny) {
#pragma unroll
      for (int q = 0; q < kSteps; ++q) {
        const int k = q * kStep / kLen, j0 = q * kStep % kLen;
        const ParamVec wq = w1, bq = b1;
        if (q + 1 < kSteps) fetch(q + 1);
        const Part at((k * lanes + lane) * kLen, anew(width));
        if (j0 == 0) x[k] = anew(x[k]);
#pragma unroll
        for (int j = 0; j < kStep; ++j)
          y[j0 + j] = fmaf(fmaf((float)x[k][j0 + j] - m0, rstd, shift), (float)wq[j], (float)bq[j]);
        if (j0 + kStep == kLen) at.store(dst, width, y);
      }
    } else {
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        const Part at((k * lanes + lane) * kLen, anew(width));
        x[k] = anew(x[k]);
        if (kKeep && !at.any()) continue;
        if (!kKeep) {
          at.param(a.weight, a.param_f32, 1.0f, width, w);
          at.param(a.bias, a.param_f32, 0.0f, width, b);
        }
#pragma unroll
        for (int j = 0; j < kLen; ++j) {
          const int p = kKeep ? k * kLen + j : j;
          y[j] = fmaf(fmaf((float)x[k][j] - m0, rstd, shift), w[p], b[p]);
        }
        at.store(dst, width, y);
      }
    }
  }
}

// ---- gradients of rows that fit a workgroup's registers ---------------------------

constexpr int kGradBlocks = 256;   // at most: each leaves a part of the parameters' sums
// Widest rows that stay in a workgroup's registers, of 32-bit and of 16-bit columns: 24
// of those a lane fill 126 registers with their sums (32 would spill 34).  2,048 x
// 24,576 bf16 82 us, read twice 114; 2,048 x 16,384 float32 95, 16,385 136.
constexpr int kGradWidth = 16 * kMaxBlock, kGradWidth16 = 24 * kMaxBlock;

__device__ __forceinline__ void store_as(int dtype, void *p, int64_t i, float v) {
  if (dtype == ML2_F32)
    static_cast<float *>(p)[i] = v;
  else if (dtype == ML2_BF16)
    static_cast<__bf16 *>(p)[i] = narrow<__bf16>(v);
  else
    static_cast<_Float16 *>(p)[i] = narrow<_Float16>(v);
}

struct GradShape {
  int lanes, log_g;   // of a row; log_g: where they are at most a wave
  int per, threads;   // rows at a time, threads of a workgroup
  int blocks;
  bool direct;        // one workgroup: it writes the parameters' sums itself
};

// Sums over a wave's groups of 2^log_g lanes, in the lanes of the first.
template <int N>
__device__ __forceinline__ void fold_groups(float (&v)[N], int log_g) {
  const auto each = [&](auto fn) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = fn(v[i]);
  };
  const auto add = [](float p, float r) { return p + r; };
  if (log_g <= 3) each([](float x) { return x + lane_swap<0x128>(x); });  // row_ror 8
  if (log_g <= 2) each([](float x) { return x + lane_swap<0x124>(x); });  // row_ror 4
  if (log_g <= 1) each([](float x) { return x + lane_swap<0x122>(x); });  // row_ror 2
  if (log_g <= 0) each([](float x) { return x + lane_swap<0x121>(x); });  // row_ror 1
  if (log_g <= 4) each([&](float x) { return join_rows(x, add); });
  each([&](float x) { return join_halves(x, add); });
}

// Sums of a lane group over all rows it takes go to part[block][0] (weight) and
// [1] (bias), float32 [width] each.
template <typename T, int E, Ends ENDS>
__global__ __launch_bounds__(kMaxBlock) void grad_kernel(NormGradArgs a, GradShape g,
                                                         float over_width, float *part) {
  constexpr int kLen = Vec<T>::kLen, kVecs = E / kLen;
  typedef Piece<T, ENDS> Part;
  // The row's sums and the weight, each lane's four by four, then the parts of the
  // gradients of weight and bias (a row as wide as a workgroup has but one part).
  constexpr bool kJoins = E <= 16;
  constexpr int kSpan = kMaxBlock * E, kWeight = kJoins ? kSpan : 128;
  __shared__ float lds[kWeight + kSpan];
  typedef float F4 __attribute__((ext_vector_type(4)));
  float (*sums)[kMaxBlock / 64][3] = reinterpret_cast<float (*)[kMaxBlock / 64][3]>(lds);
  F4 *weight = reinterpret_cast<F4 *>(lds + kWeight);
  const int lanes = g.lanes, group = (int)threadIdx.x / lanes, width = (int)a.width;
  const int lane = (int)threadIdx.x - group * lanes;
  const bool wide = lanes > 64;
  typename Vec<T>::type x1[kVecs], d1[kVecs];
  float mean1, rstd1, dw[E], db[E];
  const auto load = [&](int64_t row) {
    row = min(row, a.rows - 1);
    const T *xs = static_cast<const T *>(a.x) + row * a.ld;
    const T *ds = static_cast<const T *>(a.dout) + row * a.dout_ld;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const Part at((k * lanes + lane) * kLen, anew(width));
      x1[k] = at.load(xs, width);
      d1[k] = at.load(ds, width);
    }
    mean1 = a.mean[row];
    rstd1 = a.rstd[row];
  };
  // The next row is loaded while this one is worked on, where the registers hold both.
  constexpr bool kAhead = E * sizeof(T) <= 32;
  const int64_t step = (int64_t)gridDim.x * g.per;
  if (kAhead) load((int64_t)blockIdx.x * g.per + group);
  if (group == 0) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      float w[kLen];
      Part((k * lanes + lane) * kLen, width).param(a.weight, a.param_f32, 1.0f, width, w);
#pragma unroll
      for (int j = 0; j < kLen; j += 4)
        weight[(k * kLen + j) / 4 * lanes + lane] = F4{w[j], w[j + 1], w[j + 2], w[j + 3]};
    }
  }
#pragma unroll
  for (int i = 0; i < E; ++i) dw[i] = db[i] = 0.0f;
  __syncthreads();
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * g.per; row0 < a.rows; row0 += step, turn ^= 1) {
    if (!kAhead) load(row0 + group);
    typename Vec<T>::type x[kVecs], d[kVecs];
    const float mean = mean1, rstd = rstd1;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      x[k] = x1[k];
      d[k] = d1[k];
    }
    if (kAhead && row0 + step < a.rows) load(row0 + step + group);
    float s[3] = {0.0f, 0.0f, 0.0f};  // of x - mean, g, g (x - mean)
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const Part at((k * lanes + lane) * kLen, anew(width));
      if (!kJoins) __builtin_amdgcn_sched_barrier(0);
      float w[kLen];
#pragma unroll
      for (int j = 0; j < kLen; j += 4) {
        const F4 v = weight[(k * kLen + j) / 4 * lanes + lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[j + i] = v[i];
      }
      if (at.whole()) {
#pragma unroll
        for (int j = 0; j < kLen; ++j) {
          const float xj = (float)x[k][j] - mean, gj = (float)d[k][j] * w[j];
          s[0] += xj;
          s[1] += gj;
          s[2] = fmaf(gj, xj, s[2]);
        }
      } else if (at.any()) {
#pragma unroll
        for (int j = 0; j < kLen; ++j) {
          const bool has = at.has(j, width);
          const float xj = has ? (float)x[k][j] - mean : 0.0f;
          const float gj = has ? (float)d[k][j] * w[j] : 0.0f;
          s[0] += xj;
          s[1] += gj;
          s[2] = fmaf(gj, xj, s[2]);
        }
      }
    }
    group_sums(s, E > 8 || wide ? 6 : g.log_g);  // more than 8 columns a lane: whole waves
    if (wide) {
      // One barrier a row: the waves that still read the last row's sums have the
      // other half of the buffer.
      const int wave = (int)threadIdx.x >> 6, waves = lanes >> 6;
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < 3; ++i) sums[turn][wave][i] = s[i];
      }
      __syncthreads();
      const int w0 = group * waves;
#pragma unroll
      for (int i = 0; i < 3; ++i) s[i] = sums[turn][w0][i];
      for (int v = 1; v < waves; ++v) {
#pragma unroll
        for (int i = 0; i < 3; ++i) s[i] += sums[turn][w0 + v][i];
      }
    }
    const float delta = s[0] * over_width, g_avg = s[1] * over_width;
    const float along = (s[2] - delta * s[1]) * over_width * rstd;  // avg(g xhat)
    const float shift = -delta * rstd;
    const int64_t row = row0 + group;
    if (row < a.rows) {
      T *dst = a.dx ? static_cast<T *>(a.dx) + row * a.dx_ld : nullptr;
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        x[k] = anew(x[k]);
        d[k] = anew(d[k]);
        const Part at((k * lanes + lane) * kLen, anew(width));
        if (!at.any()) continue;
        float y[kLen];
#pragma unroll
        for (int j = 0; j < kLen; ++j) {
          const int i = k * kLen + j;
          const float w = weight[i / 4 * lanes + lane][j & 3];
          const float dj = (float)d[k][j], xhat = fmaf((float)x[k][j] - mean, rstd, shift);
          dw[i] = fmaf(dj, xhat, dw[i]);
          db[i] += dj;
          y[j] = rstd * fmaf(-along, xhat, fmaf(dj, w, -g_avg));
        }
        if (dst) at.store(dst, width, y);
        if (!kJoins) __builtin_amdgcn_sched_barrier(0);  // one vector at a time
      }
    }
  }
  if (!part) return;
  // The groups of a wave, then the waves: lane i of a wave holds the columns of
  // lane i % lanes.
  if (E == 8 && !wide && g.log_g < 6) {
    fold_groups(dw, g.log_g);
    fold_groups(db, g.log_g);
  }
  const int parts = wide ? g.per : (int)blockDim.x >> 6;
  float *to = part + (int64_t)blockIdx.x * 2 * width;
  const int own = wide ? group : (int)threadIdx.x >> 6;
  typedef float U4 __attribute__((ext_vector_type(4), aligned(4)));
  // Four sums of a piece, from its column j on.
  const auto put = [&](const Part &at, int j, F4 v, float *row) {
    float *p = row + at.col + j;
    if (at.whole()) {
      *reinterpret_cast<U4 *>(p) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (at.has(j + i, width)) p[i] = v[i];
    }
  };
  const auto four = [](const float *v) { return F4{v[0], v[1], v[2], v[3]}; };
  if (!kJoins) {
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const Part at((i / kLen * lanes + lane) * kLen, width);
      put(at, i % kLen, four(dw + i), to);
      put(at, i % kLen, four(db + i), to + width);
    }
    return;
  }
  // A part lies in LDS as the weight does, a lane's vectors `lanes` apart: stored by
  // columns, 32 bytes from lane to lane, 16 parts of 771 took 3.0 us.
  const int vecs = E / 4 * lanes;  // of a part
  F4 *joined = reinterpret_cast<F4 *>(lds);
  __syncthreads();
  if (wide || (int)(threadIdx.x & 63) < lanes) {  // at most kSpan / 4 of all parts
    F4 *mine = joined + own * vecs + lane;
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      mine[i / 4 * lanes] = four(dw + i);
      mine[i / 4 * lanes + kSpan / 4] = four(db + i);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * vecs; i += blockDim.x) {
    const int q = i >= vecs, slot = q ? i - vecs : i, nth = slot / lanes;
    const F4 *from = joined + q * (kSpan / 4) + slot;
    F4 v = from[0];
#pragma unroll 8
    for (int p = 1; p < parts; ++p) v += from[p * vecs];
    const Part at((nth * 4 / kLen * lanes + slot - nth * lanes) * kLen, width);
    const int j = nth * 4 % kLen;
    if (!g.direct) {
      put(at, j, v, to + q * width);
    } else if (void *out = q ? a.dbias : a.dweight) {
#pragma unroll
      for (int n = 0; n < 4; ++n)
        if (at.has(j + n, width)) store_as(a.grad_dtype, out, at.col + j + n, v[n]);
    }
  }
}

// ---- gradients of wider rows -------------------------------------------------------

constexpr int kStatThreads = 256, kStatVecs = 4;

// A wave a workgroup, with two vectors of a row a lane: 2,048 x 30,000 float32 234 us, of
// four waves 253, of one wave with four vectors 235; 512 x 65,536 bf16 79, 85 (and
// with one vector 79), 79.
template <typename T>
struct Wide {
  static constexpr int kThreads = 64, kVecs = 2;
  static constexpr int64_t kSlab = (int64_t)kThreads * kVecs * Vec<T>::kLen;
};

// Row sums of x - mean, g and g (x - mean) over a piece of kStatVecs vectors a
// thread: stat[row][piece][3].
template <typename T>
__global__ __launch_bounds__(kStatThreads) void stat_kernel(NormGradArgs a, int64_t pieces,
                                                            float *stat) {
  constexpr int kLen = Vec<T>::kLen;
  typedef Piece<T, kAnywhere> Part;
  __shared__ float lds[2][kStatThreads / 64][3];
  const int width = (int)a.width;
  int turn = 0;
  for (int64_t item = blockIdx.x; item < a.rows * pieces; item += gridDim.x, turn ^= 1) {
    const int64_t row = item / pieces, piece = item - row * pieces;
    const float mean = a.mean[row];
    const T *xs = static_cast<const T *>(a.x) + row * a.ld;
    const T *ds = static_cast<const T *>(a.dout) + row * a.dout_ld;
    typename Vec<T>::type x[kStatVecs], d[kStatVecs];
    const int c0 = ((int)piece * kStatVecs * kStatThreads + (int)threadIdx.x) * kLen;
#pragma unroll
    for (int k = 0; k < kStatVecs; ++k) {
      const Part at(c0 + k * kStatThreads * kLen, width);
      x[k] = at.load(xs, width);
      d[k] = at.load(ds, width);
    }
    float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < kStatVecs; ++k) {
      const Part at(c0 + k * kStatThreads * kLen, width);
      float w[kLen];
      at.param(a.weight, a.param_f32, 1.0f, width, w);
#pragma unroll
      for (int j = 0; j < kLen; ++j) {
        const bool has = at.has(j, width);
        const float v = has ? (float)x[k][j] - mean : 0.0f, g = has ? (float)d[k][j] * w[j] : 0.0f;
        s[0] += v;
        s[1] += g;
        s[2] = fmaf(g, v, s[2]);
      }
    }
    block_sums(s, lds[turn]);
    if (threadIdx.x < 3) stat[item * 3 + threadIdx.x] = s[threadIdx.x];
  }
}

// A workgroup takes a slab of columns of `chunk` rows.
template <typename T>
__global__ __launch_bounds__(Wide<T>::kThreads) void wide_kernel(NormGradArgs a, int64_t pieces,
                                                            int64_t chunk, float over_width,
                                                            const float *stat, float *part) {
  constexpr int kLen = Vec<T>::kLen, kVecs = Wide<T>::kVecs, kThreads = Wide<T>::kThreads;
  typedef Piece<T, kAnywhere> Part;
  const int width = (int)a.width;
  const int c0 = ((int)blockIdx.x * kVecs * kThreads + (int)threadIdx.x) * kLen;
  const int64_t r0 = (int64_t)blockIdx.y * chunk, r1 = min(a.rows, r0 + chunk);
  float w[kVecs][kLen], dw[kVecs][kLen], db[kVecs][kLen];
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    Part(c0 + k * kThreads * kLen, width).param(a.weight, a.param_f32, 1.0f, width, w[k]);
#pragma unroll
    for (int j = 0; j < kLen; ++j) dw[k][j] = db[k][j] = 0.0f;
  }
  // The next row is loaded before this one's gradient is written.  A lane takes one
  // piece's sums of the row.
  static_assert(ML2_MAX_WIDTH <= 16 * kStatVecs * kStatThreads * 4, "16 lanes hold the pieces");
  typename Vec<T>::type x[kVecs], d[kVecs], x1[kVecs], d1[kVecs];
  float s1[3], mean1, rstd1;
  const int lane = threadIdx.x & 15;
  const auto load = [&](int64_t row) {
    const T *xs = static_cast<const T *>(a.x) + row * a.ld;
    const T *ds = static_cast<const T *>(a.dout) + row * a.dout_ld;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const Part at(c0 + k * kThreads * kLen, width);
      x1[k] = at.load(xs, width);
      d1[k] = at.load(ds, width);
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
      s1[i] = lane < pieces ? stat[(row * pieces + lane) * 3 + i] : 0.0f;
    mean1 = a.mean[row];
    rstd1 = a.rstd[row];
  };
  load(r0);
  for (int64_t row = r0; row < r1; ++row) {
    float s[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) s[i] = s1[i];
    group_sums(s, 4);
    const float mean = mean1, rstd = rstd1;
    const float delta = s[0] * over_width, g_avg = s[1] * over_width;
    const float along = (s[2] - delta * s[1]) * over_width * rstd;
    const float shift = -delta * rstd;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      x[k] = x1[k];
      d[k] = d1[k];
    }
    if (row + 1 < r1) load(row + 1);
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      float y[kLen];
#pragma unroll
      for (int j = 0; j < kLen; ++j) {
        const float dj = (float)d[k][j], xhat = fmaf((float)x[k][j] - mean, rstd, shift);
        dw[k][j] = fmaf(dj, xhat, dw[k][j]);
        db[k][j] += dj;
        y[j] = rstd * fmaf(-along, xhat, fmaf(dj, w[k][j], -g_avg));
      }
      if (a.dx)
        Part(c0 + k * kThreads * kLen, width)
            .store(static_cast<T *>(a.dx) + row * a.dx_ld, width, y);
    }
  }
  if (!part) return;
  float *to = part + (int64_t)blockIdx.y * 2 * width;
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    const Part at(c0 + k * kThreads * kLen, width);
#pragma unroll
    for (int j = 0; j < kLen; ++j) {
      if (at.has(j, width)) {
        to[at.col + j] = dw[k][j];
        to[width + at.col + j] = db[k][j];
      }
    }
  }
}

// ---- the parameters' sums ------------------------------------------------------------

constexpr int kJoinColumns = 64, kJoinSlices = 16;
constexpr int kJoinAhead = 8;  // parts in flight

// blockIdx.y = 0: weight, 1: bias.  Slices of threads add the parts one after the
// other, then the slices.
__global__ __launch_bounds__(kJoinColumns *kJoinSlices) void join_kernel(NormGradArgs a,
                                                                         const float *part,
                                                                         int parts) {
  __shared__ float lds[kJoinSlices][kJoinColumns];
  void *to = blockIdx.y ? a.dbias : a.dweight;
  if (!to) return;
  const int lane = threadIdx.x & (kJoinColumns - 1), slice = threadIdx.x / kJoinColumns;
  const int64_t c = (int64_t)blockIdx.x * kJoinColumns + lane;
  const int slices = blockDim.x / kJoinColumns, each = (parts + slices - 1) / slices;
  const int p1 = min(parts, (slice + 1) * each);
  float v = 0.0f;
  if (c < a.width) {
    for (int p = slice * each; p < p1; p += kJoinAhead) {
      float x[kJoinAhead];
#pragma unroll
      for (int i = 0; i < kJoinAhead; ++i)
        x[i] = p + i < p1 ? part[((int64_t)(p + i) * 2 + blockIdx.y) * a.width + c] : 0.0f;
#pragma unroll
      for (int i = 0; i < kJoinAhead; ++i) v += x[i];
    }
  }
  lds[slice][lane] = v;
  __syncthreads();
  if (slice == 0 && c < a.width) {
#pragma unroll
    for (int k = 1; k < kJoinSlices; ++k) v += k < slices ? lds[k][lane] : 0.0f;
    store_as(a.grad_dtype, to, c, v);
  }
}

// ---- launches ---------------------------------------------------------------------

int log2_up(int64_t v) {
  int l = 0;
  while (((int64_t)1 << l) < v) ++l;
  return l;
}

// Rows of at most a wave, and of a workgroup.
template <typename T, int E, Ends ENDS>
hipError_t launch_narrow(const NormArgs &a, int cu_count, hipStream_t s) {
  const int log_g = log2_up((a.width + E - 1) / E);
  if (ENDS == kAnywhere && a.width == (int64_t)E << log_g)
    return launch_narrow<T, E, ENDS == kAnywhere ? kWhole : ENDS>(a, cu_count, s);
  const int64_t per = kWaveBlock >> log_g;
  const int64_t grid = std::min<int64_t>((a.rows + per - 1) / per, (int64_t)cu_count * 8);
  norm_kernel<T, E, true, ENDS, kAny><<<(uint32_t)grid, kWaveBlock, 0, s>>>(
      a, log_g, 1.0f / (float)a.width);
  return hipGetLastError();
}

// Workgroups of a row of so many waves: as many as a compute unit holds at eight waves a
// SIMD, which takes a fourth of a workgroup's waves, rounded up.  Float32 rows that fill
// their 16 columns a lane have 65 registers, so seven, and those of 64 columns a lane 99 or
// 116, so four: of these, some workgroups begin when others have ended.  2,048 x 16,384
// float32 takes 54 us, 16,380 columns (63 registers) 48, 15,360 51, 15,350 45; 8,192 x
// 8,192, of eight waves, 100, 8,190 columns 104.  (12,000 x 10,000 bf16, of ten waves: 94
// us, three a compute unit 114; 12,000 x 5,000, of five: 49, six 51; 4,096 x 9,000 31 and
// 29.)  Rows whose parameters do not stay in registers lose nothing with a workgroup of
// their own, and then a row's loads do not wait for the last one's stores: 16,384 x 20,000
// bf16 235, as above 258; 4,096 x 40,000 fp16 128 and 136.  It pays after some rows:
// 2,048 x 32,768 50 and 56, 1,536 x 50,024 70 and 68, 1,024 x 50,021 62 and 55.
int64_t wide_grid(int64_t rows, int waves, bool own, int cu_count) {
  const int64_t fit = (int64_t)cu_count * (waves <= 4 ? 32 / waves : 8 / ((waves + 3) / 4));
  return std::min(rows, own && rows > 3 * fit ? (int64_t)1 << 20 : fit);
}

template <typename T, int E>
hipError_t launch_wide(const NormArgs &a, int cu_count, hipStream_t s) {
  const int threads = (int)((a.width + 64 * E - 1) / (64 * E) * 64);
  const int64_t grid = wide_grid(a.rows, threads / 64, E > 16, cu_count);
  const float over = 1.0f / (float)a.width;
  constexpr bool kSplit = E > 16;
  const auto launch = [&](auto fn) { fn<<<(uint32_t)grid, threads, 0, s>>>(a, 0, over); };
  if (kSplit && a.weight && a.bias && a.param_f32)
    launch(norm_kernel<T, E, false, kAnywhere, kSplit ? kFloat : kAny>);
  else if (kSplit && sizeof(T) == 2 && a.weight && a.bias)
    launch(norm_kernel<T, E, false, kAnywhere, kSplit && sizeof(T) == 2 ? kSame : kAny>);
  else if (!kSplit && a.width == (int64_t)E * threads)
    launch(norm_kernel<T, E, false, kSplit ? kAnywhere : kWhole, kAny>);
  else
    launch(norm_kernel<T, E, false, kAnywhere, kAny>);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_norm(const NormArgs &a, int cu_count, hipStream_t s) {
  if (a.width < Vec<T>::kLen) return launch_narrow<T, 8, kShort>(a, cu_count, s);
  if (a.width <= 64 * 8) return launch_narrow<T, 8, kAnywhere>(a, cu_count, s);
  if (a.width <= 64 * 16) return launch_narrow<T, 16, kAnywhere>(a, cu_count, s);
  if (a.width <= kMaxBlock * 16) return launch_wide<T, 16>(a, cu_count, s);
  if (a.width <= kMaxBlock * 32) return launch_wide<T, 32>(a, cu_count, s);
  return launch_wide<T, 64>(a, cu_count, s);
}

int grad_columns(int64_t width) {
  return width <= 64 * 8 ? 8 : width <= kGradWidth ? 16 : 24;
}

GradShape grad_shape(int64_t rows, int64_t width) {
  GradShape g;
  const int64_t lanes = (width + grad_columns(width) - 1) / grad_columns(width);
  if (lanes <= 64) {
    g.log_g = log2_up(lanes);
    g.lanes = 1 << g.log_g;
    g.threads = kMaxBlock;
  } else {
    g.log_g = 6;
    g.lanes = (int)((lanes + 63) / 64 * 64);
    g.threads = kMaxBlock / g.lanes * g.lanes;
  }
  g.per = g.threads / g.lanes;
  const int64_t turns = (rows + g.per - 1) / g.per;
  // A turn costs less than the launch that joins parts: 256 x 128 float32 (4 turns)
  // 8.8 us, in two launches 10.1; 512 x 128 (8) 12.5 and 10.2; 32 x 1,024 bf16 (2) 8.5
  // and 9.8; 64 x 1,024 (4) 12.3 and 11.3; 8 x 4,096 (2) 10.2 and 11.7; 2 x 8,192 (1) 9.9
  // and 11.6; 4 x 8,192 (2) 12.2 and 11.4; 1 x 10,000 (1) 10.6 and 12.2; 1 x 16,384 14.2
  // and 12.2.
  g.direct = turns <= (grad_columns(width) == 8 ? 4 : g.lanes <= 256 ? 2 : width <= 12 * kMaxBlock);
  // Waves of a SIMD follow one another: where all rows are taken at once, as few of
  // them as make as many workgroups as there may be.  3,001 x 771 fp16 13.2 us, 16 rows a
  // workgroup 13.8; 2,048 12.0 and 12.5.  (Not where that doubles the parts, or where
  // they are wider: 256 x 4,096 bf16 13.7 and 11.6, 700 x 4,096 15.4 and 14.9.)
  if (g.lanes <= 64 && turns >= kGradBlocks / 2 && turns < kGradBlocks) {
    const int64_t few = (rows + kGradBlocks - 1) / kGradBlocks, wave = 64 / g.lanes;
    g.per = (int)((few + wave - 1) / wave * wave);
    g.threads = g.per * g.lanes;
  }
  g.blocks = g.direct ? 1 : (int)std::min<int64_t>((rows + g.per - 1) / g.per, kGradBlocks);
  return g;
}

int64_t stat_pieces(int64_t width) {  // for the smaller vectors
  const int64_t each = (int64_t)kStatVecs * kStatThreads * 4;
  return (width + each - 1) / each;
}

// A chunk has at least so many rows, and the chunks of all slabs so many workgroups at
// most: a chunk costs its part of the parameters' sums, a row of a chunk a turn.  100
// rows of 20,000 bf16 17 us, in chunks of one row 28, of 12 20; 2,048 of 30,000 float32
// 234, with 960 or 2,048 workgroups 246; 512 of 65,536 bf16 79, 82 and 82.
constexpr int64_t kLeastChunk = 4, kWideBlocks = 1280;
// Rows of more than half of kGradWidth, of which a compute unit has one or two, are read
// twice too: 200 of 10,000 bf16 19 us, in registers 21; 300 21 and 23; 400 24 and 23; of
// 16,384 float32 60 rows 15 and 15, 200 19 and 21, 300 25 and 30, 512 35 and 34.  Very
// few are done sooner with fewer launches: 5 of 10,000 14 and 12.
constexpr int64_t kTwiceFrom = 64, kTwiceTo = 320;

// Rows of a chunk.
template <typename T>
int64_t wide_chunk(int64_t rows, int64_t width) {
  const int64_t slabs = (width + Wide<T>::kSlab - 1) / Wide<T>::kSlab;
  const int64_t chunks = std::max<int64_t>(1, std::min<int64_t>(rows / kLeastChunk, kWideBlocks / slabs));
  return (rows + chunks - 1) / chunks;
}

// Whether rows are read twice.
bool grad_twice(int64_t rows, int64_t width, size_t size) {
  return width > (size == 2 ? kGradWidth16 : kGradWidth) ||
         (width > kGradWidth / 2 && rows > kTwiceFrom && rows <= kTwiceTo);
}

template <typename T>
hipError_t launch_grad(const NormGradArgs &a, void *ws, hipStream_t s) {
  const bool sums = a.dweight || a.dbias;
  const float over = 1.0f / (float)a.width;
  float *part = static_cast<float *>(ws);
  int parts = 0;
  bool done = false;
  if (a.rows > 0 && !grad_twice(a.rows, a.width, sizeof(T))) {
    const GradShape g = grad_shape(a.rows, a.width);
    parts = g.blocks;
    done = g.direct;
    const auto launch = [&](auto fn) {
      fn<<<g.blocks, g.threads, 0, s>>>(a, g, over, sums ? part : nullptr);
    };
    const bool whole = a.width == (int64_t)g.lanes * grad_columns(a.width);
    if (a.width < Vec<T>::kLen)
      launch(grad_kernel<T, 8, kShort>);
    else if (grad_columns(a.width) == 8)
      whole ? launch(grad_kernel<T, 8, kWhole>) : launch(grad_kernel<T, 8, kAnywhere>);
    else if (sizeof(T) == 4 || grad_columns(a.width) == 16)
      whole ? launch(grad_kernel<T, 16, kWhole>) : launch(grad_kernel<T, 16, kAnywhere>);
    else
      launch(grad_kernel<T, sizeof(T) == 2 ? 24 : 16, kAnywhere>);
  } else if (a.rows > 0) {
    const int64_t each = (int64_t)kStatVecs * kStatThreads * Vec<T>::kLen;
    const int64_t pieces = (a.width + each - 1) / each;
    float *stat = part;
    part += (size_t)a.rows * stat_pieces(a.width) * 3;
    const int64_t items = std::min<int64_t>(a.rows * pieces, 1 << 20);
    stat_kernel<T><<<(uint32_t)items, kStatThreads, 0, s>>>(a, pieces, stat);
    const int64_t chunk = wide_chunk<T>(a.rows, a.width);
    const dim3 grid((uint32_t)((a.width + Wide<T>::kSlab - 1) / Wide<T>::kSlab),
                    (uint32_t)((a.rows + chunk - 1) / chunk));
    parts = (int)grid.y;
    wide_kernel<T><<<grid, Wide<T>::kThreads, 0, s>>>(a, pieces, chunk, over, stat,
                                                 sums ? part : nullptr);
  }
  if (sums && !done) {
    const dim3 grid((uint32_t)((a.width + kJoinColumns - 1) / kJoinColumns), 2);
    const int slices = std::max(1, std::min(kJoinSlices, (parts + kJoinAhead - 1) / kJoinAhead));
    join_kernel<<<grid, kJoinColumns * slices, 0, s>>>(a, part, parts);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_layer_norm(int dtype, const NormArgs &a, int cu_count, hipStream_t s) {
  if (dtype == ML2_F32) return launch_norm<float>(a, cu_count, s);
  if (dtype == ML2_BF16) return launch_norm<__bf16>(a, cu_count, s);
  return launch_norm<_Float16>(a, cu_count, s);
}

size_t layer_norm_grad_workspace_bytes(int64_t rows, int64_t width) {
  if (rows <= 0 || width <= 0) return 0;
  size_t floats = 0;  // for rows of either size of columns
  if (!grad_twice(rows, width, 2))
    floats = (size_t)grad_shape(rows, width).blocks * 2 * (size_t)width;
  if (grad_twice(rows, width, 4)) {
    const int64_t chunk =
        std::min(wide_chunk<float>(rows, width), wide_chunk<__bf16>(rows, width));
    floats = std::max(floats, (size_t)rows * (size_t)stat_pieces(width) * 3 +
                                  (size_t)((rows + chunk - 1) / chunk) * 2 * (size_t)width);
  }
  return floats * sizeof(float);
}

hipError_t launch_layer_norm_grad(int dtype, const NormGradArgs &a, void *ws, hipStream_t s) {
  if (dtype == ML2_F32) return launch_grad<float>(a, ws, s);
  if (dtype == ML2_BF16) return launch_grad<__bf16>(a, ws, s);
  return launch_grad<_Float16>(a, ws, s);
}

}  // namespace ml2
