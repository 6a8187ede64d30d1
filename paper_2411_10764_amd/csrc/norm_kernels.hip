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
#include <algorithm>

#include "train.h"

namespace ml2 {
namespace {

constexpr int kWaveBlock = 256;   // threads where a row has at most a wave
constexpr int kMaxBlock = 1024;

// weight or bias (or `none` where there is none) of columns c .. c + kLen - 1
template <typename T>
__device__ __forceinline__ void load_param(const void *p, int f32, float none, int64_t c,
                                           int64_t width, float *x) {
  constexpr int kLen = Vec<T>::kLen;
  if (!p) {
#pragma unroll
    for (int j = 0; j < kLen; ++j) x[j] = none;
  } else if (f32) {
#pragma unroll
    for (int j = 0; j < kLen; j += 4) load_floats(static_cast<const float *>(p), c + j, width, x + j);
  } else {
    load_floats(static_cast<const T *>(p), c, width, x);
  }
}

// N sums over the workgroup's waves, in every thread.
template <int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float (*lds)[N]) {
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = group_sum(v[i], 6);
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

// E columns a lane.  WAVE: 2^log_g lanes share a row, else the workgroup does.
// Vector k of a lane lies at column (k * lanes + lane) * kLen.
template <typename T, int E, bool WAVE>
__global__ __launch_bounds__(WAVE ? kWaveBlock : kMaxBlock) void norm_kernel(NormArgs a,
                                                                             int log_g,
                                                                             float over_width) {
  constexpr int kLen = Vec<T>::kLen, kVecs = E / kLen;
  constexpr bool kKeep = E <= 16;  // the parameters stay in registers
  __shared__ float first[kMaxBlock / 64][1], second[kMaxBlock / 64][2];
  const int lanes = WAVE ? 1 << log_g : (int)blockDim.x;
  const int lane = WAVE ? threadIdx.x & (lanes - 1) : threadIdx.x;
  const int64_t per = WAVE ? kWaveBlock >> log_g : 1;
  const int64_t group = WAVE ? threadIdx.x >> log_g : 0;
  float w[kKeep ? E : kLen], b[kKeep ? E : kLen];
  if (kKeep) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int64_t c = ((int64_t)k * lanes + lane) * kLen;
      load_param<T>(a.weight, a.param_f32, 1.0f, c, a.width, w + k * kLen);
      load_param<T>(a.bias, a.param_f32, 0.0f, c, a.width, b + k * kLen);
    }
  }
  for (int64_t row0 = (int64_t)blockIdx.x * per; row0 < a.rows;
       row0 += (int64_t)gridDim.x * per) {
    const int64_t row = row0 + group;
    const bool in = row < a.rows;
    const T *src = static_cast<const T *>(a.x) + (in ? row : 0) * a.ld;
    float x[E];
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
      load_floats(src, ((int64_t)k * lanes + lane) * kLen, in ? a.width : 0, x + k * kLen);
    float s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < E; ++i) s[0] += x[i];
    if (WAVE)
      s[0] = group_sum(s[0], log_g);
    else
      block_sums(s, first);
    const float m0 = s[0] * over_width;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int64_t c = ((int64_t)k * lanes + lane) * kLen;
      if (c + kLen > a.width) {  // columns behind the row differ from the mean by nothing
#pragma unroll
        for (int j = 0; j < kLen; ++j)
          if (c + j >= a.width) x[k * kLen + j] = m0;
      }
    }
    float t[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < E; ++i) {
      x[i] -= m0;
      t[0] += x[i];
      t[1] = fmaf(x[i], x[i], t[1]);
    }
    if (WAVE) {
      t[0] = group_sum(t[0], log_g);
      t[1] = group_sum(t[1], log_g);
    } else {
      block_sums(t, second);
    }
    const float delta = t[0] * over_width;
    const float raw = fmaf(t[1], over_width, -delta * delta);
    const float var = raw < 0.0f ? 0.0f : raw;  // a NaN stays one
    const float rstd = 1.0f / sqrtf(var + a.eps);
    if (!in) continue;
    if (lane == 0) {
      if (a.mean) a.mean[row] = m0 + delta;
      if (a.rstd) a.rstd[row] = rstd;
    }
    T *dst = static_cast<T *>(a.out) + row * a.out_ld;
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int64_t c = ((int64_t)k * lanes + lane) * kLen;
      if (c >= a.width) continue;
      if (!kKeep) {
        load_param<T>(a.weight, a.param_f32, 1.0f, c, a.width, w);
        load_param<T>(a.bias, a.param_f32, 0.0f, c, a.width, b);
      }
      float y[kLen];
#pragma unroll
      for (int j = 0; j < kLen; ++j) {
        const int p = kKeep ? k * kLen + j : j;
        y[j] = fmaf((x[k * kLen + j] - delta) * rstd, w[p], b[p]);
      }
      store_floats(dst, c, a.width, y);
    }
  }
}

// ---- gradients of rows that fit a workgroup's registers ---------------------------

constexpr int kGradBlocks = 256;   // at most: each leaves a part of the parameters' sums
constexpr int kGradWidth = 16 * kMaxBlock;

struct GradShape {
  int lanes, log_g;   // of a row; log_g: where they are at most a wave
  int per, threads;   // rows at a time, threads of a workgroup
  int blocks;
};

// Sums of a lane group over all rows it takes go to part[block][0] (weight) and
// [1] (bias), float32 [width] each.
template <typename T, int E>
__global__ __launch_bounds__(kMaxBlock) void grad_kernel(NormGradArgs a, GradShape g,
                                                         float over_width, float *part) {
  constexpr int kLen = Vec<T>::kLen, kVecs = E / kLen;
  __shared__ float lds[kMaxBlock * E];
  float (*sums)[kMaxBlock / 64][3] = reinterpret_cast<float (*)[kMaxBlock / 64][3]>(lds);
  const int lanes = g.lanes, group = (int)threadIdx.x / lanes;
  const int lane = (int)threadIdx.x - group * lanes;
  const bool wide = lanes > 64;
  float w[E], dw[E], db[E];
#pragma unroll
  for (int k = 0; k < kVecs; ++k)
    load_param<T>(a.weight, a.param_f32, 1.0f, ((int64_t)k * lanes + lane) * kLen, a.width,
                  w + k * kLen);
#pragma unroll
  for (int i = 0; i < E; ++i) dw[i] = db[i] = 0.0f;
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * g.per; row0 < a.rows;
       row0 += (int64_t)gridDim.x * g.per, turn ^= 1) {
    const int64_t row = row0 + group;
    const bool in = row < a.rows;
    const int64_t from = in ? row : 0, width = in ? a.width : 0;
    const float mean = a.mean[from], rstd = a.rstd[from];
    const T *xs = static_cast<const T *>(a.x) + from * a.ld;
    const T *ds = static_cast<const T *>(a.dout) + from * a.dout_ld;
    float x[E], d[E];
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int64_t c = ((int64_t)k * lanes + lane) * kLen;
      load_floats(xs, c, width, x + k * kLen);
      load_floats(ds, c, width, d + k * kLen);
    }
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      const int64_t c = ((int64_t)k * lanes + lane) * kLen;
      if (c + kLen > width) {
#pragma unroll
        for (int j = 0; j < kLen; ++j)
          if (c + j >= width) x[k * kLen + j] = mean;
      }
    }
    float s[3] = {0.0f, 0.0f, 0.0f};  // of x - mean, g, g (x - mean)
#pragma unroll
    for (int i = 0; i < E; ++i) {
      x[i] -= mean;
      const float gi = d[i] * w[i];
      s[0] += x[i];
      s[1] += gi;
      s[2] = fmaf(gi, x[i], s[2]);
    }
    const int log_g = wide ? 6 : g.log_g;
#pragma unroll
    for (int i = 0; i < 3; ++i) s[i] = group_sum(s[i], log_g);
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
    if (in) {
      T *dst = a.dx ? static_cast<T *>(a.dx) + row * a.dx_ld : nullptr;
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        const int64_t c = ((int64_t)k * lanes + lane) * kLen;
        float y[kLen];
#pragma unroll
        for (int j = 0; j < kLen; ++j) {
          const int i = k * kLen + j;
          const float xhat = (x[i] - delta) * rstd;
          dw[i] = fmaf(d[i], xhat, dw[i]);
          db[i] += d[i];
          y[j] = rstd * (fmaf(d[i], w[i], -g_avg) - xhat * along);
        }
        if (dst) store_floats(dst, c, a.width, y);
      }
    }
  }
  if (!part) return;
  // The groups of a wave, then the waves: lane i of a wave holds the columns of
  // lane i % lanes.
  if (!wide) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      float v[2] = {dw[i], db[i]};
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        if (g.log_g <= 3) v[q] += lane_swap<0x128>(v[q]);  // row_ror 8
        if (g.log_g <= 2) v[q] += lane_swap<0x124>(v[q]);  // row_ror 4
        if (g.log_g <= 1) v[q] += lane_swap<0x122>(v[q]);  // row_ror 2
        if (g.log_g <= 0) v[q] += lane_swap<0x121>(v[q]);  // row_ror 1
        const auto add = [](float p, float r) { return p + r; };
        if (g.log_g <= 4) v[q] = join_rows(v[q], add);
        if (g.log_g <= 5) v[q] = join_halves(v[q], add);
      }
      dw[i] = v[0];
      db[i] = v[1];
    }
  }
  const int parts = wide ? g.per : (int)blockDim.x >> 6;
  const int own = wide ? group : (int)threadIdx.x >> 6;
  const bool has = wide || (int)(threadIdx.x & 63) < lanes;
  const int span = lanes * E;  // columns that a part holds, the row's and some behind it
  float *to = part + (int64_t)blockIdx.x * 2 * a.width;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    __syncthreads();
    if (has) {
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
#pragma unroll
        for (int j = 0; j < kLen; ++j)
          lds[own * span + (k * lanes + lane) * kLen + j] = q ? db[k * kLen + j] : dw[k * kLen + j];
      }
    }
    __syncthreads();
    for (int64_t c = threadIdx.x; c < a.width; c += blockDim.x) {
      float v = lds[c];
      for (int p = 1; p < parts; ++p) v += lds[p * span + c];
      to[q * a.width + c] = v;
    }
  }
}

// ---- gradients of wider rows -------------------------------------------------------

constexpr int kStatThreads = 256, kStatVecs = 4;
constexpr int kWideThreads = 256, kWideColumns = 8;  // a thread's columns

// Row sums of x - mean, g and g (x - mean) over a piece of kStatVecs vectors a
// thread: stat[row][piece][3].
template <typename T>
__global__ __launch_bounds__(kStatThreads) void stat_kernel(NormGradArgs a, int64_t pieces,
                                                            float *stat) {
  constexpr int kLen = Vec<T>::kLen;
  __shared__ float lds[2][kStatThreads / 64][3];
  int turn = 0;
  for (int64_t item = blockIdx.x; item < a.rows * pieces; item += gridDim.x, turn ^= 1) {
    const int64_t row = item / pieces, piece = item - row * pieces;
    const float mean = a.mean[row];
    const T *xs = static_cast<const T *>(a.x) + row * a.ld;
    const T *ds = static_cast<const T *>(a.dout) + row * a.dout_ld;
    float x[kStatVecs][kLen], d[kStatVecs][kLen];
    const int64_t c0 = (piece * kStatVecs * kStatThreads + threadIdx.x) * kLen;
#pragma unroll
    for (int k = 0; k < kStatVecs; ++k) {
      load_floats(xs, c0 + k * kStatThreads * kLen, a.width, x[k]);
      load_floats(ds, c0 + k * kStatThreads * kLen, a.width, d[k]);
    }
    float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < kStatVecs; ++k) {
      const int64_t c = c0 + k * kStatThreads * kLen;
      float w[kLen];
      if (c < a.width) {
        load_param<T>(a.weight, a.param_f32, 1.0f, c, a.width, w);
#pragma unroll
        for (int j = 0; j < kLen; ++j) {
          const float v = c + j < a.width ? x[k][j] - mean : 0.0f, g = d[k][j] * w[j];
          s[0] += v;
          s[1] += g;
          s[2] = fmaf(g, v, s[2]);
        }
      }
    }
    block_sums(s, lds[turn]);
    if (threadIdx.x < 3) stat[item * 3 + threadIdx.x] = s[threadIdx.x];
  }
}

// A workgroup takes kWideThreads * kWideColumns columns of `chunk` rows.
template <typename T>
__global__ __launch_bounds__(kWideThreads) void wide_kernel(NormGradArgs a, int64_t pieces,
                                                            int64_t chunk, float over_width,
                                                            const float *stat, float *part) {
  constexpr int kLen = Vec<T>::kLen, kVecs = kWideColumns / kLen;
  const int64_t c0 = ((int64_t)blockIdx.x * kVecs * kWideThreads + threadIdx.x) * kLen;
  const int64_t r0 = (int64_t)blockIdx.y * chunk, r1 = min(a.rows, r0 + chunk);
  float w[kVecs][kLen], dw[kVecs][kLen], db[kVecs][kLen];
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    load_param<T>(a.weight, a.param_f32, 1.0f, c0 + k * kWideThreads * kLen, a.width, w[k]);
#pragma unroll
    for (int j = 0; j < kLen; ++j) dw[k][j] = db[k][j] = 0.0f;
  }
  for (int64_t row = r0; row < r1; ++row) {
    float s[3] = {0.0f, 0.0f, 0.0f};
    for (int64_t p = 0; p < pieces; ++p) {
#pragma unroll
      for (int i = 0; i < 3; ++i) s[i] += stat[(row * pieces + p) * 3 + i];
    }
    const float mean = a.mean[row], rstd = a.rstd[row];
    const float delta = s[0] * over_width, g_avg = s[1] * over_width;
    const float along = (s[2] - delta * s[1]) * over_width * rstd;
    const T *xs = static_cast<const T *>(a.x) + row * a.ld;
    const T *ds = static_cast<const T *>(a.dout) + row * a.dout_ld;
    float x[kVecs][kLen], d[kVecs][kLen];
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      load_floats(xs, c0 + k * kWideThreads * kLen, a.width, x[k]);
      load_floats(ds, c0 + k * kWideThreads * kLen, a.width, d[k]);
    }
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      float y[kLen];
#pragma unroll
      for (int j = 0; j < kLen; ++j) {
        const float xhat = (x[k][j] - mean - delta) * rstd;
        dw[k][j] = fmaf(d[k][j], xhat, dw[k][j]);
        db[k][j] += d[k][j];
        y[j] = rstd * (fmaf(d[k][j], w[k][j], -g_avg) - xhat * along);
      }
      if (a.dx)
        store_floats(static_cast<T *>(a.dx) + row * a.dx_ld, c0 + k * kWideThreads * kLen, a.width,
                     y);
    }
  }
  if (!part) return;
  float *to = part + (int64_t)blockIdx.y * 2 * a.width;
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
#pragma unroll
    for (int j = 0; j < kLen; ++j) {
      const int64_t c = c0 + k * kWideThreads * kLen + j;
      if (c < a.width) {
        to[c] = dw[k][j];
        to[a.width + c] = db[k][j];
      }
    }
  }
}

// ---- the parameters' sums ------------------------------------------------------------

constexpr int kJoinColumns = 64, kJoinSlices = 16;

__device__ __forceinline__ void store_as(int dtype, void *p, int64_t i, float v) {
  if (dtype == ML2_F32)
    static_cast<float *>(p)[i] = v;
  else if (dtype == ML2_BF16)
    static_cast<__bf16 *>(p)[i] = narrow<__bf16>(v);
  else
    static_cast<_Float16 *>(p)[i] = narrow<_Float16>(v);
}

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
  const int each = (parts + kJoinSlices - 1) / kJoinSlices;
  const int p1 = min(parts, (slice + 1) * each);
  float v = 0.0f;
  if (c < a.width) {
#pragma unroll 8
    for (int p = slice * each; p < p1; ++p) v += part[((int64_t)p * 2 + blockIdx.y) * a.width + c];
  }
  lds[slice][lane] = v;
  __syncthreads();
  if (slice == 0 && c < a.width) {
    for (int k = 1; k < kJoinSlices; ++k) v += lds[k][lane];
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
template <typename T, int E>
hipError_t launch_narrow(const NormArgs &a, int cu_count, hipStream_t s) {
  const int log_g = log2_up((a.width + E - 1) / E);
  const int64_t per = kWaveBlock >> log_g;
  const int64_t grid = std::min<int64_t>((a.rows + per - 1) / per, (int64_t)cu_count * 8);
  norm_kernel<T, E, true><<<(uint32_t)grid, kWaveBlock, 0, s>>>(a, log_g, 1.0f / (float)a.width);
  return hipGetLastError();
}

template <typename T, int E>
hipError_t launch_wide(const NormArgs &a, int cu_count, hipStream_t s) {
  const int threads = (int)((a.width + 64 * E - 1) / (64 * E) * 64);
  const int64_t grid = std::min<int64_t>(a.rows, (int64_t)cu_count * (2048 / threads));
  norm_kernel<T, E, false><<<(uint32_t)grid, threads, 0, s>>>(a, 0, 1.0f / (float)a.width);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_norm(const NormArgs &a, int cu_count, hipStream_t s) {
  if (a.width <= 64 * 8) return launch_narrow<T, 8>(a, cu_count, s);
  if (a.width <= 64 * 16) return launch_narrow<T, 16>(a, cu_count, s);
  if (a.width <= kMaxBlock * 16) return launch_wide<T, 16>(a, cu_count, s);
  if (a.width <= kMaxBlock * 32) return launch_wide<T, 32>(a, cu_count, s);
  return launch_wide<T, 64>(a, cu_count, s);
}

int grad_columns(int64_t width) { return width <= 64 * 8 ? 8 : 16; }

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
  g.blocks = (int)std::min<int64_t>((rows + g.per - 1) / g.per, kGradBlocks);
  return g;
}

int64_t stat_pieces(int64_t width) {  // for the smaller vectors
  const int64_t each = (int64_t)kStatVecs * kStatThreads * 4;
  return (width + each - 1) / each;
}

constexpr int64_t kWideSlab = (int64_t)kWideThreads * kWideColumns;

// Rows of a chunk: enough chunks to fill the device.
int64_t wide_chunk(int64_t rows, int64_t width) {
  const int64_t slabs = (width + kWideSlab - 1) / kWideSlab;
  const int64_t chunks = std::max<int64_t>(1, std::min<int64_t>(rows, 1024 / slabs));
  return (rows + chunks - 1) / chunks;
}

template <typename T>
hipError_t launch_grad(const NormGradArgs &a, void *ws, hipStream_t s) {
  const bool sums = a.dweight || a.dbias;
  const float over = 1.0f / (float)a.width;
  float *part = static_cast<float *>(ws);
  int parts = 0;
  if (a.rows > 0 && a.width <= kGradWidth) {
    const GradShape g = grad_shape(a.rows, a.width);
    parts = g.blocks;
    if (grad_columns(a.width) == 8)
      grad_kernel<T, 8><<<g.blocks, g.threads, 0, s>>>(a, g, over, sums ? part : nullptr);
    else
      grad_kernel<T, 16><<<g.blocks, g.threads, 0, s>>>(a, g, over, sums ? part : nullptr);
  } else if (a.rows > 0) {
    const int64_t each = (int64_t)kStatVecs * kStatThreads * Vec<T>::kLen;
    const int64_t pieces = (a.width + each - 1) / each;
    float *stat = part;
    part += (size_t)a.rows * stat_pieces(a.width) * 3;
    const int64_t items = std::min<int64_t>(a.rows * pieces, 1 << 20);
    stat_kernel<T><<<(uint32_t)items, kStatThreads, 0, s>>>(a, pieces, stat);
    const int64_t chunk = wide_chunk(a.rows, a.width);
    const dim3 grid((uint32_t)((a.width + kWideSlab - 1) / kWideSlab),
                    (uint32_t)((a.rows + chunk - 1) / chunk));
    parts = (int)grid.y;
    wide_kernel<T><<<grid, kWideThreads, 0, s>>>(a, pieces, chunk, over, stat,
                                                 sums ? part : nullptr);
  }
  if (sums) {
    const dim3 grid((uint32_t)((a.width + kJoinColumns - 1) / kJoinColumns), 2);
    join_kernel<<<grid, kJoinColumns * kJoinSlices, 0, s>>>(a, part, parts);
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
  if (width <= kGradWidth)
    return (size_t)grad_shape(rows, width).blocks * 2 * (size_t)width * sizeof(float);
  const int64_t chunk = wide_chunk(rows, width);
  return ((size_t)rows * (size_t)stat_pieces(width) * 3 +
          (size_t)((rows + chunk - 1) / chunk) * 2 * (size_t)width) * sizeof(float);
}

hipError_t launch_layer_norm_grad(int dtype, const NormGradArgs &a, void *ws, hipStream_t s) {
  if (dtype == ML2_F32) return launch_grad<float>(a, ws, s);
  if (dtype == ML2_BF16) return launch_grad<__bf16>(a, ws, s);
  return launch_grad<_Float16>(a, ws, s);
}

}  // namespace ml2
