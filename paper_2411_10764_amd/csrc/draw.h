// Shared by the operators over rows of scores and over tables (sample_kernels,
// logprob_kernels, embed_kernels): element types, launch arguments, and the
// exponent every one of them takes of a score.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "ml2.h"
#include "ml2_internal.h"

namespace ml2 {

// Rows of scores with a mask (see ml2.h).
struct ScoreRows {
  const void *scores;
  int64_t n, ld, rows;
  const uint8_t *valid;  // or null
  int64_t valid_ld;
  const float *temperature;  // [rows] or null
};

struct SampleArgs {
  ScoreRows s;
  const int32_t *top_k;  // [rows] or null, as the next two
  const float *top_p, *min_p;
  const float *u;  // [rows][draws]
  int32_t draws;
  int32_t *idx;
  float *logprob;
};

struct LogprobArgs {
  ScoreRows s;
  const int32_t *targets;  // [rows][per_row]
  const float *weight;     // [rows][per_row], null without a gradient
  int32_t per_row;
  float *logprob;          // or null
  void *grad;              // or null
  int64_t grad_ld;
};

struct EmbedArgs {
  const void *table;
  int64_t table_rows, width, ld;
  const int32_t *ids;
  int64_t n;
  float scale;
  void *out;
  int64_t out_ld;
};

struct EmbedGradArgs {
  const void *dout;
  int64_t n, width, dout_ld;
  const int32_t *ids;
  float scale;
  void *grad;
  int64_t table_rows, grad_ld;
};

size_t sample_workspace_bytes(int64_t n, int64_t rows, int32_t draws);
hipError_t launch_sample(int dtype, const SampleArgs &a, void *ws, int cu_count, hipStream_t s);
size_t logprob_workspace_bytes(int64_t n, int64_t rows, int32_t per_row);
hipError_t launch_logprob(int dtype, const LogprobArgs &a, void *ws, int cu_count, hipStream_t s);
hipError_t launch_embed(int dtype, const EmbedArgs &a, int cu_count, hipStream_t s);
size_t embed_grad_workspace_bytes(int64_t n, int64_t table_rows, int64_t width);
hipError_t launch_embed_grad(int dtype, int grad_dtype, const EmbedGradArgs &a, void *ws,
                             hipStream_t s);

// ---- device helpers ---------------------------------------------------------

typedef unsigned long long u64;

// v of the lane that the DPP control names, `none` where there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lane_move(uint32_t v, uint32_t none) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xF, false);
}

template <int CTRL, int ROWS>
__device__ __forceinline__ u64 lane_move(u64 v, u64 none) {
  return ((u64)lane_move<CTRL, ROWS>((uint32_t)(v >> 32), (uint32_t)(none >> 32)) << 32) |
         lane_move<CTRL, ROWS>((uint32_t)v, (uint32_t)none);
}

// Folds v over the lanes up to and including the own one (DPP moves: shifts
// inside rows of 16 lanes, then the rows' last lanes; an LDS shuffle a step
// takes several times as long).  `none`: the neutral value.
template <typename V, typename F>
__device__ __forceinline__ V wave_fold(V v, V none, F f) {
  v = f(v, lane_move<0x111, 0xF>(v, none));
  v = f(v, lane_move<0x112, 0xF>(v, none));
  v = f(v, lane_move<0x114, 0xF>(v, none));
  v = f(v, lane_move<0x118, 0xF>(v, none));
  v = f(v, lane_move<0x142, 0xA>(v, none));
  return f(v, lane_move<0x143, 0xC>(v, none));
}

template <typename V>
__device__ __forceinline__ V wave_prefix(V v) {  // inclusive
  return wave_fold(v, (V)0, [](V a, V b) { return a + b; });
}

__device__ __forceinline__ u64 from_lane(u64 v, int lane) {
  return ((u64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}

__device__ __forceinline__ uint32_t from_lane(uint32_t v, int lane) {
  return (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

// Vectors of 16 bytes that need the alignment of one element only (the memory
// system takes any address; the type keeps the compiler from assuming more).
template <typename T>
struct Vec {
  static constexpr int kLen = 16 / (int)sizeof(T);
  typedef T type __attribute__((ext_vector_type(kLen), aligned(sizeof(T))));
};

// A float32 value rounded to an element.  (The compiler would fold a product
// and its rounding to fp16 into one instruction that rounds once, and only
// where it sees both: results would depend on the path an element takes.)
template <typename T>
__device__ __forceinline__ T narrow(float x) {
  if constexpr (sizeof(T) == 2) asm("" : "+v"(x));
  return (T)x;
}

// An element as float32, a signaling NaN made a quiet one.  The compiler turns
// fmaxf and comparisons joined by `or` into maxima, which give NaN where one
// operand is signaling; it also counts on a cast from bfloat16, which is a shift
// of the bits, to have quieted it.
template <typename T>
__device__ __forceinline__ float widen(T v) {
  float x;
  if constexpr (__is_same(T, __bf16))
    x = __uint_as_float((uint32_t)__builtin_bit_cast(uint16_t, v) << 16);
  else
    x = (float)v;
  return __builtin_canonicalizef(x);
}

// A score as float32 with -0.0 canonicalised to +0.0, and -inf where the entry
// is not included (so a NaN or a masked entry never competes).
__device__ __forceinline__ float included(float s, bool valid) {
  return valid && !__builtin_isnan(s) ? s + 0.0f : -__builtin_inff();
}

// Eight consecutive entries i .. i+7 of a row of n: -inf where not included.
template <typename T>
__device__ __forceinline__ void load8(const T *scores, const uint8_t *valid, int64_t i, int64_t n,
                                      float (&x)[8]) {
  typedef T V __attribute__((ext_vector_type(8), aligned(sizeof(T))));
  typedef unsigned long long Mask __attribute__((aligned(1)));
  if (i + 8 <= n) {
    const V v = *reinterpret_cast<const V *>(scores + i);
    const unsigned long long mask = valid ? *reinterpret_cast<const Mask *>(valid + i) : ~0ull;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = included((float)v[j], ((mask >> (8 * j)) & 0xFF) != 0);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      x[j] = i + j < n ? included((float)scores[i + j], !valid || valid[i + j] != 0)
                       : -__builtin_inff();
  }
}

__device__ __forceinline__ float inverse_temperature(const float *temperature, int64_t row,
                                                     bool *greedy) {
  const float t = temperature ? temperature[row] : 1.0f;
  *greedy = !(t > 0.0f);
  return t > 0.0f ? 1.0f / t : 1.0f;
}

}  // namespace ml2
