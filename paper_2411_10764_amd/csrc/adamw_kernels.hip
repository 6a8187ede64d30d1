// The norm of many gradients together, and a step of AdamW over many tensors.
//
//   g = grad f,  m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g g
//   p' = p - (lr decay p + lr / (1 - b1^t) m' / (sqrt(v') / sqrt(1 - b2^t) + eps))
//
// Bytes bound both.  A launch takes a table of tensors by value (no copy to the
// device, nothing to keep until it has run); a workgroup finds its tensor by one
// comparison of all first workgroups with its own number.
//
// Measured: norm of 134M bf16 elements 53 us (268 MB, 5.1 TB/s); steps of 33.5M
// float32 parameters 170 us (940 MB, 5.5 TB/s), of 12M in 60 tensors with a bf16 copy
// 75, of 134M bf16 ones with 8-bit states 250 (1.35 GB, 5.4 TB/s; where rate and number
// lie on the device 321).
#include <math.h>

#include <algorithm>

#include "train.h"

namespace ml2 {
namespace {

constexpr int kThreads = 256;
// Workgroups of a launch, about; beyond that they take several tiles each.  (More
// tiles for fewer workgroups cost: 33.5M bf16 parameters with 16,384 workgroups 134 us,
// 8,192 140, 4,096 142.)
constexpr int64_t kMostBlocks = 1 << 20;

// The last tensor of `count` whose first workgroup is not behind `block`.
template <int MOST>
__device__ __forceinline__ int find_tensor(const uint32_t (&first)[MOST], int count,
                                           uint32_t block) {
  int n = 0;
#pragma unroll
  for (int i = 0; i < MOST; i += 64) {
    const int at = i + (int)(threadIdx.x & 63);
    n += __popcll(__ballot(at < count && at < MOST && first[at < MOST ? at : 0] <= block));
  }
  return __builtin_amdgcn_readfirstlane(n - 1);
}

// ---- norm ------------------------------------------------------------------------

constexpr int kNormTensors = 128;
constexpr int kNormVecs = 4;       // vectors of a thread in flight
// About as many parts, and one for each tensor, of at least so many elements: 4M float32
// elements in 10 tensors 10.4 us, with half the parts of twice the size 12.7; 134M bf16
// ones 54 with 2,048 or 4,096 parts, 57 with 1,024.
constexpr int kNormParts = 4096;
constexpr int64_t kNormLeast = 8192;

struct NormTable {
  const void *grad[kNormTensors];
  int64_t n[kNormTensors];
  uint32_t first[kNormTensors];  // workgroup
  int count;
  int64_t chunk;                 // elements of a workgroup
  double *part;
};
static_assert(sizeof(NormTable) <= 3968, "kernel arguments");

__device__ __forceinline__ double block_sum(double v, double *lds) {
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) lds[wave] = v;
  __syncthreads();
  v = lds[0];
  for (int w = 1; w < (int)(blockDim.x >> 6); ++w) v += lds[w];
  return v;
}

// The squares of elements a .. b - 1, a thread's share.
template <typename T>
__device__ __forceinline__ double squares(const T *g, int64_t a, int64_t b) {
  constexpr int kLen = Vec<T>::kLen;
  double s[kNormVecs] = {};
  for (int64_t i = a + (int64_t)threadIdx.x * kLen; i < b;
       i += (int64_t)blockDim.x * kLen * kNormVecs) {
    float x[kNormVecs][kLen];
#pragma unroll
    for (int k = 0; k < kNormVecs; ++k)
      load_floats(g, i + (int64_t)k * blockDim.x * kLen, b, x[k]);
#pragma unroll
    for (int k = 0; k < kNormVecs; ++k) {
#pragma unroll
      for (int j = 0; j < kLen; ++j) s[k] = fma((double)x[k][j], (double)x[k][j], s[k]);
    }
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void square_kernel(NormTable t) {
  __shared__ double lds[kThreads / 64];
  const int i = find_tensor(t.first, t.count, blockIdx.x);
  const int64_t a = (int64_t)(blockIdx.x - t.first[i]) * t.chunk;
  const double s = block_sum(
      squares(static_cast<const T *>(t.grad[i]), a, min(t.n[i], a + t.chunk)), lds);
  if (threadIdx.x == 0) t.part[blockIdx.x] = s;
}

struct NormOut {
  float scale, max_norm;
  float *norm, *factor;
  int32_t *step;
};

__device__ __forceinline__ void finish(const NormOut &o, double sum) {
  const double norm = (double)o.scale * sqrt(sum);
  const bool finite = fabs((float)norm) < __builtin_inff();
  if (o.norm) *o.norm = (float)norm;
  if (o.factor)
    *o.factor = finite ? (float)((double)o.scale * fmin(1.0, (double)o.max_norm / norm))
                       : __builtin_nanf("");
  if (o.step && finite) *o.step += 1;
}

__global__ __launch_bounds__(1024) void finish_kernel(const double *part, int64_t parts,
                                                      NormOut o) {
  __shared__ double lds[16];
  double v = 0.0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < parts; i += 1024) v += part[i];
  v = block_sum(v, lds);
  if (threadIdx.x == 0) finish(o, v);
}

// Few elements in all: one workgroup, one launch.  Its waves take chunks of all
// tensors in turn (t.first: chunks).
template <typename T>
__global__ __launch_bounds__(1024) void norm_one_kernel(NormTable t, uint32_t chunks, NormOut o) {
  constexpr int kLen = Vec<T>::kLen;
  __shared__ double lds[16];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  double v = 0.0;
  for (uint32_t c = wave; c < chunks; c += 16) {
    const int i = find_tensor(t.first, t.count, c);
    const int64_t at = (int64_t)(c - t.first[i]) * t.chunk + lane * kLen;
    float x[kNormVecs][kLen];
#pragma unroll
    for (int k = 0; k < kNormVecs; ++k)
      load_floats(static_cast<const T *>(t.grad[i]), at + k * 64 * kLen, t.n[i], x[k]);
#pragma unroll
    for (int k = 0; k < kNormVecs; ++k) {
#pragma unroll
      for (int j = 0; j < kLen; ++j) v = fma((double)x[k][j], (double)x[k][j], v);
    }
  }
  v = block_sum(v, lds);
  if (threadIdx.x == 0) finish(o, v);
}

// Up to so many chunks: 65,536 float32 elements 7.2 us, in two launches 9.7; 131,072
// 10.7 and 9.9.  163,840 bf16 ones 9.8 and 8.2.
constexpr int64_t kNormOne = 64;

int64_t norm_chunk(const int64_t *sizes, int32_t count) {
  int64_t total = 0;
  for (int32_t i = 0; i < count; ++i) total += sizes[i] / kNormParts + 1;
  return std::max(kNormLeast, (total + 4095) / 4096 * 4096);
}

int64_t norm_parts(const int64_t *sizes, int32_t count, int64_t chunk) {
  int64_t parts = 0;
  for (int32_t i = 0; i < count; ++i) parts += (sizes[i] + chunk - 1) / chunk;
  return parts;
}

template <typename T>
hipError_t launch_norm(const void *const *grads, const int64_t *sizes, int32_t count,
                       const NormOut &o, double *part, hipStream_t s) {
  constexpr int64_t kChunk = 64 * kNormVecs * Vec<T>::kLen;  // of a wave
  int64_t chunks = 0;
  for (int32_t i = 0; i < count && chunks <= kNormOne; ++i)
    chunks += (sizes[i] + kChunk - 1) / kChunk;
  const bool one = chunks <= kNormOne;
  NormTable t;
  t.chunk = one ? kChunk : norm_chunk(sizes, count);
  t.part = part;
  t.count = 0;
  uint32_t blocks = 0;
  int64_t parts = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (sizes[i] == 0) continue;
    t.grad[t.count] = grads[i];
    t.n[t.count] = sizes[i];
    t.first[t.count++] = blocks;
    blocks += (uint32_t)((sizes[i] + t.chunk - 1) / t.chunk);
    if (!one && t.count == kNormTensors) {
      square_kernel<T><<<blocks, kThreads, 0, s>>>(t);
      parts += blocks;
      t.part += blocks;
      t.count = 0;
      blocks = 0;
    }
  }
  if (one) {
    norm_one_kernel<T><<<1, 1024, 0, s>>>(t, blocks, o);
    return hipGetLastError();
  }
  if (t.count > 0) square_kernel<T><<<blocks, kThreads, 0, s>>>(t);
  finish_kernel<<<1, 1024, 0, s>>>(part, parts + blocks, o);
  return hipGetLastError();
}

// ---- step ------------------------------------------------------------------------

constexpr int kTensors = 48;
constexpr int kTile = 2048;  // elements of a workgroup and turn

struct StepTable {
  void *param[kTensors];
  const void *grad[kTensors];
  void *m[kTensors], *v[kTensors];
  void *param_out[kTensors], *m_out[kTensors], *v_out[kTensors];
  void *copy[kTensors];
  int64_t n[kTensors];
  float decay[kTensors];
  uint32_t first[kTensors];  // workgroup
};

struct StepShared {
  int64_t tiles;          // of a workgroup
  double b1, b2, log_b1, log_b2;
  const float *lr_device;
  const int32_t *step_device;
  const float *factor;
  float lr, eps;
  float rate, root;       // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  uint32_t step, key;     // key: of the seed
  int32_t count, place;   // place: of the table's first tensor
};
static_assert(sizeof(StepTable) + sizeof(StepShared) <= 4096, "kernel arguments");

constexpr uint32_t kPhi = 0x9E3779B9u, kPlastic = 0xC13FA9A9u;  // 2^32 over those numbers

__host__ __device__ __forceinline__ uint32_t fold_word(uint32_t k, uint32_t word) {
  k += word + kPhi;
  k = (k ^ (k >> 16)) * kPhi;
  k = (k ^ (k >> 15)) * kPlastic;
  return k ^ (k >> 16);
}

__host__ __device__ __forceinline__ void rates(double lr, double step, double log_b1,
                                               double log_b2, float *rate, float *root) {
  *rate = (float)(lr / -expm1(step * log_b1));
  *root = (float)(1.0 / sqrt(-expm1(step * log_b2)));
}

// What a workgroup needs of the step: the same in all its threads.  Each of them works
// out rates whose rate or number lies on the device, some hundred instructions, most of
// them of 64 bits, before its tile.  Steps in 32 bits have the time: 33.5M float32
// parameters 174 us, with rates from the host 173; 12M in 60 tensors 76 and 74.  Those in
// 8 bits are bound by instructions and have not: 134M bf16 ones 321 us and 253.
struct Step {
  float f, lr, rate, root, eps;
  bool taken;  // the factor is finite
  uint32_t step;
};

__device__ __forceinline__ Step read_step(const StepShared &o) {
  Step s;
  s.f = o.factor ? *o.factor : 1.0f;
  s.taken = fabsf(s.f) < __builtin_inff();
  s.lr = o.lr;
  s.rate = o.rate;
  s.root = o.root;
  s.step = o.step;
  if (o.lr_device || o.step_device) {
    if (o.lr_device) s.lr = *o.lr_device;
    if (o.step_device) s.step = (uint32_t)max(1, *o.step_device);
    rates(s.lr, (double)s.step, o.log_b1, o.log_b2, &s.rate, &s.root);
  }
  s.eps = o.eps;
  return s;
}

// A parameter after its step; m and r = sqrt(v) are the new ones.
__device__ __forceinline__ float moved(const Step &s, float decay, float p, float m, float r) {
  return p - fmaf(decay, p, s.rate * m / fmaf(r, s.root, s.eps));
}

// LEN elements of a tile from place `at` on, and back.  A tile's array is the same
// in all lanes and a place the same in all tiles, so an address costs nothing; `left`
// elements of the tile are the tensor's, all of them where WHOLE.
template <typename T, int LEN>
struct Some {
  typedef T type __attribute__((ext_vector_type(LEN), aligned(sizeof(T))));
};

template <typename T, int LEN, bool WHOLE>
__device__ __forceinline__ void load_some(const T *tile, uint32_t at, uint32_t left, float *x) {
  if (WHOLE || at + LEN <= left) {
    const auto v = *reinterpret_cast<const typename Some<T, LEN>::type *>(tile + at);
#pragma unroll
    for (int j = 0; j < LEN; ++j) x[j] = (float)v[j];
  } else {
#pragma unroll
    for (int j = 0; j < LEN; ++j) x[j] = at + j < left ? (float)tile[at + j] : 0.0f;
  }
}

template <typename T, int LEN, bool WHOLE>
__device__ __forceinline__ void store_some(T *tile, uint32_t at, uint32_t left, const float *x) {
  if (WHOLE || at + LEN <= left) {
    typename Some<T, LEN>::type v;
#pragma unroll
    for (int j = 0; j < LEN; ++j) v[j] = narrow<T>(x[j]);
    *reinterpret_cast<typename Some<T, LEN>::type *>(tile + at) = v;
  } else {
#pragma unroll
    for (int j = 0; j < LEN; ++j)
      if (at + j < left) tile[at + j] = narrow<T>(x[j]);
  }
}

// The arrays of a tensor from element `first` on.
template <typename P, typename G, typename S>
struct Arrays {
  const P *param;
  const G *grad;
  const S *m, *v;
  P *param_out;
  S *m_out, *v_out;
  G *copy;  // or null
  __device__ __forceinline__ Arrays(const StepTable &t, int at, int64_t first)
      : param(static_cast<const P *>(t.param[at]) + first),
        grad(static_cast<const G *>(t.grad[at]) + first),
        m(static_cast<const S *>(t.m[at]) + first),
        v(static_cast<const S *>(t.v[at]) + first),
        param_out(static_cast<P *>(t.param_out[at]) + first),
        m_out(static_cast<S *>(t.m_out[at]) + first),
        v_out(static_cast<S *>(t.v_out[at]) + first),
        copy(t.copy[at] ? static_cast<G *>(t.copy[at]) + first : nullptr) {}
};

struct Rates {
  float b1, b2, a1, a2;  // a: 1 - b
};

template <typename P, typename G, bool WHOLE>
__device__ __forceinline__ void step_tile(const Arrays<P, G, float> &t, uint32_t left,
                                          const Step &s, const Rates &q, float decay) {
  constexpr int kLen = 4, kVecs = kTile / kThreads / kLen;
  float p[kVecs][kLen], g[kVecs][kLen], m[kVecs][kLen], v[kVecs][kLen];
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    const uint32_t at = threadIdx.x * kLen + k * kThreads * kLen;
    load_some<P, kLen, WHOLE>(t.param, at, left, p[k]);
    load_some<G, kLen, WHOLE>(t.grad, at, left, g[k]);
    load_some<float, kLen, WHOLE>(t.m, at, left, m[k]);
    load_some<float, kLen, WHOLE>(t.v, at, left, v[k]);
  }
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    const uint32_t at = threadIdx.x * kLen + k * kThreads * kLen;
    if (s.taken) {
#pragma unroll
      for (int j = 0; j < kLen; ++j) {
        const float gj = g[k][j] * s.f;
        m[k][j] = fmaf(q.b1, m[k][j], q.a1 * gj);
        v[k][j] = fmaf(q.b2, v[k][j], q.a2 * gj * gj);
        p[k][j] = moved(s, decay, p[k][j], m[k][j], sqrtf(v[k][j]));
      }
    }
    store_some<P, kLen, WHOLE>(t.param_out, at, left, p[k]);
    store_some<float, kLen, WHOLE>(t.m_out, at, left, m[k]);
    store_some<float, kLen, WHOLE>(t.v_out, at, left, v[k]);
    if (t.copy) store_some<G, kLen, WHOLE>(t.copy, at, left, p[k]);
  }
}

template <typename P, typename G>
__global__ __launch_bounds__(kThreads) void step_kernel(StepTable t, StepShared o) {
  const int at = find_tensor(t.first, o.count, blockIdx.x);
  const int64_t n = t.n[at];
  const Step s = read_step(o);
  const float decay = s.lr * t.decay[at];
  const Rates q = {(float)o.b1, (float)o.b2, (float)(1.0 - o.b1), (float)(1.0 - o.b2)};
  const int64_t tile0 = (int64_t)(blockIdx.x - t.first[at]) * o.tiles;
  for (int64_t tile = tile0; tile < tile0 + o.tiles && tile * kTile < n; ++tile) {
    const Arrays<P, G, float> a(t, at, tile * kTile);
    const int64_t left = n - tile * kTile;
    if (left >= kTile)
      step_tile<P, G, true>(a, kTile, s, q, decay);
    else
      step_tile<P, G, false>(a, (uint32_t)left, s, q, decay);
  }
}

// ---- states in 8 bits ----------------------------------------------------------------
//
// Half a wave holds a block of 256 elements, a lane 8 neighbouring ones, so the
// block's largest value is found without LDS.
//
// An e4m3 number is a float32 number 2^120 times as small without its last 20
// bits, denormals included; adding 20 random bits before they are cut off rounds up
// as often as the part cut off asks for.
//
// Every operation is float32's own, rounded once, as ml2.h says it: a state's codes
// are the same wherever they are worked out.  (Constants and products carried as sums
// of two numbers, so that little is rounded before the codes are, took 281 us for
// 134M bf16 elements against 250 and changed a code in two million.)

constexpr int kLane = 8;
static_assert(ML2_STATE_BLOCK == 32 * kLane, "half a wave holds a block");
constexpr float kTop = 448.0f;

typedef uint32_t Codes __attribute__((ext_vector_type(2), aligned(4)));

// 8 codes of a tile from place `at` on; 0 behind the tensor.
template <bool WHOLE>
__device__ __forceinline__ Codes load_codes(const uint8_t *tile, uint32_t at, uint32_t left) {
  if (WHOLE || at + kLane <= left) return *reinterpret_cast<const Codes *>(tile + at);
  Codes c = {0, 0};
#pragma unroll
  for (int j = 0; j < kLane; ++j)
    if (at + j < left) c[j >> 2] |= (uint32_t)tile[at + j] << (8 * (j & 3));
  return c;
}

template <bool WHOLE>
__device__ __forceinline__ void store_codes(uint8_t *tile, uint32_t at, uint32_t left, Codes c) {
  if (WHOLE || at + kLane <= left) {
    *reinterpret_cast<Codes *>(tile + at) = c;
  } else {
#pragma unroll
    for (int j = 0; j < kLane; ++j)
      if (at + j < left) tile[at + j] = (uint8_t)(c[j >> 2] >> (8 * (j & 3)));
  }
}

// The numbers that codes stand for, in units of their scale.
__device__ __forceinline__ void decode(Codes c, float (&x)[kLane]) {
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[w], true);
    x[4 * w] = lo[0];
    x[4 * w + 1] = lo[1];
    x[4 * w + 2] = hi[0];
    x[4 * w + 3] = hi[1];
  }
}

// A block's scale, and its reciprocal; `most`: the bits of the lane's largest size,
// ordered as the sizes are, NaN last.  A NaN or an infinity makes the scale NaN.
struct Scale {
  float scale, over;
};

__device__ __forceinline__ Scale block_scale(uint32_t most) {
  const float top = group_fold(__uint_as_float(most), 5, [](float a, float b) {
    return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
  });
  const float scale = fmaxf(top * (1.0f / kTop), 0x1p-100f);
  const float r = __builtin_amdgcn_rcpf(scale);  // and what it is off by
  const float over = fmaf(fmaf(-scale, r, 1.0f), r, r);
  return top < __builtin_inff() ? Scale{scale, over} : Scale{__builtin_nanf(""), 0.0f};
}

// The code of a size in units of its scale; random: 20 bits, least: the smallest
// code.
__device__ __forceinline__ uint32_t encode(float size, uint32_t random, uint32_t least) {
  const uint32_t code = (__float_as_uint(size * 0x1p-120f) + random) >> 20;
  return min(max(code, least), 0x7Eu);
}

// Scales of a tile's blocks, of m and of r: read and written.
struct Scales {
  const float *m, *r;
  float *m_out, *r_out;
};

template <typename P, typename G, bool WHOLE>
__device__ __forceinline__ void step8_tile(const Arrays<P, G, uint8_t> &t, const Scales &c,
                                           uint32_t left, const Step &s, const Rates &q,
                                           float decay, uint32_t key) {
  const uint32_t at = threadIdx.x * kLane, block = at / ML2_STATE_BLOCK;
  const bool in = WHOLE || block * ML2_STATE_BLOCK < left;  // the half wave, or none of it
  float p[kLane], g[kLane], m[kLane], r[kLane], ms = 0.0f, rs = 0.0f;
  load_some<P, kLane, WHOLE>(t.param, at, left, p);
  load_some<G, kLane, WHOLE>(t.grad, at, left, g);
  const Codes mc = load_codes<WHOLE>(t.m, at, left), rc = load_codes<WHOLE>(t.v, at, left);
  if (in) {
    ms = c.m[block];
    rs = c.r[block];
  }
  if (!s.taken) {
    store_some<P, kLane, WHOLE>(t.param_out, at, left, p);
    if (t.copy) store_some<G, kLane, WHOLE>(t.copy, at, left, p);
    store_codes<WHOLE>(t.m_out, at, left, mc);
    store_codes<WHOLE>(t.v_out, at, left, rc);
    if (in && (threadIdx.x & 31) == 0) {
      c.m_out[block] = ms;
      c.r_out[block] = rs;
    }
    return;
  }
  decode(mc, m);
  decode(rc, r);
#pragma unroll
  for (int j = 0; j < kLane; ++j) {
    const float gj = g[j] * s.f, old = r[j] * rs;
    m[j] = m[j] * ms * q.b1 + gj * q.a1;
    const float v = old * old * q.b2 + gj * q.a2 * gj;
    // The root from its reciprocal and what v lacks of its square, which the fused
    // operation finds exactly.  An infinite v gives an infinite root.
    const float y = __builtin_amdgcn_rsqf(__builtin_amdgcn_fmed3f(v, 0x1p-126f, 0x1.fffffep127f));
    const float root = v * y, lacks = fmaf(-root, root, v);
    r[j] = v < __builtin_inff() ? fmaf(lacks, 0.5f * y, root) : v;
    // A quotient by the reciprocal, which is off by at most its last place: the exact one
    // takes about ten instructions, and these bound the kernel.
    p[j] -= fmaf(decay, p[j],
                 s.rate * m[j] * __builtin_amdgcn_rcpf(fmaf(r[j], s.root, s.eps)));
    if (!WHOLE && at + j >= left) m[j] = r[j] = 0.0f;
  }
  store_some<P, kLane, WHOLE>(t.param_out, at, left, p);
  if (t.copy) store_some<G, kLane, WHOLE>(t.copy, at, left, p);
  uint32_t most_m = 0, most_r = 0;
#pragma unroll
  for (int j = 0; j < kLane; ++j) {
    most_m = max(most_m, __float_as_uint(m[j]) & 0x7FFFFFFFu);
    most_r = max(most_r, __float_as_uint(r[j]));
  }
  const Scale to_m = block_scale(most_m), to_r = block_scale(most_r);
  Codes mo = {0, 0}, ro = {0, 0};
#pragma unroll
  for (int j = 0; j < kLane; ++j) {
    uint32_t h = key + (at + (uint32_t)j) * kPhi;
    h = (h ^ (h >> 15)) * kPlastic;
    h ^= h >> 16;
    const uint32_t a = encode(fabsf(m[j]) * to_m.over, (h >> 12 & 0xFFFF0u) | 8u, 0);
    const uint32_t b = encode(r[j] * to_r.over, (h << 4 & 0xFFFF0u) | 8u,
                              min(__float_as_uint(r[j]), 1u));
    mo[j >> 2] |= (a | (__float_as_uint(m[j]) >> 24 & 0x80u)) << (8 * (j & 3));
    ro[j >> 2] |= b << (8 * (j & 3));
  }
  store_codes<WHOLE>(t.m_out, at, left, mo);
  store_codes<WHOLE>(t.v_out, at, left, ro);
  if (in && (threadIdx.x & 31) == 0) {
    c.m_out[block] = to_m.scale;
    c.r_out[block] = to_r.scale;
  }
}

template <typename P, typename G>
__global__ __launch_bounds__(kThreads) void step8_kernel(StepTable t, StepShared o) {
  const int at = find_tensor(t.first, o.count, blockIdx.x);
  const int64_t n = t.n[at];
  const Step s = read_step(o);
  const float decay = s.lr * t.decay[at];
  const Rates q = {(float)o.b1, (float)o.b2, (float)(1.0 - o.b1), (float)(1.0 - o.b2)};
  const uint32_t key = fold_word(fold_word(o.key, s.step), (uint32_t)(o.place + at));
  const int64_t codes = (n + ML2_STATE_BLOCK - 1) / ML2_STATE_BLOCK * ML2_STATE_BLOCK;
  const int64_t tile0 = (int64_t)(blockIdx.x - t.first[at]) * o.tiles;
  for (int64_t tile = tile0; tile < tile0 + o.tiles && tile * kTile < n; ++tile) {
    const int64_t first = tile * kTile, left = n - first;
    const Arrays<P, G, uint8_t> a(t, at, first);
    const auto scales = [&](void *state) {
      return reinterpret_cast<float *>(static_cast<uint8_t *>(state) + codes) +
             first / ML2_STATE_BLOCK;
    };
    const Scales c = {scales(t.m[at]), scales(t.v[at]), scales(t.m_out[at]), scales(t.v_out[at])};
    const uint32_t high = (uint32_t)(first >> 32);
    const uint32_t k = (high ? fold_word(key, high) : key) + (uint32_t)first * kPhi;
    if (left >= kTile)
      step8_tile<P, G, true>(a, c, kTile, s, q, decay, k);
    else
      step8_tile<P, G, false>(a, c, (uint32_t)left, s, q, decay, k);
  }
}

typedef void (*StepFn)(StepTable, StepShared);

template <typename P>
StepFn step_of(int grad_dtype, int bits) {
  if (grad_dtype == ML2_F32) return bits == 8 ? step8_kernel<P, float> : step_kernel<P, float>;
  if (grad_dtype == ML2_BF16) return bits == 8 ? step8_kernel<P, __bf16> : step_kernel<P, __bf16>;
  return bits == 8 ? step8_kernel<P, _Float16> : step_kernel<P, _Float16>;
}

}  // namespace

size_t grad_norm_workspace_bytes(const int64_t *sizes, int32_t count) {
  return (size_t)norm_parts(sizes, count, norm_chunk(sizes, count)) * sizeof(double);
}

hipError_t launch_grad_norm(int dtype, const void *const *grads, const int64_t *sizes,
                            int32_t count, float scale, float max_norm, float *norm,
                            float *factor, int32_t *step, void *ws, hipStream_t s) {
  const NormOut o = {scale, max_norm, norm, factor, step};
  double *part = static_cast<double *>(ws);
  if (dtype == ML2_F32) return launch_norm<float>(grads, sizes, count, o, part, s);
  if (dtype == ML2_BF16) return launch_norm<__bf16>(grads, sizes, count, o, part, s);
  return launch_norm<_Float16>(grads, sizes, count, o, part, s);
}

hipError_t launch_adamw(int param_dtype, int grad_dtype, int state_bits,
                        const ml2_adamw_tensor *tensors, int32_t count,
                        const ml2_adamw_options &o, hipStream_t s) {
  const StepFn fn = param_dtype == ML2_F32    ? step_of<float>(grad_dtype, state_bits)
                    : param_dtype == ML2_BF16 ? step_of<__bf16>(grad_dtype, state_bits)
                                              : step_of<_Float16>(grad_dtype, state_bits);
  StepTable t;
  StepShared c = {};
  c.log_b1 = log(o.beta1);
  c.log_b2 = log(o.beta2);
  c.lr_device = o.lr_device;
  c.step_device = o.step_device;
  c.factor = o.factor;
  c.lr = (float)o.lr;
  c.b1 = o.beta1;
  c.b2 = o.beta2;
  c.eps = (float)o.eps;
  c.step = (uint32_t)o.step;
  if (!o.step_device) rates(o.lr, (double)o.step, c.log_b1, c.log_b2, &c.rate, &c.root);
  c.key = fold_word(fold_word(0, (uint32_t)o.seed), (uint32_t)(o.seed >> 32));
  hipError_t e = hipSuccess;
  for (int32_t i0 = 0; i0 < count && e == hipSuccess; i0 += kTensors) {
    c.place = i0;
    c.count = std::min(count - i0, kTensors);
    int64_t tiles = 0;
    for (int32_t i = 0; i < c.count; ++i) tiles += (tensors[i0 + i].n + kTile - 1) / kTile;
    if (tiles == 0) continue;
    c.tiles = (tiles + kMostBlocks - 1) / kMostBlocks;
    uint32_t blocks = 0;
    for (int32_t i = 0; i < c.count; ++i) {
      const ml2_adamw_tensor &e = tensors[i0 + i];
      t.param[i] = e.param;
      t.grad[i] = e.grad;
      t.m[i] = e.m;
      t.v[i] = e.v;
      t.param_out[i] = e.param_out ? e.param_out : e.param;
      t.m_out[i] = e.m_out ? e.m_out : e.m;
      t.v_out[i] = e.v_out ? e.v_out : e.v;
      t.copy[i] = e.copy;
      t.n[i] = e.n;
      t.decay[i] = e.weight_decay;
      t.first[i] = blocks;
      blocks += (uint32_t)(((e.n + kTile - 1) / kTile + c.tiles - 1) / c.tiles);
    }
    fn<<<blocks, kThreads, 0, s>>>(t, c);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace ml2
