// Log-probabilities of given entries of rows of scores under the masked
// softmax, and the gradient of their weighted sum.
//
//   z_i = (s_i - m) * R,  l = sum_i exp(z_i)
//   logprob_j = z_{t_j} - log l
//   grad_i = R * (sum_{j: t_j = i} w_j - exp(z_i) / l * sum_j w_j)
//
// A row is cut into chunks.  stats_kernel reads a chunk once and keeps a
// running maximum and sum (of exp of differences to that maximum); finish and
// grad join the chunks' pairs in chunk order, so every workgroup of a row
// arrives at the same m and l.  Weights are joined in the order of j.
#include <algorithm>

#include "draw.h"

namespace ml2 {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504088896340736f;

struct Stat {
  float m, l;  // maximum of the included scores, sum of exp((s - m) * R)
};

// exp(y * ln 2) of a difference to the maximum.  Where maximum and score are
// both infinite their difference is NaN and the entry counts as the maximum.
__device__ __forceinline__ float weight_of(float x, float m, float c) {
  return fminf(__builtin_amdgcn_exp2f((x - m) * c), 1.0f);
}

__device__ __forceinline__ Stat join(Stat a, Stat b, float c) {
  const float ninf = -__builtin_inff();
  if (b.m == ninf) return a;
  if (a.m == ninf) return b;
  const float m = fmaxf(a.m, b.m);
  return {m, a.l * weight_of(a.m, m, c) + b.l * weight_of(b.m, m, c)};
}

// The workgroup's pairs joined (in thread order pairs of a tree); the result
// in every thread.
__device__ __forceinline__ Stat block_join(Stat s, float c, Stat *lds) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Stat o = {__shfl_xor(s.m, d), __shfl_xor(s.l, d)};
    s = (threadIdx.x & d) ? join(o, s, c) : join(s, o, c);
  }
  const int waves = blockDim.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  s = lds[0];
  for (int w = 1; w < waves; ++w) s = join(s, lds[w], c);
  return s;
}

struct Rows {
  LogprobArgs a;
  Stat *part;      // [rows][chunks]
  int64_t chunk;   // entries of a chunk
  int64_t chunks;
};

template <typename T>
__device__ __forceinline__ float load_score(const Rows &k, int64_t row, int64_t i) {
  const T *s = static_cast<const T *>(k.a.s.scores) + row * k.a.s.ld;
  const bool ok = !k.a.s.valid || k.a.s.valid[row * k.a.s.valid_ld + i] != 0;
  return included((float)s[i], ok);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void stats_kernel(Rows k) {
  __shared__ Stat lds[kThreads / 64];
  const int64_t row = blockIdx.x / k.chunks, chunk = blockIdx.x % k.chunks;
  const int64_t lo = chunk * k.chunk, hi = min(k.a.s.n, lo + k.chunk);
  bool greedy;
  const float c = inverse_temperature(k.a.s.temperature, row, &greedy) * kLog2e;
  Stat s = {-__builtin_inff(), 0.0f};
  for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
    const float x = load_score<T>(k, row, i);
    if (x == -__builtin_inff()) continue;
    if (x > s.m) {
      s.l = s.m == -__builtin_inff() ? 0.0f : s.l * weight_of(s.m, x, c);
      s.m = x;
    }
    s.l += weight_of(x, s.m, c);
  }
  s = block_join(s, c, lds);
  if (threadIdx.x == 0) k.part[blockIdx.x] = s;
}

// The row's maximum and sum, in every thread.
__device__ __forceinline__ Stat row_stat(const Rows &k, int64_t row, float c, Stat *lds) {
  Stat s = {-__builtin_inff(), 0.0f};
  for (int64_t i = threadIdx.x; i < k.chunks; i += blockDim.x)
    s = join(s, k.part[row * k.chunks + i], c);
  return block_join(s, c, lds);
}

template <typename T>
__device__ __forceinline__ float target_logprob(const Rows &k, int64_t row, int64_t t, Stat st,
                                                float r) {
  if (t < 0 || t >= k.a.s.n) return 0.0f;
  const float x = load_score<T>(k, row, t);
  if (x == -__builtin_inff()) return x;
  return (x == st.m ? 0.0f : (x - st.m) * r) - logf(st.l);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void finish_kernel(Rows k) {
  __shared__ Stat lds[kThreads / 64];
  const int64_t row = blockIdx.x;
  bool greedy;
  const float r = inverse_temperature(k.a.s.temperature, row, &greedy);
  const Stat st = row_stat(k, row, r * kLog2e, lds);
  for (int j = threadIdx.x; j < k.a.per_row; j += kThreads) {
    const int64_t at = row * k.a.per_row + j;
    k.a.logprob[at] = target_logprob<T>(k, row, k.a.targets[at], st, r);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void grad_kernel(Rows k) {
  __shared__ Stat lds[kThreads / 64];
  __shared__ float wsum[kThreads];
  const int64_t row = blockIdx.x / k.chunks, chunk = blockIdx.x % k.chunks;
  const int64_t lo = chunk * k.chunk, hi = min(k.a.s.n, lo + k.chunk);
  bool greedy;
  const float r = inverse_temperature(k.a.s.temperature, row, &greedy), c = r * kLog2e;
  const Stat st = row_stat(k, row, c, lds);
  // The row's weights, summed in an order that every workgroup shares.
  const int32_t *targets = k.a.targets + row * k.a.per_row;
  const float *weight = k.a.weight + row * k.a.per_row;
  float w = 0.0f;
  for (int j = threadIdx.x; j < k.a.per_row; j += kThreads) {
    const float lp = target_logprob<T>(k, row, targets[j], st, r);
    if (chunk == 0 && k.a.logprob) k.a.logprob[row * k.a.per_row + j] = lp;
    const int64_t t = targets[j];
    if (t >= 0 && t < k.a.s.n && load_score<T>(k, row, t) != -__builtin_inff()) w += weight[j];
  }
  wsum[threadIdx.x] = w;
  __syncthreads();
  for (int d = kThreads / 2; d > 0; d >>= 1) {
    if ((int)threadIdx.x < d) wsum[threadIdx.x] += wsum[threadIdx.x + d];
    __syncthreads();
  }
  const float scale = -wsum[0] / st.l;
  T *grad = static_cast<T *>(k.a.grad) + row * k.a.grad_ld;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
    const float x = load_score<T>(k, row, i);
    grad[i] = narrow<T>(x == -__builtin_inff() ? 0.0f : weight_of(x, st.m, c) * scale * r);
  }
  __syncthreads();
  // The targets of this chunk: the first of those that name an entry adds up
  // the weights of all of them.
  for (int j = threadIdx.x; j < k.a.per_row; j += kThreads) {
    const int64_t t = targets[j];
    if (t < lo || t >= hi) continue;
    const float x = load_score<T>(k, row, t);
    if (x == -__builtin_inff()) continue;
    bool first = true;
    for (int q = 0; q < j && first; ++q) first = targets[q] != t;
    if (!first) continue;
    float sum = weight[j];
    for (int q = j + 1; q < k.a.per_row; ++q)
      if (targets[q] == t) sum += weight[q];
    grad[t] = narrow<T>((weight_of(x, st.m, c) * scale + sum) * r);
  }
}

// Chunks of a row: enough workgroups for the device where rows are few, none
// of them over fewer than 4,096 entries.
void cut(int64_t n, int64_t rows, int cu_count, int64_t *chunk, int64_t *chunks) {
  const int64_t want = std::max<int64_t>(1, (int64_t)cu_count * 4 / std::max<int64_t>(1, rows));
  const int64_t most = std::max<int64_t>(1, (n + 4095) / 4096);
  const int64_t c = std::min(want, most);
  *chunk = std::max<int64_t>(1, ((n + c - 1) / c + 63) / 64 * 64);
  *chunks = std::max<int64_t>(1, (n + *chunk - 1) / *chunk);
}

template <typename T>
hipError_t launch(const LogprobArgs &a, void *ws, int cu_count, hipStream_t s) {
  Rows k{};
  k.a = a;
  k.part = static_cast<Stat *>(ws);
  cut(a.s.n, a.s.rows, cu_count, &k.chunk, &k.chunks);
  const uint32_t grid = (uint32_t)(a.s.rows * k.chunks);
  stats_kernel<T><<<grid, kThreads, 0, s>>>(k);
  if (a.grad)
    grad_kernel<T><<<grid, kThreads, 0, s>>>(k);
  else
    finish_kernel<T><<<(uint32_t)a.s.rows, kThreads, 0, s>>>(k);
  return hipGetLastError();
}

}  // namespace

size_t logprob_workspace_bytes(int64_t n, int64_t rows, int32_t per_row) {
  (void)per_row;
  // chunks: at most 4 workgroups a CU (of at most 1,024 CUs), or one a row
  const int64_t chunks = std::max<int64_t>(1, 4096 / std::max<int64_t>(1, rows));
  (void)n;
  return std::max<size_t>(256, (size_t)rows * chunks * sizeof(Stat));
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
