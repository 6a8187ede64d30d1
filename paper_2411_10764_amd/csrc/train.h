// Shared by the operators of a training step (norm_kernels, adamw_kernels):
// launch arguments and the sums that they take over lanes.
#pragma once

#include "draw.h"

namespace ml2 {

struct NormArgs {
  const void *x;
  int64_t rows, width, ld;
  const void *weight, *bias;  // or null
  int param_f32;              // their type: float32, else that of x
  float eps;
  void *out;
  int64_t out_ld;
  float *mean, *rstd;         // or null
};

struct NormGradArgs {
  const void *x;
  int64_t rows, width, ld;
  const void *dout;
  int64_t dout_ld;
  const void *weight;  // or null
  int param_f32;
  const float *mean, *rstd;
  void *dx;            // or null, as the next two
  int64_t dx_ld;
  void *dweight, *dbias;
  int grad_dtype;
};

hipError_t launch_layer_norm(int dtype, const NormArgs &a, int cu_count, hipStream_t s);
size_t layer_norm_grad_workspace_bytes(int64_t rows, int64_t width);
hipError_t launch_layer_norm_grad(int dtype, const NormGradArgs &a, void *ws, hipStream_t s);

size_t grad_norm_workspace_bytes(const int64_t *sizes, int32_t count);
hipError_t launch_grad_norm(int dtype, const void *const *grads, const int64_t *sizes,
                            int32_t count, float scale, float max_norm, float *norm,
                            float *factor, int32_t *step, void *ws, hipStream_t s);
hipError_t launch_adamw(int param_dtype, int grad_dtype, int state_bits,
                        const ml2_adamw_tensor *tensors, int32_t count,
                        const ml2_adamw_options &o, hipStream_t s);

// ---- device helpers ---------------------------------------------------------

// The value of the lane that the DPP control names (every lane has one).
template <int CTRL>
__device__ __forceinline__ float lane_swap(float v) {
  return __uint_as_float(
      (uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}

// v of the own half of 32 lanes (of the own row of 16) joined with the other's,
// in every lane; the lower one's comes first.
template <typename F>
__device__ __forceinline__ float join_halves(float v, F f) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <typename F>
__device__ __forceinline__ float join_rows(float v, F f) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// v folded over groups of 2^log_g neighbouring lanes (log_g <= 6, the same in
// every lane), in every lane of the group.  f must not care for the order of its
// two operands, so all lanes arrive at the same bits.
template <typename F>
__device__ __forceinline__ float group_fold(float v, int log_g, F f) {
  if (log_g >= 1) v = f(v, lane_swap<0xB1>(v));   // quad_perm 1 0 3 2
  if (log_g >= 2) v = f(v, lane_swap<0x4E>(v));   // quad_perm 2 3 0 1
  if (log_g >= 3) v = f(v, lane_swap<0x141>(v));  // row_half_mirror
  if (log_g >= 4) v = f(v, lane_swap<0x140>(v));  // row_mirror
  if (log_g >= 5) v = join_rows(v, f);
  if (log_g >= 6) v = join_halves(v, f);
  return v;
}

// N numbers summed over such groups: one decision a step where log_g is not known when
// this is compiled, and the steps of one sum between those of another.
template <int N>
__device__ __forceinline__ void group_sums(float (&v)[N], int log_g) {
  const auto add = [](float a, float b) { return a + b; };
  const auto step = [&](auto f) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = f(v[i]);
  };
  if (log_g >= 1) step([](float x) { return x + lane_swap<0xB1>(x); });
  if (log_g >= 2) step([](float x) { return x + lane_swap<0x4E>(x); });
  if (log_g >= 3) step([](float x) { return x + lane_swap<0x141>(x); });
  if (log_g >= 4) step([](float x) { return x + lane_swap<0x140>(x); });
  if (log_g >= 5) step([&](float x) { return join_rows(x, add); });
  if (log_g >= 6) step([&](float x) { return join_halves(x, add); });
}

// Elements c .. c + kLen - 1 of a row of `width`, zeros outside.
template <typename T>
__device__ __forceinline__ void load_floats(const T *row, int64_t c, int64_t width, float *x) {
  constexpr int kLen = Vec<T>::kLen;
  if (c + kLen <= width) {
    const typename Vec<T>::type v = *reinterpret_cast<const typename Vec<T>::type *>(row + c);
#pragma unroll
    for (int j = 0; j < kLen; ++j) x[j] = (float)v[j];
  } else {
#pragma unroll
    for (int j = 0; j < kLen; ++j) x[j] = c + j < width ? (float)row[c + j] : 0.0f;
  }
}

}  // namespace ml2
