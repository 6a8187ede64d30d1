// C-ABI entry points of the operators of a training step: argument validation
// and the launches.
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "args.h"
#include "ml2_internal.h"
#include "train.h"

using ml2::aligned;
using ml2::element_size;
using ml2::fail;
using ml2::hip_fail;
using ml2::overlap;
using ml2::size_ok;

namespace {

constexpr int64_t kMostLd = (int64_t)1 << 32;
constexpr int64_t kMostElements = (int64_t)1 << 40;

// Bytes from `at` to `end`, or nothing.
struct Range {
  uintptr_t at, end;
};

Range range(const void *p, int64_t bytes) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return {at, p && bytes > 0 ? at + (uintptr_t)bytes : at};
}

bool meet(Range a, Range b) { return a.at < b.end && b.at < a.end && a.at < a.end && b.at < b.end; }

// Rows of `bytes` bytes, `pitch` bytes apart; what lies between them is not theirs.
struct Rows {
  uintptr_t at;
  uint64_t rows, bytes, pitch;
};

Rows matrix(const void *p, int64_t rows, int64_t width, int64_t ld, size_t size) {
  const bool any = p && rows > 0 && width > 0;
  return {reinterpret_cast<uintptr_t>(p), any ? (uint64_t)rows : 0, (uint64_t)width * size,
          (uint64_t)ld * size};
}

// The row in which b begins, or behind which, or else the next one.  No end of the
// matrix is worked out: with the largest sizes it lies beyond 64 bits.
bool meet(const Rows &a, Range b) {
  if (a.rows == 0 || b.at >= b.end || b.end <= a.at) return false;
  const uint64_t from = b.at > a.at ? b.at - a.at : 0, row = from / a.pitch, in = from % a.pitch;
  if (row >= a.rows) return false;
  return in < a.bytes || (row + 1 < a.rows && b.end - b.at > a.pitch - in);
}

bool same(Range a, Range b) { return a.at == b.at && a.end == b.end; }

// Whether matrix b, which is written, is neither a itself nor apart from it.
bool shares(const void *a, int64_t lda, const void *b, int64_t ldb, int64_t rows, int64_t width,
            size_t size) {
  if (a == b && (lda == ldb || rows <= 1)) return false;
  return overlap(a, lda, b, ldb, rows, width, size);
}

// What both calls of layer norm say of their rows and parameters.
ml2_status check_norm(const char *call, int32_t dtype, const void *x, int64_t rows, int64_t width,
                      int64_t ld, int32_t param_dtype, const void *weight, const void *bias,
                      size_t *size, size_t *param_size) {
  if (!element_size(dtype, size) || !element_size(param_dtype, param_size))
    return fail(ML2_ERR_INVALID_ARG, "%s: unknown dtype %d or param_dtype %d", call, dtype,
                param_dtype);
  if (param_dtype != dtype && param_dtype != ML2_F32)
    return fail(ML2_ERR_INVALID_ARG, "%s: param_dtype %d is neither dtype %d nor ML2_F32", call,
                param_dtype, dtype);
  if (!size_ok(rows) || !size_ok(width))
    return fail(ML2_ERR_INVALID_ARG, "%s: sizes out of range", call);
  if (width > ML2_MAX_WIDTH)
    return fail(ML2_ERR_UNSUPPORTED, "%s: width = %lld > %d", call, (long long)width,
                ML2_MAX_WIDTH);
  if (ld < width || ld > kMostLd)
    return fail(ML2_ERR_INVALID_ARG, "%s: ld = %lld, width = %lld", call, (long long)ld,
                (long long)width);
  if (rows > 0 && width > 0 && !x) return fail(ML2_ERR_INVALID_ARG, "%s: x is NULL", call);
  if (!aligned(x, *size) || !aligned(weight, *param_size) || !aligned(bias, *param_size))
    return fail(ML2_ERR_INVALID_ARG, "%s: an array is not aligned to its type", call);
  return ML2_OK;
}

}  // namespace

ml2_status ml2_layer_norm(int32_t dtype, const void *x, int64_t rows, int64_t width, int64_t ld,
                          int32_t param_dtype, const void *weight, const void *bias, float eps,
                          void *out, int64_t out_ld, float *mean, float *rstd, void *stream) {
  size_t size = 0, param_size = 0;
  ml2_status st = check_norm("ml2_layer_norm", dtype, x, rows, width, ld, param_dtype, weight, bias,
                             &size, &param_size);
  if (st != ML2_OK) return st;
  if (out_ld < width || out_ld > kMostLd)
    return fail(ML2_ERR_INVALID_ARG, "ml2_layer_norm: out_ld = %lld, width = %lld",
                (long long)out_ld, (long long)width);
  if (!(eps > 0.0f) || !isfinite(eps))
    return fail(ML2_ERR_INVALID_ARG, "ml2_layer_norm: eps = %g", (double)eps);
  if (rows > 0 && width > 0 && !out)
    return fail(ML2_ERR_INVALID_ARG, "ml2_layer_norm: out is NULL");
  if (!aligned(out, size) || !aligned(mean, 4) || !aligned(rstd, 4))
    return fail(ML2_ERR_INVALID_ARG, "ml2_layer_norm: an array is not aligned to its type");
  const Range params[2] = {range(weight, width * (int64_t)param_size),
                           range(bias, width * (int64_t)param_size)};
  const Rows in = matrix(x, rows, width, ld, size), to = matrix(out, rows, width, out_ld, size);
  const Range stats[2] = {range(mean, rows * 4), range(rstd, rows * 4)};
  bool bad = shares(x, ld, out, out_ld, rows, width, size) || meet(stats[0], stats[1]);
  for (const Range &p : params) bad = bad || meet(to, p) || meet(p, stats[0]) || meet(p, stats[1]);
  for (const Range &p : stats) bad = bad || meet(in, p) || meet(to, p);
  if (bad)
    return fail(ML2_ERR_INVALID_ARG, "ml2_layer_norm: out, mean or rstd shares memory with "
                "another array");
  if (rows == 0 || width == 0) return ML2_OK;
  int dev = 0;
  st = ml2::current_device(&dev);
  if (st != ML2_OK) return st;
  const ml2::NormArgs a = {x, rows, width, ld, weight, bias, param_dtype == ML2_F32, eps,
                           out, out_ld, mean, rstd};
  const hipError_t e =
      ml2::launch_layer_norm(dtype, a, ml2::cu_count(dev), static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ML2_OK : hip_fail(e, "ml2_layer_norm: kernel launch");
}

ml2_status ml2_layer_norm_grad_workspace_bytes(int64_t rows, int64_t width, size_t *bytes) {
  if (!bytes || !size_ok(rows) || !size_ok(width))
    return fail(ML2_ERR_INVALID_ARG, "ml2_layer_norm_grad_workspace_bytes: bytes is NULL or sizes "
                "out of range");
  if (width > ML2_MAX_WIDTH)
    return fail(ML2_ERR_UNSUPPORTED, "ml2_layer_norm_grad_workspace_bytes: width = %lld > %d",
                (long long)width, ML2_MAX_WIDTH);
  *bytes = ml2::layer_norm_grad_workspace_bytes(rows, width);
  return ML2_OK;
}

ml2_status ml2_layer_norm_grad(int32_t dtype, const void *x, int64_t rows, int64_t width,
                               int64_t ld, const void *dout, int64_t dout_ld, int32_t param_dtype,
                               const void *weight, const float *mean, const float *rstd, void *dx,
                               int64_t dx_ld, int32_t grad_dtype, void *dweight, void *dbias,
                               void *workspace, size_t workspace_bytes, void *stream) {
  const char *call = "ml2_layer_norm_grad";
  size_t size = 0, param_size = 0, grad_size = 0;
  ml2_status st = check_norm(call, dtype, x, rows, width, ld, param_dtype, weight, nullptr, &size,
                             &param_size);
  if (st != ML2_OK) return st;
  if (!element_size(grad_dtype, &grad_size) || (grad_dtype != dtype && grad_dtype != ML2_F32))
    return fail(ML2_ERR_INVALID_ARG, "%s: grad_dtype %d is neither dtype %d nor ML2_F32", call,
                grad_dtype, dtype);
  if (dout_ld < width || dout_ld > kMostLd || (dx && (dx_ld < width || dx_ld > kMostLd)))
    return fail(ML2_ERR_INVALID_ARG, "%s: dout_ld = %lld, dx_ld = %lld, width = %lld", call,
                (long long)dout_ld, (long long)dx_ld, (long long)width);
  if (rows > 0 && width > 0 && (!dout || !mean || !rstd))
    return fail(ML2_ERR_INVALID_ARG, "%s: NULL dout, mean or rstd", call);
  if (!aligned(dout, size) || !aligned(dx, size) || !aligned(mean, 4) || !aligned(rstd, 4) ||
      !aligned(dweight, grad_size) || !aligned(dbias, grad_size))
    return fail(ML2_ERR_INVALID_ARG, "%s: an array is not aligned to its type", call);
  if (!workspace || !aligned(workspace, 256))
    return fail(ML2_ERR_INVALID_ARG, "%s: workspace is NULL or not 256-byte aligned", call);
  const size_t need = ml2::layer_norm_grad_workspace_bytes(rows, width);
  if (workspace_bytes < need)
    return fail(ML2_ERR_INVALID_ARG, "%s: workspace %zu < %zu bytes", call, workspace_bytes, need);
  const Rows in[2] = {matrix(x, rows, width, ld, size), matrix(dout, rows, width, dout_ld, size)};
  const Range read[3] = {range(weight, width * (int64_t)param_size), range(mean, rows * 4),
                         range(rstd, rows * 4)};
  const Range ws = range(workspace, (int64_t)need);
  const Rows to = matrix(dx, rows, width, dx_ld, size);
  const Range sums[2] = {range(dweight, width * (int64_t)grad_size),
                         range(dbias, width * (int64_t)grad_size)};
  bool bad = dx && (shares(x, ld, dx, dx_ld, rows, width, size) ||
                    shares(dout, dout_ld, dx, dx_ld, rows, width, size));
  bad = bad || meet(to, ws) || meet(sums[0], sums[1]);
  for (const Range &q : sums) {
    bad = bad || meet(q, ws) || meet(to, q);
    for (const Rows &p : in) bad = bad || meet(p, q);
    for (const Range &p : read) bad = bad || meet(p, q);
  }
  for (const Rows &p : in) bad = bad || meet(p, ws);
  for (const Range &p : read) bad = bad || meet(p, ws) || meet(to, p);
  if (bad)
    return fail(ML2_ERR_INVALID_ARG, "%s: dx, dweight, dbias or workspace shares memory with "
                "another array", call);
  if (width == 0 || (!dweight && !dbias && (!dx || rows == 0))) return ML2_OK;
  const ml2::NormGradArgs a = {x, rows, width, ld, dout, dout_ld, weight, param_dtype == ML2_F32,
                               mean, rstd, dx, dx_ld, dweight, dbias, grad_dtype};
  const hipError_t e =
      ml2::launch_layer_norm_grad(dtype, a, workspace, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ML2_OK : hip_fail(e, "ml2_layer_norm_grad: kernel launch");
}

static ml2_status check_sizes(const char *call, const int64_t *sizes, int32_t count) {
  if (count < 0 || (count > 0 && !sizes))
    return fail(ML2_ERR_INVALID_ARG, "%s: count = %d or sizes is NULL", call, count);
  if (count > ML2_MAX_TENSORS)
    return fail(ML2_ERR_UNSUPPORTED, "%s: count = %d > %d", call, count, ML2_MAX_TENSORS);
  for (int32_t i = 0; i < count; ++i) {
    if (sizes[i] < 0)
      return fail(ML2_ERR_INVALID_ARG, "%s: sizes[%d] = %lld", call, i, (long long)sizes[i]);
    if (sizes[i] > kMostElements)
      return fail(ML2_ERR_UNSUPPORTED, "%s: sizes[%d] = %lld", call, i, (long long)sizes[i]);
  }
  return ML2_OK;
}

ml2_status ml2_grad_norm_workspace_bytes(const int64_t *sizes, int32_t count, size_t *bytes) {
  if (!bytes) return fail(ML2_ERR_INVALID_ARG, "ml2_grad_norm_workspace_bytes: bytes is NULL");
  const ml2_status st = check_sizes("ml2_grad_norm_workspace_bytes", sizes, count);
  if (st == ML2_OK) *bytes = ml2::grad_norm_workspace_bytes(sizes, count);
  return st;
}

ml2_status ml2_grad_norm(int32_t dtype, const void *const *grads, const int64_t *sizes,
                         int32_t count, float scale, float max_norm, float *norm, float *factor,
                         int32_t *step, void *workspace, size_t workspace_bytes, void *stream) {
  const char *call = "ml2_grad_norm";
  size_t size = 0;
  if (!element_size(dtype, &size))
    return fail(ML2_ERR_INVALID_ARG, "%s: unknown dtype %d", call, dtype);
  const ml2_status st = check_sizes(call, sizes, count);
  if (st != ML2_OK) return st;
  if (count > 0 && !grads) return fail(ML2_ERR_INVALID_ARG, "%s: grads is NULL", call);
  if (!(scale > 0.0f) || !isfinite(scale) || !(max_norm > 0.0f))
    return fail(ML2_ERR_INVALID_ARG, "%s: scale = %g, max_norm = %g", call, (double)scale,
                (double)max_norm);
  if (!aligned(norm, 4) || !aligned(factor, 4) || !aligned(step, 4))
    return fail(ML2_ERR_INVALID_ARG, "%s: an array is not aligned to its type", call);
  if (!workspace || !aligned(workspace, 256))
    return fail(ML2_ERR_INVALID_ARG, "%s: workspace is NULL or not 256-byte aligned", call);
  const size_t need = ml2::grad_norm_workspace_bytes(sizes, count);
  if (workspace_bytes < need)
    return fail(ML2_ERR_INVALID_ARG, "%s: workspace %zu < %zu bytes", call, workspace_bytes, need);
  const Range to[4] = {range(norm, 4), range(factor, 4), range(step, 4),
                       range(workspace, (int64_t)need)};
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < i; ++j)
      if (meet(to[i], to[j]))
        return fail(ML2_ERR_INVALID_ARG, "%s: norm, factor, step or workspace share memory", call);
  for (int32_t i = 0; i < count; ++i) {
    if (sizes[i] > 0 && (!grads[i] || !aligned(grads[i], size)))
      return fail(ML2_ERR_INVALID_ARG, "%s: grads[%d] is NULL or not aligned to its type", call, i);
    for (const Range &r : to)
      if (meet(r, range(grads[i], sizes[i] * (int64_t)size)))
        return fail(ML2_ERR_INVALID_ARG, "%s: grads[%d] shares memory with what is written", call,
                    i);
  }
  if (!norm && !factor && !step) return ML2_OK;
  const hipError_t e = ml2::launch_grad_norm(dtype, grads, sizes, count, scale, max_norm, norm,
                                             factor, step, workspace,
                                             static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ML2_OK : hip_fail(e, "ml2_grad_norm: kernel launch");
}

// Bytes of m or v.
static int64_t state_bytes(int32_t bits, int64_t n) {
  const int64_t blocks = (n + ML2_STATE_BLOCK - 1) / ML2_STATE_BLOCK;
  return bits == 32 ? 4 * n : blocks * (ML2_STATE_BLOCK + 4);
}

ml2_status ml2_adamw_state_bytes(int32_t state_bits, int64_t n, size_t *bytes) {
  if (!bytes || n < 0 || (state_bits != 8 && state_bits != 32))
    return fail(ML2_ERR_INVALID_ARG, "ml2_adamw_state_bytes: state_bits = %d, n = %lld or bytes is "
                "NULL", state_bits, (long long)n);
  if (n > kMostElements)
    return fail(ML2_ERR_UNSUPPORTED, "ml2_adamw_state_bytes: n = %lld", (long long)n);
  *bytes = (size_t)state_bytes(state_bits, n);
  return ML2_OK;
}

namespace {

// The arrays of a tensor: what is read, and what is written in its place.
struct Arrays {
  Range in[4], out[4];  // param, m, v, grad; param_out, m_out, v_out, copy
};

Arrays arrays(const ml2_adamw_tensor &t, size_t param_size, size_t grad_size, int32_t bits) {
  const int64_t p = t.n * (int64_t)param_size, g = t.n * (int64_t)grad_size;
  const int64_t s = state_bytes(bits, t.n);
  return {{range(t.param, p), range(t.m, s), range(t.v, s), range(t.grad, g)},
          {range(t.param_out ? t.param_out : t.param, p), range(t.m_out ? t.m_out : t.m, s),
           range(t.v_out ? t.v_out : t.v, s), range(t.copy, g)}};
}

// The ranges of a list that are not empty, in order.  Tensors mostly lie in the order
// in which they were made, then nothing is sorted.
void put_in_order(std::vector<Range> *list, size_t from) {
  const auto before = [](Range a, Range b) { return a.at < b.at; };
  const auto begin = list->begin(), middle = begin + (ptrdiff_t)from, end = list->end();
  if (!std::is_sorted(middle, end, before)) std::sort(middle, end, before);
  std::inplace_merge(begin, middle, end, before);
}

// Whether nothing that is written shares memory with anything but its own input.
bool apart(const ml2_adamw_tensor *tensors, int32_t count, size_t param_size, size_t grad_size,
           int32_t bits) {
  std::vector<Range> written, read;
  written.reserve(4 * (size_t)count);
  for (int q = 0; q < 4; ++q) {
    const size_t w0 = written.size(), r0 = read.size();
    for (int32_t i = 0; i < count; ++i) {
      const Arrays a = arrays(tensors[i], param_size, grad_size, bits);
      if (a.out[q].at < a.out[q].end) written.push_back(a.out[q]);
      if (a.in[q].at < a.in[q].end && (q == 3 || !same(a.in[q], a.out[q])))
        read.push_back(a.in[q]);
    }
    put_in_order(&written, w0);
    put_in_order(&read, r0);
  }
  for (size_t i = 1; i < written.size(); ++i)
    if (written[i].at < written[i - 1].end) return false;
  // The written ones are apart, so their ends are in order too: the first that ends
  // behind the beginning of a read one is the only one it can meet first.
  size_t w = 0;
  for (const Range &r : read) {
    while (w < written.size() && written[w].end <= r.at) ++w;
    if (w < written.size() && written[w].at < r.end) return false;
  }
  return true;
}

}  // namespace

ml2_status ml2_adamw(int32_t param_dtype, int32_t grad_dtype, int32_t state_bits,
                     const ml2_adamw_tensor *tensors, int32_t count,
                     const ml2_adamw_options *options, void *stream) {
  const char *call = "ml2_adamw";
  size_t param_size = 0, grad_size = 0;
  if (!element_size(param_dtype, &param_size) || !element_size(grad_dtype, &grad_size))
    return fail(ML2_ERR_INVALID_ARG, "%s: unknown param_dtype %d or grad_dtype %d", call,
                param_dtype, grad_dtype);
  if (state_bits != 8 && state_bits != 32)
    return fail(ML2_ERR_INVALID_ARG, "%s: state_bits = %d is neither 8 nor 32", call, state_bits);
  if (count < 0 || (count > 0 && !tensors) || !options)
    return fail(ML2_ERR_INVALID_ARG, "%s: count = %d, or NULL tensors or options", call, count);
  if (count > ML2_MAX_TENSORS)
    return fail(ML2_ERR_UNSUPPORTED, "%s: count = %d > %d", call, count, ML2_MAX_TENSORS);
  const ml2_adamw_options &o = *options;
  if (!(o.beta1 >= 0.0 && o.beta1 < 1.0) || !(o.beta2 >= 0.0 && o.beta2 < 1.0) ||
      !((float)o.eps >= 0x1p-126f) || !isfinite((float)o.eps) || !isfinite((float)o.lr))
    return fail(ML2_ERR_INVALID_ARG, "%s: lr = %g, beta1 = %g, beta2 = %g, eps = %g", call, o.lr,
                o.beta1, o.beta2, o.eps);
  if (!o.step_device && (o.step < 1 || o.step > (int64_t)INT32_MAX))
    return fail(ML2_ERR_INVALID_ARG, "%s: step = %lld", call, (long long)o.step);
  if (!aligned(o.lr_device, 4) || !aligned(o.step_device, 4) || !aligned(o.factor, 4))
    return fail(ML2_ERR_INVALID_ARG, "%s: an option is not aligned to its type", call);
  const size_t state_align = 4;
  for (int32_t i = 0; i < count; ++i) {
    const ml2_adamw_tensor &t = tensors[i];
    if (t.n < 0) return fail(ML2_ERR_INVALID_ARG, "%s: n[%d] = %lld", call, i, (long long)t.n);
    if (t.n > kMostElements)
      return fail(ML2_ERR_UNSUPPORTED, "%s: n[%d] = %lld", call, i, (long long)t.n);
    if (!isfinite(t.weight_decay))
      return fail(ML2_ERR_INVALID_ARG, "%s: weight_decay[%d] = %g", call, i,
                  (double)t.weight_decay);
    if (t.n == 0) continue;
    if (!t.param || !t.grad || !t.m || !t.v)
      return fail(ML2_ERR_INVALID_ARG, "%s: tensor %d: NULL param, grad, m or v", call, i);
    if (!aligned(t.param, param_size) || !aligned(t.param_out, param_size) ||
        !aligned(t.grad, grad_size) || !aligned(t.copy, grad_size) || !aligned(t.m, state_align) ||
        !aligned(t.v, state_align) || !aligned(t.m_out, state_align) ||
        !aligned(t.v_out, state_align))
      return fail(ML2_ERR_INVALID_ARG, "%s: tensor %d: an array is not aligned to its type", call,
                  i);
    const Arrays a = arrays(t, param_size, grad_size, state_bits);
    for (const Range &r : a.out)
      if (meet(r, range(o.lr_device, 4)) || meet(r, range(o.step_device, 4)) ||
          meet(r, range(o.factor, 4)))
        return fail(ML2_ERR_INVALID_ARG, "%s: tensor %d shares memory with an option", call, i);
  }
  try {
    if (!apart(tensors, count, param_size, grad_size, state_bits))
      return fail(ML2_ERR_INVALID_ARG, "%s: arrays that are written share memory with others",
                  call);
  } catch (const std::bad_alloc &) {
    return fail(ML2_ERR_OUT_OF_MEMORY, "%s: no host memory", call);
  }
  const hipError_t e = ml2::launch_adamw(param_dtype, grad_dtype, state_bits, tensors, count, o,
                                         static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ML2_OK : hip_fail(e, "ml2_adamw: kernel launch");
}
