// C-ABI entry points of the operators over rows of scores and over tables:
// argument validation and the launches.
#include "draw.h"
#include "ml2_internal.h"

using ml2::fail;
using ml2::hip_fail;

namespace {

bool element_size(int32_t dtype, size_t *size) {
  if (dtype != ML2_F32 && dtype != ML2_BF16 && dtype != ML2_F16) return false;
  *size = dtype == ML2_F32 ? 4 : 2;
  return true;
}

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bool size_ok(int64_t v) { return v >= 0 && v <= (int64_t)INT32_MAX; }

ml2_status check_rows(const char *call, int32_t dtype, const ml2::ScoreRows &s, int32_t per_row,
                      const void *ws, size_t ws_bytes, size_t need) {
  size_t size = 0;
  if (!element_size(dtype, &size))
    return fail(ML2_ERR_INVALID_ARG, "%s: unknown dtype %d", call, dtype);
  if (!size_ok(s.n) || !size_ok(s.rows) || per_row < 0)
    return fail(ML2_ERR_INVALID_ARG, "%s: n = %lld, rows = %lld or %d per row out of range", call,
                (long long)s.n, (long long)s.rows, per_row);
  if (per_row > ML2_MAX_TOPK)
    return fail(ML2_ERR_UNSUPPORTED, "%s: %d per row > %d", call, per_row, ML2_MAX_TOPK);
  if (s.rows > ML2_MAX_ROWS)
    return fail(ML2_ERR_UNSUPPORTED, "%s: rows = %lld > %d", call, (long long)s.rows,
                ML2_MAX_ROWS);
  if (s.ld < s.n || s.ld > (int64_t)1 << 40)
    return fail(ML2_ERR_INVALID_ARG, "%s: ld = %lld, n = %lld", call, (long long)s.ld,
                (long long)s.n);
  if (s.rows > 0 && s.n > 0 && !s.scores)
    return fail(ML2_ERR_INVALID_ARG, "%s: scores is NULL", call);
  if (!aligned(s.scores, size))
    return fail(ML2_ERR_INVALID_ARG, "%s: scores are not aligned to their type", call);
  if (s.valid && s.valid_ld != 0 && (s.valid_ld < s.n || s.valid_ld > (int64_t)1 << 40))
    return fail(ML2_ERR_INVALID_ARG, "%s: valid_ld = %lld, n = %lld", call,
                (long long)s.valid_ld, (long long)s.n);
  if (!ws || !aligned(ws, 256))
    return fail(ML2_ERR_INVALID_ARG, "%s: workspace is NULL or not 256-byte aligned", call);
  if (ws_bytes < need)
    return fail(ML2_ERR_INVALID_ARG, "%s: workspace %zu < %zu bytes", call, ws_bytes, need);
  return ML2_OK;
}

// Whether two matrices of `rows` rows of n elements of `size` bytes, lda and ldb
// elements apart and aligned to their elements, have one in common.  Columns of
// one buffer lie between one another without that.
bool overlap(const void *a, int64_t lda, const void *b, int64_t ldb, int64_t rows, int64_t n,
             size_t size) {
  if (!a || !b || rows <= 0 || n <= 0) return false;
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
  if (pa > pb) return overlap(b, ldb, a, lda, rows, n, size);
  const uint64_t d = (pb - pa) / size;  // b's first element, counted from a's
  const uint64_t la = (uint64_t)lda, lb = (uint64_t)ldb, len = (uint64_t)n;
  if (d >= (uint64_t)(rows - 1) * la + len) return false;
  if (la == lb) {
    // row r of b begins in row r + d / la of a, or behind its end and reaches on
    // into the next
    const uint64_t at = d % la, row = d / la;
    return at < len || (row + 1 < (uint64_t)rows && at + len > la);
  }
  for (uint64_t i = 0, j = 0; i < (uint64_t)rows && j < (uint64_t)rows;) {
    const uint64_t x = i * la, y = d + j * lb;
    if (x < y + len && y < x + len) return true;
    if (x < y) ++i; else ++j;
  }
  return false;
}

// n, rows and per_row of a workspace query.
ml2_status check_sizes(const char *call, int64_t n, int64_t rows, int32_t per_row,
                       const size_t *bytes) {
  if (!bytes) return fail(ML2_ERR_INVALID_ARG, "%s: bytes is NULL", call);
  if (!size_ok(n) || !size_ok(rows) || per_row < 0)
    return fail(ML2_ERR_INVALID_ARG, "%s: sizes out of range", call);
  if (per_row > ML2_MAX_TOPK)
    return fail(ML2_ERR_UNSUPPORTED, "%s: %d per row > %d", call, per_row, ML2_MAX_TOPK);
  if (rows > ML2_MAX_ROWS)
    return fail(ML2_ERR_UNSUPPORTED, "%s: rows = %lld > %d", call, (long long)rows, ML2_MAX_ROWS);
  return ML2_OK;
}

}  // namespace

ml2_status ml2_sample_workspace_bytes(int64_t n, int64_t rows, int32_t draws, size_t *bytes) {
  const ml2_status st = check_sizes("ml2_sample_workspace_bytes", n, rows, draws, bytes);
  if (st == ML2_OK) *bytes = ml2::sample_workspace_bytes(n, rows, draws);
  return st;
}

ml2_status ml2_sample(int32_t dtype, const void *scores, int64_t n, int64_t ld, int64_t rows,
                      const uint8_t *valid, int64_t valid_ld, const float *temperature,
                      const int32_t *top_k, const float *top_p, const float *min_p,
                      const float *u, int32_t draws, int32_t *idx, float *logprob,
                      void *workspace, size_t workspace_bytes, void *stream) {
  const ml2::ScoreRows s = {scores, n, ld, rows, valid, valid_ld, temperature};
  size_t need = 0;
  if (size_ok(n) && size_ok(rows) && rows <= ML2_MAX_ROWS && draws >= 0 && draws <= ML2_MAX_TOPK)
    need = ml2::sample_workspace_bytes(n, rows, draws);
  ml2_status st = check_rows("ml2_sample", dtype, s, draws, workspace, workspace_bytes, need);
  if (st != ML2_OK) return st;
  if (rows > 0 && draws > 0 && (!u || !idx || !logprob))
    return fail(ML2_ERR_INVALID_ARG, "ml2_sample: u, idx or logprob is NULL");
  if (rows == 0 || draws == 0) return ML2_OK;
  int dev = 0;
  st = ml2::current_device(&dev);
  if (st != ML2_OK) return st;
  const ml2::SampleArgs a = {s, top_k, top_p, min_p, u, draws, idx, logprob};
  const hipError_t e = ml2::launch_sample(dtype, a, workspace, ml2::cu_count(dev),
                                          static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ML2_OK : hip_fail(e, "ml2_sample: kernel launch");
}

ml2_status ml2_logprob_workspace_bytes(int64_t n, int64_t rows, int32_t per_row, size_t *bytes) {
  const ml2_status st = check_sizes("ml2_logprob_workspace_bytes", n, rows, per_row, bytes);
  if (st == ML2_OK) *bytes = ml2::logprob_workspace_bytes(n, rows, per_row);
  return st;
}

static ml2_status logprob(const char *call, int32_t dtype, const ml2::LogprobArgs &a,
                          void *workspace, size_t workspace_bytes, void *stream) {
  size_t need = 0;
  if (size_ok(a.s.n) && size_ok(a.s.rows) && a.s.rows <= ML2_MAX_ROWS && a.per_row >= 0 && a.per_row <= ML2_MAX_TOPK)
    need = ml2::logprob_workspace_bytes(a.s.n, a.s.rows, a.per_row);
  ml2_status st = check_rows(call, dtype, a.s, a.per_row, workspace, workspace_bytes, need);
  if (st != ML2_OK) return st;
  if (a.s.rows > 0 && a.per_row > 0 && !a.targets)
    return fail(ML2_ERR_INVALID_ARG, "%s: targets is NULL", call);
  if (a.s.rows == 0 || (!a.grad && (!a.logprob || a.per_row == 0))) return ML2_OK;
  int dev = 0;
  st = ml2::current_device(&dev);
  if (st != ML2_OK) return st;
  const hipError_t e = ml2::launch_logprob(dtype, a, workspace, ml2::cu_count(dev),
                                           static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(ML2_ERR_HIP, "%s: kernel launch: %s", call, hipGetErrorString(e));
  return ML2_OK;
}

ml2_status ml2_logprob(int32_t dtype, const void *scores, int64_t n, int64_t ld, int64_t rows,
                       const uint8_t *valid, int64_t valid_ld, const float *temperature,
                       const int32_t *targets, int32_t per_row, float *logprob_out,
                       void *workspace, size_t workspace_bytes, void *stream) {
  if (rows > 0 && per_row > 0 && !logprob_out)
    return fail(ML2_ERR_INVALID_ARG, "ml2_logprob: logprob is NULL");
  const ml2::LogprobArgs a = {{scores, n, ld, rows, valid, valid_ld, temperature},
                              targets, nullptr, per_row, logprob_out, nullptr, 0};
  return logprob("ml2_logprob", dtype, a, workspace, workspace_bytes, stream);
}

ml2_status ml2_logprob_grad(int32_t dtype, const void *scores, int64_t n, int64_t ld,
                            int64_t rows, const uint8_t *valid, int64_t valid_ld,
                            const float *temperature, const int32_t *targets,
                            const float *weight, int32_t per_row, float *logprob_out, void *grad,
                            int64_t grad_ld, void *workspace, size_t workspace_bytes,
                            void *stream) {
  size_t size = 0;
  if (!element_size(dtype, &size))
    return fail(ML2_ERR_INVALID_ARG, "ml2_logprob_grad: unknown dtype %d", dtype);
  if (rows > 0 && n > 0 && !grad)
    return fail(ML2_ERR_INVALID_ARG, "ml2_logprob_grad: grad is NULL");
  if (grad_ld < n || grad_ld > (int64_t)1 << 40 || !aligned(grad, size))
    return fail(ML2_ERR_INVALID_ARG, "ml2_logprob_grad: grad_ld = %lld, n = %lld, or grad is "
                "not aligned to its type", (long long)grad_ld, (long long)n);
  if (rows > 0 && per_row > 0 && !weight)
    return fail(ML2_ERR_INVALID_ARG, "ml2_logprob_grad: weight is NULL");
  const bool sizes = size_ok(n) && size_ok(rows) && rows <= ML2_MAX_ROWS && per_row >= 0 &&
                     per_row <= ML2_MAX_TOPK && ld >= n && ld <= (int64_t)1 << 40;  // else refused below
  if (sizes && overlap(scores, ld, grad, grad_ld, rows, n, size))
    return fail(ML2_ERR_INVALID_ARG, "ml2_logprob_grad: grad overlaps scores");
  const int64_t items = sizes ? rows * per_row : 0;
  if (overlap(logprob_out, items, targets, items, 1, items, 4) ||
      overlap(logprob_out, items, weight, items, 1, items, 4))
    return fail(ML2_ERR_INVALID_ARG, "ml2_logprob_grad: logprob overlaps targets or weight");
  // n = 0: no gradient to write, log-probabilities all the same
  const ml2::LogprobArgs a = {{scores, n, ld, rows, valid, valid_ld, temperature},
                              targets, weight, per_row, logprob_out, grad, grad_ld};
  return logprob("ml2_logprob_grad", dtype, a, workspace, workspace_bytes, stream);
}

ml2_status ml2_embed(int32_t dtype, const void *table, int64_t table_rows, int64_t width,
                     int64_t ld, const int32_t *ids, int64_t n, float scale, void *out,
                     int64_t out_ld, void *stream) {
  size_t size = 0;
  if (!element_size(dtype, &size))
    return fail(ML2_ERR_INVALID_ARG, "ml2_embed: unknown dtype %d", dtype);
  if (!size_ok(table_rows) || !size_ok(width) || !size_ok(n))
    return fail(ML2_ERR_INVALID_ARG, "ml2_embed: sizes out of range");
  if (width > ML2_MAX_WIDTH)
    return fail(ML2_ERR_UNSUPPORTED, "ml2_embed: width = %lld > %d", (long long)width,
                ML2_MAX_WIDTH);
  if (ld < width || out_ld < width || ld > (int64_t)1 << 32 || out_ld > (int64_t)1 << 32)
    return fail(ML2_ERR_INVALID_ARG, "ml2_embed: ld = %lld, out_ld = %lld, width = %lld",
                (long long)ld, (long long)out_ld, (long long)width);
  if (n > 0 && width > 0 && (!ids || !out || (!table && table_rows > 0)))
    return fail(ML2_ERR_INVALID_ARG, "ml2_embed: NULL table, ids or out");
  if (!aligned(table, size) || !aligned(out, size) || !aligned(ids, 4))
    return fail(ML2_ERR_INVALID_ARG, "ml2_embed: an array is not aligned to its type");
  if (n == 0 || width == 0) return ML2_OK;
  int dev = 0;
  const ml2_status st = ml2::current_device(&dev);
  if (st != ML2_OK) return st;
  const ml2::EmbedArgs a = {table, table_rows, width, ld, ids, n, scale, out, out_ld};
  const hipError_t e =
      ml2::launch_embed(dtype, a, ml2::cu_count(dev), static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ML2_OK : hip_fail(e, "ml2_embed: kernel launch");
}

static ml2_status check_grad_sizes(const char *call, int64_t n, int64_t table_rows,
                                   int64_t width) {
  if (!size_ok(table_rows) || !size_ok(width) || !size_ok(n))
    return fail(ML2_ERR_INVALID_ARG, "%s: sizes out of range", call);
  if (width > ML2_MAX_WIDTH)
    return fail(ML2_ERR_UNSUPPORTED, "%s: width = %lld > %d", call, (long long)width,
                ML2_MAX_WIDTH);
  if (n > ML2_MAX_TOKENS)
    return fail(ML2_ERR_UNSUPPORTED, "%s: n = %lld > %d", call, (long long)n, ML2_MAX_TOKENS);
  return ML2_OK;
}

ml2_status ml2_embed_grad_workspace_bytes(int64_t n, int64_t table_rows, int64_t width,
                                          size_t *bytes) {
  if (!bytes)
    return fail(ML2_ERR_INVALID_ARG, "ml2_embed_grad_workspace_bytes: bytes is NULL");
  const ml2_status st = check_grad_sizes("ml2_embed_grad_workspace_bytes", n, table_rows, width);
  if (st == ML2_OK) *bytes = ml2::embed_grad_workspace_bytes(n, table_rows, width);
  return st;
}

ml2_status ml2_embed_grad(int32_t dtype, const void *dout, int64_t n, int64_t width,
                          int64_t dout_ld, const int32_t *ids, float scale, int32_t grad_dtype,
                          void *grad, int64_t table_rows, int64_t grad_ld, void *workspace,
                          size_t workspace_bytes, void *stream) {
  size_t size = 0, grad_size = 0;
  if (!element_size(dtype, &size) || !element_size(grad_dtype, &grad_size))
    return fail(ML2_ERR_INVALID_ARG, "ml2_embed_grad: unknown dtype %d or grad_dtype %d", dtype,
                grad_dtype);
  if (grad_dtype != dtype && grad_dtype != ML2_F32)
    return fail(ML2_ERR_INVALID_ARG, "ml2_embed_grad: grad_dtype %d is neither dtype %d nor "
                "ML2_F32", grad_dtype, dtype);
  ml2_status st = check_grad_sizes("ml2_embed_grad", n, table_rows, width);
  if (st != ML2_OK) return st;
  if (dout_ld < width || grad_ld < width || dout_ld > (int64_t)1 << 32 ||
      grad_ld > (int64_t)1 << 32)
    return fail(ML2_ERR_INVALID_ARG, "ml2_embed_grad: dout_ld = %lld, grad_ld = %lld, "
                "width = %lld", (long long)dout_ld, (long long)grad_ld, (long long)width);
  if (width > 0 && ((n > 0 && (!dout || !ids)) || (table_rows > 0 && !grad)))
    return fail(ML2_ERR_INVALID_ARG, "ml2_embed_grad: NULL dout, ids or grad");
  if (!aligned(dout, size) || !aligned(grad, grad_size) || !aligned(ids, 4))
    return fail(ML2_ERR_INVALID_ARG, "ml2_embed_grad: an array is not aligned to its type");
  if (!workspace || !aligned(workspace, 256))
    return fail(ML2_ERR_INVALID_ARG, "ml2_embed_grad: workspace is NULL or not 256-byte aligned");
  const size_t need = ml2::embed_grad_workspace_bytes(n, table_rows, width);
  if (workspace_bytes < need)
    return fail(ML2_ERR_INVALID_ARG, "ml2_embed_grad: workspace %zu < %zu bytes", workspace_bytes,
                need);
  if (table_rows == 0 || width == 0) return ML2_OK;
  const ml2::EmbedGradArgs a = {dout, n, width, dout_ld, ids, scale, grad, table_rows, grad_ld};
  const hipError_t e = ml2::launch_embed_grad(dtype, grad_dtype, a, workspace,
                                              static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ML2_OK : hip_fail(e, "ml2_embed_grad: kernel launch");
}
