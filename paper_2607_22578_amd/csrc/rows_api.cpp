// Host side of the row-table operators: argument validation and launches behind the
// C ABI declared in include/hs_merge.h, with the conventions of api.cpp (everything is
// validated before anything is enqueued; nothing is allocated).
#include <hip/hip_runtime_api.h>

#include "../../include/hs_merge.h"
#include "status.h"

namespace hs {
hipError_t launch_pack_rows(const void *src, int src_dtype, int64_t rows, int64_t dim, int group,
                            int scale_dtype, void *codes, void *scales, hipStream_t st);
hipError_t launch_embed(const hs_row_table *t, const void *ids, int is64, int64_t n, float scale,
                        int64_t pad, void *out, int out_dtype, hipStream_t st);
size_t embed_grad_workspace_bytes(int64_t n, int64_t rows, int64_t dim);
hipError_t launch_embed_grad(const void *grad, int grad_dtype, const void *ids, int is64,
                             int64_t n, int64_t rows, int64_t dim, float scale, int64_t pad,
                             int add, void *table, int table_dtype, void *ws, hipStream_t st);
hipError_t launch_score_packed(const hs_row_table *t, const void *x, int x_dtype, int64_t n_x,
                               void *out, int out_dtype, int64_t out_stride, hipStream_t st);
hipError_t launch_adjust(const hs_adjust *a, const void *in, int64_t stride, void *out,
                         int64_t out_stride, int dtype, int64_t n_rows, int64_t n_cols,
                         hipStream_t st);
size_t topk_rows_workspace_bytes(int64_t n_rows, int64_t n_cols, int k);
hipError_t launch_topk_rows(const void *scores, int dtype, int64_t stride, int64_t n_rows,
                            int64_t n_cols, int k, float *out_s, int32_t *out_i, void *ws,
                            hipStream_t st);
}  // namespace hs

using hs::aligned;
using hs::device_status;
using hs::fail;
using hs::ok;

// (int64 sizes of one array stay far below 2^63 within these)
static const int64_t kRowsMax = INT32_MAX, kDimMax = 16384, kIdsMax = (int64_t)1 << 30,
                     kBatchMax = (int64_t)1 << 20, kCellsMax = (int64_t)1 << 40;

static bool float_type(int32_t t) { return t == HS_F32 || t == HS_BF16; }
static size_t elem(int32_t t) { return t == HS_F32 ? 4 : 2; }

static bool overlap(const void *a, uint64_t an, const void *b, uint64_t bn) {
  const uint64_t x = (uint64_t)(uintptr_t)a, y = (uint64_t)(uintptr_t)b;
  return an > 0 && bn > 0 && x < y + bn && y < x + an;
}

// The same for n rows of `row` bytes that start `step` >= row bytes apart: what lies between
// them does not count.
static bool on_rows(const void *rows, uint64_t row, uint64_t step, int64_t n, const void *b,
                    uint64_t bn) {
  if (n <= 0 || !overlap(rows, (uint64_t)(n - 1) * step + row, b, bn)) return false;
  const uint64_t x = (uint64_t)(uintptr_t)rows, y = (uint64_t)(uintptr_t)b;
  const uint64_t i = y > x ? (y - x) / step : 0;   // the last row that starts at b or before
  return overlap(b, bn, (const void *)(uintptr_t)(x + i * step), row) ||
         (i + 1 < (uint64_t)n &&
          overlap(b, bn, (const void *)(uintptr_t)(x + (i + 1) * step), row));
}

static hs_status check_shape(int64_t rows, int64_t dim, const char *who) {
  if (rows < 0 || rows > kRowsMax)
    return fail(HS_ERR_INVALID_ARG, "%s: rows %lld out of [0, 2^31-1]", who, (long long)rows);
  if (dim < 1 || dim > kDimMax)
    return fail(HS_ERR_INVALID_ARG, "%s: dim %lld out of [1, 16384]", who, (long long)dim);
  return HS_OK;
}

static hs_status check_group(int64_t dim, int32_t group, int32_t scale_dtype, const char *who) {
  if (group != 32 && group != 64 && group != 128)
    return fail(HS_ERR_UNSUPPORTED, "%s: group %d is not 32, 64 or 128", who, group);
  if (dim % group != 0)
    return fail(HS_ERR_UNSUPPORTED, "%s: dim %lld is no multiple of the group's %d columns", who,
                (long long)dim, group);
  if (!float_type(scale_dtype))
    return fail(HS_ERR_UNSUPPORTED, "%s: scale_dtype %d unsupported", who, scale_dtype);
  return HS_OK;
}

static hs_status check_table(const hs_row_table *t, const char *who) {
  if (!t) return fail(HS_ERR_INVALID_ARG, "%s: null table", who);
  hs_status s = check_shape(t->rows, t->dim, who);
  if (s != HS_OK) return s;
  size_t align = 4;
  switch (t->dtype) {
    case HS_F32:
    case HS_BF16:
      break;
    case HS_FP8_E4M3:
      if (t->rows > 0 && !t->scale)
        return fail(HS_ERR_INVALID_ARG, "%s: an FP8 table needs scales", who);
      break;
    case HS_FP4_E2M1:
      s = check_group(t->dim, t->group, t->scale_dtype, who);
      if (s != HS_OK) return s;
      if (t->rows > 0 && !t->scale)
        return fail(HS_ERR_INVALID_ARG, "%s: an FP4 table needs scales", who);
      align = elem(t->scale_dtype);
      break;
    default:
      return fail(HS_ERR_UNSUPPORTED, "%s: table dtype %d unsupported", who, t->dtype);
  }
  if (t->rows > 0 && !t->data) return fail(HS_ERR_INVALID_ARG, "%s: null table data", who);
  if (!aligned(t->data, 16))
    return fail(HS_ERR_ALIGNMENT, "%s: table data must be 16-byte aligned", who);
  if (t->dtype >= HS_FP8_E4M3 && !aligned(t->scale, align))
    return fail(HS_ERR_ALIGNMENT, "%s: misaligned table scales", who);
  return HS_OK;
}

static uint64_t table_bytes(const hs_row_table *t) {
  const uint64_t cells = (uint64_t)t->rows * (uint64_t)t->dim;
  return t->dtype == HS_F32 ? cells * 4 : t->dtype == HS_BF16 ? cells * 2
         : t->dtype == HS_FP8_E4M3 ? cells : cells / 2;
}

// Whether out[bytes] overlaps the table's rows or scales.
static bool on_table(const hs_row_table *t, const void *out, uint64_t bytes) {
  const uint64_t rows = (uint64_t)t->rows;
  const uint64_t scales = t->dtype == HS_FP8_E4M3 ? rows * 4
                          : t->dtype == HS_FP4_E2M1
                              ? rows * (uint64_t)(t->dim / t->group) * elem(t->scale_dtype)
                              : 0;
  return overlap(t->data, table_bytes(t), out, bytes) || overlap(t->scale, scales, out, bytes);
}

static hs_status check_ids(const void *ids, int32_t is64, int64_t n, const char *who) {
  if (n < 0 || n > kIdsMax)
    return fail(HS_ERR_INVALID_ARG, "%s: n %lld out of [0, 2^30]", who, (long long)n);
  if (is64 != 0 && is64 != 1)
    return fail(HS_ERR_INVALID_ARG, "%s: ids_is_i64 must be 0 or 1", who);
  if (n > 0 && !ids) return fail(HS_ERR_INVALID_ARG, "%s: null ids", who);
  if (!aligned(ids, is64 ? 8 : 4)) return fail(HS_ERR_ALIGNMENT, "%s: misaligned ids", who);
  return HS_OK;
}

static hs_status check_scale(float scale, const char *who) {
  if (!(scale - scale == 0.0f)) return fail(HS_ERR_INVALID_ARG, "%s: scale is not finite", who);
  return HS_OK;
}

extern "C" {

hs_status hs_pack_rows(const void *src, int32_t src_dtype, int64_t rows, int64_t dim,
                       int32_t group, int32_t scale_dtype, void *codes, void *scale,
                       void *stream) {
  const char *who = "hs_pack_rows";
  hs_status s = check_shape(rows, dim, who);
  if (s != HS_OK) return s;
  if (!float_type(src_dtype))
    return fail(HS_ERR_UNSUPPORTED, "%s: src_dtype %d unsupported", who, src_dtype);
  s = check_group(dim, group, scale_dtype, who);
  if (s != HS_OK) return s;
  if (rows > 0 && (!src || !codes || !scale))
    return fail(HS_ERR_INVALID_ARG, "%s: null argument", who);
  if (!aligned(src, 16) || !aligned(codes, 16) || !aligned(scale, elem(scale_dtype)))
    return fail(HS_ERR_ALIGNMENT, "%s: src and codes must be 16-byte aligned, scale to its "
                "element", who);
  const uint64_t sb = (uint64_t)rows * (uint64_t)dim * elem(src_dtype),
                 cb = (uint64_t)rows * (uint64_t)(dim / 2),
                 gb = (uint64_t)rows * (uint64_t)(dim / group) * elem(scale_dtype);
  if (overlap(src, sb, codes, cb) || overlap(src, sb, scale, gb) || overlap(codes, cb, scale, gb))
    return fail(HS_ERR_INVALID_ARG, "%s: src, codes and scale overlap", who);
  return device_status(hs::launch_pack_rows(src, src_dtype, rows, dim, group, scale_dtype, codes,
                                            scale, (hipStream_t)stream),
                       "hs_pack_rows launch");
}

hs_status hs_embed(const hs_row_table *table, const void *ids, int32_t ids_is_i64, int64_t n,
                   float scale, int64_t pad_id, void *out, int32_t out_dtype, void *stream) {
  const char *who = "hs_embed";
  hs_status s = check_table(table, who);
  if (s == HS_OK) s = check_ids(ids, ids_is_i64, n, who);
  if (s == HS_OK) s = check_scale(scale, who);
  if (s != HS_OK) return s;
  if (!float_type(out_dtype))
    return fail(HS_ERR_UNSUPPORTED, "%s: out_dtype %d unsupported", who, out_dtype);
  if (n > 0 && !out) return fail(HS_ERR_INVALID_ARG, "%s: null out", who);
  if (!aligned(out, elem(out_dtype))) return fail(HS_ERR_ALIGNMENT, "%s: misaligned out", who);
  const uint64_t ob = (uint64_t)n * (uint64_t)table->dim * elem(out_dtype);
  if (on_table(table, out, ob) || overlap(ids, (uint64_t)n * (ids_is_i64 ? 8 : 4), out, ob))
    return fail(HS_ERR_INVALID_ARG, "%s: out overlaps the table or ids", who);
  return device_status(hs::launch_embed(table, ids, ids_is_i64, n, scale, pad_id, out, out_dtype,
                                        (hipStream_t)stream),
                       "hs_embed launch");
}

hs_status hs_embed_grad_bytes(int64_t n, int64_t rows, int64_t dim, size_t *bytes) {
  const char *who = "hs_embed_grad_bytes";
  if (!bytes) return fail(HS_ERR_INVALID_ARG, "%s: null argument", who);
  hs_status s = check_shape(rows, dim, who);
  if (s != HS_OK) return s;
  if (n < 0 || n > kIdsMax)
    return fail(HS_ERR_INVALID_ARG, "%s: n %lld out of [0, 2^30]", who, (long long)n);
  *bytes = hs::embed_grad_workspace_bytes(n, rows, dim);
  return ok();
}

hs_status hs_embed_grad(const void *d_out, int32_t d_out_dtype, const void *ids,
                        int32_t ids_is_i64, int64_t n, int64_t rows, int64_t dim, float scale,
                        int64_t pad_id, int32_t accumulate, void *d_table,
                        int32_t d_table_dtype, void *ws, size_t ws_bytes, void *stream) {
  const char *who = "hs_embed_grad";
  hs_status s = check_shape(rows, dim, who);
  if (s == HS_OK) s = check_ids(ids, ids_is_i64, n, who);
  if (s == HS_OK) s = check_scale(scale, who);
  if (s != HS_OK) return s;
  if (!float_type(d_out_dtype) || !float_type(d_table_dtype))
    return fail(HS_ERR_UNSUPPORTED, "%s: dtypes %d and %d unsupported", who, d_out_dtype,
                d_table_dtype);
  if (accumulate != 0 && accumulate != 1)
    return fail(HS_ERR_INVALID_ARG, "%s: accumulate must be 0 or 1", who);
  if ((n > 0 && !d_out) || (rows > 0 && !d_table))
    return fail(HS_ERR_INVALID_ARG, "%s: null argument", who);
  if (!aligned(d_out, elem(d_out_dtype)) || !aligned(d_table, elem(d_table_dtype)))
    return fail(HS_ERR_ALIGNMENT, "%s: misaligned d_out or d_table", who);
  const size_t need = hs::embed_grad_workspace_bytes(n, rows, dim);
  if (!ws || ws_bytes < need)
    return fail(HS_ERR_WORKSPACE, "%s: workspace %zu bytes, need %zu", who, ws_bytes, need);
  if (!aligned(ws, 256))
    return fail(HS_ERR_ALIGNMENT, "%s: workspace must be 256-byte aligned", who);
  const uint64_t gb = (uint64_t)n * (uint64_t)dim * elem(d_out_dtype),
                 tb = (uint64_t)rows * (uint64_t)dim * elem(d_table_dtype),
                 ib = (uint64_t)n * (ids_is_i64 ? 8 : 4);
  if (overlap(d_out, gb, d_table, tb))
    return fail(HS_ERR_INVALID_ARG, "%s: d_out and d_table overlap", who);
  // (a call that writes nothing writes nothing of its workspace either)
  if (rows > 0 && (n > 0 || !accumulate)) {
    if (overlap(ids, ib, d_table, tb))
      return fail(HS_ERR_INVALID_ARG, "%s: ids and d_table overlap", who);
    if (overlap(ws, need, d_out, gb) || overlap(ws, need, ids, ib) || overlap(ws, need, d_table, tb))
      return fail(HS_ERR_INVALID_ARG, "%s: the workspace overlaps d_out, ids or d_table", who);
  }
  return device_status(hs::launch_embed_grad(d_out, d_out_dtype, ids, ids_is_i64, n, rows, dim,
                                             scale, pad_id, accumulate, d_table, d_table_dtype,
                                             ws, (hipStream_t)stream),
                       "hs_embed_grad launch");
}

hs_status hs_score_packed(const hs_row_table *table, const void *x, int32_t x_dtype, int64_t n_x,
                          void *out, int32_t out_dtype, int64_t out_stride, void *stream) {
  const char *who = "hs_score_packed";
  hs_status s = check_table(table, who);
  if (s != HS_OK) return s;
  if (table->dtype != HS_FP4_E2M1)
    return fail(HS_ERR_UNSUPPORTED, "%s: the table must be packed (HS_FP4_E2M1)", who);
  if (!float_type(x_dtype) || !float_type(out_dtype))
    return fail(HS_ERR_UNSUPPORTED, "%s: dtypes %d and %d unsupported", who, x_dtype, out_dtype);
  if (n_x < 0 || n_x > kBatchMax)
    return fail(HS_ERR_INVALID_ARG, "%s: n_x %lld out of [0, 2^20]", who, (long long)n_x);
  if (out_stride < table->rows || out_stride > kCellsMax)
    return fail(HS_ERR_INVALID_ARG, "%s: out_stride %lld below the table's %lld rows (or above "
                "2^40)", who, (long long)out_stride, (long long)table->rows);
  if (n_x > 0 && table->rows > 0 && (!x || !out))
    return fail(HS_ERR_INVALID_ARG, "%s: null argument", who);
  if (!aligned(x, 16) || !aligned(out, elem(out_dtype)))
    return fail(HS_ERR_ALIGNMENT, "%s: x must be 16-byte aligned, out to its element", who);
  if (n_x > 0 && table->rows > 0) {
    const uint64_t ob = ((uint64_t)(n_x - 1) * (uint64_t)out_stride + (uint64_t)table->rows) *
                        elem(out_dtype);
    if (on_table(table, out, ob) ||
        overlap(x, (uint64_t)n_x * (uint64_t)table->dim * elem(x_dtype), out, ob))
      return fail(HS_ERR_INVALID_ARG, "%s: out overlaps the table or x", who);
  }
  return device_status(hs::launch_score_packed(table, x, x_dtype, n_x, out, out_dtype, out_stride,
                                               (hipStream_t)stream),
                       "hs_score_packed launch");
}

static hs_status check_scores(const void *scores, int32_t dtype, int64_t stride, int64_t n_rows,
                              int64_t n_cols, const char *who) {
  if (!float_type(dtype)) return fail(HS_ERR_UNSUPPORTED, "%s: dtype %d unsupported", who, dtype);
  if (n_rows < 0 || n_rows > kBatchMax || n_cols < 0 || n_cols > kRowsMax ||
      n_rows * n_cols > kCellsMax)
    return fail(HS_ERR_INVALID_ARG, "%s: %lld rows of %lld columns out of [0, 2^20], [0, 2^31-1] "
                "or 2^40 in all", who, (long long)n_rows, (long long)n_cols);
  if (stride < n_cols || stride > kCellsMax)
    return fail(HS_ERR_INVALID_ARG, "%s: stride %lld below n_cols %lld (or above 2^40)", who,
                (long long)stride, (long long)n_cols);
  if (n_rows > 0 && n_cols > 0 && !scores)
    return fail(HS_ERR_INVALID_ARG, "%s: null scores", who);
  if (!aligned(scores, elem(dtype)))
    return fail(HS_ERR_ALIGNMENT, "%s: misaligned scores", who);
  return HS_OK;
}

hs_status hs_adjust_scores(const hs_adjust *adjust, const void *scores, int64_t stride, void *out,
                           int64_t out_stride, int32_t dtype, int64_t n_rows, int64_t n_cols,
                           void *stream) {
  const char *who = "hs_adjust_scores";
  if (!adjust) return fail(HS_ERR_INVALID_ARG, "%s: null adjust", who);
  hs_status s = check_scores(scores, dtype, stride, n_rows, n_cols, who);
  if (s == HS_OK) s = check_scores(out, dtype, out_stride, n_rows, n_cols, who);
  if (s != HS_OK) return s;
  const hs_adjust &a = *adjust;
  if (a.n_seen < 0 || a.n_seen > kIdsMax || a.n_bias < 0 || a.n_bias > kIdsMax)
    return fail(HS_ERR_INVALID_ARG, "%s: n_seen %lld or n_bias %lld out of [0, 2^30]", who,
                (long long)a.n_seen, (long long)a.n_bias);
  if (a.seen_off && a.n_seen > 0 && !a.seen)
    return fail(HS_ERR_INVALID_ARG, "%s: seen_off without seen", who);
  if (a.bias_off && a.n_bias > 0 && (!a.bias_id || !a.bias))
    return fail(HS_ERR_INVALID_ARG, "%s: bias_off without bias_id and bias", who);
  if (a.allow && (a.allow_stride < 0 || a.allow_stride > kCellsMax ||
                  (a.allow_stride > 0 && a.allow_stride < (n_cols + 31) / 32)))
    return fail(HS_ERR_INVALID_ARG, "%s: allow_stride %lld is neither 0 nor at least %lld words",
                who, (long long)a.allow_stride, (long long)((n_cols + 31) / 32));
  if (!aligned(a.seen_off, 8) || !aligned(a.bias_off, 8) || !aligned(a.seen, 4) ||
      !aligned(a.prompt_len, 4) || !aligned(a.repetition, 4) || !aligned(a.frequency, 4) ||
      !aligned(a.presence, 4) || !aligned(a.bias_id, 4) || !aligned(a.bias, 4) ||
      !aligned(a.allow, 4))
    return fail(HS_ERR_ALIGNMENT, "%s: misaligned list or array", who);
  if (n_rows > 0 && n_cols > 0) {
    const uint64_t row = (uint64_t)n_cols * elem(dtype), step = (uint64_t)out_stride * elem(dtype),
                   n = (uint64_t)n_rows, words = ((uint64_t)n_cols + 31) / 32;
    auto on_out = [&](const void *p, uint64_t bytes) {
      return p && on_rows(out, row, step, n_rows, p, bytes);
    };
    bool on = on_out(a.prompt_len, n * 4) || on_out(a.repetition, n * 4) ||
              on_out(a.frequency, n * 4) || on_out(a.presence, n * 4);
    if (a.seen_off)
      on = on || on_out(a.seen_off, (n + 1) * 8) || on_out(a.seen, (uint64_t)a.n_seen * 4);
    if (a.bias_off)
      on = on || on_out(a.bias_off, (n + 1) * 8) || on_out(a.bias_id, (uint64_t)a.n_bias * 4) ||
           on_out(a.bias, (uint64_t)a.n_bias * 4);
    // (the masks may lie between the rows, one behind each: looked at one by one if so)
    const uint64_t masks = a.allow && a.allow_stride > 0 ? n : 1;
    if (on_out(a.allow, ((masks - 1) * (uint64_t)a.allow_stride + words) * 4))
      for (uint64_t r = 0; r < masks && !on; ++r)
        on = on_out(a.allow + r * (uint64_t)a.allow_stride, words * 4);
    if (on) return fail(HS_ERR_INVALID_ARG, "%s: out overlaps a list, an array or a mask", who);
  }
  if (n_rows > 0 && n_cols > 0 && !(scores == out && stride == out_stride)) {
    const uint64_t es = elem(dtype);
    const uint64_t ib = ((uint64_t)(n_rows - 1) * (uint64_t)stride + (uint64_t)n_cols) * es,
                   ob = ((uint64_t)(n_rows - 1) * (uint64_t)out_stride + (uint64_t)n_cols) * es;
    if (overlap(scores, ib, out, ob))
      return fail(HS_ERR_INVALID_ARG, "%s: scores and out overlap without being the same", who);
  }
  return device_status(hs::launch_adjust(adjust, scores, stride, out, out_stride, dtype, n_rows,
                                         n_cols, (hipStream_t)stream),
                       "hs_adjust_scores launch");
}

static hs_status check_k(int32_t k, const char *who) {
  if (k < 1 || k > 1024) return fail(HS_ERR_INVALID_ARG, "%s: k %d out of [1, 1024]", who, k);
  return HS_OK;
}

hs_status hs_topk_rows_bytes(int64_t n_rows, int64_t n_cols, int32_t k, size_t *bytes) {
  const char *who = "hs_topk_rows_bytes";
  if (!bytes) return fail(HS_ERR_INVALID_ARG, "%s: null argument", who);
  if (n_rows < 0 || n_rows > kBatchMax || n_cols < 0 || n_cols > kRowsMax)
    return fail(HS_ERR_INVALID_ARG, "%s: %lld rows of %lld columns out of range", who,
                (long long)n_rows, (long long)n_cols);
  hs_status s = check_k(k, who);
  if (s != HS_OK) return s;
  *bytes = hs::topk_rows_workspace_bytes(n_rows, n_cols, k);
  return ok();
}

hs_status hs_topk_rows(const void *scores, int32_t dtype, int64_t stride, int64_t n_rows,
                       int64_t n_cols, int32_t k, float *topk_score, int32_t *topk_index,
                       void *ws, size_t ws_bytes, void *stream) {
  const char *who = "hs_topk_rows";
  hs_status s = check_scores(scores, dtype, stride, n_rows, n_cols, who);
  if (s == HS_OK) s = check_k(k, who);
  if (s != HS_OK) return s;
  if (n_rows > 0 && (!topk_score || !topk_index))
    return fail(HS_ERR_INVALID_ARG, "%s: null output", who);
  if (!aligned(topk_score, 4) || !aligned(topk_index, 4))
    return fail(HS_ERR_ALIGNMENT, "%s: misaligned output", who);
  const uint64_t sb = n_rows > 0 && n_cols > 0
                          ? ((uint64_t)(n_rows - 1) * (uint64_t)stride + (uint64_t)n_cols) *
                                elem(dtype)
                          : 0,
                 kb = (uint64_t)n_rows * (uint64_t)k * 4;
  if (overlap(scores, sb, topk_score, kb) || overlap(scores, sb, topk_index, kb) ||
      overlap(topk_score, kb, topk_index, kb))
    return fail(HS_ERR_INVALID_ARG, "%s: scores and the outputs overlap", who);
  const size_t need = hs::topk_rows_workspace_bytes(n_rows, n_cols, k);
  if (!ws || ws_bytes < need)
    return fail(HS_ERR_WORKSPACE, "%s: workspace %zu bytes, need %zu", who, ws_bytes, need);
  if (!aligned(ws, 256))
    return fail(HS_ERR_ALIGNMENT, "%s: workspace must be 256-byte aligned", who);
  if (n_rows > 0 &&
      (on_rows(scores, (uint64_t)n_cols * elem(dtype), (uint64_t)stride * elem(dtype), n_rows, ws,
               need) ||
       overlap(ws, need, topk_score, kb) || overlap(ws, need, topk_index, kb)))
    return fail(HS_ERR_INVALID_ARG, "%s: the workspace overlaps scores or an output", who);
  return device_status(hs::launch_topk_rows(scores, dtype, stride, n_rows, n_cols, k, topk_score,
                                            topk_index, ws, (hipStream_t)stream),
                       "hs_topk_rows launch");
}

}  // extern "C"
