// Entry points of what brings tokens to experts and back: argument checks and launches (experts.hip).
#include "checks.h"
#include "experts.h"

namespace {

stem_status check_choices(stem_ctx* c, const char* who, int64_t T, int k) {
  if (k < 1 || k > STEM_EXPERTS_MAX_CHOICES) return stem_fail(c, STEM_ERR_SHAPE, "%s: k = %d is not in 1 .. %d", who, k, STEM_EXPERTS_MAX_CHOICES);
  if (T > ((int64_t)1 << 30) / k) return stem_fail(c, STEM_ERR_SHAPE, "%s: %lld tokens of %d choices are over 2^30", who, (long long)T, k);
  return STEM_OK;
}

stem_status check_rows(stem_ctx* c, const char* who, int64_t rows, int64_t width) {
  if (rows < 0 || rows > ((int64_t)1 << 30)) return stem_fail(c, STEM_ERR_SHAPE, "%s: %lld rows", who, (long long)rows);
  if (width < 0 || width > ((int64_t)1 << 30)) return stem_fail(c, STEM_ERR_SHAPE, "%s: rows of %lld elements", who, (long long)width);
  return STEM_OK;
}

ExpertsRowsArgs rows_args(const stem_ctx* c, int64_t T, int64_t rows, int64_t width, int k) {
  ExpertsRowsArgs a = {};
  a.es = c->desc.dtype == STEM_BF16 ? 2 : 4;
  a.T = T; a.rows = rows; a.width = width; a.k = k;
  a.flag = c->flag;
  return a;
}

}  // namespace

extern "C" {

stem_status stem_experts_sort(stem_ctx* c, const int32_t* experts, int64_t T, int k, int n_experts, int32_t* src, int32_t* place, int32_t* offsets,
                              void* stream) {
  static const char who[] = "stem_experts_sort";
  STEM_TRY(stem_enter(c, T));
  STEM_TRY(check_choices(c, who, T, k));
  if (n_experts < 1 || n_experts > STEM_EXPERTS_MAX) return stem_fail(c, STEM_ERR_SHAPE, "%s: %d experts; 1 to %d", who, n_experts, STEM_EXPERTS_MAX);
  if (!offsets || (T > 0 && (!experts || !src || !place))) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  STEM_TRY(check_words(c, who, {experts, src, place, offsets}));
  const size_t pairs = (size_t)(T * k) * 4;
  STEM_TRY(check_apart(c, who, {{experts, pairs}}, {{src, pairs}, {place, pairs}, {offsets, (size_t)(n_experts + 1) * 4}}));
  const ExpertsSortArgs a = {experts, (int32_t)(T * k), n_experts, c->experts_counts, src, place, offsets, c->flag};
  HIP_TRY(c, stem_experts_sort_launch(c, a, static_cast<hipStream_t>(stream)));
  return STEM_OK;
}

stem_status stem_experts_dispatch(stem_ctx* c, const void* x, int64_t T, int64_t width, const int32_t* src, int64_t rows, int k, const int32_t* ids,
                                  void* xs, int32_t* ids_out, void* stream) {
  static const char who[] = "stem_experts_dispatch";
  STEM_TRY(stem_enter(c, T));
  STEM_TRY(check_choices(c, who, T, k));
  STEM_TRY(check_rows(c, who, rows, width));
  if (T == 0 || rows == 0) return STEM_OK;
  if (!src || (width > 0 && (!x || !xs))) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  if (!ids != !ids_out) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: ids and ids_out go together", who);
  ExpertsRowsArgs a = rows_args(c, T, rows, width, k);
  const size_t row = width * a.es;
  STEM_TRY(check_words(c, who, {src, ids, ids_out}));
  STEM_TRY(check_buffers(c, who, {{x, T * row}}, {{xs, rows * row}}, false));
  STEM_TRY(check_apart(c, who, {{x, T * row}, {src, (size_t)rows * 4}, {ids, (size_t)T * 4}}, {{xs, rows * row}, {ids_out, (size_t)rows * 4}}));
  a.x = x; a.src = src; a.ids = ids; a.xs = xs; a.ids_out = ids_out;
  HIP_TRY(c, stem_experts_dispatch_launch(c, a, static_cast<hipStream_t>(stream)));
  return STEM_OK;
}

stem_status stem_experts_combine(stem_ctx* c, const void* ys, int64_t rows, int64_t width, const int32_t* place, const float* weights, int64_t T, int k,
                                 const void* residual, void* y, void* stream) {
  static const char who[] = "stem_experts_combine";
  STEM_TRY(stem_enter(c, T));
  STEM_TRY(check_choices(c, who, T, k));
  STEM_TRY(check_rows(c, who, rows, width));
  if (T == 0 || width == 0) return STEM_OK;
  if (!place || (rows > 0 && !ys) || !y) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  ExpertsRowsArgs a = rows_args(c, T, rows, width, k);
  const size_t row = width * a.es, pairs = (size_t)(T * k) * 4;
  STEM_TRY(check_words(c, who, {place, weights}));
  STEM_TRY(check_buffers(c, who, {{residual, T * row}}, {{y, T * row}}, true));
  STEM_TRY(check_buffers(c, who, {{ys, rows * row}}, {{y, T * row}}, false));
  STEM_TRY(check_apart(c, who, {{place, pairs}, {weights, pairs}}, {{y, T * row}}));
  a.ys = ys; a.place = place; a.weights = weights; a.residual = residual; a.y = y;
  HIP_TRY(c, stem_experts_combine_launch(c, a, static_cast<hipStream_t>(stream)));
  return STEM_OK;
}

stem_status stem_experts_combine_backward(stem_ctx* c, const void* dy, const void* ys, int64_t rows, int64_t width, const int32_t* place,
                                          const float* weights, int64_t T, int k, void* dys, float* dweights, void* stream) {
  static const char who[] = "stem_experts_combine_backward";
  STEM_TRY(stem_enter(c, T));
  STEM_TRY(check_choices(c, who, T, k));
  STEM_TRY(check_rows(c, who, rows, width));
  if (T == 0 || (!dys && !dweights)) return STEM_OK;
  if (!place || (width > 0 && !dy)) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  if (dweights && rows > 0 && width > 0 && !ys) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: the weights' gradient needs ys", who);
  ExpertsRowsArgs a = rows_args(c, T, rows, width, k);
  const size_t row = width * a.es, pairs = (size_t)(T * k) * 4;
  STEM_TRY(check_words(c, who, {place, weights, dweights}));
  // (a row of ys is read by the token that writes the same row of dys, but not before)
  STEM_TRY(check_buffers(c, who, {{dy, T * row}, {dweights ? ys : nullptr, rows * row}}, {{dys, rows * row}}, false));
  STEM_TRY(check_apart(c, who, {{place, pairs}, {weights, pairs}, {dy, T * row}, {dweights ? ys : nullptr, rows * row}}, {{dys, rows * row}, {dweights, pairs}}));
  a.x = dy; a.ys = ys; a.place = place; a.weights = weights; a.dys = dys; a.dweights = dweights;
  HIP_TRY(c, stem_experts_combine_backward_launch(c, a, static_cast<hipStream_t>(stream)));
  return STEM_OK;
}

}  // extern "C"
