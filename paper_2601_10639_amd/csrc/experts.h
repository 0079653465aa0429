// Tokens to experts and back (experts.hip), called by its entry points (api_experts.hip).
#pragma once
#include "stem_internal.h"

// (token, choice) pairs up to which a workgroup of the sort has 1024 of them, and 4096 beyond; and rows of counts that sorts of up to this many need: one for each
// segment, and the totals
#define EXPERTS_SMALL 65536
inline int64_t stem_experts_segments(int64_t pairs) { return EXPERTS_SMALL / 1024 + pairs / 4096; }

struct ExpertsSortArgs {
  const int32_t* experts;   // [pairs]
  int32_t pairs, n;
  int32_t* counts;          // [segments + 1][n + 1]: of more than one segment
  int32_t *src, *place, *offsets;
  int32_t* flag;
};
hipError_t stem_experts_sort_launch(stem_ctx* ctx, const ExpertsSortArgs& a, hipStream_t s);

struct ExpertsRowsArgs {
  int es;                   // bytes of an element: 2 (bf16) or 4 (fp32)
  int64_t T, rows, width;   // tokens, sorted rows, elements of a row
  int k;
  const void* x;            // dispatch: [T, width]; combine's backward: dy
  const void* ys;           // [rows, width]
  const int32_t *src, *place, *ids;
  const float* weights;     // [T, k], may be null
  const void* residual;
  void *xs, *y, *dys;
  int32_t* ids_out;
  float* dweights;
  int32_t* flag;
};
hipError_t stem_experts_dispatch_launch(stem_ctx* ctx, const ExpertsRowsArgs& a, hipStream_t s);
hipError_t stem_experts_combine_launch(stem_ctx* ctx, const ExpertsRowsArgs& a, hipStream_t s);
hipError_t stem_experts_combine_backward_launch(stem_ctx* ctx, const ExpertsRowsArgs& a, hipStream_t s);
