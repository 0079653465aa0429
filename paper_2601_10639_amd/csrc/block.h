// Arguments of the kernels around the layer (block.hip), filled in by their entry points (api_block.hip).
#pragma once
#include "stem_internal.h"

#define STEM_BLOCK_MAX_WIDTH 16384   // a row's values stay in a workgroup's registers
#define STEM_BLOCK_WIDE 4096         // longer rows take workgroups of 1024 lanes in the backward pass, of which a compute unit holds one
// Workgroups of a launch of the backward pass, and so partial sums of a gradient that is a sum over tokens
inline int stem_block_grid(int d) { return d > STEM_BLOCK_WIDE ? 256 : 512; }
#define STEM_BLOCK_GRID 512          // at most

struct DropArgs {
  uint32_t threshold;   // of 65536: dropped below it; 0 = nothing is
  float scale;          // of what is kept
  uint64_t seed, offset;
  const uint64_t* step; // device, added to offset; may be null
};

struct BlockArgs {
  int64_t T;
  int d;
  float inv_d;
  const void *f, *x;            // the block's output and the residual stream; backward: x is y, which the next norm was taken of
  stem_norm out, next;
  float residual_scale, branch_scale;
  int gate_kind;
  const void* gate;
  DropArgs drop;
  void *y, *n;                  // forward
  const void *dy, *dn;          // backward: either may be null
  void *dx, *df, *dgate;        // dgate: of a token or an element
  int accumulate;
  float* part_of[3];            // where sums over tokens go (dw_next, dw_out, a channel's gate); null = not wanted
  float* part[3];               // [0]: room for their partial sums
};

hipError_t stem_block_forward_launch(stem_ctx* ctx, int is_bf16, bool branch, const BlockArgs& a, hipStream_t s);
hipError_t stem_block_backward_launch(stem_ctx* ctx, int is_bf16, bool branch, const BlockArgs& a, hipStream_t s);
hipError_t stem_dropout_launch(stem_ctx* ctx, int is_bf16, const void* x, int64_t T, int64_t d, const DropArgs& drop, void* y, hipStream_t s);
