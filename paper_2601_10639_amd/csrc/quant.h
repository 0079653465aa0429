// 8-bit integer products: layout, arguments and launches (quant.hip, gemm_int8.hip), called by their entry points (api_block.hip).
//
// Layout.  A matrix [rows, K] is kept as blocks of 32 rows x 32 k, 1 KB each: chunk h of row r, 16 bytes of k = 16 h .. 16 h + 15, lies at
// (32 h + r) * 16, so that a block is one operand of v_mfma_i32_32x32x32_i8 with lane l's 16 bytes at 16 l, and a load of it is 1 KB in a
// row wherever it is made from.  The blocks of 32 rows follow each other along k; k is padded with zeros to a multiple of 128 and the
// rows to one of 32.
#pragma once
#include "stem_internal.h"

inline int64_t stem_quant_pitch(int64_t K) { return (K + 127) / 128 * 128; }
inline int64_t stem_quant_size(int64_t rows, int64_t K) { return (rows + 31) / 32 * 32 * stem_quant_pitch(K); }
// Tokens whose hidden values a layer call has in fp32 at a time: up to 128 MiB, so that they are in the memory-side cache when they are read again
inline int64_t stem_quant_chunk(int64_t F) {
  const int64_t n = ((int64_t)128 << 20) / (4 * stem_quant_pitch(F)) / 256 * 256;
  return n < 256 ? 256 : n;
}

struct QuantRowsArgs {
  const bf16_t* x;     // [rows, K]
  int64_t rows;
  int K;
  int pad_rows;        // write zeros for the rows that fill the last block
  stem_norm norm;      // of a row, before it is quantised (bf16 weight)
  int8_t* q;
  float* scale;        // [rows]
  uint32_t* clear;     // set to zero besides; may be null
  int64_t clear_words;
};
hipError_t stem_quant_rows_launch(stem_ctx* ctx, int kid, const QuantRowsArgs& a, hipStream_t s);

struct QuantGemmArgs {
  const int8_t *A, *B;              // tokens [M, K] and weights [N, K], in the layout above
  const float *scale_a, *scale_b;
  int M, N, K;                      // K: padded
  bf16_t* y;                        // [M, N], or null: a gate product
  const bf16_t* residual;           // [M, N], may be null
  float* h;                         // SiLU(product) * E[ids], blocks of 32 tokens x 32 channels, 4 KB: the four channels 8 g + 4 (l / 32) ..
                                    // of token l % 32 at (64 g + l) * 16; channels up to the pitch of N
  uint32_t* amax;                   // [M], zero: takes the bits of each token's largest magnitude
  const int32_t* ids;
  const bf16_t* E;
  int E_rows;
  int32_t* flag;
};
hipError_t stem_quant_gemm_launch(stem_ctx* ctx, int kid, const QuantGemmArgs& a, hipStream_t s);

struct QuantHiddenArgs {
  const float* h;                   // as a gate product leaves them
  const uint32_t* amax;
  int M, blocks;                    // blocks of 32 channels a row
  int8_t* q;                        // tokens of the next product
  float* scale;
};
hipError_t stem_quant_hidden_launch(stem_ctx* ctx, const QuantHiddenArgs& a, hipStream_t s);
