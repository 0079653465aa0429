// 8-bit integer products: layout, arguments and launches (quant.hip, gemm_int8.hip, gemm_int8_decode.hip), called by their entry points (api_block.hip).
//
// Layout.  A matrix [rows, K] is kept as blocks of 32 rows x 32 k, 1 KB each: chunk h of row r, 16 bytes of k = 16 h .. 16 h + 15, lies at
// (32 h + r) * 16, so that a block is one operand of v_mfma_i32_32x32x32_i8 with lane l's 16 bytes at 16 l, and a load of it is 1 KB in a
// row wherever it is made from.  The blocks of 32 rows follow each other along k; k is padded to a multiple of 128 and the rows to one of
// 32.  Weights are padded with zeros.  What tokens have there is any integer, of hidden values in blocks that no kernel wrote too: behind a row's
// end in k it meets the weights' zeros, and rows past the last one are in no output.
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
  int64_t all_rows;    // with those that fill the last block: by the launcher
};
hipError_t stem_quant_rows_launch(stem_ctx* ctx, int kid, const QuantRowsArgs& a, hipStream_t s);

struct QuantGemmArgs {
  const int8_t *A, *B;              // tokens [M, K] and weights [N, K], in the layout above
  const float *scale_a, *scale_b;
  int M, N, K;                      // K: padded
  int* ws;                          // room for the sums of K slices
  size_t ws_bytes;
  int32_t* tickets;                 // the context's
  int ksplit;                       // by the launcher
  bf16_t* y;                        // [M, N], or null: a gate product
  const bf16_t* residual;           // [M, N], may be null
  float* h;                         // SiLU(product) * E[ids], blocks of 32 tokens x 32 channels, 4 KB: the four channels 8 g + 4 (l / 32) ..
                                    // of token l % 32 at (64 g + l) * 16; blocks of a row: up to the pitch of N
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
  int stride;                       // of amax
  int M, blocks;                    // blocks of 32 channels a row
  int8_t* q;                        // tokens of the next product
  float* scale;
};
hipError_t stem_quant_hidden_launch(stem_ctx* ctx, const QuantHiddenArgs& a, hipStream_t s);

#define STEM_QUANT_DECODE_TOKENS 64
#define QUANT_WS (256 * 128 * 64 * 4)   // bytes: a product is cut into 256 workgroups at most, of tiles of up to 128 x 64
// Every workgroup of a few tokens' product has all of them: their maxima lie in lines of their own, or the atomics of 256 workgroups on one line
// take longer than the product (16 tokens of 2048 x 8192: the gate product 65 us instead of 10)
#define QUANT_AMAX_STRIDE 32
// Products of up to 64 tokens.  Tokens: A and scale_a, or up to 8 that are quantised in place (stem_quant_decode_inline): rows x of row_K
// elements behind a norm, or hidden values h with `maxima` figures for each token.
struct QuantDecodeArgs {
  const int8_t *A, *B;
  const float *scale_a, *scale_b;
  int M, N, K, ksplit;
  const bf16_t* x;
  int row_K;
  stem_norm norm;
  const float* h;
  const uint32_t* max_in;           // [maxima][8]
  int maxima;
  bf16_t* y;                        // [M, N], or null: a gate product
  const bf16_t* residual;
  float* h_out;
  uint32_t* max_out;                // [tiles of 32 channels][8], or null:
  uint32_t* amax;                   // [M] of QUANT_AMAX_STRIDE words, zero: takes the bits of each token's largest magnitude
  const int32_t* ids;
  const bf16_t* E;
  int E_rows;
  int32_t* flag;
  int* ws;                          // partial sums of the K slices
  int32_t* tickets;                 // the context's
};
bool stem_quant_decode_inline(int64_t T, int64_t K);
int stem_quant_decode_slices(int N, int K, size_t ws_bytes, int M);
hipError_t stem_quant_decode_launch(stem_ctx* ctx, int kid, const QuantDecodeArgs& a, hipStream_t s);

// ---- device code of both: 16 elements of a row, as they lie in memory, to integers -------------------------------------
struct QuantChunk { uint32_t w[8]; };
// those past the row's end (`left` elements on) are zero
__device__ __forceinline__ QuantChunk quant_load_chunk(const bf16_t* p, int left) {
  QuantChunk c = {};
  if (left >= 16) {
    __builtin_memcpy(c.w, p, 32);        // (rows of an odd K begin at any 2-byte address)
  } else {
#pragma unroll
    for (int q = 0; q < 16; ++q)
      if (q < left) c.w[q >> 1] |= (uint32_t)p[q] << (16 * (q & 1));
  }
  return c;
}
__device__ __forceinline__ float quant_element(const QuantChunk& c, int q) {
  return __uint_as_float(q & 1 ? c.w[q >> 1] & 0xffff0000u : c.w[q >> 1] << 16);
}
// The low byte is that of rint(v inv), |v inv| at most 127 and a rounding: next to 1.5 x 2^23 a float's last digit is 1.  In two roundings,
// as rint(v inv) has them.
__device__ __forceinline__ uint32_t quant_integer(float v, float inv) {
#pragma clang fp contract(off)
  const float m = v * inv;
  return __float_as_uint(m + 12582912.f);
}
__device__ __forceinline__ uint32_t quant_four_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400), __builtin_amdgcn_perm(b, a, 0x0c0c0400), 0x05040100);
}
// Scale of a row from the bits of its largest magnitude.  A row that holds a NaN or an infinity has none: its integers are zero and its scale
// NaN, so that what is made of it is NaN and nothing else is.  A row of zeros, or of values so small that their scale would be subnormal, has
// the scale 2^-126.
struct QuantScale { float scale, inv; uint32_t mask; };
__device__ __forceinline__ QuantScale quant_scale(uint32_t top) {
  const bool finite = top < 0x7f800000u;
  const float s = fmaxf(__uint_as_float(top) / 127.0f, 0x1p-126f);
  return {finite ? s : __uint_as_float(0x7fc00000u), 1.0f / s, finite ? ~0u : 0u};
}
