// Rows to 8-bit integers, for products with a scale for each token and each channel (gemm_int8.hip).
//
//     s_t = max_k |x_tk| / 127,  q_tk = rint(x_tk / s_t);   y_tn = s_t s_n sum_k q_tk q_nk
//
// The sums are exact in 32 bits up to K = 133 000 (127^2 K < 2^31).
#include "quant.h"

typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;

namespace {

// ---- rows to integers -------------------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }

// LPR neighbouring lanes have a row (256: the workgroup).  f: of two values in each lane's place, given and taken as bits.
template <int LPR, class F>
__device__ __forceinline__ uint32_t over_row(uint32_t v, uint32_t* red, F f) {
  v = f(v, dpp<0xb1>(v));                                   // quad_perm 1 0 3 2
  v = f(v, dpp<0x4e>(v));                                   // quad_perm 2 3 0 1
  v = f(v, dpp<0x141>(v));                                  // row_half_mirror
  if (LPR > 8) v = f(v, dpp<0x140>(v));                     // row_mirror
  if (LPR > 16) v = f(v, (uint32_t)__shfl_xor((int)v, 16));
  if (LPR > 32) v = f(v, (uint32_t)__shfl_xor((int)v, 32));
  if (LPR > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = f(f(red[0], red[1]), f(red[2], red[3]));
  }
  return v;
}
template <int LPR>
__device__ __forceinline__ float sum_row(float v, uint32_t* red) {
  return __uint_as_float(over_row<LPR>(__float_as_uint(v), red, [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// A row's chunks lie 512 bytes apart in its block row, and 8 neighbouring rows' chunks in a line.  With few lanes a
// row a wavefront stores longer pieces of a line, and waits for more of its loads before it has a row.  us, 16 / 32 / 64 / 256 lanes a row, behind a
// norm: 16384 x 2048 32 / 28 / 32 / 46, 1000 x 2048 12 / 9 / 8 / 9; without one, 16384 x 4096 - / 47 / 59 / 75, 8192 x 8192 - / - / 61 / 77.
// CPT: chunks a lane holds, in fp32; 0: the row is longer and is read again for each step.
template <int LPR, int CPT>
__global__ __launch_bounds__(256) void quant_rows_kernel(QuantRowsArgs p) {
  __shared__ uint32_t red[4];
  constexpr int ROWS = 256 / LPR, HELD = CPT ? CPT : 1;
  // a norm's weight, read by every row: from LDS where a workgroup has several
  constexpr bool SHARED = LPR <= 64;
  __shared__ QuantChunk weight[SHARED ? LPR * HELD : 1];
  const int l = threadIdx.x % LPR;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR;
  if (p.clear)
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.clear_words; i += (int64_t)gridDim.x * 256) p.clear[i] = 0;
  const int chunks = (p.K + 127) / 128 * 8;
  const bool live = row < p.rows;
  const bf16_t* const x = p.x + (live ? row : 0) * p.K;
  auto fetch = [&](int t) __attribute__((always_inline)) {
    const int c = t * LPR + l;
    return live && c * 16 < p.K ? quant_load_chunk(x + c * 16, p.K - c * 16) : QuantChunk{};
  };
  QuantChunk raw[HELD] = {};
  if constexpr (CPT > 0) {
#pragma unroll
    for (int t = 0; t < CPT; ++t)
      if (t * LPR < chunks) raw[t] = fetch(t);
  }
  if (SHARED && p.norm.weight) {
    for (int c = threadIdx.x; c * 16 < p.K; c += 256) weight[c] = quant_load_chunk(static_cast<const bf16_t*>(p.norm.weight) + c * 16, p.K - c * 16);
    __syncthreads();
  }
  if (LPR <= 64 && row >= p.all_rows) return;               // (whole groups of lanes that exchange nothing with others)
  // f on each step's values, which it may change where the lane holds them; otherwise they are made again
  float v[HELD][16];
  auto elements = [&](const QuantChunk& c, float (&u)[16]) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < 16; ++q) u[q] = quant_element(c, q);
  };
  if constexpr (CPT > 0) {
#pragma unroll
    for (int t = 0; t < CPT; ++t) elements(raw[t], v[t]);
  }
  // zeros behind the row's end
  auto cut = [&](int t, float (&u)[16]) __attribute__((always_inline)) {
    const int left = p.K - (t * LPR + l) * 16;
    if (left < 16)
#pragma unroll
      for (int q = 0; q < 16; ++q) u[q] = q < left ? u[q] : 0.f;
  };
  float mean = 0.f, r = 1.f;
  // the values a step has after its norm so far (stage 1: centred, 2: normed and weighted)
  auto advance = [&](int stage, int t, float (&u)[16]) __attribute__((always_inline)) {
    if (stage == 1) {
#pragma unroll
      for (int q = 0; q < 16; ++q) u[q] -= mean;
    } else {
      const int at = t * LPR + l;
      if (p.norm.weight) {
        const QuantChunk w = at * 16 >= p.K ? QuantChunk{} : SHARED ? weight[at] : quant_load_chunk(static_cast<const bf16_t*>(p.norm.weight) + at * 16, p.K - at * 16);
#pragma unroll
        for (int q = 0; q < 16; ++q) u[q] = u[q] * r * quant_element(w, q);
      } else {
#pragma unroll
        for (int q = 0; q < 16; ++q) u[q] *= r;
      }
    }
    cut(t, u);
  };
  const bool centred = p.norm.kind == STEM_NORM_LAYER, normed = p.norm.kind != STEM_NORM_NONE || p.norm.weight;
  // f(t, values) for every step, after `stage` steps of the norm, the last of them taken now
  auto each_step = [&](int stage, auto f) __attribute__((always_inline)) {
    if constexpr (CPT > 0) {
#pragma unroll
      for (int t = 0; t < CPT; ++t)
        if (t * LPR < chunks) {
          if (stage == 1 && centred) advance(1, t, v[t]);
          if (stage == 2 && normed) advance(2, t, v[t]);
          f(t, v[t]);
        }
    } else {
      for (int t = 0; t * LPR < chunks; ++t) {
        elements(fetch(t), v[0]);
        if (stage >= 1 && centred) advance(1, t, v[0]);
        if (stage >= 2 && normed) advance(2, t, v[0]);
        f(t, v[0]);
      }
    }
  };
  if (p.norm.kind != STEM_NORM_NONE) {
    float s = 0.f;
    if (centred) {
      each_step(0, [&](int, float (&u)[16]) {
#pragma unroll
        for (int q = 0; q < 16; ++q) s += u[q];
      });
      mean = sum_row<LPR>(s, red) / (float)p.K;
      s = 0.f;
    }
    each_step(1, [&](int, float (&u)[16]) {
#pragma unroll
      for (int q = 0; q < 16; ++q) s += u[q] * u[q];
    });
    r = 1.0f / sqrtf(sum_row<LPR>(s, red) / (float)p.K + p.norm.eps);
  }
  uint32_t top = 0;
  each_step(2, [&](int, float (&u)[16]) {
#pragma unroll
    for (int q = 0; q < 16; q += 2) top = max(max(top, __float_as_uint(u[q]) & 0x7fffffffu), __float_as_uint(u[q + 1]) & 0x7fffffffu);
  });
  top = over_row<LPR>(top, red, [](uint32_t a, uint32_t b) { return max(a, b); });
  const QuantScale s = quant_scale(top);
  if (l == 0 && live) p.scale[row] = s.scale;
  int8_t* const out = p.q + (row >> 5) * 32 * (int64_t)chunks * 16 + (row & 31) * 16;
  each_step(CPT ? 3 : 2, [&](int t, float (&u)[16]) {
    const int c = t * LPR + l;
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      w[q] = quant_four_bytes(quant_integer(u[4 * q], s.inv), quant_integer(u[4 * q + 1], s.inv), quant_integer(u[4 * q + 2], s.inv), quant_integer(u[4 * q + 3], s.inv)) & s.mask;
    if (c < chunks) *reinterpret_cast<u32x4_t*>(out + (int64_t)(c >> 1) * 1024 + (c & 1) * 512) = u32x4_t{w[0], w[1], w[2], w[3]};
  });
}

// ---- hidden values to integers ---------------------------------------------------------------------------------
// A wavefront takes RUN blocks of 32 tokens x 32 channels as the gate product left them: a lane has 16 values of one token, and after a swap
// of half rows (v_permlane32_swap) the 16 that are one chunk of the next product's operand, in the order of the lanes: loads and stores of
// 1 KB throughout.  Measured: 27 us for 4096 x 8192 values, 6.2 TB/s read and written, the values still in the memory-side cache for half of them.
constexpr int RUN = 4;   // (rows are whole 128 channels)
__global__ __launch_bounds__(256) void quant_hidden_kernel(QuantHiddenArgs p) {
  const int lane = threadIdx.x & 63;
  const int runs = p.blocks / RUN, groups = (p.M + 31) / 32;
  const int64_t run = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (run >= (int64_t)runs * groups) return;
  const int group = (int)(run / runs), first = (int)(run % runs) * RUN, m = group * 32 + (lane & 31);
  const float* const h = p.h + ((size_t)group * p.blocks + first) * 1024 + lane * 4;
  f32x4_t v[RUN][4];
#pragma unroll
  for (int b = 0; b < RUN; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) v[b][g] = *reinterpret_cast<const f32x4_t*>(h + b * 1024 + g * 256);
  const QuantScale s = quant_scale(p.amax[(m < p.M ? m : p.M - 1) * p.stride]);
  if (first == 0 && lane < 32 && m < p.M) p.scale[m] = s.scale;
  int8_t* const q = p.q + ((size_t)group * p.blocks + first) * 1024 + lane * 16;
#pragma unroll
  for (int b = 0; b < RUN; ++b) {
    uint32_t w[4];
#pragma unroll
    for (int g = 0; g < 4; ++g)
      w[g] = quant_four_bytes(quant_integer(v[b][g][0], s.inv), quant_integer(v[b][g][1], s.inv), quant_integer(v[b][g][2], s.inv), quant_integer(v[b][g][3], s.inv)) & s.mask;
    const u32x2_t lo = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), hi = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    *reinterpret_cast<u32x4_t*>(q + b * 1024) = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
  }
}

template <int LPR, int CPT>
void launch_rows(const QuantRowsArgs& a, hipStream_t s) {
  quant_rows_kernel<LPR, CPT><<<(unsigned)((a.all_rows * LPR + 255) / 256), 256, 0, s>>>(a);
}

}  // namespace

hipError_t stem_quant_rows_launch(stem_ctx* ctx, int kid, const QuantRowsArgs& p, hipStream_t s) {
  ProfScope prof(ctx, kid, s);
  QuantRowsArgs a = p;
  a.all_rows = a.pad_rows ? (a.rows + 31) / 32 * 32 : a.rows;
  if (a.K <= 2048) a.all_rows >= 2048 ? launch_rows<32, 4>(a, s) : launch_rows<64, 2>(a, s);
  else if (a.K <= 4096) a.all_rows >= 2048 ? launch_rows<32, 8>(a, s) : launch_rows<256, 1>(a, s);
  else if (a.K <= 8192) a.all_rows >= 1024 ? launch_rows<64, 8>(a, s) : launch_rows<256, 2>(a, s);
  else launch_rows<256, 0>(a, s);
  return hipGetLastError();
}

hipError_t stem_quant_hidden_launch(stem_ctx* ctx, const QuantHiddenArgs& a, hipStream_t s) {
  ProfScope prof(ctx, K_QUANT_HIDDEN, s);
  const int64_t runs = (int64_t)(a.blocks / RUN) * ((a.M + 31) / 32);
  quant_hidden_kernel<<<(unsigned)((runs + 3) / 4), 256, 0, s>>>(a);
  return hipGetLastError();
}
