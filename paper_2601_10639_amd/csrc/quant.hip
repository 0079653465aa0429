// Rows to 8-bit integers, for products with a scale for each token and each channel (gemm_int8.hip).
//
//     s_t = max_k |x_tk| / 127,  q_tk = rint(x_tk / s_t);   y_tn = s_t s_n sum_k q_tk q_nk
//
// The sums are exact in 32 bits up to K = 133 000 (127^2 K < 2^31).  A row that holds a NaN or an infinity has no scale: its
// integers are zero and its scale NaN, so that what is made of it is NaN and nothing else is.  A row of zeros, or of values so small that
// their scale would be subnormal, has the scale 2^-126.
#include "quant.h"

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;

namespace {

// ---- rows to integers -------------------------------------------------------------------------------------
// 16 elements of a row from p on, of which `left` are the row's; the others read as zero.  VEC: rows are multiples of 8 elements.
template <bool VEC>
__device__ __forceinline__ void load16(const bf16_t* p, int left, float (&v)[16]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (VEC) {
      bf16x8_t u = {};
      if (left > 8 * h) u = *reinterpret_cast<const bf16x8_t*>(p + 8 * h);
#pragma unroll
      for (int q = 0; q < 8; ++q) v[8 * h + q] = (float)u[q];
    } else {
#pragma unroll
      for (int q = 8 * h; q < 8 * h + 8; ++q) v[q] = q < left ? __uint_as_float((uint32_t)p[q] << 16) : 0.f;
    }
  }
}
__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* red) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return max(max(red[0], red[1]), max(red[2], red[3]));
}

// A workgroup has a row.  VPT: chunks of 16 elements a thread holds; 0: the row is longer than that and is read again for each step.
template <bool VEC, int VPT>
__global__ __launch_bounds__(256) void quant_rows_kernel(QuantRowsArgs p) {
  __shared__ float red[4];
  __shared__ uint32_t redm[4];
  const int64_t row = blockIdx.x;
  const int chunks = (int)((p.K + 127) / 128 * 8);
  int8_t* const out = p.q + (row >> 5) * 32 * (int64_t)chunks * 16 + (row & 31) * 16;
  const bf16_t* const x = p.x + row * p.K;
  constexpr int HELD = VPT ? VPT : 1;
  float v[HELD][16];
  const bool live = row < p.rows;
  if (p.clear)
    for (int64_t i = row * 256 + threadIdx.x; i < p.clear_words; i += (int64_t)gridDim.x * 256) p.clear[i] = 0;
  const int steps = VPT ? VPT : (chunks + 255) / 256;
  auto fetch = [&](int t, float (&u)[16]) {
    const int c = t * 256 + threadIdx.x;
    if (live && c * 16 < p.K) load16<VEC>(x + c * 16, p.K - c * 16, u);
    else
#pragma unroll
      for (int q = 0; q < 16; ++q) u[q] = 0.f;
  };
  if (VPT) {
#pragma unroll
    for (int t = 0; t < HELD; ++t) fetch(t, v[t]);
  }
  // what the row's values are before they are quantised: a norm's mean and factor, and its weight
  float mean = 0.f, r = 1.f;
  if (p.norm.kind != STEM_NORM_NONE) {
    if (p.norm.kind == STEM_NORM_LAYER) {
      float s = 0.f;
      for (int t = 0; t < steps; ++t) {
        if (!VPT) fetch(t, v[0]);
#pragma unroll
        for (int q = 0; q < 16; ++q) s += v[VPT ? t : 0][q];
      }
      mean = block_sum(s, red) / (float)p.K;
    }
    float s = 0.f;
    for (int t = 0; t < steps; ++t) {
      if (!VPT) fetch(t, v[0]);
      const int left = p.K - (t * 256 + (int)threadIdx.x) * 16;
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const float c = q < left ? v[VPT ? t : 0][q] - mean : 0.f;
        s += c * c;
      }
    }
    r = 1.0f / sqrtf(block_sum(s, red) / (float)p.K + p.norm.eps);
  }
  auto finish = [&](int t, float (&u)[16]) {
    if (p.norm.kind == STEM_NORM_NONE) return;
    const int c = t * 256 + threadIdx.x, left = p.K - c * 16;
    float w[16];
    if (p.norm.weight && left > 0) load16<VEC>(static_cast<const bf16_t*>(p.norm.weight) + c * 16, left, w);
#pragma unroll
    for (int q = 0; q < 16; ++q) u[q] = q < left ? (u[q] - mean) * r * (p.norm.weight ? w[q] : 1.f) : 0.f;
  };
  uint32_t top = 0;
  for (int t = 0; t < steps; ++t) {
    if (!VPT) fetch(t, v[0]);
    float (&u)[16] = v[VPT ? t : 0];
    finish(t, u);
#pragma unroll
    for (int q = 0; q < 16; ++q) top = max(top, __float_as_uint(u[q]) & 0x7fffffffu);
  }
  top = block_max(top, redm);
  const bool finite = top < 0x7f800000u;
  const float s = fmaxf(__uint_as_float(top) / 127.0f, 0x1p-126f), inv = finite ? 1.0f / s : 0.f;
  if (threadIdx.x == 0 && live) p.scale[row] = finite ? s : __uint_as_float(0x7fc00000u);
  for (int t = 0; t < steps; ++t) {
    const int c = t * 256 + threadIdx.x;
    if (c >= chunks) break;
    float (&u)[16] = v[VPT ? t : 0];
    if (!VPT) {
      fetch(t, u);
      finish(t, u);
    }
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      w[q] = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        // |u / s| is at most 127 and a rounding
        const int i = finite ? (int)fminf(fmaxf(rintf(u[4 * q + k] * inv), -127.f), 127.f) : 0;
        w[q] |= (uint32_t)(i & 0xff) << (8 * k);
      }
    }
    *reinterpret_cast<uint4*>(out + (int64_t)(c >> 1) * 1024 + (c & 1) * 512) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// ---- hidden values to integers ---------------------------------------------------------------------------------
// A wavefront takes RUN blocks of 32 tokens x 32 channels as the gate product left them: a lane has 16 values of one token, and after a swap
// of half rows (v_permlane32_swap) the 16 that are one chunk of the next product's operand, in the order of the lanes: loads and stores of
// 1 KB throughout.
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
  const uint32_t top = p.amax[m < p.M ? m : p.M - 1];
  const bool finite = top < 0x7f800000u;
  const float s = fmaxf(__uint_as_float(top) / 127.0f, 0x1p-126f), inv = finite ? 1.0f / s : 0.f;
  if (first == 0 && lane < 32 && m < p.M) p.scale[m] = finite ? s : __uint_as_float(0x7fc00000u);
  int8_t* const q = p.q + ((size_t)group * p.blocks + first) * 1024 + lane * 16;
#pragma unroll
  for (int b = 0; b < RUN; ++b) {
    uint32_t w[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      // |v inv| is at most 127 and a rounding: next to 1.5 x 2^23 a float's last digit is 1, and the low byte the integer's
      uint32_t c[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) c[k] = __float_as_uint(__builtin_fmaf(v[b][g][k], inv, 12582912.f));
      w[g] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[3], c[2], 0x0c0c0400), __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400), 0x05040100);
    }
    const u32x2_t lo = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), hi = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    *reinterpret_cast<u32x4_t*>(q + b * 1024) = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
  }
}

template <bool VEC>
hipError_t rows(const QuantRowsArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)(a.pad_rows ? (a.rows + 31) / 32 * 32 : a.rows);
  if (a.K <= 4096) quant_rows_kernel<VEC, 1><<<grid, 256, 0, s>>>(a);
  else if (a.K <= 8192) quant_rows_kernel<VEC, 2><<<grid, 256, 0, s>>>(a);
  else quant_rows_kernel<VEC, 0><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t stem_quant_rows_launch(stem_ctx* ctx, int kid, const QuantRowsArgs& a, hipStream_t s) {
  ProfScope prof(ctx, kid, s);
  return a.K % 8 == 0 ? rows<true>(a, s) : rows<false>(a, s);
}

hipError_t stem_quant_hidden_launch(stem_ctx* ctx, const QuantHiddenArgs& a, hipStream_t s) {
  ProfScope prof(ctx, K_QUANT_HIDDEN, s);
  const int64_t runs = (int64_t)(a.blocks / RUN) * ((a.M + 31) / 32);
  quant_hidden_kernel<<<(unsigned)((runs + 3) / 4), 256, 0, s>>>(a);
  return hipGetLastError();
}
