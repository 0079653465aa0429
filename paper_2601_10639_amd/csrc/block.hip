// What a decoder block does around the layer: the norm in front of it, and behind it the norm, dropout, gate and residual
// joined with the norm in front of the next block; their backward passes; and dropout by itself.
//
//     u = N_out(f) * w_out;   y = a x + b g * D(u);   n = N_next(y) * w_next
//
// N is v / sqrt(mean v^2 + eps), or (v - mean) / sqrt(var + eps).  With v^ = N(v) and r = 1 / sqrt(...), the gradient of N's
// input for the gradient h of its output is  r (h - v^ mean(h v^))  and for the second kind  r (h - mean(h) - v^ mean(h v^)).
// So the backward pass is, with h1 = dn * w_next:
//     G = dy + N_next'(h1);  dx = a G;  h = b G;  dg = h * D(u);  du = mask * (h * g);  df = N_out'(du * w_out);
//     dw_next = sum over tokens of dn * y^;  dw_out = sum over tokens of du * f^.
// The statistics are taken again from f and y, which the backward pass reads anyway: storing them would save a reduction
// over registers and cost the caller two buffers.
#include "block.h"

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;

namespace {

// ---- eight consecutive elements of a row, in fp32 --------------------------------------------------
// `left`: elements of the row from p on, 4 or more (an fp32 row ends on a multiple of 4, a bf16 row on one of 64)
__device__ __forceinline__ void load8(const bf16_t* p, int, float (&v)[8]) {
  const bf16x8_t u = *reinterpret_cast<const bf16x8_t*>(p);
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = (float)u[q];
}
__device__ __forceinline__ void load8(const float* p, int left, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p);
  const float4 b = left > 4 ? *reinterpret_cast<const float4*>(p + 4) : make_float4(0.f, 0.f, 0.f, 0.f);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store8(bf16_t* p, int, const float (&v)[8]) {
  bf16x8_t u;
#pragma unroll
  for (int q = 0; q < 8; ++q) u[q] = (__bf16)v[q];
  *reinterpret_cast<bf16x8_t*>(p) = u;
}
__device__ __forceinline__ void store8(float* p, int left, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  if (left > 4) *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ float load1(const bf16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ void store1(bf16_t* p, float v) { *reinterpret_cast<__bf16*>(p) = (__bf16)v; }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

// ---- dropout's generator -----------------------------------------------------------------------------
// Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): a bijection
// of the counter (column / 8, row, offset) keyed by the seed.  The 128 bits of a counter serve eight neighbouring elements,
// 16 each: a call for four elements, 32 bits each, would make the generator and not memory the bound of the dropout kernel.
struct Bits { uint32_t w[4]; };
__device__ __forceinline__ Bits philox(uint32_t c0, uint32_t c1, uint64_t offset, uint64_t seed) {
  uint32_t c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32), k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}
__device__ __forceinline__ bool kept(const Bits& r, int q, uint32_t threshold) {
  return (q & 1 ? r.w[q >> 1] >> 16 : r.w[q >> 1] & 0xffffu) >= threshold;
}
__device__ __forceinline__ uint64_t offset_of(const DropArgs& d) { return d.offset + (d.step ? *d.step : 0); }

// ---- sums over a row ---------------------------------------------------------------------------------
// LPR neighbouring lanes hold a row (a power of two; more than 64: whole wavefronts).  Every lane gets every sum.  `red` has
// room for two sets of partial sums, taken in turn, so that one barrier a reduction is enough.
template <int LPR>
struct RowSum {
  static constexpr int WPR = LPR > 64 ? LPR / 64 : 1;   // wavefronts that share a row
  float (*red)[WPR][2];
  int turn;
  template <int N>
  __device__ __forceinline__ void operator()(float (&v)[N]) {
    static_assert(N <= 2, "room in red");
#pragma unroll
    for (int o = 1; o < (LPR < 64 ? LPR : 64); o <<= 1)
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], o);
    if (WPR > 1) {
      const int wave = (threadIdx.x >> 6) % WPR;
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < N; ++k) red[turn][wave][k] = v[k];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < N; ++k) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < WPR; ++w) s += red[turn][w][k];
        v[k] = s;
      }
      turn ^= 1;
    }
  }
};

template <int LPR, int VPT>
struct Shape {
  static constexpr int THREADS = LPR > 256 ? LPR : 256;
  static constexpr int SLOTS = THREADS / LPR;             // rows a workgroup has in hand
  static constexpr int WPR = RowSum<LPR>::WPR;
};

// v <- N(v), and 1 / sqrt(...).  Elements past the row's end are zero and stay zero.  The variance is of the centred values: the
// difference of two sums of squares would lose what a large mean shifts out.
template <int LPR, int VPT>
__device__ __forceinline__ float normalise(float (&v)[VPT][8], const bool (&in)[VPT], const int (&left)[VPT], int kind, float eps, float inv_d,
                                           RowSum<LPR>& row_sum) {
  if (kind == STEM_NORM_NONE) return 1.f;
  if (kind == STEM_NORM_LAYER) {
    float s[1] = {0.f};
#pragma unroll
    for (int t = 0; t < VPT; ++t)
#pragma unroll
      for (int q = 0; q < 8; ++q) s[0] += v[t][q];
    row_sum(s);
    const float mean = s[0] * inv_d;
#pragma unroll
    for (int t = 0; t < VPT; ++t)
#pragma unroll
      for (int q = 0; q < 8; ++q) v[t][q] = in[t] && q < left[t] ? v[t][q] - mean : 0.f;
  }
  float s[1] = {0.f};
#pragma unroll
  for (int t = 0; t < VPT; ++t)
#pragma unroll
    for (int q = 0; q < 8; ++q) s[0] += v[t][q] * v[t][q];
  row_sum(s);
  const float r = 1.0f / sqrtf(s[0] * inv_d + eps);
#pragma unroll
  for (int t = 0; t < VPT; ++t)
#pragma unroll
    for (int q = 0; q < 8; ++q) v[t][q] *= r;
  return r;
}

// h <- the gradient of N's input, h being that of its output v^ (past the row's end zero, and again afterwards)
template <int LPR, int VPT>
__device__ __forceinline__ void normalise_back(float (&h)[VPT][8], const float (&v)[VPT][8], const bool (&in)[VPT], const int (&left)[VPT], float r,
                                               int kind, float inv_d, RowSum<LPR>& row_sum) {
  if (kind == STEM_NORM_NONE) return;
  float s[2] = {0.f, 0.f};
#pragma unroll
  for (int t = 0; t < VPT; ++t)
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      s[0] += h[t][q] * v[t][q];
      s[1] += h[t][q];
    }
  row_sum(s);
  const float along = s[0] * inv_d, mean = kind == STEM_NORM_LAYER ? s[1] * inv_d : 0.f;
#pragma unroll
  for (int t = 0; t < VPT; ++t)
#pragma unroll
    for (int q = 0; q < 8; ++q) h[t][q] = in[t] && q < left[t] ? r * (h[t][q] - mean - v[t][q] * along) : 0.f;
}

// ---- forward -------------------------------------------------------------------------------------------
// BRANCH: the end of a block; without it y is x and only n is written.  One pass: a row's values stay in registers from its loads
// to its stores.
template <class E, int LPR, int VPT, bool BRANCH>
__global__ __launch_bounds__((Shape<LPR, VPT>::THREADS)) void block_forward_kernel(BlockArgs p) {
  typedef Shape<LPR, VPT> S;
  __shared__ float red[S::SLOTS][2][S::WPR][2];
  const int slot = threadIdx.x / LPR, lane = threadIdx.x % LPR;
  RowSum<LPR> row_sum{red[slot], 0};
  bool in[VPT];
  int col[VPT], left[VPT];
#pragma unroll
  for (int t = 0; t < VPT; ++t) {
    col[t] = (t * LPR + lane) * 8;
    in[t] = col[t] < p.d;
    left[t] = p.d - col[t];
  }
  const uint64_t offset = BRANCH && p.drop.threshold ? offset_of(p.drop) : 0;
  for (int64_t base = (int64_t)blockIdx.x * S::SLOTS; base < p.T; base += (int64_t)gridDim.x * S::SLOTS) {
    const int64_t row = base + slot;
    const bool live = row < p.T;
    const size_t at = (size_t)(live ? row : p.T - 1) * p.d;
    float y[VPT][8], f[VPT][8];
#pragma unroll
    for (int t = 0; t < VPT; ++t) {
#pragma unroll
      for (int q = 0; q < 8; ++q) y[t][q] = f[t][q] = 0.f;
      if (in[t]) load8(static_cast<const E*>(p.x) + at + col[t], left[t], y[t]);
      if (BRANCH && in[t]) load8(static_cast<const E*>(p.f) + at + col[t], left[t], f[t]);
    }
    if (BRANCH) {
      normalise<LPR, VPT>(f, in, left, p.out.kind, p.out.eps, p.inv_d, row_sum);
      const float of_token = p.gate_kind == STEM_GATE_TOKEN ? load1(static_cast<const E*>(p.gate) + (live ? row : p.T - 1)) : 1.f;
#pragma unroll
      for (int t = 0; t < VPT; ++t) {
        if (!in[t]) continue;
        if (p.out.weight) {
          float w[8];
          load8(static_cast<const E*>(p.out.weight) + col[t], left[t], w);
#pragma unroll
          for (int q = 0; q < 8; ++q) f[t][q] *= w[q];
        }
        if (p.drop.threshold) {
          const Bits r = philox((uint32_t)(col[t] >> 3), (uint32_t)row, offset, p.drop.seed);
#pragma unroll
          for (int q = 0; q < 8; ++q) f[t][q] = kept(r, q, p.drop.threshold) ? f[t][q] * p.drop.scale : 0.f;
        }
        if (p.gate_kind == STEM_GATE_CHANNEL || p.gate_kind == STEM_GATE_FULL) {
          float g[8];
          load8(static_cast<const E*>(p.gate) + (p.gate_kind == STEM_GATE_FULL ? at : 0) + col[t], left[t], g);
#pragma unroll
          for (int q = 0; q < 8; ++q) f[t][q] *= g[q];
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) y[t][q] = p.residual_scale * y[t][q] + p.branch_scale * (f[t][q] * of_token);
        if (live) store8(static_cast<E*>(p.y) + at + col[t], left[t], y[t]);
      }
    }
    if (p.n) {
      normalise<LPR, VPT>(y, in, left, p.next.kind, p.next.eps, p.inv_d, row_sum);
#pragma unroll
      for (int t = 0; t < VPT; ++t) {
        if (!in[t]) continue;
        if (p.next.weight) {
          float w[8];
          load8(static_cast<const E*>(p.next.weight) + col[t], left[t], w);
#pragma unroll
          for (int q = 0; q < 8; ++q) y[t][q] *= w[q];
        }
        if (live) store8(static_cast<E*>(p.n) + at + col[t], left[t], y[t]);
      }
    }
  }
}

// ---- backward ------------------------------------------------------------------------------------------
// Sums over tokens (of dw_next, dw_out and a gate a channel) are held in registers over a workgroup's rows and written as one partial
// sum a workgroup, [sum][workgroup][d]; block_sums_kernel adds those in order.  No atomics: the same bits on every run.
template <class E, int LPR, int VPT, bool BRANCH>
__global__ __launch_bounds__((Shape<LPR, VPT>::THREADS)) void block_backward_kernel(BlockArgs p) {
  typedef Shape<LPR, VPT> S;
  __shared__ float red[S::SLOTS][2][S::WPR][2];
  __shared__ float sums[S::SLOTS > 1 ? S::THREADS * VPT * 8 : 1];
  const int slot = threadIdx.x / LPR, lane = threadIdx.x % LPR;
  RowSum<LPR> row_sum{red[slot], 0};
  bool in[VPT];
  int col[VPT], left[VPT];
#pragma unroll
  for (int t = 0; t < VPT; ++t) {
    col[t] = (t * LPR + lane) * 8;
    in[t] = col[t] < p.d;
    left[t] = p.d - col[t];
  }
  const uint64_t offset = BRANCH && p.drop.threshold ? offset_of(p.drop) : 0;
  float sum_next[VPT][8], sum_out[VPT][8], sum_gate[VPT][8];
#pragma unroll
  for (int t = 0; t < VPT; ++t)
#pragma unroll
    for (int q = 0; q < 8; ++q) sum_next[t][q] = sum_out[t][q] = sum_gate[t][q] = 0.f;
  for (int64_t base = (int64_t)blockIdx.x * S::SLOTS; base < p.T; base += (int64_t)gridDim.x * S::SLOTS) {
    const int64_t row = base + slot;
    const bool live = row < p.T;
    const size_t at = (size_t)(live ? row : p.T - 1) * p.d;
    float G[VPT][8];
#pragma unroll
    for (int t = 0; t < VPT; ++t) {
#pragma unroll
      for (int q = 0; q < 8; ++q) G[t][q] = 0.f;
      if (p.dy && in[t]) load8(static_cast<const E*>(p.dy) + at + col[t], left[t], G[t]);
    }
    if (p.dn) {
      float y[VPT][8], h[VPT][8];
#pragma unroll
      for (int t = 0; t < VPT; ++t) {
#pragma unroll
        for (int q = 0; q < 8; ++q) y[t][q] = h[t][q] = 0.f;
        if (in[t]) {
          load8(static_cast<const E*>(p.x) + at + col[t], left[t], y[t]);
          load8(static_cast<const E*>(p.dn) + at + col[t], left[t], h[t]);
        }
      }
      const float r = normalise<LPR, VPT>(y, in, left, p.next.kind, p.next.eps, p.inv_d, row_sum);
#pragma unroll
      for (int t = 0; t < VPT; ++t) {
        if (live)
#pragma unroll
          for (int q = 0; q < 8; ++q) sum_next[t][q] += h[t][q] * y[t][q];
        if (p.next.weight && in[t]) {
          float w[8];
          load8(static_cast<const E*>(p.next.weight) + col[t], left[t], w);
#pragma unroll
          for (int q = 0; q < 8; ++q) h[t][q] *= w[q];
        }
      }
      normalise_back<LPR, VPT>(h, y, in, left, r, p.next.kind, p.inv_d, row_sum);
#pragma unroll
      for (int t = 0; t < VPT; ++t)
#pragma unroll
        for (int q = 0; q < 8; ++q) G[t][q] += h[t][q];
    }
    auto store_dx = [&](int t) {   // of a vector whose inputs have all been read: dx may be any of them
      if (!p.dx || !live) return;
      float o[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) o[q] = p.residual_scale * G[t][q];
      store8(static_cast<E*>(p.dx) + at + col[t], left[t], o);
    };
    if (!BRANCH) {
#pragma unroll
      for (int t = 0; t < VPT; ++t)
        if (in[t]) store_dx(t);
      continue;
    }
    float f[VPT][8];
#pragma unroll
    for (int t = 0; t < VPT; ++t) {
#pragma unroll
      for (int q = 0; q < 8; ++q) f[t][q] = 0.f;
      if (p.f && in[t]) load8(static_cast<const E*>(p.f) + at + col[t], left[t], f[t]);
    }
    const float r = normalise<LPR, VPT>(f, in, left, p.out.kind, p.out.eps, p.inv_d, row_sum);
    const float of_token = p.gate_kind == STEM_GATE_TOKEN ? load1(static_cast<const E*>(p.gate) + (live ? row : p.T - 1)) : 1.f;
    float of_gate[1] = {0.f};
#pragma unroll
    for (int t = 0; t < VPT; ++t) {
      if (!in[t]) continue;
      float w[8], g[8], keep[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) { w[q] = 1.f; g[q] = of_token; keep[q] = 1.f; }
      if (p.out.weight) load8(static_cast<const E*>(p.out.weight) + col[t], left[t], w);
      if (p.gate_kind == STEM_GATE_CHANNEL || p.gate_kind == STEM_GATE_FULL)
        load8(static_cast<const E*>(p.gate) + (p.gate_kind == STEM_GATE_FULL ? at : 0) + col[t], left[t], g);
      if (p.drop.threshold) {
        const Bits b = philox((uint32_t)(col[t] >> 3), (uint32_t)row, offset, p.drop.seed);
#pragma unroll
        for (int q = 0; q < 8; ++q) keep[q] = kept(b, q, p.drop.threshold) ? p.drop.scale : 0.f;
      }
      store_dx(t);
      float dg[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float h = p.branch_scale * G[t][q];
        // (what is dropped counts for nothing, whatever f holds there)
        const float u = keep[q] != 0.f ? f[t][q] * w[q] * keep[q] : 0.f, du = keep[q] != 0.f ? h * g[q] * keep[q] : 0.f;
        dg[q] = h * u;
        if (live) {
          sum_out[t][q] += du * f[t][q];
          sum_gate[t][q] += dg[q];
        }
        of_gate[0] += q < left[t] ? dg[q] : 0.f;
        G[t][q] = du * w[q];
      }
      if (p.gate_kind == STEM_GATE_FULL && p.dgate && live) store8(static_cast<E*>(p.dgate) + at + col[t], left[t], dg);
    }
    if (p.gate_kind == STEM_GATE_TOKEN && p.dgate) {
      row_sum(of_gate);
      if (live && lane == 0) store1(static_cast<E*>(p.dgate) + row, of_gate[0]);
    }
    if (p.df) {
      normalise_back<LPR, VPT>(G, f, in, left, r, p.out.kind, p.inv_d, row_sum);
      if (live)
#pragma unroll
        for (int t = 0; t < VPT; ++t)
          if (in[t]) store8(static_cast<E*>(p.df) + at + col[t], left[t], G[t]);
    }
  }
  auto write = [&](float (&sum)[VPT][8], float* part) {
    if (!part) return;
    float* const to = part + (size_t)blockIdx.x * p.d;
    if (S::SLOTS == 1) {
#pragma unroll
      for (int t = 0; t < VPT; ++t)
        if (in[t]) store8(to + col[t], left[t], sum[t]);
      return;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < VPT; ++t)
#pragma unroll
      for (int q = 0; q < 8; ++q) sums[(slot * VPT + t) * LPR * 8 + lane * 8 + q] = sum[t][q];
    __syncthreads();
    for (int c = threadIdx.x; c < p.d; c += S::THREADS) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < S::SLOTS; ++k) s += sums[k * VPT * LPR * 8 + c];
      to[c] = s;
    }
  };
  write(sum_next, p.part[0]);
  if (BRANCH) {
    write(sum_out, p.part[1]);
    write(sum_gate, p.part[2]);
  }
}

// out[c] (+)= sum of part[k][c] over k < n, for up to three sums: four stretches of k, each in order, these in order
struct SumArgs { const float* part[3]; float* out[3]; int n, d, accumulate; };
__global__ __launch_bounds__(256) void block_sums_kernel(SumArgs p) {
  __shared__ float s[4][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), k = threadIdx.x >> 6, which = blockIdx.y;
  const float* const part = which == 0 ? p.part[0] : which == 1 ? p.part[1] : p.part[2];
  float* const out = which == 0 ? p.out[0] : which == 1 ? p.out[1] : p.out[2];
  float v = 0.f;
  if (c < p.d)
    for (int i = k * p.n / 4; i < (k + 1) * p.n / 4; ++i) v += part[(size_t)i * p.d + c];
  s[k][threadIdx.x & 63] = v;
  __syncthreads();
  if (k == 0 && c < p.d) {
    v = (s[0][threadIdx.x] + s[1][threadIdx.x]) + (s[2][threadIdx.x] + s[3][threadIdx.x]);
    out[c] = p.accumulate ? out[c] + v : v;
  }
}

// ---- dropout by itself -------------------------------------------------------------------------------------
// A thread has the eight elements of a counter; `tx` (a power of two) threads lie along a row.
template <class E>
__global__ __launch_bounds__(256) void dropout_kernel(const E* x, E* y, int64_t T, int64_t d, int tx_log, DropArgs drop,
                                                      int vectors) {
  const int tx = 1 << tx_log;
  const int64_t columns = (d + 7) / 8;
  const int64_t tiles = (columns + tx - 1) >> tx_log;
  const int64_t row = (int64_t)(blockIdx.x / tiles) * (256 >> tx_log) + (threadIdx.x >> tx_log);
  const int64_t c = ((int64_t)(blockIdx.x % tiles) << tx_log) + (threadIdx.x & (tx - 1));
  if (row >= T || c >= columns) return;
  const Bits r = philox((uint32_t)c, (uint32_t)row, offset_of(drop), drop.seed);
  const int64_t at = row * d + c * 8;
  if (vectors) {
    float v[8];
    load8(x + at, 8, v);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = kept(r, q, drop.threshold) ? v[q] * drop.scale : 0.f;
    store8(y + at, 8, v);
  } else {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (c * 8 + q < d) store1(y + at + q, kept(r, q, drop.threshold) ? load1(x + at + q) * drop.scale : 0.f);
  }
}

// ---- launches ------------------------------------------------------------------------------------------------
template <class E, int LPR, int VPT, bool BRANCH, bool BACK>
hipError_t launch(const BlockArgs& a, int64_t most, hipStream_t s, int* grid_out) {
  typedef Shape<LPR, VPT> S;
  const int64_t groups = (a.T + S::SLOTS - 1) / S::SLOTS;
  const int grid = (int)(groups < most ? groups : most);
  if (grid_out) *grid_out = grid;
  BlockArgs p = a;
  if (BACK) {
    float* to = a.part[0];
    const bool want[3] = {a.part_of[0] != nullptr, a.part_of[1] != nullptr, a.part_of[2] != nullptr};
    for (int k = 0; k < 3; ++k) {
      p.part[k] = want[k] ? to : nullptr;
      if (want[k]) to += (size_t)grid * a.d;
    }
    block_backward_kernel<E, LPR, VPT, BRANCH><<<grid, S::THREADS, 0, s>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    SumArgs q = {};
    int n = 0;
    for (int k = 0; k < 3; ++k)
      if (want[k]) { q.part[n] = p.part[k]; q.out[n++] = a.part_of[k]; }
    if (n == 0) return hipSuccess;
    q.n = grid; q.d = a.d; q.accumulate = a.accumulate;
    block_sums_kernel<<<dim3((a.d + 63) / 64, n), 256, 0, s>>>(q);
  } else {
    block_forward_kernel<E, LPR, VPT, BRANCH><<<grid, S::THREADS, 0, s>>>(p);
  }
  return hipGetLastError();
}

template <class E, bool BRANCH, bool BACK>
hipError_t by_width(const BlockArgs& a, hipStream_t s) {
  const int most = STEM_BLOCK_GRID;
  if (a.d <= 64) return launch<E, 8, 1, BRANCH, BACK>(a, most, s, nullptr);
  if (a.d <= 128) return launch<E, 16, 1, BRANCH, BACK>(a, most, s, nullptr);
  if (a.d <= 256) return launch<E, 32, 1, BRANCH, BACK>(a, most, s, nullptr);
  if (a.d <= 512) return launch<E, 64, 1, BRANCH, BACK>(a, most, s, nullptr);
  if (a.d <= 1024) return launch<E, 64, 2, BRANCH, BACK>(a, most, s, nullptr);
  if (a.d <= 2048) return launch<E, 256, 1, BRANCH, BACK>(a, most, s, nullptr);
  if (a.d <= 4096) return launch<E, 256, 2, BRANCH, BACK>(a, most, s, nullptr);
  if (a.d <= 8192) return launch<E, 1024, 1, BRANCH, BACK>(a, most, s, nullptr);
  return launch<E, 1024, 2, BRANCH, BACK>(a, most, s, nullptr);
}

}  // namespace

hipError_t stem_block_forward_launch(stem_ctx* ctx, int is_bf16, bool branch, const BlockArgs& a, hipStream_t s) {
  ProfScope prof(ctx, branch ? K_BLOCK_LEAVE : K_BLOCK_ENTER, s);
  if (is_bf16) return branch ? by_width<bf16_t, true, false>(a, s) : by_width<bf16_t, false, false>(a, s);
  return branch ? by_width<float, true, false>(a, s) : by_width<float, false, false>(a, s);
}

hipError_t stem_block_backward_launch(stem_ctx* ctx, int is_bf16, bool branch, const BlockArgs& a, hipStream_t s) {
  ProfScope prof(ctx, branch ? K_BLOCK_LEAVE_BACK : K_BLOCK_ENTER_BACK, s);
  if (is_bf16) return branch ? by_width<bf16_t, true, true>(a, s) : by_width<bf16_t, false, true>(a, s);
  return branch ? by_width<float, true, true>(a, s) : by_width<float, false, true>(a, s);
}

hipError_t stem_dropout_launch(stem_ctx* ctx, int is_bf16, const void* x, int64_t T, int64_t d, const DropArgs& drop, void* y, hipStream_t s) {
  ProfScope prof(ctx, K_DROPOUT, s);
  const int64_t columns = (d + 7) / 8;
  int tx_log = 0;
  while (tx_log < 8 && ((int64_t)1 << tx_log) < columns) ++tx_log;
  const int64_t tiles = (columns + (1 << tx_log) - 1) >> tx_log, rows = (T + (256 >> tx_log) - 1) / (256 >> tx_log);
  const int vectors = d % 8 == 0;
  if (is_bf16)
    dropout_kernel<bf16_t><<<(unsigned)(tiles * rows), 256, 0, s>>>(static_cast<const bf16_t*>(x), static_cast<bf16_t*>(y), T, d, tx_log, drop, vectors);
  else
    dropout_kernel<float><<<(unsigned)(tiles * rows), 256, 0, s>>>(static_cast<const float*>(x), static_cast<float*>(y), T, d, tx_log, drop, vectors);
  return hipGetLastError();
}
