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
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
typedef __amdgpu_buffer_rsrc_t rsrc_t;

namespace {

constexpr uint32_t OOB = 0x80000000u;   // a buffer offset beyond any row: reads as zero, is not stored

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
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
template <int LPR>
struct RowSum {
  static constexpr int WPR = LPR > 64 ? LPR / 64 : 1;   // wavefronts that share a row
  float (*red)[WPR][2];
  int turn;
  template <int N>
  __device__ __forceinline__ void operator()(float (&v)[N]) {
    static_assert(N <= 2, "room in red");
#pragma unroll
    for (int k = 0; k < N; ++k) {
      v[k] = add_dpp<0xb1>(v[k]);                      // quad_perm 1 0 3 2
      v[k] = add_dpp<0x4e>(v[k]);                      // quad_perm 2 3 0 1
      v[k] = add_dpp<0x141>(v[k]);                     // row_half_mirror
      if (LPR > 8) v[k] = add_dpp<0x140>(v[k]);        // row_mirror
      if (LPR > 16) {                                  // rows 0, 1 and 2, 3 against each other, then the halves
        const u32x2_t w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[k]), __float_as_uint(v[k]), false, false);
        v[k] = __uint_as_float(w[0]) + __uint_as_float(w[1]);
      }
      if (LPR > 32) {
        const u32x2_t w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[k]), __float_as_uint(v[k]), false, false);
        v[k] = __uint_as_float(w[0]) + __uint_as_float(w[1]);
      }
    }
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

// THREADS of a workgroup: several rows of up to 64 lanes, or of 256 (two in the backward pass, whose sums over tokens then take half
// as many partial sums)
template <class E, int LPR, int VPT, bool BACK>
struct Shape {
  static constexpr int THREADS = LPR > 256 ? LPR : BACK ? 512 : 256;
  static constexpr int SLOTS = THREADS / LPR;             // rows a workgroup has in hand
  static constexpr int WPR = RowSum<LPR>::WPR;
  static constexpr bool WHOLE = sizeof(E) == 2;           // rows are whole vectors of 8
};

template <int VPT>
__device__ __forceinline__ float sum(const float (&v)[VPT][8]) {
  float s = 0.f;
#pragma unroll
  for (int t = 0; t < VPT; ++t)
#pragma unroll
    for (int q = 0; q < 8; ++q) s += v[t][q];
  return s;
}
template <int VPT>
__device__ __forceinline__ float dot(const float (&v)[VPT][8], const float (&w)[VPT][8]) {
  float s = 0.f;
#pragma unroll
  for (int t = 0; t < VPT; ++t)
#pragma unroll
    for (int q = 0; q < 8; ++q) s += v[t][q] * w[t][q];
  return s;
}
// The rows that a workgroup has in hand, of one tensor: a buffer that ends behind them and behind the tensor, so that a slot without a row
// reads zeros and stores nothing, as do lanes behind a row's end, and all of a tensor that is not there.  No branches.
template <class E>
__device__ __forceinline__ rsrc_t rows_of(const void* p, int64_t base, int slots, const BlockArgs& a) {
  const int64_t left = a.T - base;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<E*>(static_cast<const E*>(p)) + base * a.d, 0,
                                           p ? (int)((left < slots ? left : slots) * a.d * sizeof(E)) : 0, 0x00020000);
}

// This lane's vectors of a row
template <class E, int LPR, int VPT, bool BACK>
struct Columns {
  bool in[VPT];
  int col[VPT], left[VPT];
  uint32_t off[VPT], off2[VPT];     // of the vector in rows_of(), and of its second half
  __device__ __forceinline__ Columns(int slot, int lane, int d) {
#pragma unroll
    for (int t = 0; t < VPT; ++t) {
      col[t] = (t * LPR + lane) * 8;
      in[t] = col[t] < d;
      left[t] = d - col[t];
      off[t] = in[t] ? (uint32_t)((slot * d + col[t]) * sizeof(E)) : OOB;
      off2[t] = left[t] > 4 ? off[t] + 16 : OOB;
    }
  }
  // v where the first or second four elements of vector t are the row's, else 0
  __device__ __forceinline__ float where(int t, int half, float v) const { return in[t] && (Shape<E, LPR, VPT, BACK>::WHOLE || !half || left[t] > 4) ? v : 0.f; }
  // a vector as it lies in memory, and its values
  struct Raw { u32x4_t a, b; };
  __device__ __forceinline__ Raw request(rsrc_t r, int t) const {
    Raw w;
    w.a = __builtin_amdgcn_raw_buffer_load_b128(r, off[t], 0, 0);
    if (sizeof(E) == 4) w.b = __builtin_amdgcn_raw_buffer_load_b128(r, off2[t], 0, 0);
    return w;
  }
  static __device__ __forceinline__ void values(const Raw& w, float (&v)[8]) {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      v[q] = __uint_as_float(sizeof(E) == 4 ? (q < 4 ? w.a[q & 3] : w.b[q & 3]) : q & 1 ? w.a[q >> 1] & 0xffff0000u : w.a[q >> 1] << 16);
  }
  __device__ __forceinline__ void load1(rsrc_t r, int t, float (&v)[8]) const { values(request(r, t), v); }
  __device__ __forceinline__ void load(rsrc_t r, float (&v)[VPT][8]) const {
#pragma unroll
    for (int t = 0; t < VPT; ++t) load1(r, t, v[t]);
  }
  __device__ __forceinline__ void store(rsrc_t r, int t, const float (&v)[8]) const {
    if (sizeof(E) == 2) {
      bf16x8_t u;
#pragma unroll
      for (int q = 0; q < 8; ++q) u[q] = (__bf16)v[q];
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, u), r, off[t], 0, 0);
    } else {
      const float4 a = make_float4(v[0], v[1], v[2], v[3]), b = make_float4(v[4], v[5], v[6], v[7]);
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, a), r, off[t], 0, 0);
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, b), r, off2[t], 0, 0);
    }
  }
  // a weight of each channel, 1 where there is none
  __device__ __forceinline__ void weight(const void* p, float (&v)[VPT][8]) const {
#pragma unroll
    for (int t = 0; t < VPT; ++t) {
#pragma unroll
      for (int q = 0; q < 8; ++q) v[t][q] = 1.f;
      if (p && in[t]) load8(static_cast<const E*>(p) + col[t], left[t], v[t]);
    }
  }
  // v <- v - mean of a row whose sum this is; elements past the row's end are zero and stay zero
  __device__ __forceinline__ void centre(float (&v)[VPT][8], float mean) const {
#pragma unroll
    for (int t = 0; t < VPT; ++t) {
      const float m[2] = {where(t, 0, mean), where(t, 1, mean)};
#pragma unroll
      for (int q = 0; q < 8; ++q) v[t][q] -= m[q >> 2];
    }
  }
  // G += the gradient of N's input for the gradient h of its output v^; r = 1 / sqrt(...)
  __device__ __forceinline__ void add_back(float (&G)[VPT][8], const float (&h)[VPT][8], const float (&v)[VPT][8], float r, int kind, float inv_d,
                                           RowSum<LPR>& row_sum) const {
    float s[2] = {dot(h, v), 0.f};
    if (kind == STEM_NORM_LAYER) {
      s[1] = sum(h);
      row_sum(s);
      const float mean = r * s[1] * inv_d;
#pragma unroll
      for (int t = 0; t < VPT; ++t) {
        const float m[2] = {where(t, 0, mean), where(t, 1, mean)};
#pragma unroll
        for (int q = 0; q < 8; ++q) G[t][q] -= m[q >> 2];
      }
    } else {
      float one[1] = {s[0]};
      row_sum(one);
      s[0] = one[0];
    }
    const float along = -r * s[0] * inv_d;
#pragma unroll
    for (int t = 0; t < VPT; ++t)
#pragma unroll
      for (int q = 0; q < 8; ++q) G[t][q] = __builtin_fmaf(along, v[t][q], __builtin_fmaf(r, h[t][q], G[t][q]));
  }
};

template <int VPT>
__device__ __forceinline__ void scale_by(float (&v)[VPT][8], float r) {
#pragma unroll
  for (int t = 0; t < VPT; ++t)
#pragma unroll
    for (int q = 0; q < 8; ++q) v[t][q] *= r;
}

// 1 / sqrt(mean of squares + eps), v centred before for the second kind.  The variance is of the centred values: the difference of two sums
// of squares would lose what a large mean shifts out.
template <class C, int LPR, int VPT>
__device__ __forceinline__ float factor(const C& c, float (&v)[VPT][8], const stem_norm& n, float inv_d, RowSum<LPR>& row_sum) {
  if (n.kind == STEM_NORM_LAYER) {
    float s[1] = {sum(v)};
    row_sum(s);
    c.centre(v, s[0] * inv_d);
  }
  float s[1] = {dot(v, v)};
  row_sum(s);
  return 1.0f / sqrtf(s[0] * inv_d + n.eps);
}

// ---- forward -------------------------------------------------------------------------------------------
// BRANCH: the end of a block; without it y is x and only n is written.  One pass: a row's values stay in registers from its loads
// to its stores.  A workgroup keeps what is the same for all rows (w_out times a gate a channel, w_next) in registers and takes as many rows
// as leave 8 workgroups to a compute unit.
// Measured, 16384 x 2048 in bf16, both norms, a gate a channel, p 0.1: 53 to 55 us, 5 TB/s of the 268 MB that have to move (a copy reaches 6.0).
// Arithmetic is nearly as long: about 15 million VALU instructions, 26 us of all SIMDs, 13 more for the generator's wide multiplications.  One token: the launch.
template <class E, int LPR, int VPT, bool BRANCH>
__global__ __launch_bounds__((Shape<E, LPR, VPT, false>::THREADS)) void block_forward_kernel(BlockArgs p) {
  typedef Shape<E, LPR, VPT, false> S;
  __shared__ float red[S::SLOTS][2][S::WPR][2];
  const int slot = threadIdx.x / LPR, lane = threadIdx.x % LPR;
  RowSum<LPR> row_sum{red[slot], 0};
  const Columns<E, LPR, VPT, false> c(slot, lane, p.d);
  const uint64_t offset = BRANCH && p.drop.threshold ? offset_of(p.drop) : 0;
  const bool by_channel = p.gate_kind == STEM_GATE_CHANNEL, by_element = p.gate_kind == STEM_GATE_FULL, by_token = p.gate_kind == STEM_GATE_TOKEN;
  float branch[VPT][8], after[VPT][8];
  if (BRANCH) {
    c.weight(p.out.weight, branch);
    if (by_channel) {
      float g[VPT][8];
      c.weight(p.gate, g);
#pragma unroll
      for (int t = 0; t < VPT; ++t)
#pragma unroll
        for (int q = 0; q < 8; ++q) branch[t][q] *= g[t][q];
    }
  }
  c.weight(p.next.weight, after);
  const float of_branch = p.branch_scale * (p.drop.threshold ? p.drop.scale : 1.f);
  for (int64_t base = (int64_t)blockIdx.x * S::SLOTS; base < p.T; base += (int64_t)gridDim.x * S::SLOTS) {
    const int64_t row = base + slot;
    float y[VPT][8];
    c.load(rows_of<E>(p.x, base, S::SLOTS, p), y);
    if (BRANCH) {
      float f[VPT][8];
      c.load(rows_of<E>(p.f, base, S::SLOTS, p), f);
      float r = of_branch;
      if (by_token) r *= load1(static_cast<const E*>(p.gate) + (row < p.T ? row : p.T - 1));
      if (by_element) {
        float g[VPT][8];
        c.load(rows_of<E>(p.gate, base, S::SLOTS, p), g);
        if (p.out.kind != STEM_NORM_NONE) r *= factor(c, f, p.out, p.inv_d, row_sum);
#pragma unroll
        for (int t = 0; t < VPT; ++t)
#pragma unroll
          for (int q = 0; q < 8; ++q) f[t][q] *= g[t][q];
      } else if (p.out.kind != STEM_NORM_NONE) {
        r *= factor(c, f, p.out, p.inv_d, row_sum);
      }
      const rsrc_t ry = rows_of<E>(p.y, base, S::SLOTS, p);
#pragma unroll
      for (int t = 0; t < VPT; ++t) {
        if (p.drop.threshold) {
          const Bits b = philox((uint32_t)(c.col[t] >> 3), (uint32_t)row, offset, p.drop.seed);
#pragma unroll
          for (int q = 0; q < 8; ++q) y[t][q] = p.residual_scale * y[t][q] + (kept(b, q, p.drop.threshold) ? f[t][q] * branch[t][q] * r : 0.f);
        } else {
#pragma unroll
          for (int q = 0; q < 8; ++q) y[t][q] = p.residual_scale * y[t][q] + f[t][q] * branch[t][q] * r;
        }
        c.store(ry, t, y[t]);
      }
    }
    if (p.n) {
      if (p.next.kind != STEM_NORM_NONE) scale_by(y, factor(c, y, p.next, p.inv_d, row_sum));
      const rsrc_t rn = rows_of<E>(p.n, base, S::SLOTS, p);
#pragma unroll
      for (int t = 0; t < VPT; ++t) {
#pragma unroll
        for (int q = 0; q < 8; ++q) y[t][q] *= after[t][q];
        c.store(rn, t, y[t]);
      }
    }
  }
}

// ---- backward ------------------------------------------------------------------------------------------
// Sums over tokens are held in registers over a workgroup's rows and written as one partial sum a workgroup, [sum][workgroup][d];
// block_sums_kernel adds those in order.  No atomics: the same bits on every run.  dw_out and the gradient of a gate a channel are the same
// sum, of h times the kept N_out(f), times the gate and times w_out: it is held once.  All of a row is requested before its first reduction.
// Measured, 16384 x 2048 in bf16, both norms, a gate a channel, p 0.1: 83 us and 4 for the sums, 4.6 TB/s of the 403 MB that have to move;
// the arithmetic alone is about 60 us (29.3 million VALU instructions), and 115 registers leave 16 wavefronts a compute unit to hide the rest.
// Without BRANCH, the same shape: 56 us, 4.8 TB/s; 16384 x 2048 in fp32 100 us, with BRANCH 158.
// Workgroups of 512, two rows of 2048 each: 512 of them are all resident, and write half as many partial sums as 1024 of 256 would.  Of 1024
// a compute unit holds one: 256 (512 take two turns: 4096 x 8192 119 us instead of 112, 1024 x 8192 46.7 / 37.2, 2048 x 16384 157 / 139).
template <class E, int LPR, int VPT, bool BRANCH>
__global__ __launch_bounds__((Shape<E, LPR, VPT, true>::THREADS)) void block_backward_kernel(BlockArgs p) {
  typedef Shape<E, LPR, VPT, true> S;
  __shared__ float red[S::SLOTS][2][S::WPR][2];
  __shared__ float sums[S::SLOTS > 1 ? S::THREADS * VPT * 8 : 1];
  const int slot = threadIdx.x / LPR, lane = threadIdx.x % LPR;
  RowSum<LPR> row_sum{red[slot], 0};
  const Columns<E, LPR, VPT, true> c(slot, lane, p.d);
  const uint64_t offset = BRANCH && p.drop.threshold ? offset_of(p.drop) : 0;
  const bool by_channel = p.gate_kind == STEM_GATE_CHANNEL, by_element = p.gate_kind == STEM_GATE_FULL, by_token = p.gate_kind == STEM_GATE_TOKEN;
  // The next row is requested before this one's first reduction where registers allow it (16384 x 2048 96 -> 91 us; fp32 gains nothing).
  constexpr bool EARLY = VPT == 1 && LPR < 1024 && sizeof(E) == 2;
  // Rows of two vectors a lane (1024 lanes, 128 registers): the weights are read again for each row, and the sums over tokens lie in LDS
  // where there are two, each lane's own (2048 x 16384 in bf16 306 us with all in registers and scratch memory, 157 so).
  constexpr bool AGAIN = VPT == 2, IN_LDS = AGAIN && BRANCH;
  __shared__ float4 lds_sum[IN_LDS ? 4 * VPT * S::THREADS : 1];
  enum { NEXT, OUT };
  float sum[2][VPT][8] = {};
  auto place = [&](int which, int t, int half) __attribute__((always_inline)) {
    return lds_sum + (IN_LDS ? ((which * VPT + t) * 2 + half) * S::THREADS + threadIdx.x : 0);
  };
  auto add = [&](int which, int t, auto product) __attribute__((always_inline)) {
    float(&v)[8] = sum[which][t];
    float4 w[2];
    if (IN_LDS) { w[0] = *place(which, t, 0); w[1] = *place(which, t, 1); memcpy(v, w, 32); }
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = product(q, v[q]);
    if (IN_LDS) { memcpy(w, v, 32); *place(which, t, 0) = w[0]; *place(which, t, 1) = w[1]; }
  };
  if (IN_LDS)
#pragma unroll
    for (int k = 0; k < 4 * VPT; ++k) lds_sum[k * S::THREADS + threadIdx.x] = make_float4(0.f, 0.f, 0.f, 0.f);
  // w_next; w_out times a gate a channel
  float after[VPT][8], branch[VPT][8];
  if (!AGAIN) c.weight(p.next.weight, after);
  auto branch_weight = [&](float (&w)[VPT][8], bool weight, bool gate) __attribute__((always_inline)) {
    c.weight(weight ? p.out.weight : nullptr, w);
    if (gate && by_channel) {
      float g[VPT][8];
      c.weight(p.gate, g);
#pragma unroll
      for (int t = 0; t < VPT; ++t)
#pragma unroll
        for (int q = 0; q < 8; ++q) w[t][q] *= g[t][q];
    }
  };
  if (BRANCH && !AGAIN) branch_weight(branch, true, true);
  const float of_branch = p.branch_scale * (p.drop.threshold ? p.drop.scale : 1.f);
  typedef typename Columns<E, LPR, VPT, true>::Raw Raw;
  struct Row { Raw dy[VPT], f[VPT], y[VPT], dn[VPT]; };
  auto request = [&](int64_t base) __attribute__((always_inline)) {
    auto rows = [&](const void* t) __attribute__((always_inline)) { return rows_of<E>(base < p.T ? t : nullptr, base < p.T ? base : 0, S::SLOTS, p); };
    Row r;
#pragma unroll
    for (int t = 0; t < VPT; ++t) {
      r.dy[t] = c.request(rows(p.dy), t);
      r.y[t] = c.request(rows(p.dn ? p.x : nullptr), t);
      r.dn[t] = c.request(rows(p.dn), t);
      if (BRANCH) r.f[t] = c.request(rows(p.f), t);
    }
    return r;
  };
  const int64_t step = (int64_t)gridDim.x * S::SLOTS;
  Row next = request((int64_t)blockIdx.x * S::SLOTS);
  for (int64_t base = (int64_t)blockIdx.x * S::SLOTS; base < p.T; base += step) {
    const int64_t row = base + slot;
    const bool live = row < p.T;            // a slot without a row has zeros in all places, and adds zeros
    auto rows = [&](const void* t) __attribute__((always_inline)) { return rows_of<E>(t, base, S::SLOTS, p); };
    const Row in = next;
    if (EARLY) next = request(base + step);
    float G[VPT][8], f[VPT][8];
#pragma unroll
    for (int t = 0; t < VPT; ++t) {
      c.values(in.dy[t], G[t]);
      if (BRANCH) c.values(in.f[t], f[t]);
    }
    if (p.dn) {
      float y[VPT][8], h[VPT][8];
#pragma unroll
      for (int t = 0; t < VPT; ++t) {
        c.values(in.y[t], y[t]);
        c.values(in.dn[t], h[t]);
      }
      const float r = factor(c, y, p.next, p.inv_d, row_sum), r_live = live ? r : 0.f;
      scale_by(y, r_live);
      if (AGAIN) c.weight(p.next.weight, after);
#pragma unroll
      for (int t = 0; t < VPT; ++t) {
        add(NEXT, t, [&](int q, float v) __attribute__((always_inline)) { return __builtin_fmaf(h[t][q], y[t][q], v); });
#pragma unroll
        for (int q = 0; q < 8; ++q) h[t][q] *= after[t][q];
      }
      c.add_back(G, h, y, r_live, p.next.kind, p.inv_d, row_sum);
    }
    const rsrc_t rdx = rows(p.dx);
    auto store_dx = [&](int t) __attribute__((always_inline)) {   // of a vector whose inputs have all been read: dx may be any of them
      float o[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) o[q] = p.residual_scale * G[t][q];
      c.store(rdx, t, o);
    };
    if (!BRANCH) {
#pragma unroll
      for (int t = 0; t < VPT; ++t) store_dx(t);
      if (!EARLY) next = request(base + step);
      continue;
    }
    // (f stays as the norm leaves it: f^ without what follows)
    float r = 1.f;
    if (p.f && p.out.kind != STEM_NORM_NONE) {
      r = factor(c, f, p.out, p.inv_d, row_sum);
      if (!live) r = 0.f;
      scale_by(f, r);
    }
    const float gate_of_row = by_token ? load1(static_cast<const E*>(p.gate) + (live ? row : p.T - 1)) : 1.f, of_row = live ? gate_of_row : 1.f;
    float token_gate = 0.f;
    if (AGAIN) branch_weight(branch, true, true);
#pragma unroll
    for (int t = 0; t < VPT; ++t) {
      float g[8], dg[8];
      if (by_element) c.load1(rows(p.gate), t, g);
      store_dx(t);
#pragma unroll
      for (int q = 0; q < 8; ++q) G[t][q] *= of_branch;
      // What is dropped counts for nothing, whatever h, f, the gate or w_out hold there: each product is cut where it is complete.  (Without
      // dropout the threshold is 0 and all is kept.)
      Bits bits = {};
      if (p.drop.threshold) bits = philox((uint32_t)(c.col[t] >> 3), (uint32_t)row, offset, p.drop.seed);
      if (by_token || by_element) {          // (branch is w_out alone)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          dg[q] = kept(bits, q, p.drop.threshold) ? G[t][q] * (f[t][q] * branch[t][q]) : 0.f;
          token_gate += dg[q];
          G[t][q] *= by_element ? g[q] : of_row;
        }
        if (by_element) c.store(rows(p.dgate), t, dg);
      }
      add(OUT, t, [&](int q, float v) __attribute__((always_inline)) {
        const float sum = __builtin_fmaf(G[t][q], f[t][q], v);
        return kept(bits, q, p.drop.threshold) ? sum : v;
      });
#pragma unroll
      for (int q = 0; q < 8; ++q) G[t][q] = kept(bits, q, p.drop.threshold) ? G[t][q] * branch[t][q] : 0.f;
    }
    if (by_token && p.dgate) {
      float s[1] = {token_gate};
      row_sum(s);
      if (live && lane == 0) store1(static_cast<E*>(p.dgate) + row, s[0]);
    }
    if (p.df) {
      if (p.out.kind != STEM_NORM_NONE) {
        float o[VPT][8] = {};
        c.add_back(o, G, f, r, p.out.kind, p.inv_d, row_sum);
#pragma unroll
        for (int t = 0; t < VPT; ++t) c.store(rows(p.df), t, o[t]);
      } else {
#pragma unroll
        for (int t = 0; t < VPT; ++t) c.store(rows(p.df), t, G[t]);
      }
    }
    if (!EARLY) next = request(base + step);
  }
  auto write = [&](const float (&sum)[VPT][8], float* part) __attribute__((always_inline)) {
    float* const to = part + (size_t)blockIdx.x * p.d;
    if (S::SLOTS == 1) {
#pragma unroll
      for (int t = 0; t < VPT; ++t)
        if (c.in[t]) store8(to + c.col[t], c.left[t], sum[t]);
      return;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < VPT; ++t)
#pragma unroll
      for (int q = 0; q < 8; ++q) sums[(slot * VPT + t) * LPR * 8 + lane * 8 + q] = sum[t][q];
    __syncthreads();
    for (int k = threadIdx.x; k < p.d; k += S::THREADS) {
      float s = 0.f;
#pragma unroll
      for (int n = 0; n < S::SLOTS; ++n) s += sums[n * VPT * LPR * 8 + k];
      to[k] = s;
    }
  };
  if (IN_LDS)
#pragma unroll
    for (int k = 0; k < 2 * VPT; ++k) {
      const float4 w[2] = {*place(k / VPT, k % VPT, 0), *place(k / VPT, k % VPT, 1)};
      memcpy(sum[k / VPT][k % VPT], w, 32);
    }
  if (p.part[0]) write(sum[NEXT], p.part[0]);
  if (BRANCH) {
#pragma unroll 1
    for (int which = 1; which < 3; ++which) {
      if (!p.part[which]) continue;
      float w[VPT][8];
      branch_weight(w, which == 2, which == 1);
#pragma unroll
      for (int t = 0; t < VPT; ++t)
#pragma unroll
        for (int q = 0; q < 8; ++q) w[t][q] *= sum[OUT][t][q];
      write(w, p.part[which]);
    }
  }
}

// out[c] (+)= sum of part[k][c] over k < n, for up to three sums: a thread has every 32nd k, in order, and 32 threads a column, in order
struct SumArgs { const float* part[3]; float* out[3]; int n, d, accumulate; };
__global__ __launch_bounds__(1024) void block_sums_kernel(SumArgs p) {
  __shared__ float s[32][33];
  const int x = threadIdx.x & 31, k = threadIdx.x >> 5, c = blockIdx.x * 32 + x, which = blockIdx.y;
  const float* const part = which == 0 ? p.part[0] : which == 1 ? p.part[1] : p.part[2];
  float* const out = which == 0 ? p.out[0] : which == 1 ? p.out[1] : p.out[2];
  float v[STEM_BLOCK_GRID / 32];   // all in flight together
#pragma unroll
  for (int i = 0; i < STEM_BLOCK_GRID / 32; ++i) v[i] = c < p.d && i * 32 + k < p.n ? part[(size_t)(i * 32 + k) * p.d + c] : 0.f;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < STEM_BLOCK_GRID / 32; ++i) sum += v[i];
  s[k][x] = sum;
  __syncthreads();
  if (k == 0 && c < p.d) {
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) sum += s[i][x];
    out[c] = p.accumulate ? out[c] + sum : sum;
  }
}

// ---- dropout by itself -------------------------------------------------------------------------------------
// A thread has the eight elements of a counter; `tx` (a power of two) threads lie along a row.  Measured: 65536 x 1024 in bf16 44.5 us, 6.0 TB/s,
// what a copy reaches; the generator takes about 39 of them beside.  999 x 1001 in fp32, element by element, 5.0 to 5.2.
template <class E>
__global__ __launch_bounds__(256) void dropout_kernel(const E* x, E* y, int64_t T, int64_t d, int64_t row0, int tx_log, DropArgs drop,
                                                      int vectors) {
  const int tx = 1 << tx_log;
  const int64_t columns = (d + 7) / 8;
  const int64_t tiles = (columns + tx - 1) >> tx_log;
  const int64_t row = row0 + (int64_t)(blockIdx.x / tiles) * (256 >> tx_log) + (threadIdx.x >> tx_log);
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
hipError_t launch(const BlockArgs& a, hipStream_t s) {
  typedef Shape<E, LPR, VPT, BACK> S;
  const int64_t groups = (a.T + S::SLOTS - 1) / S::SLOTS, most = BACK ? stem_block_grid(a.d) : 2048 * 256 / S::THREADS;
  // Up to 512 workgroups of the backward pass are done in one round either way: 385 and more take two rows in turn, and write half as many partial
  // sums.  us, one each / two in turn, with BRANCH: bf16 4000 x 512 12.6 / 12.1, 2000 x 1024 14.4 / 13.7, 1024 x 2048 17.4 / 15.2, 512 x 4096 22.0 / 19.2;
  // fp32 4000 x 512 15.2 / 14.4, 2000 x 1024 17.1 / 18.0, 800 x 2048 17.8 / 16.6, 1024 x 2048 19.0 / 19.1, 512 x 4096 21.3 / 20.4.  Without: bf16 512 x 4096
  // 11.3 / 10.1, fp32 13.3 / 11.4, the others within 0.5 of each other.  (Fewer workgroups gain nothing: 512 x 2048 12.9 / 13.5.)
  const bool in_turn = BACK && groups > 384 && groups <= STEM_BLOCK_GRID;
  const int grid = (int)(in_turn ? (groups + 1) / 2 : groups < most ? groups : most);
  if constexpr (BACK) {
    BlockArgs p = a;
    SumArgs q = {};
    int n = 0;
    for (int k = 0; k < 3; ++k) {
      p.part[k] = a.part_of[k] ? a.part[0] + (size_t)n * grid * a.d : nullptr;
      if (a.part_of[k]) { q.part[n] = p.part[k]; q.out[n++] = a.part_of[k]; }
    }
    block_backward_kernel<E, LPR, VPT, BRANCH><<<grid, S::THREADS, 0, s>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || n == 0) return e;
    q.n = grid; q.d = a.d; q.accumulate = a.accumulate;
    block_sums_kernel<<<dim3((a.d + 31) / 32, n), 1024, 0, s>>>(q);
  } else {
    block_forward_kernel<E, LPR, VPT, BRANCH><<<grid, S::THREADS, 0, s>>>(a);
  }
  return hipGetLastError();
}

// Lanes a row and vectors a lane.  A lane has one vector where it can: more wavefronts wait for memory at a time.  Two vectors halve what a
// row's reduction costs besides, and pay where a row would take more than a wavefront and the tensors stream from memory.  us, one vector /
// two, bf16, both norms, p 0.1: forward 32768 x 1024 56 / 54, 4096 x 2048 14.9 / 16.6, 16384 x 2048 58 / 54.7 (4096 x 2048 in fp32 24.3 / 26.5, 16384 108 / 103),
// 8192 x 4096 57 / 52, 512 x 8192 11.9 / 10.7, 4096 x 8192 70 / 56; the norm alone 1024 x 8192 7.2 / 7.5; backward, whose
// registers are its sums', 65536 x 512 86 / 86, 16384 x 2048 87 / 104, 8192 x 4096 88 / 109, 256 x 8192 24.5 / 25.4.
template <class E, bool BRANCH, bool BACK>
hipError_t by_width(const BlockArgs& a, hipStream_t s) {
  if (a.d <= 64) return launch<E, 8, 1, BRANCH, BACK>(a, s);
  if (a.d <= 128) return launch<E, 16, 1, BRANCH, BACK>(a, s);
  if (a.d <= 256) return launch<E, 32, 1, BRANCH, BACK>(a, s);
  if (a.d <= 512) return launch<E, 64, 1, BRANCH, BACK>(a, s);
  if (a.d <= 1024) return launch<E, BACK ? 128 : 64, BACK ? 1 : 2, BRANCH, BACK>(a, s);
  if constexpr (BRANCH && !BACK)
    if (a.d > 1024 && a.d <= 2048 && a.T * a.d * (int64_t)sizeof(E) >= (64 << 20)) return launch<E, 128, 2, BRANCH, BACK>(a, s);
  if (a.d <= 2048) return launch<E, 256, 1, BRANCH, BACK>(a, s);
  if (a.d <= STEM_BLOCK_WIDE) return launch<E, BACK ? 512 : 256, BACK ? 1 : 2, BRANCH, BACK>(a, s);
  if (a.d <= 8192) return launch<E, BRANCH && !BACK ? 512 : 1024, BRANCH && !BACK ? 2 : 1, BRANCH, BACK>(a, s);
  return launch<E, 1024, 2, BRANCH, BACK>(a, s);
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

// A launch has fewer than 2^32 threads: longer tensors are done in several, of as many rows each.
constexpr int64_t DROPOUT_GRID = 1 << 23;
hipError_t stem_dropout_launch(stem_ctx* ctx, int is_bf16, const void* x, int64_t T, int64_t d, const DropArgs& drop, void* y, hipStream_t s) {
  ProfScope prof(ctx, K_DROPOUT, s);
  const int64_t columns = (d + 7) / 8;
  int tx_log = 0;
  while (tx_log < 8 && ((int64_t)1 << tx_log) < columns) ++tx_log;
  const int64_t tiles = (columns + (1 << tx_log) - 1) >> tx_log, rows = 256 >> tx_log;   // workgroups along a row, rows of a workgroup
  const int vectors = d % 8 == 0;
  const int64_t most = DROPOUT_GRID / tiles * rows;   // rows of a launch
  for (int64_t row0 = 0; row0 < T; row0 += most) {
    const unsigned grid = (unsigned)(tiles * (((T - row0 < most ? T - row0 : most) + rows - 1) / rows));
    if (is_bf16)
      dropout_kernel<bf16_t><<<grid, 256, 0, s>>>(static_cast<const bf16_t*>(x), static_cast<bf16_t*>(y), T, d, row0, tx_log, drop, vectors);
    else
      dropout_kernel<float><<<grid, 256, 0, s>>>(static_cast<const float*>(x), static_cast<float*>(y), T, d, row0, tx_log, drop, vectors);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
