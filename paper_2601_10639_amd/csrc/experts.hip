// Tokens to experts and back.  A token has k choices, each an expert or none; a pair is a token and one of its choices.
//
//     sort:      row r of the sorted order has pair src[r] = t k + j, pairs ascending by expert and then by themselves; place[src[r]] = r
//     dispatch:  xs[r] = x[src[r] / k]                  (its backward pass is combine without weights)
//     combine:   y_t = residual_t + sum_j w_tj ys[place_tj]
//     backward:  dys[place_tj] = w_tj dy_t,  dw_tj = <dy_t, ys[place_tj]>
//
// All of them move rows and are bound by memory, or by the launch where rows are few.
#include <type_traits>

#include "experts.h"

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;

namespace {

// ---- sort ------------------------------------------------------------------------------------------------------------------
// A workgroup has a segment of the pairs, 64 a wavefront and turn; lanes with one expert find each other by ballots over the bits of
// its number, so every pair's rank among its wavefront's is a popcount, and a table in LDS has how many each wavefront has seen.  No
// atomics: the order is the pairs' own.  Pairs of no expert (negative, or none of the n, which is reported) are kept as expert n: they get
// place -1, and the rows behind the last expert's get src -1.
// PLACE: the counts are taken again and the pairs placed; otherwise they are stored for the kernel that does.
constexpr int WAVES = EXPERTS_SEGMENT / 256, TURNS = EXPERTS_SEGMENT / 64 / WAVES;

__device__ __forceinline__ void in_order() {                // of LDS, within the wavefront
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <bool PLACE>
__global__ __launch_bounds__(WAVES * 64) void sort_kernel(ExpertsSortArgs p, int segments, int bits) {
  extern __shared__ int32_t table[];                        // [WAVES][n + 1], then [n + 1] of first rows
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = p.n, pitch = n + 1;
  int32_t* const mine = table + wave * pitch;
  int32_t* const first = table + WAVES * pitch;
  const int at = blockIdx.x * EXPERTS_SEGMENT + wave * (64 * TURNS) + lane;
  for (int e = threadIdx.x; e < WAVES * pitch; e += WAVES * 64) table[e] = 0;
  int expert[TURNS], rank[TURNS];
#pragma unroll
  for (int t = 0; t < TURNS; ++t) {
    const int i = at + t * 64;
    int e = i < p.pairs ? p.experts[i] : -1;
    if (e >= n) *p.flag = 1;
    expert[t] = (unsigned)e < (unsigned)n ? e : n;
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < TURNS; ++t) {
    const bool live = at + t * 64 < p.pairs;
    uint64_t same = __ballot(live);
    for (int b = 0; b < bits; ++b) {
      const bool set = expert[t] >> b & 1;
      const uint64_t with = __ballot(set);
      same &= set ? with : ~with;
    }
    const int before = mine[expert[t]];                     // (LDS is in order within a wavefront)
    const int below = __popcll(same & ((1ull << lane) - 1));
    rank[t] = before + below;   // of the lanes that are live
    in_order();
    if (live && below == 0) mine[expert[t]] = before + __popcll(same);
    in_order();
  }
  __syncthreads();
  // each expert's pairs in front of every wavefront's, and the segment's
  for (int e = threadIdx.x; e <= n; e += WAVES * 64) {
    int sum = 0;
    for (int w = 0; w < WAVES; ++w) {
      const int c = table[w * pitch + e];
      table[w * pitch + e] = sum;
      sum += c;
    }
    if (!PLACE) p.counts[(int64_t)blockIdx.x * pitch + e] = sum;
    first[e] = sum;
  }
  if (!PLACE) return;
  __syncthreads();
  // the rows in front of each expert's: in all segments, and of the expert itself in those before this one
  if (segments > 1)
    for (int e = threadIdx.x; e <= n; e += WAVES * 64) {
      int all = 0, before = 0;
      for (int s = 0; s < segments; ++s) {
        const int c = p.counts[(int64_t)s * pitch + e];
        before += s < (int)blockIdx.x ? c : 0;
        all += c;
      }
      first[e] = all;
      for (int w = 0; w < WAVES; ++w) table[w * pitch + e] += before;
    }
  __syncthreads();
  if (wave == 0) {
    int sum = 0;
    for (int e0 = 0; e0 <= n; e0 += 64) {
      const int e = e0 + lane, c = e <= n ? first[e] : 0;
      int scan = c;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int up = __shfl_up(scan, d);
        scan += lane >= d ? up : 0;
      }
      if (e <= n) {
        first[e] = sum + scan - c;
        if (blockIdx.x == 0) p.offsets[e] = sum + scan - c;
      }
      sum += __shfl(scan, 63);
    }
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < TURNS; ++t) {
    const int i = at + t * 64, e = expert[t];
    if (i >= p.pairs) continue;
    const int row = first[e] + mine[e] + rank[t];
    p.place[i] = e < n ? row : -1;
    p.src[row] = e < n ? i : -1;
  }
}

// ---- rows ------------------------------------------------------------------------------------------------------------------
// BYTES: 16 where rows are whole vectors, else one element
template <class E>
__device__ __forceinline__ float to_float(E v) {
  if constexpr (sizeof(E) == 2) return __uint_as_float((uint32_t)v << 16);
  else return v;
}
template <class E>
__device__ __forceinline__ E from_float(float v) {
  if constexpr (sizeof(E) == 2) return __builtin_bit_cast(uint16_t, (__bf16)v);
  else return v;
}
template <class E, int V>
struct Piece { E v[V]; };
template <class E, int V>
__device__ __forceinline__ Piece<E, V> load(const void* base, int64_t at) {   // V elements from element `at` on
  Piece<E, V> p;
  __builtin_memcpy(&p, __builtin_assume_aligned(static_cast<const E*>(base) + at, V * sizeof(E)), sizeof p);
  return p;
}
template <class E, int V>
__device__ __forceinline__ void store(void* base, int64_t at, const Piece<E, V>& p) {
  __builtin_memcpy(__builtin_assume_aligned(static_cast<E*>(base) + at, V * sizeof(E)), &p, sizeof p);
}

// a wavefront has a row
template <class E, int V>
__global__ __launch_bounds__(256) void dispatch_kernel(ExpertsRowsArgs p) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= p.rows) return;
  const int pair = p.src[row];
  if (pair < 0) return;
  int64_t t = pair / p.k;
  if (t >= p.T) {
    if (lane == 0) *p.flag = 1;
    t = p.T - 1;
  }
  if (p.ids && lane == 0) p.ids_out[row] = p.ids[t];
  for (int64_t c = lane * V; c < p.width; c += 64 * V) store<E, V>(p.xs, row * p.width + c, load<E, V>(p.x, t * p.width + c));
}

// a wavefront has a token
template <class E, int V>
__global__ __launch_bounds__(256) void combine_kernel(ExpertsRowsArgs p) {
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= p.T) return;
  for (int64_t c = lane * V; c < p.width; c += 64 * V) {
    float sum[V] = {};
    if (p.residual) {
      const Piece<E, V> r = load<E, V>(p.residual, t * p.width + c);
#pragma unroll
      for (int q = 0; q < V; ++q) sum[q] = to_float(r.v[q]);
    }
    for (int j = 0; j < p.k; ++j) {
      int64_t row = p.place[t * p.k + j];
      if (row < 0) continue;
      if (row >= p.rows) {
        if (lane == 0) *p.flag = 1;
        if (p.rows == 0) continue;
        row = p.rows - 1;
      }
      const float w = p.weights ? p.weights[t * p.k + j] : 1.f;
      const Piece<E, V> v = load<E, V>(p.ys, row * p.width + c);
#pragma unroll
      for (int q = 0; q < V; ++q) sum[q] = __builtin_fmaf(w, to_float(v.v[q]), sum[q]);
    }
    Piece<E, V> out;
#pragma unroll
    for (int q = 0; q < V; ++q) out.v[q] = from_float<E>(sum[q]);
    store<E, V>(p.y, t * p.width + c, out);
  }
}

// a wavefront has a token
template <class E, int V>
__global__ __launch_bounds__(256) void combine_backward_kernel(ExpertsRowsArgs p) {
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= p.T) return;
  for (int j = 0; j < p.k; ++j) {
    int64_t row = p.place[t * p.k + j];
    if (row < 0) {
      if (p.dweights && lane == 0) p.dweights[t * p.k + j] = 0.f;
      continue;
    }
    if (row >= p.rows) {
      if (lane == 0) {
        *p.flag = 1;
        if (p.dweights) p.dweights[t * p.k + j] = 0.f;
      }
      continue;
    }
    const float w = p.weights ? p.weights[t * p.k + j] : 1.f;
    float sum = 0.f;
    for (int64_t c = lane * V; c < p.width; c += 64 * V) {
      const Piece<E, V> g = load<E, V>(p.x, t * p.width + c);
      if (p.dweights) {
        const Piece<E, V> v = load<E, V>(p.ys, row * p.width + c);
#pragma unroll
        for (int q = 0; q < V; ++q) sum = __builtin_fmaf(to_float(g.v[q]), to_float(v.v[q]), sum);
      }
      if (p.dys) {
        Piece<E, V> out;
#pragma unroll
        for (int q = 0; q < V; ++q) out.v[q] = from_float<E>(w * to_float(g.v[q]));
        store<E, V>(p.dys, row * p.width + c, out);
      }
    }
    if (!p.dweights) continue;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) p.dweights[t * p.k + j] = sum;
  }
}

template <class F>
hipError_t by_type(const ExpertsRowsArgs& a, int64_t waves, F f) {
  const unsigned grid = (unsigned)((waves + 3) / 4);
  const bool whole = a.width * a.es % 16 == 0;
  if (a.es == 2) whole ? f(bf16_t{}, std::integral_constant<int, 8>{}, grid) : f(bf16_t{}, std::integral_constant<int, 1>{}, grid);
  else whole ? f(float{}, std::integral_constant<int, 4>{}, grid) : f(float{}, std::integral_constant<int, 1>{}, grid);
  return hipGetLastError();
}

}  // namespace

hipError_t stem_experts_sort_launch(stem_ctx* ctx, const ExpertsSortArgs& a, hipStream_t s) {
  ProfScope prof(ctx, K_EXPERTS_SORT, s);
  const int segments = a.pairs ? (a.pairs + EXPERTS_SEGMENT - 1) / EXPERTS_SEGMENT : 1;
  int bits = 1;
  while (a.n >> bits) ++bits;
  const size_t lds = (size_t)(WAVES + 1) * (a.n + 1) * 4;
  if (segments > 1) sort_kernel<false><<<segments, WAVES * 64, lds, s>>>(a, segments, bits);
  sort_kernel<true><<<segments, WAVES * 64, lds, s>>>(a, segments, bits);
  return hipGetLastError();
}

hipError_t stem_experts_dispatch_launch(stem_ctx* ctx, const ExpertsRowsArgs& a, hipStream_t s) {
  ProfScope prof(ctx, K_EXPERTS_DISPATCH, s);
  return by_type(a, a.rows, [&](auto e, auto v, unsigned grid) { dispatch_kernel<decltype(e), decltype(v)::value><<<grid, 256, 0, s>>>(a); });
}
hipError_t stem_experts_combine_launch(stem_ctx* ctx, const ExpertsRowsArgs& a, hipStream_t s) {
  ProfScope prof(ctx, K_EXPERTS_COMBINE, s);
  return by_type(a, a.T, [&](auto e, auto v, unsigned grid) { combine_kernel<decltype(e), decltype(v)::value><<<grid, 256, 0, s>>>(a); });
}
hipError_t stem_experts_combine_backward_launch(stem_ctx* ctx, const ExpertsRowsArgs& a, hipStream_t s) {
  ProfScope prof(ctx, K_EXPERTS_COMBINE_BACK, s);
  return by_type(a, a.T, [&](auto e, auto v, unsigned grid) { combine_backward_kernel<decltype(e), decltype(v)::value><<<grid, 256, 0, s>>>(a); });
}
