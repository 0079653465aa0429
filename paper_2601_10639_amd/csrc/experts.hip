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
// PLACE: the counts are taken again and the pairs placed; otherwise they are stored for the kernel that does.  Bound by latency: 128 pairs 3.7 us, 32768 pairs and 64
// experts 5.0 and 6.3 in two launches.
// Up to SUMMED segments each placing workgroup adds up all segments' counts itself, which grows with their square; beyond, a kernel between the two leaves what is in front of
// each segment, and the totals.  us, added up by each / by a kernel, pairs and experts: 2^17 and 64 13.8 / 16.4, 2^19 and 64 18.3 / 19.3, 2^19 and 512 29.8 / 24.5, 2^20 and 64
// 29.7 / 24.1, 2^24 and 64 1470 / 187, 2^24 and 512 3730 / 250.
constexpr int TURNS = 4, SUMMED = 128;

__device__ __forceinline__ void in_order() {                // of LDS, within the wavefront
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int WAVES, bool PLACE>
__global__ __launch_bounds__(WAVES * 64) void sort_kernel(ExpertsSortArgs p, int segments, int bits, bool summed) {
  extern __shared__ int32_t table[];                        // [WAVES][n + 1], then [n + 1] of first rows
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = p.n, pitch = n + 1;
  int32_t* const mine = table + wave * pitch;
  int32_t* const first = table + WAVES * pitch;
  const int at = blockIdx.x * (WAVES * 64 * TURNS) + wave * (64 * TURNS) + lane;
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
  if (summed)
    for (int e = threadIdx.x; e <= n; e += WAVES * 64) {
      const int before = p.counts[(int64_t)blockIdx.x * pitch + e];
      first[e] = p.counts[(int64_t)segments * pitch + e];
      for (int w = 0; w < WAVES; ++w) table[w * pitch + e] += before;
    }
  else if (segments > 1)
    for (int e = threadIdx.x; e <= n; e += WAVES * 64) {
      int all = 0, before = 0;
      for (int s0 = 0; s0 < segments; s0 += 16) {              // 16 under way together
        int c[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) c[u] = p.counts[(int64_t)min(s0 + u, segments - 1) * pitch + e];
#pragma unroll
        for (int u = 0; u < 16; ++u) {
          all += s0 + u < segments ? c[u] : 0;
          before += s0 + u < (int)blockIdx.x ? c[u] : 0;
        }
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

// Counts of the segments to what is in front of each, and the totals behind them.  A workgroup has 64 experts, a lane each, and its 16 wavefronts a strip of segments each, which they
// read twice: what is in front of a strip is known once all are added up.
__global__ __launch_bounds__(1024) void sum_kernel(ExpertsSortArgs p, int segments) {
  constexpr int STRIPS = 16, TOGETHER = 16;
  __shared__ int32_t sums[STRIPS][64];
  const int lane = threadIdx.x & 63, strip = threadIdx.x >> 6, pitch = p.n + 1, e = blockIdx.x * 64 + lane;
  const int per = (segments + STRIPS - 1) / STRIPS, lo = min(strip * per, segments), hi = min(lo + per, segments);
  int32_t* const at = p.counts + min(e, p.n);
  auto each = [&](auto f) __attribute__((always_inline)) {
    for (int s0 = lo; s0 < hi; s0 += TOGETHER) {
      int c[TOGETHER];
#pragma unroll
      for (int u = 0; u < TOGETHER; ++u) c[u] = at[(int64_t)min(s0 + u, hi - 1) * pitch];
#pragma unroll
      for (int u = 0; u < TOGETHER; ++u)
        if (s0 + u < hi) f(s0 + u, c[u]);
    }
  };
  int sum = 0;
  each([&](int, int c) __attribute__((always_inline)) { sum += c; });
  sums[strip][lane] = sum;
  __syncthreads();
  int before = 0, all = 0;
  for (int s = 0; s < STRIPS; ++s) {
    before += s < strip ? sums[s][lane] : 0;
    all += sums[s][lane];
  }
  if (e > p.n) return;
  each([&](int s, int c) __attribute__((always_inline)) {
    at[(int64_t)s * pitch] = before;
    before += c;
  });
  if (strip == 0) at[(int64_t)segments * pitch] = all;
}

// ---- rows ------------------------------------------------------------------------------------------------------------------
// LPR neighbouring lanes have a row or a token, pieces of V elements (16 bytes, at any element's address; rows of fewer elements: one) a lane at a time, and U of
// them are under way together: loads behind a store that may lie over what they read would wait for it.  A row's last piece ends where the row does and
// has elements of the one before it again where the row is no whole number of pieces; pieces beyond it are loaded as it is, so that no load has a branch, and
// not stored.
// (vectors, not arrays of elements: those the compiler keeps in LDS)
// 16384 tokens of 2048, two of 64 experts each: dispatch 39 to 40 us (126 MB read, the second reading of a row from the last level mostly, and 126 written: 6.3 TB/s), combine
// with the residual 48 to 50 (190 + 67 MB, 5.2 TB/s); the fp32 gradients of 1999 x 1001, three of 5 experts, 9 to 10.8.  Residual and output in one, whose long rows of no whole
// number of pieces go an element at a time: 16384 tokens of 4097 bf16 114 us and in one 109, of 8191 220 and 221.
template <int BYTES> struct RawOf;
template <> struct RawOf<16> { typedef u32x4_t type; };
template <> struct RawOf<4> { typedef uint32_t type; };
template <> struct RawOf<2> { typedef uint16_t type; };
template <class E, int V>
using Raw = typename RawOf<V * sizeof(E)>::type;
template <class E, int V>
__device__ __forceinline__ float element(const Raw<E, V>& p, int q) {
  uint32_t w;
  if constexpr (V > 1) w = p[q * sizeof(E) / 4];
  else w = p;
  if constexpr (sizeof(E) == 2) return __uint_as_float(q & 1 ? w & 0xffff0000u : w << 16);
  else return __uint_as_float(w);
}
template <class E, int V>
__device__ __forceinline__ Raw<E, V> pack(const float (&f)[V]) {
  Raw<E, V> p;
  if constexpr (sizeof(E) == 4) {
    if constexpr (V == 1) p = __float_as_uint(f[0]);
    else
#pragma unroll
      for (int q = 0; q < V; ++q) p[q] = __float_as_uint(f[q]);
  } else if constexpr (V == 1) {
    p = __builtin_bit_cast(uint16_t, (__bf16)f[0]);
  } else {
#pragma unroll
    for (int q = 0; q < V; q += 2)
      p[q / 2] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f[q]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f[q + 1]) << 16;
  }
  return p;
}
// U pieces of a row from element c on, `step` apart
template <class E, int V, int U>
__device__ __forceinline__ void load(const void* base, int64_t row, int width, int c, int step, Raw<E, V> (&p)[U]) {
  const E* const from = static_cast<const E*>(base) + row * width;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    Raw<E, V> v;
    __builtin_memcpy(&v, from + min(c + u * step, width - V), sizeof v);
    p[u] = v;
  }
}
template <class E, int V, int U>
__device__ __forceinline__ void store(void* base, int64_t row, int width, int c, int step, const Raw<E, V> (&p)[U]) {
  E* const to = static_cast<E*>(base) + row * width;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const Raw<E, V> v = p[u];
    if (c + u * step < width) __builtin_memcpy(to + min(c + u * step, width - V), &v, sizeof v);
  }
}

template <class E, int V, int LPR>
__global__ __launch_bounds__(256) void dispatch_kernel(ExpertsRowsArgs p) {
  constexpr int STEP = LPR * V, U = 4;
  const int l = threadIdx.x % LPR, width = (int)p.width;
  const int64_t row = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
  if (row >= p.rows) return;
  const int pair = p.src[row];
  if (pair < 0) return;
  int64_t t = pair / p.k;
  if (t >= p.T) {
    if (l == 0) *p.flag = 1;
    t = p.T - 1;
  }
  if (p.ids && l == 0) p.ids_out[row] = p.ids[t];
  for (int c = 0; c < width; c += U * STEP) {
    Raw<E, V> v[U];
    load<E, V, U>(p.x, t, width, c + l * V, STEP, v);
    store<E, V, U>(p.xs, row, width, c + l * V, STEP, v);
  }
}

// Places and weights of a token's choices, lane j of its lanes having the j-th (and the LPR + j-th)
template <int LPR>
struct Choices {
  static constexpr int N = LPR < STEM_EXPERTS_MAX_CHOICES ? 2 : 1;
  int place[N];
  float weight[N];
  __device__ __forceinline__ void load(const ExpertsRowsArgs& p, int64_t t, int l) {
#pragma unroll
    for (int h = 0; h < N; ++h) {
      const int j = h * LPR + l;
      place[h] = j < p.k ? p.place[t * p.k + j] : -1;
      weight[h] = j < p.k && p.weights ? p.weights[t * p.k + j] : 1.f;
    }
  }
  __device__ __forceinline__ int row(int j) const { return __shfl(N > 1 && j >= LPR ? place[N - 1] : place[0], j % LPR, LPR); }
  __device__ __forceinline__ float of(int j) const { return __shfl(N > 1 && j >= LPR ? weight[N - 1] : weight[0], j % LPR, LPR); }
};

template <class E, int V, int LPR>
__global__ __launch_bounds__(256) void combine_kernel(ExpertsRowsArgs p) {
  constexpr int STEP = LPR * V, U = 4;
  const int l = threadIdx.x % LPR, width = (int)p.width;
  const int64_t t = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
  if (t >= p.T) return;
  Choices<LPR> choices;
  choices.load(p, t, l);
  // (a place behind the rows is the last of them, and reported)
#pragma unroll
  for (int& place : choices.place)
    if (place >= p.rows) {
      *p.flag = 1;
      place = (int)p.rows - 1;
    }
  for (int c0 = 0; c0 < width; c0 += U * STEP) {
    const int c = c0 + l * V;
    float sum[U][V];
    if (p.residual) {
      Raw<E, V> v[U];
      load<E, V, U>(p.residual, t, width, c, STEP, v);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < V; ++q) sum[u][q] = element<E, V>(v[u], q);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < V; ++q) sum[u][q] = 0.f;
    }
    for (int j = 0; j < p.k; ++j) {
      const int row = choices.row(j);
      const float w = choices.of(j);
      if (row < 0) continue;
      Raw<E, V> v[U];
      load<E, V, U>(p.ys, row, width, c, STEP, v);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < V; ++q) sum[u][q] = __builtin_fmaf(w, element<E, V>(v[u], q), sum[u][q]);
    }
    Raw<E, V> out[U];
#pragma unroll
    for (int u = 0; u < U; ++u) out[u] = pack<E, V>(sum[u]);
    store<E, V, U>(p.y, t, width, c, STEP, out);
  }
}

template <class E, int V, int LPR>
__global__ __launch_bounds__(256) void combine_backward_kernel(ExpertsRowsArgs p) {
  constexpr int STEP = LPR * V, U = 4;
  const int l = threadIdx.x % LPR, width = (int)p.width;
  const int64_t t = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
  if (t >= p.T) return;
  Choices<LPR> choices;
  choices.load(p, t, l);
  const bool whole = width <= U * STEP;                        // dy's row stays in registers
  Raw<E, V> g[U];
  if (whole && width > 0) load<E, V, U>(p.x, t, width, l * V, STEP, g);
  for (int j = 0; j < p.k; ++j) {
    int row = choices.row(j);
    if (row >= p.rows) {                                       // reported, and none
      if (l == 0) *p.flag = 1;
      row = -1;
    }
    const float w = choices.of(j);
    float sum = 0.f;
    if (row >= 0)
      for (int c0 = 0; c0 < width; c0 += U * STEP) {
        const int c = c0 + l * V;
        Raw<E, V> v[U];
        if (p.dweights) load<E, V, U>(p.ys, row, width, c, STEP, v);
        if (!whole) load<E, V, U>(p.x, t, width, c, STEP, g);
        if (p.dweights)
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int at = c + u * STEP, again = at - min(at, width - V);   // elements that other pieces have
#pragma unroll
            for (int q = 0; q < V; ++q) sum = q >= again ? __builtin_fmaf(element<E, V>(g[u], q), element<E, V>(v[u], q), sum) : sum;
          }
        if (p.dys) {
#pragma unroll
          for (int u = 0; u < U; ++u) {
            float f[V];
#pragma unroll
            for (int q = 0; q < V; ++q) f[q] = w * element<E, V>(g[u], q);
            v[u] = pack<E, V>(f);
          }
          store<E, V, U>(p.dys, row, width, c, STEP, v);
        }
      }
    if (!p.dweights) continue;
#pragma unroll
    for (int d = 1; d < LPR; d <<= 1) sum += __shfl_xor(sum, d);
    if (l == 0) p.dweights[t * p.k + j] = sum;
  }
}

template <int N>
using Int = std::integral_constant<int, N>;
// alone: elements may not be stored twice (in place, an element that two pieces have would be read behind its store where they are not under way together)
template <class F>
hipError_t by_type(const ExpertsRowsArgs& a, int64_t n, bool alone, F f) {
  const int64_t pieces = (a.width * a.es + 15) / 16;
  auto of = [&](auto e, auto v) {
    if (pieces <= 8) f(e, v, Int<8>{}, (unsigned)((n + 31) / 32));
    else if (pieces <= 64) f(e, v, Int<16>{}, (unsigned)((n + 15) / 16));
    else f(e, v, Int<64>{}, (unsigned)((n + 3) / 4));
  };
  const bool one = a.width * a.es < 16 || (alone && a.width * a.es % 16 && pieces > 256);
  if (a.es == 2) one ? of(bf16_t{}, Int<1>{}) : of(bf16_t{}, Int<8>{});
  else one ? of(float{}, Int<1>{}) : of(float{}, Int<4>{});
  return hipGetLastError();
}

template <int WAVES>
void launch_sort(const ExpertsSortArgs& a, const int32_t* route, hipStream_t s) {
  const int segments = route[1];
  const bool summed = route[2] == 3;
  int bits = 1;
  while (a.n >> bits) ++bits;
  const size_t lds = (size_t)(WAVES + 1) * (a.n + 1) * 4;
  if (segments > 1) sort_kernel<WAVES, false><<<segments, WAVES * 64, lds, s>>>(a, segments, bits, false);
  if (summed) sum_kernel<<<a.n / 64 + 1, 1024, 0, s>>>(a, segments);
  sort_kernel<WAVES, true><<<segments, WAVES * 64, lds, s>>>(a, segments, bits, summed);
}

}  // namespace

// {wavefronts of a workgroup, segments, launches}: one workgroup where it is enough, then segments whose counts are few to add and whose pairs are few to rank
extern "C" void stem_route_experts_sort(int32_t pairs, int32_t* route) {
  route[0] = pairs <= 256 ? 1 : pairs <= 1024 || (pairs > 4096 && pairs <= EXPERTS_SMALL) ? 4 : 16;
  const int segment = route[0] * 64 * TURNS;
  route[1] = pairs ? (pairs + segment - 1) / segment : 1;
  route[2] = route[1] > SUMMED ? 3 : route[1] > 1 ? 2 : 1;
}

hipError_t stem_experts_sort_launch(stem_ctx* ctx, const ExpertsSortArgs& a, hipStream_t s) {
  ProfScope prof(ctx, K_EXPERTS_SORT, s);
  int32_t route[3];
  stem_route_experts_sort(a.pairs, route);
  if (route[0] == 1) launch_sort<1>(a, route, s);
  else if (route[0] == 4) launch_sort<4>(a, route, s);
  else launch_sort<16>(a, route, s);
  return hipGetLastError();
}

hipError_t stem_experts_dispatch_launch(stem_ctx* ctx, const ExpertsRowsArgs& a, hipStream_t s) {
  ProfScope prof(ctx, K_EXPERTS_DISPATCH, s);
  return by_type(a, a.rows, false, [&](auto e, auto v, auto l, unsigned grid) { dispatch_kernel<decltype(e), decltype(v)::value, decltype(l)::value><<<grid, 256, 0, s>>>(a); });
}
hipError_t stem_experts_combine_launch(stem_ctx* ctx, const ExpertsRowsArgs& a, hipStream_t s) {
  ProfScope prof(ctx, K_EXPERTS_COMBINE, s);
  return by_type(a, a.T, a.y == a.residual, [&](auto e, auto v, auto l, unsigned grid) { combine_kernel<decltype(e), decltype(v)::value, decltype(l)::value><<<grid, 256, 0, s>>>(a); });
}
hipError_t stem_experts_combine_backward_launch(stem_ctx* ctx, const ExpertsRowsArgs& a, hipStream_t s) {
  ProfScope prof(ctx, K_EXPERTS_COMBINE_BACK, s);
  return by_type(a, a.T, false, [&](auto e, auto v, auto l, unsigned grid) { combine_backward_kernel<decltype(e), decltype(v)::value, decltype(l)::value><<<grid, 256, 0, s>>>(a); });
}
