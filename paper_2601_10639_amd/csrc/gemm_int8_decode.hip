// 8-bit products of a few tokens (up to 64), gfx950: bound by how early and how densely the weights are requested.
//
// A workgroup has 32 channels and a slice of K; its 8 wavefronts take the slice's blocks in turn, straight from memory to registers: a
// block of the weights (32 rows x 32 k, 1 KB) is one operand of v_mfma_i32_32x32x32_i8 as it lies there (quant.h).  Up to 8 tokens whose rows
// fit 1024 chunks of 16 are quantised by every workgroup for itself, from x behind its norm or from the hidden values of the gate
// product, while its weights are on their way: reading them costs less than a launch and its wait.  More tokens come quantised.
// Measured: one token of 1024 -> 4096 4.3 us (its 4.2 MB at the rate of a long read: 0.6); a layer of 2048 x 8192, norm to residual, 16.8 us with
// one token, 20.8 with 8, 23.2 with 16, 25.4 with 48 (33.5 MB: 4.7).  A launch, the first loads' way and the tokens' figures are most of each.
// The bf16 layer, one launch up to 32 tokens, behind the norm's call is faster there.  us a layer in a graph, weights of 16 layers in turn, bf16 /
// 8 bits: 2048 x 8192 17.5 / 18.8 at one token, 17.9 / 22.4 at 8, 24.7 / 25.7 at 32, 30.3 / 28.3 at 64; 1024 x 4096 10.1 / 12.9, 10.4 / 15.0, 13.4 / 18.2, 16.3 / 20.6.
//
// Sums are integers: the wavefronts' parts are added through LDS, the slices' by the workgroup that finishes last, in any order.
#include "quant.h"

typedef __attribute__((ext_vector_type(4))) int i32x4_t;
typedef __attribute__((ext_vector_type(16))) int i32x16_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4_t;
typedef __amdgpu_buffer_rsrc_t rsrc_t;

namespace {

constexpr uint32_t OOB = 0x80000000u;
constexpr int SC1 = 16;            // device scope: the slices of a tile run on different XCDs, whose L2s don't see each other's lines
constexpr int WAVES = 8, THREADS = 64 * WAVES, DEPTH = 8;
constexpr int MAX_CHUNKS = 1024;   // of all rows that are quantised in place: two a thread

__device__ __forceinline__ float sigmoidf_fast(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
__device__ __forceinline__ rsrc_t resource(const void* p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000); }

// v over all 64 lanes
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  return v;
}
__device__ __forceinline__ u32x4_t integers(const float (&v)[16], float inv, uint32_t mask) {
  u32x4_t w;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) b[k] = quant_integer(v[4 * q + k], inv);
    w[q] = quant_four_bytes(b[0], b[1], b[2], b[3]) & mask;
  }
  return w;
}

// FROM: where the tokens come from
enum { FROM_INTEGERS = 0, FROM_ROWS, FROM_HIDDEN };

// Tokens to integers in LDS: chunk (16 k) c of this workgroup's slice of token t at ((c << rows_log) + t) * 16, and its scale.
template <int FROM>
struct Inline {
  float v[2][16];
  QuantChunk raw[2], weight[2];   // of x, of the norm's weight
  uint32_t tops[4];               // of this wavefront's token: the first 256 tiles' maxima
  int row[2], at[2];              // of the chunk that v holds: token, chunk of the row; token -1 for none
  // In front of the weights' loads: loads return in order, and all this is there before the first weights are.
  __device__ __forceinline__ void load(const QuantDecodeArgs& p, int k0, int chunks, int tid) {   // chunks of a row
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int idx = h * THREADS + tid, r = idx / chunks;
      row[h] = r < p.M ? r : -1;
      at[h] = idx - r * chunks;
#pragma unroll
      for (int q = 0; q < 16; ++q) v[h][q] = 0.f;
      if (row[h] < 0) continue;
      if (FROM == FROM_ROWS) {
        const int left = p.row_K - at[h] * 16;
        raw[h] = left > 0 ? quant_load_chunk(p.x + (size_t)r * p.row_K + at[h] * 16, left) : QuantChunk{};
        if (p.norm.weight) weight[h] = left > 0 ? quant_load_chunk(static_cast<const bf16_t*>(p.norm.weight) + at[h] * 16, left) : QuantChunk{};
      } else {
        // two groups of 8 channels, four of each in lanes r and r + 32 of the gate product's layout
        const int c = k0 / 16 + at[h];
        const float* const from = p.h + ((size_t)(c >> 1) * 4 + (c & 1) * 2) * 256 + r * 4;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4_t u = *reinterpret_cast<const f32x4_t*>(from + (q >> 1) * 256 + (q & 1) * 128);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[h][4 * q + k] = u[k];
        }
      }
    }
    if (FROM == FROM_HIDDEN) {
      const int t = tid >> 6, lane = tid & 63;
#pragma unroll
      for (int i = 0; i < 4; ++i) tops[i] = t < p.M && i * 64 + lane < p.maxima ? p.max_in[(i * 64 + lane) * 8 + t] : 0;
    }
  }
  // a figure of each token, from one of each chunk: part[] in LDS takes them, wavefront t adds up token t's, stat[t] is the result
  template <class F, class R>
  __device__ __forceinline__ void reduce(int M, int chunks, int tid, float* part, float* stat, F f, R over) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (row[h] >= 0) part[h * THREADS + tid] = f(h);
    __syncthreads();
    const int t = tid >> 6;
    if (t < M) over(t, part + t * chunks);
    __syncthreads();
  }
  __device__ __forceinline__ void quantise(const QuantDecodeArgs& p, int k0, int K, int chunks, int tid, float* part, float* stat, char* q, int rows_log,
                                           float* scale) {
    const int lane = tid & 63;
    if (FROM == FROM_ROWS)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (row[h] >= 0)
#pragma unroll
          for (int q = 0; q < 16; ++q) v[h][q] = quant_element(raw[h], q);
    auto total = [&](int t, const float* from) {
      float s = 0.f;
      for (int c = lane; c < chunks; c += 64) s += from[c];
      s = wave_sum(s);
      if (lane == 0) stat[t] = s;
    };
    if (FROM == FROM_ROWS && (p.norm.kind != STEM_NORM_NONE || p.norm.weight)) {
      if (p.norm.kind == STEM_NORM_LAYER) {
        reduce(p.M, chunks, tid, part, stat, [&](int h) { float s = 0.f;
#pragma unroll
          for (int e = 0; e < 16; ++e) s += v[h][e];
          return s; }, total);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (row[h] < 0) continue;
          const float mean = stat[row[h]] / (float)p.row_K;
#pragma unroll
          for (int e = 0; e < 16; ++e) v[h][e] = at[h] * 16 + e < p.row_K ? v[h][e] - mean : 0.f;
        }
      }
      if (p.norm.kind != STEM_NORM_NONE)
        reduce(p.M, chunks, tid, part, stat, [&](int h) { float s = 0.f;
#pragma unroll
          for (int e = 0; e < 16; ++e) s += v[h][e] * v[h][e];
          return s; }, total);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (row[h] < 0) continue;
        const float r = p.norm.kind == STEM_NORM_NONE ? 1.f : 1.0f / sqrtf(stat[row[h]] / (float)p.row_K + p.norm.eps);
        const int left = p.row_K - at[h] * 16;
        if (p.norm.weight) {
#pragma unroll
          for (int e = 0; e < 16; ++e) v[h][e] = e < left ? v[h][e] * r * quant_element(weight[h], e) : 0.f;
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) v[h][e] *= r;
        }
      }
    }
    if (FROM == FROM_ROWS) {
      reduce(p.M, chunks, tid, part, stat, [&](int h) { uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) m = max(m, __float_as_uint(v[h][e]) & 0x7fffffffu);
        return __uint_as_float(m); }, [&](int t, const float* from) {
          uint32_t m = 0;
          for (int c = lane; c < chunks; c += 64) m = max(m, __float_as_uint(from[c]));
          m = wave_max(m);
          if (lane == 0) stat[t] = __uint_as_float(m);
        });
    } else {
      const int t = tid >> 6;
      if (t < p.M) {
        uint32_t m = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
        for (int g = 256 + lane; g < p.maxima; g += 64) m = max(m, p.max_in[g * 8 + t]);
        m = wave_max(m);
        if (lane == 0) stat[t] = __uint_as_float(m);
      }
      __syncthreads();
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (row[h] < 0) continue;
      const QuantScale s = quant_scale(__float_as_uint(stat[row[h]]));
      if (at[h] == 0) scale[row[h]] = s.scale;
      const int c = at[h] - (FROM == FROM_ROWS ? k0 / 16 : 0);
      if (c >= 0 && c < K / 16) *reinterpret_cast<u32x4_t*>(q + ((c << rows_log) + row[h]) * 16) = integers(v[h], s.inv, s.mask);
    }
  }
};

template <bool GATE, int FROM, int MT>
__global__ __launch_bounds__(THREADS) void gemm_int8_decode_kernel(QuantDecodeArgs p) {
  static_assert(FROM == FROM_INTEGERS || MT == 1, "up to 8 tokens");
  constexpr bool INLINE = FROM != FROM_INTEGERS;
  // The wavefronts' sums; before, the tokens' integers, up to 1024 chunks, or twice that with the rows between their number and the next
  // power of two.  Behind them the chunks' figures.
  constexpr int SUMS = WAVES * MT * 4096, PART = INLINE ? MAX_CHUNKS * 4 : 0;
  static_assert(!INLINE || SUMS >= 2 * MAX_CHUNKS * 16, "room for the integers");
  __shared__ __attribute__((aligned(16))) char smem[SUMS + PART + 64 + 272];
  float* const part = reinterpret_cast<float*>(smem + SUMS);
  float* const scale = reinterpret_cast<float*>(smem + SUMS + PART);   // [8], and as many figures of whole rows
  uint32_t* const misc = reinterpret_cast<uint32_t*>(smem + SUMS + PART + 64);
  const int rows_log = p.M > 4 ? 3 : p.M > 2 ? 2 : p.M > 1 ? 1 : 0;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tiles = (p.N + 31) / 32;
  const int slice = blockIdx.x / tiles, tile = blockIdx.x - slice * tiles;
  const int all = p.K / 32, per = (all / 4 + p.ksplit - 1) / p.ksplit * 4, b0 = slice * per, nb = all - b0 < per ? all - b0 : per;   // blocks
  const rsrc_t rb = resource(p.B + (size_t)tile * 32 * p.K, 32 * p.K);
  const rsrc_t ra = resource(p.A, INLINE ? 0 : (p.M + 31) / 32 * 32 * p.K);
  const uint32_t la = (lane & 31) < p.M ? lane * 16 : OOB, lb = 32 + (lane & 31) < p.M ? 32 * p.K + lane * 16 : OOB;
  i32x4_t w[DEPTH], a[INLINE ? 1 : DEPTH][MT];
  auto request = [&](int from) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
      const int b = from + i * WAVES + wave;
      const int at = b < nb ? (b0 + b) * 1024 : 0;
      const uint32_t none = b < nb ? 0u : OOB;
      w[i] = __builtin_bit_cast(i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rb, (lane * 16) | none, at, 0));
      if constexpr (!INLINE) {
        a[i][0] = __builtin_bit_cast(i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(ra, la | none, at, 0));
        if (MT > 1) a[i][MT - 1] = __builtin_bit_cast(i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(ra, lb | none, at, 0));
      }
    }
  };
  const int chunks = FROM == FROM_ROWS ? p.K / 16 : nb * 2;
  Inline<INLINE ? FROM : FROM_ROWS> in;
  if constexpr (INLINE) in.load(p, b0 * 32, chunks, tid);
  __builtin_amdgcn_sched_barrier(0);
  request(0);
  // the gate product's epilogue multiplies by a row of the table
  const int u_lane = tid & 63, u_group = tid >> 6 & 3, u_half = tid >> 8;   // of the tile in lanes' layout: 4 channels of a token
  const int tok = u_half * 32 + (u_lane & 31), ch = tile * 32 + 8 * u_group + 4 * (u_lane >> 5);
  const bool mine = u_half < MT && tok < p.M && ch < p.N;
  u32x2_t e = {};
  if (GATE && mine) {
    int id = p.ids[tok];
    if ((unsigned)id >= (unsigned)p.E_rows) {   // reported to the host, clamped so no access leaves the table
      *p.flag = 1;
      id = id < 0 ? 0 : p.E_rows - 1;
    }
    e = *reinterpret_cast<const u32x2_t*>(p.E + (size_t)id * p.N + ch);
  }
  if constexpr (INLINE) {
    in.quantise(p, b0 * 32, nb * 32, chunks, tid, part, scale + 8, smem, rows_log, scale);
    __syncthreads();
  }
  i32x16_t acc[MT] = {};
  // (the lanes of further tokens repeat the first ones: their sums are not read)
  const char* const tokens = smem + (((lane >> 5) << rows_log) + (lane & ((1 << rows_log) - 1))) * 16;
  for (int from = 0; from < nb; from += DEPTH * WAVES) {
    i32x4_t wc[DEPTH], ac[INLINE ? 1 : DEPTH][MT];
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
      wc[i] = w[i];
      if constexpr (!INLINE)
#pragma unroll
        for (int t = 0; t < MT; ++t) ac[i][t] = a[i][t];
    }
    if (from + DEPTH * WAVES < nb) request(from + DEPTH * WAVES);
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
      const int b = from + i * WAVES + wave;
      if constexpr (INLINE) {
        const i32x4_t t = *reinterpret_cast<const i32x4_t*>(tokens + ((b < nb ? b : 0) << (rows_log + 5)));   // past the slice: weights of zero
        acc[0] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wc[i], t, acc[0], 0, 0, 0);
      } else {
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[t] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wc[i], ac[i][t], acc[t], 0, 0, 0);
      }
    }
  }
  if (INLINE) __syncthreads();   // the integers have been read
  i32x4_t* const sums = reinterpret_cast<i32x4_t*>(smem);
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      sums[((wave * MT + t) * 4 + g) * 64 + lane] = i32x4_t{acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]};
  if (GATE && tid < 64) misc[tid] = 0;
  __syncthreads();
  i32x4_t sum = {};
  if (mine)
#pragma unroll
    for (int v = 0; v < WAVES; ++v) sum += sums[((v * MT + u_half) * 4 + u_group) * 64 + u_lane];
  if (p.ksplit > 1) {
    const int units = MT * 256;
    const rsrc_t rw = resource(p.ws, p.ksplit * tiles * units * 16);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, sum), rw, mine ? ((slice * tiles + tile) * units + tid) * 16 : OOB, 0, SC1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int* const ticket = reinterpret_cast<int*>(misc + 64);
    if (tid == 0) *ticket = __hip_atomic_fetch_add(p.tickets + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (*ticket != p.ksplit - 1) return;
    if (tid == 0) __hip_atomic_store(p.tickets + tile, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next launch
    asm volatile("" ::: "memory");
    i32x4_t v[8];   // all in flight together; what is beyond the last slice, or this workgroup's own, reads as zero
#pragma unroll
    for (int s = 0; s < 8; ++s)
      v[s] = __builtin_bit_cast(i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rw, mine && s < p.ksplit && s != slice ? ((s * tiles + tile) * units + tid) * 16 : OOB, 0, SC1));
#pragma unroll
    for (int s = 0; s < 8; ++s) sum += v[s];
  }
  if (mine) {
    const float sa = INLINE ? scale[tok] : p.scale_a[tok];
    float z[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) z[q] = ch + q < p.N ? (float)sum[q] * (sa * p.scale_b[ch + q]) : 0.f;
    if (GATE) {
      const float u[4] = {__uint_as_float(e[0] << 16), __uint_as_float(e[0] & 0xffff0000u), __uint_as_float(e[1] << 16), __uint_as_float(e[1] & 0xffff0000u)};
      f32x4_t h;
      uint32_t top = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        h[q] = z[q] * sigmoidf_fast(z[q]) * u[q];
        top = max(top, __float_as_uint(h[q]) & 0x7fffffffu);
      }
      const int blocks = (p.N + 127) / 128 * 4;
      *reinterpret_cast<f32x4_t*>(p.h_out + (((size_t)u_half * blocks + tile) * 4 + u_group) * 256 + u_lane * 4) = h;
      atomicMax(misc + tok, top);
    } else {
      const size_t at = (size_t)tok * p.N + ch;
      if (p.N % 4 == 0) {
        if (p.residual) {
          const u32x2_t r = *reinterpret_cast<const u32x2_t*>(p.residual + at);
          z[0] += __uint_as_float(r[0] << 16); z[1] += __uint_as_float(r[0] & 0xffff0000u);
          z[2] += __uint_as_float(r[1] << 16); z[3] += __uint_as_float(r[1] & 0xffff0000u);
        }
        bf16x4_t o;
#pragma unroll
        for (int q = 0; q < 4; ++q) o[q] = (__bf16)z[q];
        *reinterpret_cast<bf16x4_t*>(p.y + at) = o;
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (ch + q < p.N) {
            if (p.residual) z[q] += __uint_as_float((uint32_t)p.residual[at + q] << 16);
            reinterpret_cast<__bf16*>(p.y)[at + q] = (__bf16)z[q];
          }
      }
    }
  }
  if (GATE) {
    __syncthreads();
    if (p.max_out) {
      if (tid < 8) p.max_out[tile * 8 + tid] = misc[tid];
    } else if (tid < p.M) {
      __hip_atomic_fetch_max(p.amax + tid * QUANT_AMAX_STRIDE, misc[tid], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    // d_ff may end inside the last 128 channels of the next product's K: zeros, by the last tile (any number would do: quant.h)
    if (tile == tiles - 1) {
      const int blocks = (p.N + 127) / 128 * 4;
      for (int t = 0; t < MT; ++t)
        for (int b = tiles * 1024 + tid; b < blocks * 1024; b += THREADS) p.h_out[(size_t)t * blocks * 1024 + b] = 0.f;
    }
  }
}

}  // namespace

bool stem_quant_decode_inline(int64_t T, int64_t K) { return T <= 8 && T * (stem_quant_pitch(K) / 16) <= MAX_CHUNKS; }

int stem_quant_decode_slices(int N, int K, size_t ws_bytes, int M) {
  // at most one workgroup a compute unit, and 4 blocks a wavefront or more
  const int tiles = (N + 31) / 32, blocks = K / 32, mt = M > 32 ? 2 : 1;
  if (tiles > STEM_TICKETS) return 1;
  int s = 256 / tiles;
  s = s < 1 ? 1 : s > 8 ? 8 : s;
  while (s > 1 && (blocks / s < 4 * WAVES || (size_t)s * tiles * mt * 4096 > ws_bytes)) --s;
  // every slice has blocks: they are cut by fours
  while (s > 1 && (blocks / 4 + s - 1) / s * (s - 1) >= blocks / 4) --s;
  return s;
}

hipError_t stem_quant_decode_launch(stem_ctx* ctx, int kid, const QuantDecodeArgs& a, hipStream_t s) {
  ProfScope prof(ctx, kid, s);
  const int grid = (a.N + 31) / 32 * a.ksplit;
  const bool gate = !a.y;
  if (a.x) {
    if (gate) gemm_int8_decode_kernel<true, FROM_ROWS, 1><<<grid, THREADS, 0, s>>>(a);
    else gemm_int8_decode_kernel<false, FROM_ROWS, 1><<<grid, THREADS, 0, s>>>(a);
  } else if (a.h) {
    gemm_int8_decode_kernel<false, FROM_HIDDEN, 1><<<grid, THREADS, 0, s>>>(a);
  } else if (a.M <= 32) {
    if (gate) gemm_int8_decode_kernel<true, FROM_INTEGERS, 1><<<grid, THREADS, 0, s>>>(a);
    else gemm_int8_decode_kernel<false, FROM_INTEGERS, 1><<<grid, THREADS, 0, s>>>(a);
  } else {
    if (gate) gemm_int8_decode_kernel<true, FROM_INTEGERS, 2><<<grid, THREADS, 0, s>>>(a);
    else gemm_int8_decode_kernel<false, FROM_INTEGERS, 2><<<grid, THREADS, 0, s>>>(a);
  }
  return hipGetLastError();
}
