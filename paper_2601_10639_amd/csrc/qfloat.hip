// bf16 rows and tiles to 8-bit floating point with a scale for each block of 128 (qfloat.h).
//
// A block's scale depends on nothing but the block, so a kernel reads each value once: a row's 128 values are eight neighbouring lanes', a tile of
// 128 x 128 is a workgroup's.  Bound by memory: 2 bytes read and 1 (or 2) written a value.
#include "qfloat.h"
#include "quant.h"   // chunks of a bf16 row

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;

namespace {

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t max_of_eight(uint32_t v) {   // neighbouring lanes
  v = max(v, dpp<0xb1>(v));    // quad_perm 1 0 3 2
  v = max(v, dpp<0x4e>(v));    // quad_perm 2 3 0 1
  return max(v, dpp<0x141>(v));   // row_half_mirror
}
template <int LPR>
__device__ __forceinline__ float sum_row(float v, float* red) {
#pragma unroll
  for (int d = 1; d < (LPR < 64 ? LPR : 64); d <<= 1) v += __shfl_xor(v, d);
  if (LPR > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (red[0] + red[1]) + (red[2] + red[3]);
  }
  return v;
}

// ---- rows without a norm ----------------------------------------------------------------------------------------------------------
// A workgroup has 32 rows and up to 4 blocks of each: a lane the 16 values of row t / 8, chunk t % 8, so that eight lanes read 256 bytes of a row and store, with
// the seven other rows of their wavefront, whole lines of the form.  16384 x 8192: 64 to 67 us, 6.1 TB/s, a copy's rate; 123 with a wavefront a row, whose 16-byte
// stores are 512 apart.
constexpr int BLOCKS = 4;
template <bool HIDDEN>
__global__ __launch_bounds__(256) void chunks_kernel(QfloatRowsArgs p) {
  const int lane = threadIdx.x & 63, c = threadIdx.x & 7, nkb = (p.K + 127) / 128, parts = (nkb + BLOCKS - 1) / BLOCKS;
  const int group = blockIdx.x / parts, kb0 = (blockIdx.x - group * parts) * BLOCKS, row = group * 32 + (threadIdx.x >> 3);
  const bool live = row < p.groups.T;
  const int64_t first = (int64_t)(live ? row : 0) * p.K;
  QuantChunk raw[HIDDEN ? 1 : BLOCKS];
  f32x4_t hid[HIDDEN ? BLOCKS : 1][4];
#pragma unroll
  for (int u = 0; u < BLOCKS; ++u) {
    const int at = (kb0 + u) * 128 + c * 16;
    if constexpr (HIDDEN) {
#pragma unroll
      for (int g = 0; g < 4; ++g) hid[u][g] = live && at < p.K ? *reinterpret_cast<const f32x4_t*>(p.h + first + at + 4 * g) : f32x4_t{};   // (d_ff: multiples of 64)
    } else {
      raw[u] = qfloat_fetch(p.x + first, at, p.K);
    }
  }
  if constexpr (!HIDDEN)
#pragma unroll
    for (int u = 0; u < BLOCKS; ++u) qfloat_settle(raw[u], p.K - (kb0 + u) * 128 - c * 16);
  auto value = [&](int u, int q) __attribute__((always_inline)) {
    if constexpr (HIDDEN) return hid[u][q >> 2][q & 3];
    else return quant_element(raw[u], q);
  };
  int place = live ? row : -1;
  if (p.groups.offsets) place = qfloat_place<8>(p.groups, row, lane);
  uint8_t* const out = p.q + ((int64_t)(place >> 5) * nkb * 4 + (c >> 1)) * 1024 + (c & 1) * 512 + (place & 31) * 16;
#pragma unroll
  for (int u = 0; u < BLOCKS; ++u) {
    const int kb = kb0 + u;
    float v[16];
#pragma unroll
    for (int q = 0; q < 16; ++q) v[q] = value(u, q);
    const QfloatScale s = qfloat_scale(max_of_eight(qfloat_top(v)));
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = qfloat_four(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3], s);
    if (place < 0 || kb >= nkb) continue;
    *reinterpret_cast<u32x4_t*>(out + (int64_t)kb * 4096) = u32x4_t{w[0], w[1], w[2], w[3]};
    if (c == 0) p.scale[qfloat_scale_at(place, kb, nkb)] = (uint8_t)s.byte;
  }
}

// ---- rows behind a norm ---------------------------------------------------------------------------------------------
// LPR neighbouring lanes have a row (256: the workgroup), CPT chunks of 16 values each (0: as many as there are, read again for each use).  A row's chunks lie 512
// bytes apart in the form, so the workgroup's rows are collected in LDS and stored together: 4 neighbouring rows are 64 bytes.  Few chunks a lane, so that many
// wavefronts hide the loads: us with rms norm, of 16384 rows unless other
//   K             512   1024   2048   2048 of 2048   4096   8192
//   <32, 2>       8.3   12.1
//   <64, 2>      12.5   12.5   19.8   5.8
//   <32, 4>       8.7   12.4   21.0   7.2                          (<16, 8>: 9.0, 13.5, 24.4, 10.2)
//   <64, 4>                                          35.3          (<32, 8>: 40.3)
//   <64, 8>                                                 83     (103 without LDS)
// A large copy moves what K 4096 reads and writes in 33 us.
template <int LPR, int CPT>
__global__ __launch_bounds__(256) void rows_kernel(QfloatRowsArgs p) {
  constexpr int ROWS = 256 / LPR, HELD = CPT ? CPT : 1;
  __shared__ float red[4];
  __shared__ int places[ROWS];
  __shared__ __attribute__((aligned(16))) u32x4_t out[256 * HELD];
  const int l = threadIdx.x % LPR, lane = threadIdx.x & 63;
  const int row = blockIdx.x * ROWS + threadIdx.x / LPR;
  const int chunks = (p.K + 127) / 128 * 8, nkb = chunks / 8;
  const bool live = row < p.groups.T;
  const bf16_t* const x = p.x + (int64_t)(live ? row : 0) * p.K;
  auto fetch = [&](int t) __attribute__((always_inline)) { return qfloat_fetch(x, (t * LPR + l) * 16, p.K); };
  auto settle = [&](int t, QuantChunk c) __attribute__((always_inline)) {
    qfloat_settle(c, p.K - (t * LPR + l) * 16);
    return c;
  };
  QuantChunk raw[HELD] = {};
  if constexpr (CPT > 0) {
#pragma unroll
    for (int t = 0; t < CPT; ++t)
      if (t * LPR < chunks) raw[t] = fetch(t);
#pragma unroll
    for (int t = 0; t < CPT; ++t)
      if (t * LPR < chunks) raw[t] = settle(t, raw[t]);
  }
  int place = live ? row : -1;
  if (p.groups.offsets) place = qfloat_place<(LPR < 64 ? LPR : 64)>(p.groups, row, lane);
  // (values are made of the packed ones at each use: held as floats they would cost half of the wavefronts)
  auto chunk = [&](int t) __attribute__((always_inline)) {
    if constexpr (CPT > 0) return raw[t];
    else return settle(t, fetch(t));
  };
  auto each_chunk = [&](auto f) __attribute__((always_inline)) {
    if constexpr (CPT > 0) {
#pragma unroll
      for (int t = 0; t < CPT; ++t)
        if (t * LPR < chunks) f(t);
    } else {
      for (int t = 0; t * LPR < chunks; ++t) f(t);
    }
  };
  float mean = 0.f, r = 1.f;
  auto total = [&](bool squares) __attribute__((always_inline)) {
    float s = 0.f;
    each_chunk([&](int t) __attribute__((always_inline)) {
      const QuantChunk c = chunk(t);
      const int in = p.K - (t * LPR + l) * 16;
      float u[16];
#pragma unroll
      for (int q = 0; q < 16; ++q) u[q] = quant_element(c, q);
      if (p.norm.kind == STEM_NORM_LAYER && squares) {
#pragma unroll
        for (int q = 0; q < 16; ++q) u[q] -= mean;
        if (in < 16)
#pragma unroll
          for (int q = 0; q < 16; ++q) u[q] = q < in ? u[q] : 0.f;
      }
#pragma unroll
      for (int q = 0; q < 16; ++q) s = squares ? __builtin_fmaf(u[q], u[q], s) : s + u[q];
    });
    return sum_row<LPR>(s, red) / (float)p.K;
  };
  if (p.norm.kind == STEM_NORM_LAYER) mean = total(false);
  if (p.norm.kind != STEM_NORM_NONE) r = 1.0f / sqrtf(total(true) + p.norm.eps);
  auto to = [&](int at, int c) __attribute__((always_inline)) {
    return reinterpret_cast<u32x4_t*>(p.q + (int64_t)(at >> 5) * 32 * chunks * 16 + (at & 31) * 16 + (int64_t)(c >> 1) * 1024 + (c & 1) * 512);
  };
  // chunk c of the workgroup's row `of` until all are there (rotated: lanes that write a row's chunks, or read a chunk's rows, are on different banks)
  auto kept = [&](int of, int c) __attribute__((always_inline)) -> u32x4_t& { return out[c * ROWS + ((of + c) & (ROWS - 1))]; };
  each_chunk([&](int t) __attribute__((always_inline)) {
    const int c = t * LPR + l, in = p.K - c * 16;
    const QuantChunk x = chunk(t);
    QuantChunk g = {};
    if (p.norm.weight) {
      g = qfloat_fetch(static_cast<const bf16_t*>(p.norm.weight), c * 16, p.K);
      qfloat_settle(g, in);
    }
    float u[16];
#pragma unroll
    for (int q = 0; q < 16; ++q) u[q] = quant_element(x, q);
    if (p.norm.kind == STEM_NORM_LAYER)
#pragma unroll
      for (int q = 0; q < 16; ++q) u[q] -= mean;
#pragma unroll
    for (int q = 0; q < 16; ++q) u[q] *= r;
    if (p.norm.weight)
#pragma unroll
      for (int q = 0; q < 16; ++q) u[q] *= quant_element(g, q);
    if (in < 16)                                               // zeros behind the row's end
#pragma unroll
      for (int q = 0; q < 16; ++q) u[q] = q < in ? u[q] : 0.f;
    const QfloatScale s = qfloat_scale(max_of_eight(qfloat_top(u)));
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = qfloat_four(u[4 * q], u[4 * q + 1], u[4 * q + 2], u[4 * q + 3], s);
    if (c >= chunks) return;
    const u32x4_t four = {w[0], w[1], w[2], w[3]};
    if (CPT > 0) kept(threadIdx.x / LPR, c) = four;
    else if (place >= 0) *to(place, c) = four;
    if ((c & 7) == 0 && place >= 0) p.scale[qfloat_scale_at(place, c >> 3, nkb)] = (uint8_t)s.byte;
  });
  if constexpr (CPT > 0) {
    if (l == 0) places[threadIdx.x / LPR] = place;
    __syncthreads();
    const int of = threadIdx.x % ROWS, at = places[of];
    if (at < 0) return;
    for (int c = threadIdx.x / ROWS; c < chunks; c += LPR) *to(at, c) = kept(of, c);
  }
}

// ---- tiles of 128 x 128 -----------------------------------------------------------------------------------------------------------
// Lane t of the workgroup has rows 4 (t / 8) .. + 3 and columns 16 (t % 8) .. + 15: a row's magnitudes are eight neighbouring lanes'.  Four rows of a
// column are a word (8 bits) or two (bf16) of the transpose, which goes through LDS to lie as that form does.  Columns' words are a pitch apart that keeps
// 16-byte pieces whole, and some more every 16 columns, so that the lanes' stores fall into different banks.  Both transposes of a weight gradient, and the gradient's
// form, of 16384 x (2001 + 2100): 60 us, 5 TB/s; of values rounded to 8 bits, 16384 x (1024 + 4096) 71 to 77 and 16384 x (2048 + 8192) 146 to 149, 5.3 TB/s both; weights of
// 8192 x 2048 to both forms 14 to 15 one after another, 19 to 20 from memory.
__device__ __forceinline__ void load_tile(const bf16_t* x, int cols, int rows, int quad, int col, QuantChunk (&raw)[4]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    raw[r] = qfloat_fetch(x + (int64_t)min(quad * 4 + r, rows - 1) * cols, col, cols);
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) qfloat_settle(raw[r], quad * 4 + r < rows ? cols - col : 0);
}
// a lane's four rows of a form whose rows have nkb blocks
__device__ __forceinline__ void store_rows(uint8_t* q, uint8_t* scale, int nkb, int row0, int kb, int c, const float (&v)[4][16], const QfloatScale (&s)[4]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int row = row0 + r;
    uint32_t w[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) w[g] = qfloat_four(v[r][4 * g], v[r][4 * g + 1], v[r][4 * g + 2], v[r][4 * g + 3], s[r]);
    *reinterpret_cast<u32x4_t*>(q + ((int64_t)(row >> 5) * (nkb * 4) + (kb * 4 + (c >> 1))) * 1024 + (c & 1) * 512 + (row & 31) * 16) = u32x4_t{w[0], w[1], w[2], w[3]};
    if (c == 0) scale[qfloat_scale_at(row, kb, nkb)] = (uint8_t)s[r].byte;
  }
}

__global__ __launch_bounds__(256) void weights_kernel(QfloatTilesArgs p) {
  constexpr int PITCH = 36;
  __shared__ uint32_t tops[4];
  __shared__ __attribute__((aligned(16))) uint32_t words[128 * PITCH + 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, quad = t >> 3, c = t & 7;
  const int nkb = (p.cols + 127) / 128, nkb_t = (p.rows + 127) / 128, tr = blockIdx.x / nkb, tc = blockIdx.x - tr * nkb;
  const int64_t form = (int64_t)nkb * nkb_t * (16384 + 128), elements = (int64_t)nkb * nkb_t * 16384;
  float v[4][16];
  {
    QuantChunk raw[4];
    load_tile(p.x + ((int64_t)blockIdx.y * p.rows + tr * 128) * p.cols, p.cols, p.rows - tr * 128, quad, tc * 128 + c * 16, raw);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int q = 0; q < 16; ++q) v[r][q] = quant_element(raw[r], q);
  }
  uint32_t m = 0;
#pragma unroll
  for (int r = 0; r < 4; ++r) m = max(m, qfloat_top(v[r]));
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
  if (lane == 0) tops[wave] = m;
  __syncthreads();
  const QfloatScale one = qfloat_scale(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
  if (p.q) {
    const QfloatScale s[4] = {one, one, one, one};
    uint8_t* const q = p.q + blockIdx.y * form;
    store_rows(q, q + elements, nkb, tr * 128 + quad * 4, tc, c, v, s);
  }
  if (!p.qt) return;
  uint8_t* const qt = p.qt + blockIdx.y * form;
#pragma unroll
  for (int q = 0; q < 16; ++q) {
    const int at = c * 16 + q;
    words[at * PITCH + c * 8 + quad] = qfloat_four(v[0][q], v[1][q], v[2][q], v[3][q], one);
    if (quad == 0) qt[elements + qfloat_scale_at(tc * 128 + at, tr, nkb_t)] = (uint8_t)one.byte;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 4; ++u) {                             // column block u, row block `wave`
    const int at = u * 32 + (lane & 31);
    *reinterpret_cast<u32x4_t*>(qt + ((int64_t)(tc * 4 + u) * (nkb_t * 4) + tr * 4 + wave) * 1024 + lane * 16) =
        *reinterpret_cast<const u32x4_t*>(words + at * PITCH + (at >> 4) * 8 + (wave * 2 + (lane >> 5)) * 4);
  }
}

// The largest magnitude of each of a lane's 16 columns over the tile's 128 rows, numbers alone, as bits of bf16, two columns a word
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2_t;
__device__ __forceinline__ void column_tops(const QuantChunk (&raw)[4], uint32_t (&top)[8], u32x4_t (&red)[4][8][2]) {
  auto larger = [](uint32_t a, uint32_t b) __attribute__((always_inline)) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a), __builtin_bit_cast(u16x2_t, b)));
  };
  auto number = [](uint32_t v) __attribute__((always_inline)) {
    return ((v & 0x7fffu) < 0x7f80u ? v & 0x7fffu : 0u) | ((v & 0x7fff0000u) < 0x7f800000u ? v & 0x7fff0000u : 0u);
  };
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = threadIdx.x & 7;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    top[w] = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) top[w] = larger(top[w], number(raw[r].w[w]));
#pragma unroll
    for (int d = 8; d < 64; d <<= 1) top[w] = larger(top[w], (uint32_t)__shfl_xor((int)top[w], d));
  }
  if (lane < 8) {
    red[wave][c][0] = u32x4_t{top[0], top[1], top[2], top[3]};
    red[wave][c][1] = u32x4_t{top[4], top[5], top[6], top[7]};
  }
  __syncthreads();
#pragma unroll
  for (int v = 0; v < 4; ++v)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x4_t other = red[v][c][h];
#pragma unroll
      for (int q = 0; q < 4; ++q) top[4 * h + q] = larger(top[4 * h + q], other[q]);
    }
}

template <bool ROUNDED>
__global__ __launch_bounds__(256) void turn_kernel(QfloatTurnArgs first, QfloatTurnArgs second, int blocks) {
  constexpr int PITCH = 68;
  __shared__ __attribute__((aligned(16))) uint32_t words[128 * PITCH + 128];
  __shared__ __attribute__((aligned(16))) u32x4_t red[ROUNDED ? 4 : 1][8][2];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, quad = t >> 3, c = t & 7;
  const QfloatTurnArgs& p = (int)blockIdx.x < blocks ? first : second;
  const int b = (int)blockIdx.x < blocks ? blockIdx.x : blockIdx.x - blocks;
  const int nkb = (p.cols + 127) / 128, tr = b / nkb, tc = b - tr * nkb;
  QfloatTile tile;
  if (!qfloat_tile<128>(p.groups, tr, lane, tile)) return;
  QuantChunk raw[4];
  load_tile(p.x + (int64_t)tile.row * p.cols, p.cols, tile.rows, quad, tc * 128 + c * 16, raw);
  uint32_t top[8];
  if constexpr (ROUNDED) column_tops(raw, top, red);
#pragma unroll
  for (int w = 0; w < 8; ++w) {                             // two columns at a time
    const int at = c * 16 + 2 * w;
    uint32_t* const to = words + at * PITCH + c * 16 + quad * 2;
    if constexpr (ROUNDED) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const QfloatScale s = qfloat_scale(h ? top[w] & 0xffff0000u : top[w] << 16);
        const uint32_t four = qfloat_four(quant_element(raw[0], 2 * w + h), quant_element(raw[1], 2 * w + h), quant_element(raw[2], 2 * w + h),
                                          quant_element(raw[3], 2 * w + h), s);
        to[h * PITCH] = qfloat_two_of<0>(four, s);
        to[h * PITCH + 1] = qfloat_two_of<1>(four, s);
      }
      continue;
    }
    to[0] = __builtin_amdgcn_perm(raw[1].w[w], raw[0].w[w], 0x05040100);
    to[1] = __builtin_amdgcn_perm(raw[3].w[w], raw[2].w[w], 0x05040100);
    to[PITCH] = __builtin_amdgcn_perm(raw[1].w[w], raw[0].w[w], 0x07060302);
    to[PITCH + 1] = __builtin_amdgcn_perm(raw[3].w[w], raw[2].w[w], 0x07060302);
  }
  if (p.q) {
    float v[4][16];
    QfloatScale s[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
      for (int q = 0; q < 16; ++q) v[r][q] = quant_element(raw[r], q);
      s[r] = qfloat_scale(max_of_eight(qfloat_top(v[r])));
    }
    store_rows(p.q, p.scale, nkb, tile.padded + quad * 4, tc, c, v, s);
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 8; ++u) {                             // column block u / 2, 16 rows 2 wave + (u & 1)
    const int at = (u >> 1) * 32 + (lane & 31), rows = wave * 2 + (u & 1);
    *reinterpret_cast<u32x4_t*>(p.turned + ((int64_t)(tc * 4 + (u >> 1)) * (p.pitch / 32) + (tile.padded >> 4) + rows) * 1024 + lane * 16) =
        *reinterpret_cast<const u32x4_t*>(words + at * PITCH + (at >> 4) * 16 + (rows * 2 + (lane >> 5)) * 4);
  }
}

template <int LPR, int CPT>
void launch_rows(const QfloatRowsArgs& a, hipStream_t s) {
  rows_kernel<LPR, CPT><<<(unsigned)(((int64_t)a.groups.T * LPR + 255) / 256), 256, 0, s>>>(a);
}

}  // namespace

hipError_t stem_qfloat_rows_launch(stem_ctx* ctx, const QfloatRowsArgs& a, hipStream_t s) {
  ProfScope prof(ctx, K_QFLOAT_ROWS, s);
  const int rows = a.groups.T;
  if (a.norm.kind == STEM_NORM_NONE && !a.norm.weight) {
    const int64_t nkb = (a.K + 127) / 128;
    const unsigned grid = (unsigned)((rows + 31) / 32 * ((nkb + BLOCKS - 1) / BLOCKS));
    if (a.h) chunks_kernel<true><<<grid, 256, 0, s>>>(a);
    else chunks_kernel<false><<<grid, 256, 0, s>>>(a);
  } else if (a.K <= 1024 && rows >= 8192) launch_rows<32, 2>(a, s);
  else if (a.K <= 2048) launch_rows<64, 2>(a, s);
  else if (a.K <= 4096) rows >= 2048 ? launch_rows<64, 4>(a, s) : launch_rows<256, 1>(a, s);
  else if (a.K <= 8192) rows >= 1024 ? launch_rows<64, 8>(a, s) : launch_rows<256, 2>(a, s);
  else launch_rows<256, 0>(a, s);
  return hipGetLastError();
}

hipError_t stem_qfloat_weights_launch(stem_ctx* ctx, const QfloatTilesArgs& a, hipStream_t s) {
  ProfScope prof(ctx, K_QFLOAT_WEIGHTS, s);
  const dim3 grid((unsigned)(stem_qfloat_size(a.rows, a.cols) / 16384), a.batch);
  weights_kernel<<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t stem_qfloat_turn_launch(stem_ctx* ctx, const QfloatTurnArgs& a, const QfloatTurnArgs& b, bool rounded, hipStream_t s) {
  ProfScope prof(ctx, K_QFLOAT_TURN, s);
  const int64_t rows = stem_qfloat_rows(a.groups.T, a.groups.n) / 128, first = rows * ((a.cols + 127) / 128), second = rows * ((b.cols + 127) / 128);
  if (rounded) turn_kernel<true><<<(unsigned)(first + second), 256, 0, s>>>(a, b, (int)first);
  else turn_kernel<false><<<(unsigned)(first + second), 256, 0, s>>>(a, b, (int)first);
  return hipGetLastError();
}
