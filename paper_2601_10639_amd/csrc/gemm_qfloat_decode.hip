// 8-bit floating point products of few rows: weights straight from memory to registers (qfloat.h has the layout, gemm_qfloat.hip the products of many rows).
//
// Bound by the weights' bytes, and by the launch where they are few.  A workgroup has 8, 16 or 32 channels and up to 16 NT rows of one group; its 8 wavefronts share K
// by blocks of 128, each of which is one v_mfma_scale_f32_16x16x128_f8f6f4: a lane's 32 bytes are two 16-byte pieces of a form, sixteen lanes' 256 bytes in a row.
// A wavefront requests all of its weights at once.  A block's scale depends on the block alone, so up to 16 rows need no kernel in front: while the
// weights are under way the workgroup makes the rows' 8-bit values in LDS, a wavefront a row behind a norm, otherwise a lane 16 values.
#include "qfloat.h"
#include "quant.h"

typedef __attribute__((ext_vector_type(8))) int i32x8_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __amdgpu_buffer_rsrc_t rsrc_t;

namespace {

constexpr uint32_t OOB = 0x80000000u;
constexpr int WAVES = 8;
enum Source { FORM, ROWS, HIDDEN };   // of the rows: a form, bf16 rows (behind a norm), fp32 hidden values

__device__ __forceinline__ float sigmoidf_fast(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
__device__ __forceinline__ rsrc_t resource(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t max_of_eight(uint32_t v) {   // neighbouring lanes
  v = max(v, dpp<0xb1>(v));    // quad_perm 1 0 3 2
  v = max(v, dpp<0x4e>(v));    // quad_perm 2 3 0 1
  return max(v, dpp<0x141>(v));   // row_half_mirror
}

// KPW: blocks of 128 whose weights a wavefront holds at a time.  CH channels: 8 (half of the products count), 16 or 32
template <int CH, int NT, Source SRC, int KPW, bool GATE>
__global__ __launch_bounds__(WAVES * 64, SRC == FORM && KPW <= 2 ? 4 : 2) void decode_kernel(QfloatDecodeArgs p) {
  static_assert(SRC == FORM || NT == 1, "rows are made to operands 16 at a time");
  constexpr int TM = 16 * NT, CB = CH == 32 ? 2 : 1;
  static_assert(CB * NT <= WAVES, "a wavefront joins the sums of 16 x 16 results");
  __shared__ __attribute__((aligned(16))) f32x4_t part[WAVES][CB * NT][64];
  __shared__ float sums[WAVES];
  extern __shared__ __attribute__((aligned(16))) uint8_t held[];   // [16][K + 16] values, then [16][blocks] scales
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, c = lane >> 4;
  const int ntn = (p.N + CH - 1) / CH, nkb = p.K / 128, tm = blockIdx.x / ntn, n0 = (blockIdx.x - tm * ntn) * CH;
  QfloatTile tile;
  if (!qfloat_tile<TM>(p.groups, tm, lane, tile)) return;
  const int rows = tile.rows < TM ? tile.rows : TM;
  // ---- requests: the weights, what the result meets
  const int64_t b_bytes = stem_qfloat_pitch(p.N) * p.K;
  const rsrc_t rb = resource(p.B + tile.group * p.stride_b, b_bytes), rs = resource(p.sb + tile.group * p.stride_b, b_bytes / 128);
  const rsrc_t ra = resource(p.A, SRC == FORM ? p.a_bytes : 0), rsa = resource(p.sa, SRC == FORM ? p.a_bytes / 128 : 0);
  // (channels past the last ones of the form are read as zeros)
  const int n = n0 + (CH == 8 ? r & 7 : r);
  const uint32_t at_b = r < CH ? (uint32_t)((n >> 5) * 32 * p.K + (n & 31) * 16 + c * 1024) : OOB;   // (a workgroup's channels are of one block of 32)
  const uint32_t at_s = (uint32_t)(((n >> 7) * nkb * 32 + (n & 31)) * 4);
  const int shift = (n >> 5 & 3) * 8;
  u32x4_t w[KPW][CB][2];
  uint32_t sw[KPW];
  auto weights = [&](int kb0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < KPW; ++u) {
      const int kb = kb0 + wave + u * WAVES;
#pragma unroll
      for (int h = 0; h < 2 * CB; ++h) w[u][h >> 1][h & 1] = __builtin_amdgcn_raw_buffer_load_b128(rb, kb < nkb ? at_b + (h & 1) * 512 + (h >> 1) * 256 : OOB, kb * 4096, 0);
      sw[u] = __builtin_amdgcn_raw_buffer_load_b32(rs, kb < nkb ? at_s : OOB, kb * 128, 0);
    }
  };
  // lane l of wavefront CB t + b has row 16 t + l % 16 and channels 16 b + 4 (l / 16) .. + 3 of the result
  const int out_row = wave / CB * 16 + r, out_n = n0 + wave % CB * 16 + c * 4, left = p.N - out_n;
  const bool mine = wave < CB * NT && out_row < rows && c * 4 < CH && left > 0;
  const int64_t to = (int64_t)(tile.row + out_row) * p.N + out_n;
  uint16_t meet[4] = {};
  int id = 0;
  if (GATE && mine) id = p.ids[tile.row + out_row];            // (first of all: what waits for a load waits for those in front of it)
  auto meeting = [&]() __attribute__((always_inline)) {
    if (!mine) return;
    const bf16_t* from = nullptr;
    if (GATE) {
      if ((unsigned)id >= (unsigned)p.E_rows) {   // reported to the host, clamped so no access leaves the table
        *p.flag = 1;
        id = id < 0 ? 0 : p.E_rows - 1;
      }
      from = p.E + (int64_t)id * p.N + out_n;
    } else if (p.residual) {
      from = p.residual + to;
    }
    if (!from) return;
    if (left >= 4) __builtin_memcpy(meet, from, 8);
    else
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < left) meet[q] = from[q];
  };
  // ---- the rows' 8-bit values, where they are not there yet
  const int pitch = p.K + 16;
  uint8_t* const scales = held + 16 * pitch;
  if constexpr (SRC != FORM) {
    // 16 values of a row, eight neighbouring lanes a block; zeros behind the row's end (quant_load_chunk's branch is the shorter code: with qfloat_fetch the layer of
    // 2048 x 8192 takes 13.5 us on one token, so 12.7)
    float v[16];
    QuantChunk raw;
    f32x4_t hid[4];
    auto request = [&](int row, int chunk) __attribute__((always_inline)) {
      const int k = chunk * 16;
      const int64_t at = (int64_t)(tile.row + row) * p.row_K + k;
      if constexpr (SRC == ROWS) {
        raw = k < p.row_K ? quant_load_chunk(p.x + at, p.row_K - k) : QuantChunk{};
      } else {
#pragma unroll
        for (int h = 0; h < 4; ++h) hid[h] = k < p.row_K ? *reinterpret_cast<const f32x4_t*>(p.h + at + h * 4) : f32x4_t{};   // (d_ff is a multiple of 64)
      }
    };
    auto unpack = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < 16; ++q) v[q] = SRC == ROWS ? quant_element(raw, q) : hid[q >> 2][q & 3];
    };
    auto keep = [&](int row, int chunk) __attribute__((always_inline)) {
      const QfloatScale s = qfloat_scale(max_of_eight(qfloat_top(v)));
      u32x4_t o;
#pragma unroll
      for (int q = 0; q < 4; ++q) o[q] = qfloat_four(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3], s);
      if (chunk >= nkb * 8) return;
      *reinterpret_cast<u32x4_t*>(held + row * pitch + chunk * 16) = o;
      if ((lane & 7) == 0) scales[row * nkb + (chunk >> 3)] = (uint8_t)s.byte;
    };
    const bool normed = SRC == ROWS && (p.norm.kind != STEM_NORM_NONE || p.norm.weight);
    if (normed) {
      // 8, 4, 2 wavefronts a row or one.  In loops: values that are read again from the nearest cache cost less than the instructions that would hold them, whose
      // first fetch is what short kernels wait for (one row of K 2048 with all chunks held and unrolled: 10.2 us against 9.5).
      const int share = p.share, turns = (rows * share + WAVES - 1) / WAVES, first = wave % share * 64 + lane;
      const bool once = turns == 1 && p.K <= 1024 * share;     // a lane has one chunk: it is loaded in front of the weights, and once (2048 -> 8192, one row of
                                                               // rms norm 5.5 us, so 5.0; the layer of 1536 x 5120 11.5 and 10.8)
      QuantChunk weight = {};
      if (once) {
        request(wave / share < rows ? wave / share : 0, first);
        if (p.norm.weight && first * 16 < p.row_K) weight = quant_load_chunk(static_cast<const bf16_t*>(p.norm.weight) + first * 16, p.row_K - first * 16);
        weights(0);
      }
      for (int turn = 0; turn < turns; ++turn) {
        const int at = turn * (WAVES / share) + wave / share, row = at < rows ? at : 0;
        float mean = 0.f, scale = 1.f;
        auto total = [&](bool squares) __attribute__((always_inline)) {
          float s = 0.f;
          for (int chunk = first; chunk * 16 < p.row_K; chunk += 64 * share) {
            if (!once) request(row, chunk);
            unpack();
            const int in = p.row_K - chunk * 16;
#pragma unroll
            for (int q = 0; q < 16; ++q) {
              const float d = q < in ? v[q] - mean : 0.f;
              s = squares ? __builtin_fmaf(d, d, s) : s + d;
            }
          }
#pragma unroll
          for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d);
          if (share > 1) {
            __syncthreads();
            if (lane == 0) sums[wave] = s;
            __syncthreads();
            s = 0.f;
            for (int u = 0; u < share; ++u) s += sums[wave / share * share + u];
          }
          return s / (float)p.row_K;
        };
        if (p.norm.kind == STEM_NORM_LAYER) mean = total(false);
        if (p.norm.kind != STEM_NORM_NONE) scale = 1.0f / sqrtf(total(true) + p.norm.eps);
        if (turn == 0) {                                       // (behind the rows, which are waited for first)
          if (!once) weights(0);
          meeting();
        }
        for (int chunk = first; chunk - lane < nkb * 8; chunk += 64 * share) {
          if (!once) request(row, chunk);
          unpack();
          const int in = p.row_K - chunk * 16;
          if (!once && p.norm.weight && in > 0) weight = quant_load_chunk(static_cast<const bf16_t*>(p.norm.weight) + chunk * 16, in);
#pragma unroll
          for (int q = 0; q < 16; ++q) {
            float x = v[q];
            if (p.norm.kind == STEM_NORM_LAYER) x -= mean;
            x *= scale;
            if (p.norm.weight) x *= quant_element(weight, q);
            v[q] = q < in ? x : 0.f;
          }
          keep(row, at < rows ? chunk : nkb * 8);
        }
      }
    } else {
      weights(0);
      meeting();
      const int per = nkb * 8, all = rows * per;
      for (int i = threadIdx.x; i - (int)threadIdx.x < all; i += WAVES * 64) {
        const int row = min(i / per, rows - 1), chunk = i - row * per;   // (beyond the last row: chunks of it that are not kept)
        request(row, chunk);
        unpack();
        keep(row, chunk);
      }
    }
    __syncthreads();
  } else {
    weights(0);
    meeting();
  }
  // ---- products
  f32x4_t acc[CB * NT];
#pragma unroll
  for (int t = 0; t < CB * NT; ++t) acc[t] = f32x4_t{};
  for (int kb0 = 0;;) {
#pragma unroll
    for (int u = 0; u < KPW; ++u) {
      const int kb = kb0 + wave + u * WAVES;
      if (kb >= nkb) break;                                    // (the same for all lanes)
      i32x8_t a[CB];
#pragma unroll
      for (int q = 0; q < 8 * CB; ++q) a[q >> 3][q & 7] = (int)w[u][q >> 3][q >> 2 & 1][q & 3];
      const int s = (int)(sw[u] >> shift);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        i32x8_t b;
        int sx;
        if constexpr (SRC == FORM) {
          const int place = tile.padded + t * 16 + r;
          const uint32_t at = t * 16 < rows ? (uint32_t)((place >> 5) * 32 * p.K + (place & 31) * 16 + c * 1024) : OOB;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(ra, at + h * 512, kb * 4096, 0);
#pragma unroll
            for (int q = 0; q < 4; ++q) b[4 * h + q] = (int)v[q];
          }
          sx = (int)(__builtin_amdgcn_raw_buffer_load_b32(rsa, (uint32_t)(((place >> 7) * nkb * 32 + (place & 31)) * 4), kb * 128, 0) >> ((place >> 5 & 3) * 8));
        } else {                                               // (rows that are not there: whatever LDS holds, in columns that are not used)
          const uint8_t* const at = held + r * pitch + kb * 128 + c * 32;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const u32x4_t v = *reinterpret_cast<const u32x4_t*>(at + h * 16);
#pragma unroll
            for (int q = 0; q < 4; ++q) b[4 * h + q] = (int)v[q];
          }
          sx = scales[r * nkb + kb];
        }
#pragma unroll
        for (int d = 0; d < CB; ++d) acc[t * CB + d] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a[d], b, acc[t * CB + d], 0, 0, 0, s, 0, sx);
      }
    }
    kb0 += KPW * WAVES;
    if (kb0 >= nkb) break;
    weights(kb0);
  }
  // ---- the wavefronts' sums, in their order
#pragma unroll
  for (int t = 0; t < CB * NT; ++t) part[wave][t][lane] = acc[t];
  __syncthreads();
  if (!mine) return;
  f32x4_t z = {};
#pragma unroll
  for (int v = 0; v < WAVES; ++v) z += part[v][wave][lane];
  float o[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float m = __uint_as_float((uint32_t)meet[q] << 16);
    o[q] = GATE ? z[q] * sigmoidf_fast(z[q]) * m : z[q] + m;
  }
  if (GATE) {
    __builtin_memcpy(p.h_out + to, o, 16);                     // (d_ff is a multiple of 64)
  } else if (left >= 4) {
    uint16_t y[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] = __builtin_bit_cast(uint16_t, (__bf16)o[q]);
    __builtin_memcpy(p.y + to, y, 8);
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (q < left) p.y[to + q] = __builtin_bit_cast(uint16_t, (__bf16)o[q]);
  }
}

template <int CH, int NT, Source SRC, bool GATE>
void by_depth(const QfloatDecodeArgs& a, int depth, unsigned grid, hipStream_t s) {
  const size_t lds = SRC == FORM ? 0 : 16 * (size_t)(a.K + 16 + a.K / 128);
  if (depth == 1) decode_kernel<CH, NT, SRC, 1, GATE><<<grid, WAVES * 64, lds, s>>>(a);
  else if (depth == 2) decode_kernel<CH, NT, SRC, 2, GATE><<<grid, WAVES * 64, lds, s>>>(a);
  else if (depth == 4) decode_kernel<CH, NT, SRC, 4, GATE><<<grid, WAVES * 64, lds, s>>>(a);
  else decode_kernel<CH, NT, SRC, 8, GATE><<<grid, WAVES * 64, lds, s>>>(a);
}

template <int NT, Source SRC, bool GATE>
void by_channels(const QfloatDecodeArgs& a, const int32_t* route, hipStream_t s) {
  const int64_t n = a.groups.n < a.groups.T ? a.groups.n : a.groups.T, tiles = (a.groups.T + 16 * NT - 1) / (16 * NT) + (a.groups.offsets ? n - 1 : 0);
  const unsigned grid = (unsigned)(tiles * ((a.N + route[0] - 1) / route[0]));
  if constexpr (NT == 1) {
    if (route[0] == 8) return by_depth<8, NT, SRC, GATE>(a, route[2], grid, s);
    if (route[0] == 16) return by_depth<16, NT, SRC, GATE>(a, route[2], grid, s);
  }
  by_depth<32, NT, SRC, GATE>(a, route[2], grid, s);
}

}  // namespace

// Few rows are 16 rows, or those whose product takes as long as its launch: us, here / on tiles: 64 rows of 2048 x 8192 10.8 / 13.3, 96 13.0 / 13.4, 256 22 / 15.5; 64 of
// N 8192, K 2048 8.2 / 9.9, 96 11.9 / 10.1; 256 of N 1024, K 4096 8.6 / 12; 128 of 4096 x 1024 6.7 / 8.3.  By groups every one has tiles of its own, most of them nearly
// empty here too: 4 rows of 16 groups of 4096 x 1024 6.9 / 11.2, 16 rows 17.6 / 14.9, 64 17.5 / 16.8; 128 rows of 8 groups of 2048 x 8192 37 / 26.
extern "C" int stem_route_qfloat_few(int64_t T, int grouped, int N, int K) {
  if (grouped) return T <= 8;
  return T <= 16 || (T <= 256 && T * N * K <= (int64_t)1 << 30);
}

// {channels and 16-row tiles of a workgroup, blocks of K that a wavefront has under way}.  About as many workgroups as compute units, if need be of 8 channels, half of whose
// products count; of 32 rows, and then 32 channels, where there are more workgroups than that helps (us, 16 / 32 rows: 64 of N 8192, K 2048 9.9 / 8.2, 256 of 1024 x 4096 9.5 / 8.6, 64 of
// 1024 x 4096 6.4 / 8.0).
extern "C" void stem_route_qfloat_decode(int64_t T, int groups, int N, int K, int form, int32_t* route) {
  const int64_t n16 = (N + 15) / 16;
  route[1] = form && (T + 15) / 16 * n16 >= 1024 ? 2 : 1;
  const int64_t tiles = (T + 16 * route[1] - 1) / (16 * route[1]) + (groups < T ? groups : T) - 1, wgs = tiles * n16;
  route[0] = route[1] == 2 ? 32 : wgs <= 128 ? 8 : wgs <= 256 ? 16 : 32;   // (two tiles of rows: 512 workgroups of 16 channels at least)
  const int per = ((K + 127) / 128 + WAVES - 1) / WAVES;
  route[2] = per <= 1 ? 1 : per <= 2 ? 2 : per <= 4 ? 4 : 8;
}

// LDS has room for 16 rows' values
bool stem_qfloat_decode_inline(int64_t rows, int64_t K) { return rows <= 16 && K <= 8192; }

hipError_t stem_qfloat_decode_launch(stem_ctx* ctx, int kid, const QfloatDecodeArgs& p, hipStream_t s) {
  ProfScope prof(ctx, kid, s);
  QfloatDecodeArgs a = p;
  a.share = a.groups.T > 4 ? 1 : a.groups.T > 2 ? 2 : a.groups.T > 1 ? 4 : 8;
  int32_t route[3];
  stem_route_qfloat_decode(a.groups.T, a.groups.offsets ? a.groups.n : 1, a.N, a.K, !a.x && !a.h, route);
  if (a.h_out) by_channels<1, ROWS, true>(a, route, s);        // (a gate product)
  else if (a.x) by_channels<1, ROWS, false>(a, route, s);
  else if (a.h) by_channels<1, HIDDEN, false>(a, route, s);
  else if (route[1] == 1) by_channels<1, FORM, false>(a, route, s);
  else by_channels<2, FORM, false>(a, route, s);
  return hipGetLastError();
}
