// 8-bit floating point products of few rows: weights straight from memory to registers (qfloat.h has the layout, gemm_qfloat.hip the products of many rows).
//
// Bound by the weights' bytes, and by the launch where they are few.  A workgroup has 16 (or 8) channels and up to 16 NT rows of one group; its 8 wavefronts share K
// by blocks of 128, each of which is one v_mfma_scale_f32_16x16x128_f8f6f4: a lane's 32 bytes are two 16-byte pieces of a form, sixteen lanes' 256 bytes in a row.
// A wavefront requests all of its weights at once.  A block's scale depends on the block alone, so up to 16 rows need no kernel in front: a
// wavefront reads the values of its blocks, behind a norm after the workgroup has the row's sums, and makes the operand in its registers.
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
__device__ __forceinline__ uint32_t over_block(uint32_t v) {   // the largest of the four lanes of a row
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max((uint32_t)a[0], (uint32_t)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max((uint32_t)b[0], (uint32_t)b[1]);
}
__device__ __forceinline__ float over_four(float v) {          // their sum
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// KPW: blocks of 128 a wavefront holds at a time.  CH channels: 8 (half of the products count), 16 or 32
template <int CH, int NT, Source SRC, int KPW, bool GATE>
__global__ __launch_bounds__(WAVES * 64, SRC == FORM && KPW <= 2 ? 4 : 2) void decode_kernel(QfloatDecodeArgs p) {
  static_assert(SRC == FORM || NT == 1, "rows are made to operands 16 at a time");
  constexpr int TM = 16 * NT, CB = CH == 32 ? 2 : 1;
  static_assert(CB * NT <= WAVES, "a wavefront joins the sums of 16 x 16 results");
  __shared__ __attribute__((aligned(16))) f32x4_t part[WAVES][CB * NT][64];
  __shared__ float sums[2][WAVES][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, c = lane >> 4;
  const int ntn = (p.N + CH - 1) / CH, nkb = p.K / 128, tm = blockIdx.x / ntn, n0 = (blockIdx.x - tm * ntn) * CH;
  QfloatTile tile;
  if (!qfloat_tile<TM>(p.groups, tm, lane, tile)) return;
  const int rows = tile.rows < TM ? tile.rows : TM;
  // ---- requests: the rows, the weights, what the result meets
  const int64_t b_bytes = stem_qfloat_pitch(p.N) * p.K;
  const rsrc_t rb = resource(p.B + tile.group * p.stride_b, b_bytes), rs = resource(p.sb + tile.group * p.stride_b, b_bytes / 128);
  const rsrc_t ra = resource(p.A, SRC == FORM ? p.a_bytes : 0), rsa = resource(p.sa, SRC == FORM ? p.a_bytes / 128 : 0);
  // (channels past the last ones of the form are read as zeros)
  const int n = n0 + (CH == 8 ? r & 7 : r);
  const uint32_t at_b = r < CH ? (uint32_t)((n >> 5) * 32 * p.K + (n & 31) * 16 + c * 1024) : OOB;   // (a workgroup's channels are of one block of 32)
  const uint32_t at_s = (uint32_t)(((n >> 7) * nkb * 32 + (n & 31)) * 4);
  const int shift = (n >> 5 & 3) * 8;
  constexpr int HELD = SRC == FORM ? 1 : KPW;
  constexpr int AHEAD = SRC == ROWS && KPW <= 2 ? KPW : 1;   // blocks of a norm's weight that registers have room for
  u32x4_t xq[SRC == ROWS ? HELD : 1][4], gq[AHEAD][4];
  auto norm_weight = [&](int u, int kb) __attribute__((always_inline)) {
    const int k = kb * 128 + c * 32;
#pragma unroll
    for (int h = 0; h < 4; ++h)
      gq[u][h] = k + h * 8 < p.row_K ? *reinterpret_cast<const u32x4_t*>(static_cast<const bf16_t*>(p.norm.weight) + k + h * 8) : u32x4_t{};
  };
  f32x4_t hq[SRC == HIDDEN ? HELD : 1][8];
  const int64_t row = tile.row + (r < rows ? r : 0);
  auto fetch = [&](int u, int kb) __attribute__((always_inline)) {
    const int k = kb * 128 + c * 32;
    if constexpr (SRC == ROWS) {                               // (rows of whole 16 values)
#pragma unroll
      for (int h = 0; h < 4; ++h) xq[u][h] = r < rows && k + h * 8 < p.row_K ? *reinterpret_cast<const u32x4_t*>(p.x + row * p.row_K + k + h * 8) : u32x4_t{};
      if (AHEAD == KPW && p.norm.weight) norm_weight(u, kb);
    } else if constexpr (SRC == HIDDEN) {
#pragma unroll
      for (int h = 0; h < 8; ++h)
        hq[u][h] = r < rows && k + h * 4 < p.row_K ? *reinterpret_cast<const f32x4_t*>(p.h + row * p.row_K + k + h * 4) : f32x4_t{};
    }
  };
  if constexpr (SRC != FORM) {
#pragma unroll
    for (int u = 0; u < KPW; ++u) fetch(u, wave + u * WAVES);
  }
  auto element = [](const u32x4_t (&v)[4], int q) __attribute__((always_inline)) {
    const uint32_t word = v[q >> 3][q >> 1 & 3];
    return __uint_as_float(q & 1 ? word & 0xffff0000u : word << 16);
  };
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
  weights(0);
  // what this lane's results meet: lane l of wavefront CB t + b has row 16 t + l % 16 and channels 16 b + 4 (l / 16) .. + 3
  const int out_row = wave / CB * 16 + r, out_n = n0 + wave % CB * 16 + c * 4, left = p.N - out_n;
  const bool mine = wave < CB * NT && out_row < rows && c * 4 < CH && left > 0;
  const int64_t to = (int64_t)(tile.row + out_row) * p.N + out_n;
  uint16_t meet[4] = {};
  if (mine) {
    const bf16_t* from = nullptr;
    if (GATE) {
      int id = p.ids[tile.row + out_row];
      if ((unsigned)id >= (unsigned)p.E_rows) {   // reported to the host, clamped so no access leaves the table
        *p.flag = 1;
        id = id < 0 ? 0 : p.E_rows - 1;
      }
      from = p.E + (int64_t)id * p.N + out_n;
    } else if (p.residual) {
      from = p.residual + to;
    }
    if (from) {
      if (left >= 4) __builtin_memcpy(meet, from, 8);
      else
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (q < left) meet[q] = from[q];
    }
  }
  // ---- the rows' norm
  float mean = 0.f, scale = 1.f;
  if constexpr (SRC == ROWS) {
    if (p.norm.kind != STEM_NORM_NONE) {
      auto total = [&](int turn, bool squares) __attribute__((always_inline)) {
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < KPW; ++u)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const bool in = (wave + u * WAVES) * 128 + c * 32 + h * 16 < p.row_K;
            float part = 0.f;
#pragma unroll
            for (int q = 0; q < 16; ++q) {
              const float v = element(xq[u], h * 16 + q) - mean;
              part += squares ? v * v : v;
            }
            s += in ? part : 0.f;
          }
        s = over_four(s);
        if (lane < 16) sums[turn][wave][lane] = s;
        __syncthreads();
        s = 0.f;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) s += sums[turn][v][r];
        return s / (float)p.row_K;
      };
      if (p.norm.kind == STEM_NORM_LAYER) mean = total(0, false);
      scale = 1.0f / sqrtf(total(1, true) + p.norm.eps);
    }
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
      if constexpr (SRC == FORM) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const int place = tile.padded + t * 16 + r;
          const uint32_t at = t * 16 < rows ? (uint32_t)((place >> 5) * 32 * p.K + (place & 31) * 16 + c * 1024) : OOB;
          i32x8_t b;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(ra, at + h * 512, kb * 4096, 0);
#pragma unroll
            for (int q = 0; q < 4; ++q) b[4 * h + q] = (int)v[q];
          }
          const uint32_t sx = __builtin_amdgcn_raw_buffer_load_b32(rsa, (uint32_t)(((place >> 7) * nkb * 32 + (place & 31)) * 4), kb * 128, 0);
#pragma unroll
          for (int d = 0; d < CB; ++d)
            acc[t * CB + d] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a[d], b, acc[t * CB + d], 0, 0, 0, s, 0, (int)(sx >> ((place >> 5 & 3) * 8)));
        }
      } else {
        float v[32];
        if constexpr (SRC == ROWS) {
          const bool normed = p.norm.kind != STEM_NORM_NONE, weighted = p.norm.weight != nullptr;
          if (AHEAD < KPW && weighted) norm_weight(0, kb);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const bool in = kb * 128 + c * 32 + h * 16 < p.row_K;
#pragma unroll
            for (int q = h * 16; q < h * 16 + 16; ++q) {
              float x = element(xq[u], q);
              if (normed) x = (x - mean) * scale;
              if (weighted) x *= element(gq[AHEAD < KPW ? 0 : u], q);
              v[q] = in ? x : 0.f;
            }
          }
        } else {
#pragma unroll
          for (int q = 0; q < 32; ++q) v[q] = hq[u][q >> 2][q & 3];
        }
        uint32_t top = 0;
#pragma unroll
        for (int q = 0; q < 32; ++q) top = max(top, qfloat_magnitude(v[q]));
        const QfloatScale sx = qfloat_scale(over_block(top));
        i32x8_t b;
#pragma unroll
        for (int q = 0; q < 8; ++q) b[q] = (int)qfloat_four(v[4 * q] * sx.inv, v[4 * q + 1] * sx.inv, v[4 * q + 2] * sx.inv, v[4 * q + 3] * sx.inv);
#pragma unroll
        for (int d = 0; d < CB; ++d) acc[d] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a[d], b, acc[d], 0, 0, 0, s, 0, (int)sx.byte);
      }
    }
    kb0 += KPW * WAVES;
    if (kb0 >= nkb) break;
    if constexpr (SRC != FORM) {                               // (without a norm: its sums need the whole row at once)
#pragma unroll
      for (int u = 0; u < KPW; ++u) fetch(u, kb0 + wave + u * WAVES);
    }
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
void by_depth(const QfloatDecodeArgs& a, int64_t tiles, hipStream_t s) {
  const unsigned grid = (unsigned)(tiles * ((a.N + CH - 1) / CH));
  const int per = (a.K / 128 + WAVES - 1) / WAVES;
  if (per <= 1) decode_kernel<CH, NT, SRC, 1, GATE><<<grid, WAVES * 64, 0, s>>>(a);
  else if (per <= 2) decode_kernel<CH, NT, SRC, 2, GATE><<<grid, WAVES * 64, 0, s>>>(a);
  else if constexpr (SRC == FORM) {
    if (per <= 4) decode_kernel<CH, NT, SRC, 4, GATE><<<grid, WAVES * 64, 0, s>>>(a);
    else decode_kernel<CH, NT, SRC, 8, GATE><<<grid, WAVES * 64, 0, s>>>(a);
  } else if constexpr (CH < 32) {   // (values held as they are need registers)
    decode_kernel<CH, NT, SRC, 4, GATE><<<grid, WAVES * 64, 0, s>>>(a);
  }
}

template <int NT, Source SRC, bool GATE>
void by_channels(const QfloatDecodeArgs& a, int64_t tiles, hipStream_t s) {
  // about as many workgroups as compute units
  const int64_t wgs = tiles * ((a.N + 15) / 16);
  const bool room = SRC == FORM || a.K <= 256 * WAVES;   // for the weights of 32 channels beside values held as they are
  if (wgs <= 128) by_depth<8, NT, SRC, GATE>(a, tiles, s);
  else if (wgs <= 256 || !room) by_depth<16, NT, SRC, GATE>(a, tiles, s);
  else by_depth<32, NT, SRC, GATE>(a, tiles, s);
}

}  // namespace

// A norm's sums need the row in registers: 4 blocks a wavefront
bool stem_qfloat_decode_inline(int64_t rows, int64_t K, bool normed) { return rows <= 16 && K % 16 == 0 && (!normed || K <= 4096); }

hipError_t stem_qfloat_decode_launch(stem_ctx* ctx, int kid, const QfloatDecodeArgs& a, hipStream_t s) {
  ProfScope prof(ctx, kid, s);
  const int nt = a.x || a.h ? 1 : a.nt;
  const int64_t tiles = (a.groups.T + 16 * nt - 1) / (16 * nt) + (a.groups.offsets ? (a.groups.n < a.groups.T ? a.groups.n : a.groups.T) - 1 : 0);
  if (a.h_out) {
    if (a.x) by_channels<1, ROWS, true>(a, tiles, s);
    else if (nt == 1) by_channels<1, FORM, true>(a, tiles, s);
    else if (nt == 2) by_channels<2, FORM, true>(a, tiles, s);
    else by_channels<4, FORM, true>(a, tiles, s);
  } else {
    if (a.x) by_channels<1, ROWS, false>(a, tiles, s);
    else if (a.h) by_channels<1, HIDDEN, false>(a, tiles, s);
    else if (nt == 1) by_channels<1, FORM, false>(a, tiles, s);
    else if (nt == 2) by_channels<2, FORM, false>(a, tiles, s);
    else by_channels<4, FORM, false>(a, tiles, s);
  }
  return hipGetLastError();
}
