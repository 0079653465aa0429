// 8-bit floating point MFMA products for gfx950: C[m,n] = sum_k a_mk b_nk of two forms (qfloat.h), the scales of their blocks of 128 multiplied in by
// the matrix instruction.
//
// A weight gradient's products are of bf16 values (qfloat.h says why), in blocks of the same bytes, and go through the same loops with the bf16 instruction.
//
// A form's blocks lie in memory as the instruction takes them, so a tile of an operand is 4 KB for each 32 rows and 128 k, in a row; it goes to LDS as it
// is (buffer_load ... lds), a fragment is the 32 bytes of two blocks at 16 x lane: no swizzle, no bank conflict.  The scales of a K tile are a word a
// lane for each 128 rows of an operand, which goes straight to a register some K tiles ahead.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "qfloat.h"

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) int i32x4_t;
typedef __attribute__((ext_vector_type(8))) int i32x8_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef __amdgpu_buffer_rsrc_t rsrc_t;

namespace {

constexpr uint32_t OOB = 0x80000000u;   // a buffer offset beyond any operand: reads as zero, is not stored
constexpr int SC1 = 16;                 // cache policy bit of the buffer instructions: device scope
constexpr int MAX_SLICES = 4, MAX_WEIGHT_SLICES = 8;

__device__ __forceinline__ float sigmoidf_fast(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
__device__ __forceinline__ void lds_dma_16(rsrc_t rs, char* lds_dst, uint32_t off, int soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr_t)lds_dst, 16, off, soff, 0, 0);
}
__device__ __forceinline__ rsrc_t resource(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}
// 16 bytes to a buffer, all of the address in the vector offset (with a scalar register as the other one the compiler has let the next vector
// instruction write the data's registers)
template <int POLICY = 0>
__device__ __forceinline__ void store_16(u32x4_t v, rsrc_t r, uint32_t off) {
  __builtin_amdgcn_raw_buffer_store_b128(v, r, off, 0, POLICY);
}
__device__ __forceinline__ void in_order() {   // of LDS, within the wavefront
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
__device__ __forceinline__ i32x8_t join(i32x4_t lo, i32x4_t hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }
__device__ __forceinline__ f32x16_t mma_bf16(i32x8_t a, i32x8_t b, f32x16_t c) {   // 32 k
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a, a, 0, 1, 2, 3)),
                                              __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(b, b, 0, 1, 2, 3)), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a, a, 4, 5, 6, 7)),
                                                 __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(b, b, 4, 5, 6, 7)), c, 0, 0, 0);
}
// 32 channels (a) x 32 tokens (b) x 64 k; the scales are byte A and byte B of their words
template <int A, int B>
__device__ __forceinline__ f32x16_t mma(i32x8_t a, i32x8_t b, f32x16_t c, uint32_t sa, uint32_t sb) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, A, (int)sa, B, (int)sb);
}

template <class F, int... U>
__device__ __forceinline__ void each(F f, std::integer_sequence<int, U...>) { (f(std::integral_constant<int, U>{}), ...); }

// Workgroup -> tile: the workgroups of an XCD take a contiguous run of tiles, walked in bands of 4 row tiles.
__device__ __forceinline__ void tile_of(int b, int nb, int ntm, int ntn, int& tm, int& tn) {
  const int q = nb >> 3, r = nb & 7, xcd = b & 7;
  const int L = xcd * q + (xcd < r ? xcd : r) + (b >> 3);
  const int per = 4 * ntn, group = L / per, first = group * 4, rows = ntm - first < 4 ? ntm - first : 4, in = L - group * per;
  tm = first + in % rows;
  tn = in / rows;
}

// What a workgroup computes
struct Work {
  int m0, rows;        // first row of the output, and how many there are from it on (in the group)
  int pa;              // the same in the form of A
  int n0;
  int k0, nk;          // K tiles
  int group;
  int tile, tiles, slice;   // of all outputs, of K slices
};
template <int TM, int TN, bool BY_K>
__device__ __forceinline__ bool find_work(const QfloatGemmArgs& p, int lane, Work& w) {
  const int ntn = (p.N + TN - 1) / TN, nk_all = p.K / 128;
  const bool grouped = p.groups.offsets != nullptr;
  int tm = 0, tn = 0, tiles = 0, part = 0, k0 = 0, nk = nk_all;   // part: of K, a group or a slice
  QfloatTile t;
  if (!BY_K && grouped) {
    if (!qfloat_tile_of<TM>(p.groups, lane, t, [&](int ntm) __attribute__((always_inline)) {
          tiles = ntm * ntn;
          if ((int)blockIdx.x >= tiles) return -1;
          tile_of(blockIdx.x, tiles, ntm, ntn, tm, tn);
          return tm;
        }))
      return false;
  } else {
    const int ntm = (p.M + TM - 1) / TM;
    tiles = ntm * ntn;
    part = blockIdx.x / tiles;
    tile_of(blockIdx.x - part * tiles, tiles, ntm, ntn, tm, tn);
    t = {0, tm * TM, p.M - tm * TM, tm * TM};
    if (BY_K && grouped) {                                   // all of the output for each group of K
      t.group = part / p.ksplit;
      part -= t.group * p.ksplit;
      qfloat_group(p.groups, t.group, lane, k0, nk);
      k0 /= 64;                                              // (bf16: 64 rows a K tile)
      nk = (nk + 63) / 64;
    }
    if (p.ksplit > 1) {                                      // (a group's may be without any)
      const int per = (nk + p.ksplit - 1) / p.ksplit;
      k0 += part * per;
      nk = min(max(nk - part * per, 0), per);
    }
  }
  w = {t.row, t.rows, t.padded, tn * TN, k0, nk, t.group, BY_K ? (t.group * tiles) + tm * ntn + tn : tm * ntn + tn, BY_K && grouped ? tiles * p.groups.n : tiles, part};
  return true;
}

// The operand tiles of a workgroup: EDGE rows x 128 k, LOADS loads of 1 KB for each of LOADERS wavefronts
template <int EDGE, int LOADERS>
struct Loader {
  static constexpr int LOADS = EDGE * 128 / 1024 / LOADERS;
  rsrc_t r;
  uint32_t off[(LOADS + 3) / 4];   // of the 32-row groups this wavefront loads from
  // rows from row0 on, `rows` of them
  __device__ __forceinline__ void init(const uint8_t* p, int64_t bytes, int rows, int K, int row0, int wave, int lane) {
    r = resource(p, bytes);
#pragma unroll
    for (int i = 0; i < (LOADS + 3) / 4; ++i) {
      const int group = (wave * LOADS + i * 4) / 4;
      off[i] = group * 32 < rows ? (uint32_t)((row0 + group * 32) * K + lane * 16) : OOB;
    }
  }
  // load i of the K tile at byte `k` of a group
  __device__ __forceinline__ void issue(int i, char* tile, int wave, int k) const {
    const int piece = wave * LOADS + i;
    lds_dma_16(r, tile + piece * 1024, off[LOADS < 4 ? 0 : i / 4], k + (piece & 3) * 1024);
  }
};

// The scale words of ROWS rows from `row` on (within 128), one K tile after another; byte 0 is the first 32 rows'
struct Scales {
  rsrc_t r;
  uint32_t off;
  int shift;
  __device__ __forceinline__ void init(const uint8_t* p, int64_t bytes, int row, int nkb, int lane) {
    r = resource(p, bytes);
    off = (uint32_t)(((row >> 7) * nkb * 32 + (lane & 31)) * 4);
    shift = (row >> 5 & 3) * 8;
  }
  __device__ __forceinline__ uint32_t load(int kt) const { return __builtin_amdgcn_raw_buffer_load_b32(r, off, kt * 128, 0); }
};

// ---- epilogue: a wavefront's 32 MI x 32 NJ results, 32 rows at a time through LDS ------------------------------------------------------
// acc[i][j]: row block i, column block j; a lane holds row lane & 31 and columns 8 g + 4 (lane >> 5) + 0..3 of each.
template <int MI, int NJ, bool F32>
struct Output {
  static constexpr int COLS = 32 * NJ, PITCH = COLS + 4;       // of a staged row, in words
  static constexpr int BYTES = 32 * PITCH * 4;                 // of LDS, for each wavefront
  static constexpr int V = F32 ? 4 : 8, LPR = COLS / V, RPP = 64 / LPR, PASSES = 32 / RPP;

  // What a block of 32 rows is added to, requested before the block in front of it is stored: a load behind a store that may lie over it waits for it.
  struct Before {
    u32x4_t pass[PASSES], edge;
  };
  // 16 bytes of results z and of what they are added to
  static __device__ __forceinline__ u32x4_t sum(const float (&z)[V], u32x4_t v) {
    if constexpr (F32) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = __float_as_uint(z[q] + __uint_as_float(v[q]));
      return v;
    } else {
      bf16x8_t o;
#pragma unroll
      for (int q = 0; q < 8; ++q) o[q] = (__bf16)(z[q] + __uint_as_float(q & 1 ? v[q >> 1] & 0xffff0000u : v[q >> 1] << 16));
      return __builtin_bit_cast(u32x4_t, o);
    }
  }

  // rows from m0 on, how many there are of them, columns from n0 on
  static __device__ __forceinline__ void run(const QfloatGemmArgs& p, const f32x16_t (&acc)[MI][NJ], char* stg, int64_t m0, int n0, int rows, int64_t base, int lane) {
    typedef typename std::conditional<F32, float, bf16_t>::type E;
    const int lim = p.N - n0 < COLS ? p.N - n0 : COLS;
    if (rows <= 0 || lim <= 0) return;
    float* const st = reinterpret_cast<float*>(stg);
    const int srow = lane / LPR, scol = (lane % LPR) * V;
    const bool adds = F32 ? p.accumulate != 0 : p.residual != nullptr;
    // columns behind the last whole V: rows take one lane each, for the row's last V (some of them again), or one by one where there are fewer
    const bool edge = lim % V != 0;
    E* const out = (F32 ? reinterpret_cast<E*>(p.c) : reinterpret_cast<E*>(p.y)) + base + m0 * p.N + n0;
    const E* const in = (F32 ? reinterpret_cast<const E*>(p.c) : reinterpret_cast<const E*>(p.residual)) + base + m0 * p.N + n0;
    auto fetch = [&](int i, Before& b) __attribute__((always_inline)) {
      if (!adds || lim < V) return;
#pragma unroll
      for (int pass = 0; pass < PASSES; ++pass)
        __builtin_memcpy(&b.pass[pass], in + (int64_t)min(i * 32 + pass * RPP + srow, rows - 1) * p.N + min(scol, lim - V), 16);
      if (edge) __builtin_memcpy(&b.edge, in + (int64_t)min(i * 32 + (lane & 31), rows - 1) * p.N + lim - V, 16);
    };
    Before before[2] = {};
    fetch(0, before[0]);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      if (i * 32 >= rows) return;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4_t w = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
          *reinterpret_cast<f32x4_t*>(st + (lane & 31) * PITCH + j * 32 + g * 8 + (lane >> 5) * 4) = w;
        }
      in_order();
      if (i + 1 < MI) fetch(i + 1, before[(i + 1) & 1]);
      const Before& b = before[i & 1];
#pragma unroll
      for (int pass = 0; pass < PASSES; ++pass) {
        const int r = i * 32 + pass * RPP + srow;
        float z[V];
        __builtin_memcpy(z, st + (pass * RPP + srow) * PITCH + scol, sizeof z);
        const u32x4_t v = sum(z, b.pass[pass]);
        if (r < rows && scol + V <= lim) __builtin_memcpy(out + (int64_t)r * p.N + scol, &v, 16);
      }
      if (edge) {
        const int r = i * 32 + (lane & 31);
        const float* const from = st + (lane & 31) * PITCH;
        if (lim >= V) {
          float z[V];
#pragma unroll
          for (int q = 0; q < V; ++q) z[q] = from[lim - V + q];
          const u32x4_t v = sum(z, b.edge);
          if (lane < 32 && r < rows) __builtin_memcpy(out + (int64_t)r * p.N + lim - V, &v, 16);
        } else if (lane < 32 && r < rows) {
          for (int q = 0; q < lim; ++q) {
            const int64_t to = (int64_t)r * p.N + q;
            if constexpr (F32) out[to] = adds ? in[to] + from[q] : from[q];
            else out[to] = __builtin_bit_cast(uint16_t, (__bf16)(from[q] + (adds ? __uint_as_float((uint32_t)in[to] << 16) : 0.f)));
          }
        }
      }
      in_order();   // all have read the rows before they are staged over
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// ---- epilogue of the gate product: the form of SiLU(z) * E[ids] ----------------------------------------------------------------------------
// A wavefront has 128 channels, a block of each of its tokens: the magnitude is over a lane's registers and one other lane's, and the
// values go to the next product's operand from here; nothing is rounded before they are.  The table rows are what moves: they go to LDS as they
// are gathered, 16 bytes a lane, chunk c of row r at chunk c ^ r % 16 so that 16 rows' reads fall into 16 chunk columns.
template <int MI>
struct Hidden {
  static constexpr int NJ = 4, CH = 16;
  static constexpr int BYTES = 32 * MI * CH * 16;              // of LDS, for each wavefront
  static __device__ __forceinline__ void run(const QfloatGemmArgs& p, f32x16_t (&acc)[MI][NJ], const int (&row_id)[(MI + 1) / 2], char* lds, int pa, int n0,
                                             int rows, int lane) {
    if (rows <= 0 || n0 >= p.N) return;
#pragma unroll
    for (int q = 0; q < MI * CH / 2; ++q) {
      const int r = q * 4 + lane / CH, col = n0 + ((lane % CH) ^ (r & 15)) * 8;
      const int id = __builtin_amdgcn_ds_bpermute((r & 63) * 4, row_id[(q * 4) >> 6]);
      const bf16_t* const at = p.E + (size_t)id * p.N + (col < p.N ? col : 0);
      __builtin_amdgcn_global_load_lds(const_cast<bf16_t*>(at), (lds_ptr_t)(lds + q * 1024), 16, 0, 0);
    }
    const int pitch = (p.N + 127) / 128 * 128, nkb = pitch / 128;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int m = i * 32 + (lane & 31);
      uint32_t top = 0;
#pragma unroll
      for (int t = 0; t < 4 * NJ; ++t) {                       // 8 channels a step
        const int j = t >> 2, g = t & 3;
        const u32x2_t e = *reinterpret_cast<const u32x2_t*>(lds + m * (CH * 16) + ((t ^ (m & 15)) << 4) + (lane >> 5) * 8);
        const float u[4] = {__uint_as_float(e[0] << 16), __uint_as_float(e[0] & 0xffff0000u), __uint_as_float(e[1] << 16), __uint_as_float(e[1] & 0xffff0000u)};
        const bool inside = n0 + 32 * j < p.N;                 // d_ff is a multiple of 64; what is behind it counts as zero
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float z = acc[i][j][4 * g + q], h = inside ? z * sigmoidf_fast(z) * u[q] : 0.f;
          acc[i][j][4 * g + q] = h;
          top = max(top, __float_as_uint(h) & 0x7fffffffu);
        }
        __builtin_amdgcn_sched_barrier(0);                     // (all steps' reads at once would not fit the registers)
      }
      if (__ballot(top >= 0x7f800000u)) {                      // (seldom: numbers alone count)
        top = 0;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int q = 0; q < 16; ++q) top = max(top, qfloat_magnitude(acc[i][j][q]));
      }
      const auto both = __builtin_amdgcn_permlane32_swap(top, top, false, false);
      const QfloatScale s = qfloat_scale(max((uint32_t)both[0], (uint32_t)both[1]));
      if (i * 32 >= rows) return;                              // (the next rows of the form are another group's)
      uint8_t* const out = p.hq + ((int64_t)((pa >> 5) + i) * (pitch / 32) + (n0 >> 5)) * 1024 + lane * 16;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        uint32_t w[4];
#pragma unroll
        for (int g = 0; g < 4; ++g)
          w[g] = qfloat_four(acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3], s);
        // halves of the lanes have halves of 8 channels: they exchange, and have 16 in a row
        const auto lo = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false), hi = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
        *reinterpret_cast<u32x4_t*>(out + j * 1024) = u32x4_t{(uint32_t)lo[0], (uint32_t)lo[1], (uint32_t)hi[0], (uint32_t)hi[1]};
      }
      if (lane < 32) p.hs[qfloat_scale_at(pa + m, n0 >> 7, nkb)] = (uint8_t)s.byte;
    }
  }
};

// ids of the table rows of a wavefront's tokens, lane l having rows l and 64 + l
template <int MI>
__device__ __forceinline__ void load_ids(const QfloatGemmArgs& p, int m0, int rows, int lane, int (&id)[(MI + 1) / 2]) {
#pragma unroll
  for (int h = 0; h < (MI + 1) / 2; ++h) {
    const int at = h * 64 + lane;
    int v = p.ids[m0 + (at < rows ? at : rows - 1)];   // (none: the last row of the group)
    if ((unsigned)v >= (unsigned)p.E_rows) {   // reported to the host, clamped so no access leaves the table
      *p.flag = 1;
      v = v < 0 ? 0 : p.E_rows - 1;
    }
    id[h] = v;
  }
}

// ---- 256 x 256 ----------------------------------------------------------------------------------------------------------------
// 4 wavefronts of 4 x 4 accumulators, a ring of five 32 KB slots of one operand tile each: the loop of the 8-bit integer products (gemm_int8.hip), whose
// instruction takes as long for the same bytes.  16384 x 8192 -> 2048: 206 to 220 us, 2.5 to 2.67 10^15 a second, matrix units busy 78 % of the clocks: the chip's
// power sets the rate.
constexpr int SLOT = 32768;

__global__ __launch_bounds__(256) void ring_kernel(QfloatGemmArgs p) {
  typedef Output<4, 4, false> Out;
  static_assert(4 * Out::BYTES <= 5 * SLOT, "room for the epilogue");
  __shared__ __attribute__((aligned(16))) char smem[5 * SLOT];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  Work w;
  if (!find_work<256, 256, false>(p, lane, w)) return;
  const int nk = p.K / 128, kbytes = nk * 4096;
  const int64_t b_bytes = stem_qfloat_pitch(p.N) * p.K;
  const uint8_t *const B = p.B + w.group * p.stride_b, *const sb = p.sb + w.group * p.stride_b;
  Loader<256, 4> la, lb;
  la.init(p.A, p.a_bytes, w.rows, p.K, w.pa, wave, lane);
  lb.init(B, b_bytes, p.N - w.n0, p.K, w.n0, wave, lane);
  const rsrc_t none = resource(p.A, 0);
  Scales ca, cb;
  ca.init(p.sa, p.a_bytes / 128, w.pa + wm * 128, nk, lane);
  cb.init(sb, b_bytes / 128, w.n0 + wn * 128, nk, lane);
  // every XCD starts at another eighth of K: the rows' groups are a power of two apart where K is, and so their blocks at one k in the
  // same few memory channels
  const int start = nk >= 16 ? (int)(blockIdx.x & 7) * nk / 8 : 0;
  int ka = start * 4096, kb = ka, ks = start;
  int left_a = nk, left_b = nk;   // tiles still to be requested; requests beyond the last one read nothing
  auto next = [&](int& k, int& left, auto& l) __attribute__((always_inline)) {
    k += 4096;
    if (k >= kbytes) k = 0;
    if (--left <= 0) l.r = none;
  };
  f32x16_t acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x16_t{};
  i32x8_t xa[4], xb[4], ya[4], yb[4];
  const uint32_t fa = wm * 16384 + lane * 16, fb = wn * 16384 + lane * 16;
  auto frag = [&](int slot, uint32_t f, int ks, int i) __attribute__((always_inline)) {
    const char* const at = smem + slot * SLOT + f + i * 4096 + ks * 2048;
    return join(*reinterpret_cast<const i32x4_t*>(at), *reinterpret_cast<const i32x4_t*>(at + 1024));
  };
  uint32_t sa, sb_, na_, nb_;
  // order of a k-step's fragments and of the products that use them, two a fragment
  auto mma2 = [&](auto Q, i32x8_t(&a)[4], i32x8_t(&b)[4]) __attribute__((always_inline)) {
    constexpr int ii[16] = {0, 0, 1, 1, 0, 1, 0, 1, 2, 2, 2, 2, 3, 3, 3, 3};
    constexpr int jj[16] = {0, 1, 0, 1, 2, 2, 3, 3, 0, 1, 2, 3, 0, 1, 2, 3};
    constexpr int h = 2 * decltype(Q)::value;
    acc[ii[h]][jj[h]] = mma<jj[h], ii[h]>(b[jj[h]], a[ii[h]], acc[ii[h]][jj[h]], sb_, sa);
    acc[ii[h + 1]][jj[h + 1]] = mma<jj[h + 1], ii[h + 1]>(b[jj[h + 1]], a[ii[h + 1]], acc[ii[h + 1]][jj[h + 1]], sb_, sa);
  };
  auto read = [&](int sa, int sb, int ks, int q, i32x8_t(&a)[4], i32x8_t(&b)[4]) __attribute__((always_inline)) {
    constexpr int isA[8] = {1, 0, 0, 1, 0, 0, 1, 1};
    constexpr int idx[8] = {0, 0, 1, 1, 2, 3, 2, 3};
    if (isA[q]) a[idx[q]] = frag(sa, fa, ks, idx[q]);
    else b[idx[q]] = frag(sb, fb, ks, idx[q]);
  };
  // Operand tiles alternate through the slots: A of K tile t in slot 2t mod 5, B in 2t+1 mod 5.  A(t+2) is requested during the first
  // k-step of tile t, behind the scales of t+1, and B(t+2) behind the barrier before its last: whole K tiles before they are needed, and the wait in front
  // of the barrier leaves the youngest 8 loads in flight.
  sa = ca.load(ks);
  sb_ = cb.load(ks);
#pragma unroll
  for (int h = 0; h < 4; ++h) {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      if (h & 1) lb.issue(q, smem + h * SLOT, wave, kb);
      else la.issue(q, smem + h * SLOT, wave, ka);
    }
    if (h & 1) next(kb, left_b, lb); else next(ka, left_a, la);
  }
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(16) : "memory");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int q = 0; q < 8; ++q) read(0, 1, 0, q, xa, xb);
  auto ring_iteration = [&](const int tmod) __attribute__((always_inline)) {
    const int s0 = (2 * tmod) % 5, s1 = (2 * tmod + 1) % 5, n0 = (2 * tmod + 2) % 5, n1 = (2 * tmod + 3) % 5, in = (2 * tmod + 4) % 5;
    if (++ks >= nk) ks = 0;
    na_ = ca.load(ks);
    nb_ = cb.load(ks);
    __builtin_amdgcn_sched_barrier(0);
    each([&](auto Q) __attribute__((always_inline)) {
      constexpr int q = decltype(Q)::value;
      read(s0, s1, 1, q, ya, yb);
      la.issue(q, smem + in * SLOT, wave, ka);
      mma2(Q, xa, xb);
      __builtin_amdgcn_sched_barrier(0);
    }, std::make_integer_sequence<int, 8>{});
    next(ka, left_a, la);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(8) : "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    each([&](auto Q) __attribute__((always_inline)) {
      constexpr int q = decltype(Q)::value;
      read(n0, n1, 0, q, xa, xb);
      lb.issue(q, smem + s0 * SLOT, wave, kb);
      mma2(Q, ya, yb);
      __builtin_amdgcn_sched_barrier(0);
    }, std::make_integer_sequence<int, 8>{});
    next(kb, left_b, lb);
    sa = na_;
    sb_ = nb_;
  };
  int kt = 0;
  for (; kt + 5 <= nk; kt += 5) {
    ring_iteration(0);
    ring_iteration(1);
    ring_iteration(2);
    ring_iteration(3);
    ring_iteration(4);
  }
  if (kt < nk) ring_iteration(0);
  if (kt + 1 < nk) ring_iteration(1);
  if (kt + 2 < nk) ring_iteration(2);
  if (kt + 3 < nk) ring_iteration(3);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  Out::run(p, acc, smem + wave * Out::BYTES, w.m0 + wm * 128, w.n0 + wn * 128, w.rows - wm * 128, 0, lane);
}

// ---- 128 x 256, two workgroups a compute unit -----------------------------------------------------------------------------------------
// 4 wavefronts of 2 x 4 accumulators, K tiles of 64 in a ring of three 24 KB slots: one workgroup's first loads and epilogue, which the gate product has a long
// one of, run beside the other's products.  A K tile is one k-step: its fragments are read while the one before is multiplied, and its slot is free then.
// The gate product of 16384 tokens of 2048 x 8192: 244 to 253 us (2.2 10^15 a second, matrix units busy 65 % of the clocks);
// 8192 rows of 1024 x 4096 in 16 uneven groups 50 to 56.
constexpr int PAIR_A = 8192, PAIR_SLOT = 24576;

template <QfloatOut OUT>
__global__ __launch_bounds__(256, 2) void pair_kernel(QfloatGemmArgs p) {
  constexpr bool HALF = OUT == QFLOAT_F32;
  typedef Output<2, 4, HALF> Out;
  typedef Hidden<2> Hid;
  static_assert(4 * Hid::BYTES <= 3 * PAIR_SLOT && 4 * Out::BYTES <= 3 * PAIR_SLOT, "room for the epilogue");
  __shared__ __attribute__((aligned(16))) char smem[3 * PAIR_SLOT];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  Work w;
  if (!find_work<128, 256, HALF>(p, lane, w)) return;
  const int nkb = p.K / 128, nk = w.nk * 2, kbytes = p.K * 32;
  const int64_t b_bytes = stem_qfloat_pitch(p.N) * p.K;
  const uint8_t *const B = p.B + (HALF ? 0 : w.group * p.stride_b), *const sb = p.sb + (HALF ? 0 : w.group * p.stride_b);
  int id[1];
  if (OUT == QFLOAT_HIDDEN) load_ids<2>(p, w.m0 + wm * 64, w.rows - wm * 64, lane, id);
  const rsrc_t none = resource(p.A, 0);
  rsrc_t ra = nk ? resource(p.A, p.a_bytes) : none, rb = nk ? resource(B, b_bytes) : none;
  Scales ca, cb;
  if constexpr (!HALF) {
    ca.init(p.sa, p.a_bytes / 128, w.pa + wm * 64, nkb, lane);
    cb.init(sb, b_bytes / 128, w.n0 + wn * 128, nkb, lane);
  }
  // a wavefront loads one 32-row group of the tokens and two of the weights: 2 KB of each and K tile
  const uint32_t oa = wave * 32 < w.rows ? (uint32_t)((w.pa + wave * 32) * p.K + lane * 16) : OOB;
  uint32_t ob[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) ob[h] = w.n0 + wave * 64 + h * 32 < p.N ? (uint32_t)((w.n0 + wave * 64 + h * 32) * p.K + lane * 16) : OOB;
  int ks = HALF ? w.k0 : nk >= 32 ? (int)(blockIdx.x & 7) * (nk >> 4) : 0, k = ks * 4096, left = nk;   // (blocks of 128)
  auto issue = [&](int q, char* slot) __attribute__((always_inline)) {   // load q of 6
    if (q < 2) lds_dma_16(ra, slot + (wave * 2 + q) * 1024, oa, k + q * 1024);
    else lds_dma_16(rb, slot + PAIR_A + (wave * 4 + q - 2) * 1024, ob[(q - 2) >> 1], k + (q & 1) * 1024);
  };
  auto next = [&]() __attribute__((always_inline)) {
    k += 2048;
    if (k >= kbytes) k = 0;
    if (--left <= 0) ra = rb = none;
  };
  f32x16_t acc[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x16_t{};
  i32x8_t xa[2], xb[4], ya[2], yb[4];
  const char* const fa = smem + wm * 4096 + lane * 16;
  const char* const fb = smem + PAIR_A + wn * 8192 + lane * 16;
  auto read = [&](int slot, int q, i32x8_t(&a)[2], i32x8_t(&b)[4]) __attribute__((always_inline)) {   // a0 b0 b1 a1 b2 b3
    constexpr int isA[6] = {1, 0, 0, 1, 0, 0}, idx[6] = {0, 0, 1, 1, 2, 3};
    const char* const at = (isA[q] ? fa : fb) + slot * PAIR_SLOT + idx[q] * 2048;
    (isA[q] ? a[idx[q]] : b[idx[q]]) = join(*reinterpret_cast<const i32x4_t*>(at), *reinterpret_cast<const i32x4_t*>(at + 1024));
  };
  uint32_t sa = 0, sb_ = 0, na = 0, nb = 0;
  if constexpr (!HALF) {
    sa = ca.load(ks) >> ca.shift;
    sb_ = cb.load(ks);
  }
#pragma unroll
  for (int st = 0; st < 3; ++st) {
#pragma unroll
    for (int q = 0; q < 6; ++q) issue(q, smem + st * PAIR_SLOT);
    next();
  }
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(12) : "memory");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int q = 0; q < 6; ++q) read(0, q, xa, xb);
  // K tile t in slot t mod 3.  Its turn begins when its fragments are in everybody's registers and t + 1 has landed: t + 3 is requested into its slot.
  auto iteration = [&](const int st, const bool even, i32x8_t(&a)[2], i32x8_t(&b)[4], i32x8_t(&c)[2], i32x8_t(&d)[4]) __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(6) : "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (!HALF && even) {
      if (++ks >= nkb) ks = 0;
      na = ca.load(ks);
      nb = cb.load(ks);
      __builtin_amdgcn_sched_barrier(0);
    }
    each([&](auto U) __attribute__((always_inline)) {
      constexpr int u = decltype(U)::value;
      constexpr int ii[8] = {0, 0, 1, 1, 0, 1, 0, 1}, jj[8] = {0, 1, 0, 1, 2, 2, 3, 3};
      if (u < 6) {
        read((st + 1) % 3, u, c, d);
        issue(u, smem + st * PAIR_SLOT);
      }
      if constexpr (HALF) acc[ii[u]][jj[u]] = mma_bf16(b[jj[u]], a[ii[u]], acc[ii[u]][jj[u]]);
      else acc[ii[u]][jj[u]] = mma<jj[u], ii[u]>(b[jj[u]], a[ii[u]], acc[ii[u]][jj[u]], sb_, sa);
      __builtin_amdgcn_sched_barrier(0);
    }, std::make_integer_sequence<int, 8>{});
    next();
    if (!HALF && !even) {
      sa = na >> ca.shift;
      sb_ = nb;
    }
  };
  int kt = 0;
  for (; kt + 6 <= nk; kt += 6) {
    iteration(0, true, xa, xb, ya, yb);
    iteration(1, false, ya, yb, xa, xb);
    iteration(2, true, xa, xb, ya, yb);
    iteration(0, false, ya, yb, xa, xb);
    iteration(1, true, xa, xb, ya, yb);
    iteration(2, false, ya, yb, xa, xb);
  }
  if (kt < nk) {                                               // (an even number is left)
    iteration(0, true, xa, xb, ya, yb);
    iteration(1, false, ya, yb, xa, xb);
    if (kt + 2 < nk) {
      iteration(2, true, xa, xb, ya, yb);
      iteration(0, false, ya, yb, xa, xb);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if constexpr (OUT == QFLOAT_HIDDEN) Hid::run(p, acc, id, smem + wave * Hid::BYTES, w.pa + wm * 64, w.n0 + wn * 128, w.rows - wm * 64, lane);
  else Out::run(p, acc, smem + wave * Out::BYTES, w.m0 + wm * 64, w.n0 + wn * 128, w.rows - wm * 64, HALF ? (int64_t)w.group * p.M * p.N : 0, lane);
}

// ---- tiles with wavefronts that load: STAGES whole K tiles in LDS ----------------------------------------------------------------------
template <int MI_, int NJ_, int WM_, int WN_, int STAGES_, int LW_>
struct Tiling {
  static constexpr int MI = MI_, NJ = NJ_, WM = WM_, WN = WN_, STAGES = STAGES_, LW = LW_, WAVES = WM * WN;
  static constexpr int TM = 32 * MI * WM, TN = 32 * NJ * WN;
  static constexpr int A_BYTES = TM * 128, STAGE = (TM + TN) * 128;
};

// Split K (few tiles): every slice writes its sums in the lanes' layout and takes a ticket of its tile; the workgroup that takes the last one adds them in
// the order of the slices, so that the result does not depend on who is last.  Nobody waits for anybody.  The slices run on different XCDs, whose L2s
// don't see each other's lines: stores and loads carry the device scope bit, and a wavefront's stores are there for the device when they
// leave its counter, which is before the workgroup's ticket is taken.  `at`: this wavefront's place among all of a slice's, `stride` apart.
template <int MI, int NJ>
__device__ __forceinline__ bool last_slice(const QfloatGemmArgs& p, f32x16_t (&acc)[MI][NJ], char* smem, int at, int stride, int slice, int tile, int lane) {
  constexpr int BYTES = MI * NJ * 4096, N = MI * NJ * 4;
  const rsrc_t rw = resource(p.ws, p.ws_bytes);                // (of the room's size, not of what the slices would need: nothing leads behind it)
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const f32x16_t& a = acc[k / 4 / NJ][k / 4 % NJ];
    const f32x4_t v = {a[4 * (k % 4)], a[4 * (k % 4) + 1], a[4 * (k % 4) + 2], a[4 * (k % 4) + 3]};
    store_16<SC1>(__builtin_bit_cast(u32x4_t, v), rw, (uint32_t)((at + slice * stride) * BYTES + lane * 16) + k * 1024u);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  int* const ticket = reinterpret_cast<int*>(smem);
  if (threadIdx.x == 0) *ticket = __hip_atomic_fetch_add(p.tickets + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  const bool last = *ticket == p.ksplit - 1;
  if (!last) return false;
  if (threadIdx.x == 0) __hip_atomic_store(p.tickets + tile, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next launch
  asm volatile("" ::: "memory");
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x16_t{};
  constexpr int SLICES = 32 / N;                               // whose loads are under way together
  for (int s = 0; s < p.ksplit; s += SLICES) {
    f32x4_t v[SLICES][N];
#pragma unroll
    for (int u = 0; u < SLICES; ++u)
#pragma unroll
      for (int k = 0; k < N; ++k)
        v[u][k] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rw, (uint32_t)(lane * 16), (at + min(s + u, p.ksplit - 1) * stride) * BYTES + k * 1024, SC1));
#pragma unroll
    for (int u = 0; u < SLICES; ++u) {
      if (s + u >= p.ksplit) break;
#pragma unroll
      for (int k = 0; k < N; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[k / 4 / NJ][k / 4 % NJ][4 * (k % 4) + q] += v[u][k][q];
    }
  }
  __syncthreads();   // the ticket has been read: LDS may be used again
  return true;
}

template <QfloatOut OUT, class C>
__global__ __launch_bounds__((C::WAVES + C::LW) * 64) void tile_kernel(QfloatGemmArgs p) {
  constexpr int MI = C::MI, NJ = C::NJ, S = C::STAGES, STAGE = C::STAGE;
  typedef Output<MI, NJ, OUT == QFLOAT_F32> Out;
  typedef Hidden<MI> Hid;
  constexpr int EPI = C::WAVES * (OUT == QFLOAT_HIDDEN ? Hid::BYTES : Out::BYTES);
  constexpr int LDS = S * STAGE > EPI ? S * STAGE : EPI;
  __shared__ __attribute__((aligned(16))) char smem[LDS];
  const int lane = threadIdx.x & 63, wave_id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool load_wave = wave_id >= C::WAVES;
  const int wave = load_wave ? wave_id - C::WAVES : wave_id, wm = wave / C::WN, wn = wave % C::WN;
  Work w;
  constexpr bool HALF = OUT == QFLOAT_F32;
  if (!find_work<C::TM, C::TN, HALF>(p, lane, w)) return;
  const int nk = w.nk, k0 = w.k0, nkb = p.K / 128;
  const int64_t b_bytes = stem_qfloat_pitch(p.N) * p.K;
  const uint8_t *const B = p.B + (HALF ? 0 : w.group * p.stride_b), *const sb = p.sb + (HALF ? 0 : w.group * p.stride_b);
  if (load_wave) {
    Loader<C::TM, C::LW> la;
    Loader<C::TN, C::LW> lb;
    constexpr int LOADS = la.LOADS + lb.LOADS;
    la.init(p.A, p.a_bytes, w.rows, p.K, w.pa, wave, lane);
    lb.init(B, b_bytes, p.N - w.n0, p.K, w.n0, wave, lane);
    int k = k0 * 4096, left = nk;
    auto request = [&](const int st) __attribute__((always_inline)) {
      if (left <= 0) { la.r = resource(p.A, 0); lb.r = resource(p.A, 0); }
#pragma unroll
      for (int q = 0; q < la.LOADS; ++q) la.issue(q, smem + st * STAGE, wave, k);
#pragma unroll
      for (int q = 0; q < lb.LOADS; ++q) lb.issue(q, smem + st * STAGE + C::A_BYTES, wave, k);
      k += 4096;
      --left;
    };
#pragma unroll
    for (int st = 0; st < S; ++st) request(st);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 1) * LOADS) : "memory");
    __builtin_amdgcn_s_barrier();
    auto load_iteration = [&](const int st) __attribute__((always_inline)) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 2) * LOADS) : "memory");
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      request(st);
      __builtin_amdgcn_sched_barrier(0);
    };
    int kt = 0;
    for (; kt + S <= nk; kt += S) {
#pragma unroll
      for (int st = 0; st < S; ++st) load_iteration(st);
    }
#pragma unroll
    for (int st = 0; st < S - 1; ++st)
      if (kt + st < nk) load_iteration(st);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing lands in LDS once the epilogue uses it
    __syncthreads();
    return;                                            // (barriers are of the wavefronts that are left)
  }
  int id[(MI + 1) / 2];
  if (OUT == QFLOAT_HIDDEN) load_ids<MI>(p, w.m0 + wm * MI * 32, w.rows - wm * MI * 32, lane, id);
  Scales ca, cb;
  uint32_t sca[S], scb[S];
  if constexpr (!HALF) {
    ca.init(p.sa, p.a_bytes / 128, w.pa + wm * MI * 32, nkb, lane);
    cb.init(sb, b_bytes / 128, w.n0 + wn * NJ * 32, nkb, lane);
#pragma unroll
    for (int st = 0; st < S; ++st) {
      sca[st] = ca.load(k0 + st);
      scb[st] = cb.load(k0 + st);
    }
  }
  f32x16_t acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = f32x16_t{};
  i32x8_t xa[MI], xb[NJ], ya[MI], yb[NJ];
  const char* const fa = smem + wm * MI * 4096 + lane * 16;
  const char* const fb = smem + C::A_BYTES + wn * NJ * 4096 + lane * 16;
  constexpr int NFRAG = MI + NJ, NMMA = MI * NJ;
  auto frag = [&](const char* f) __attribute__((always_inline)) {
    return join(*reinterpret_cast<const i32x4_t*>(f), *reinterpret_cast<const i32x4_t*>(f + 1024));
  };
  auto read = [&](int st, int ks, int q, i32x8_t(&a)[MI], i32x8_t(&b)[NJ]) __attribute__((always_inline)) {   // order a0, b0, b1, .., a1, ..
    if (q == 0) a[0] = frag(fa + st * STAGE + ks * 2048);
    else if (q <= NJ) b[q - 1] = frag(fb + st * STAGE + (q - 1) * 4096 + ks * 2048);
    else a[q - NJ] = frag(fa + st * STAGE + (q - NJ) * 4096 + ks * 2048);
  };
  auto kstep = [&](int st, int ks_next, i32x8_t(&a)[MI], i32x8_t(&b)[NJ], i32x8_t(&na)[MI], i32x8_t(&nb)[NJ], uint32_t sa, uint32_t sb) __attribute__((always_inline)) {
    auto one = [&](auto U) __attribute__((always_inline)) {
      constexpr int u = decltype(U)::value;
#pragma unroll
      for (int q = u * NFRAG / NMMA; q < (u + 1) * NFRAG / NMMA; ++q) read(st, ks_next, q, na, nb);
      if constexpr (HALF) acc[u / NJ][u % NJ] = mma_bf16(b[u % NJ], a[u / NJ], acc[u / NJ][u % NJ]);
      else acc[u / NJ][u % NJ] = mma<u % NJ, u / NJ>(b[u % NJ], a[u / NJ], acc[u / NJ][u % NJ], sb, sa);
      __builtin_amdgcn_sched_barrier(0);
    };
    each(one, std::make_integer_sequence<int, NMMA>{});
  };
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int q = 0; q < NFRAG; ++q) read(0, 0, q, xa, xb);
  // One barrier a K tile, before its last k-step: the load wavefronts have seen the next tile land, the others have read the last of this.
  int kt = 0;
  auto stage_iteration = [&](const int st) __attribute__((always_inline)) {
    uint32_t sa = 0, sb = 0;
    if constexpr (!HALF) {
      sa = sca[st] >> ca.shift;
      sb = scb[st] >> cb.shift;
      sca[st] = ca.load(k0 + kt + st + S);
      scb[st] = cb.load(k0 + kt + st + S);
    }
    kstep(st, 1, xa, xb, ya, yb, sa, sb);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    kstep((st + 1) % S, 0, ya, yb, xa, xb, sa, sb);
  };
  for (; kt + S <= nk; kt += S) {
#pragma unroll
    for (int st = 0; st < S; ++st) stage_iteration(st);
  }
#pragma unroll
  for (int st = 0; st < S - 1; ++st)
    if (kt + st < nk) stage_iteration(st);
  __syncthreads();
  if constexpr (OUT == QFLOAT_F32 || (OUT == QFLOAT_BF16 && C::TN == 64))   // (only these are cut)
    if (p.ksplit > 1 && !last_slice<MI, NJ>(p, acc, smem, w.tile * C::WAVES + wave, w.tiles * C::WAVES, w.slice, w.tile, lane)) return;
  if constexpr (OUT == QFLOAT_HIDDEN) Hid::run(p, acc, id, smem + wave * Hid::BYTES, w.pa + wm * MI * 32, w.n0 + wn * NJ * 32, w.rows - wm * MI * 32, lane);
  else Out::run(p, acc, smem + wave * Out::BYTES, w.m0 + wm * MI * 32, w.n0 + wn * NJ * 32, w.rows - wm * MI * 32, HALF ? (int64_t)w.group * p.M * p.N : 0, lane);
}

typedef Tiling<2, 2, 2, 2, 4, 4> Tile128;       // 128 x 128, 128 KB of LDS
typedef Tiling<2, 1, 2, 2, 6, 4> Tile128x64;    // 144 KB
typedef Tiling<1, 4, 4, 1, 4, 4> Hidden128;     // 128 x 128, a wavefront with whole blocks of 128 channels
typedef Tiling<1, 4, 2, 1, 6, 4> Hidden64;      // 64 x 128

template <QfloatOut OUT>
unsigned grid_of(const QfloatGemmArgs& a, int tm, int tn) {
  const int64_t ntn = (a.N + tn - 1) / tn, ntm = (a.M + tm - 1) / tm;
  if (OUT == QFLOAT_F32) return (unsigned)(ntm * ntn * (a.groups.offsets ? a.groups.n : 1) * a.ksplit);
  if (a.groups.offsets) return (unsigned)(((a.groups.T + tm - 1) / tm + std::min(a.groups.n, a.groups.T) - 1) * ntn);   // at most: each group may have a tile not full
  return (unsigned)(ntm * ntn * a.ksplit);
}

template <QfloatOut OUT, class C>
hipError_t launch(const QfloatGemmArgs& a, hipStream_t s) {
  const unsigned tiles = grid_of<OUT>(a, C::TM, C::TN);
  tile_kernel<OUT, C><<<tiles, (C::WAVES + C::LW) * 64, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

// ---- choice of the tile and of the K slices ----------------------------------------------------------------------------------------
// The largest tile that leaves no compute unit idle: operand bytes go down with it, and the time with the number of rounds.  us of a product alone, rows x K -> N:
//                              128 x 64   128 x 128   128 x 256   256 x 256
//   1024 x 2048 -> 2048           8.6        10.2
//   512 x 8192 -> 2048           18.7        23.1
//   8192 x 1024 -> 640                       14.1        10.6        16.4
//   8192 x 4096 -> 1100                      48.9        45.4        42.8
//   8192 x 8192 -> 640                       53.1        44.4        69.1
//   4096 x 4096 -> 4096                      72.0        55.8        51.8
//   2000 x 1024 -> 1024, 16 groups 11.5       7.5        10.3
// and of the gate product, whose tiles have whole blocks of 128 channels, 64 x 128 / 128 x 128 / 128 x 256: 64 x 2048 -> 8192 9.6 / 10.9, 1024 x 1024 -> 4096
// 16.3 / 11.2, 8192 x 1024 -> 640 - / 16.8 / 13.2, 2048 x 2048 -> 3200 - / 24.9 / 19.4.
// K slices fill what few tiles leave idle, where K is long: 700 x 8192 -> 200 whole 17.8, in 2, 3, 4 14.2, 11.7, 11.2; 1500 x 4096 -> 600 with its rows 20.8 and 20.0; 512 x
// 8192 -> 2048 whole 18.7, in 2 16.8, but 1024 x 4096 -> 1024, also of 128 tiles, 11.4 and 11.9; 700 x 1999 -> 1001 7.5 and 9.1.  Weight gradients, us whole, in 4, 8, 16
// slices: 14460 rows of 114 x 211 65, 24, 19, 20; 3344 of 327 x 74 18.5, 13.3, 12.7, 12.9; 8000 of 700 x 900 43, 22.5.
extern "C" void stem_route_qfloat(int64_t T, int groups, int N, int K, int out, int64_t ws_bytes, int32_t* route) {
  const int64_t per_group = (T + groups - 1) / groups;       // of an average group, which is all that is known here: uneven ones have more tiles that are not full
  auto tiles_of = [&](int64_t rows, int tm, int tn) { return (rows + tm - 1) / tm * ((N + tn - 1) / tn); };
  auto tiles = [&](int tm, int tn) {
    return std::max((per_group + tm - 1) / tm * groups, groups > 1 ? (T + tm * (int64_t)groups / 2) / tm : 0) * ((N + tn - 1) / tn);
  };
  const int nk = K / 128;
  int rows = 128, cols = 128, slices = 1;
  if (out == QFLOAT_HIDDEN) {
    if (tiles(64, 128) <= 256) rows = 64;
    else if (tiles(128, 128) > 256) cols = 256;
  } else if (out == QFLOAT_BF16) {
    if (tiles(128, 64) <= 256) cols = 64;
    else if (tiles(128, 128) > 256) cols = 256;
    if (cols == 256 && nk >= 32) {
      // rounds of 256 x 256, and of 128 x 256 in their terms: two of these a compute unit, and the last round's alone are faster
      const int64_t pair = tiles(128, 256), last = pair % 512;
      const double few = 1.1 * (double)(pair / 512) + (last == 0 ? 0 : last <= 256 ? 0.72 : 1.1);
      if ((double)((tiles(256, 256) + 255) / 256) <= few) rows = 256;
    }
  }
  if (out == QFLOAT_F32) {
    // T: rows of the output, all of it for each group; K: of an average group
    const int64_t n = tiles_of(T, 128, 128) * groups;
    if (n > 256) {
      // us: tiles of 128 x 128 one a compute unit, in rounds of 256; of 128 x 256 two, whose last round's alone are faster (4096 x 2001 x 2100 58 us and 47,
      // 5178 x 2816 x 256 in 6 groups 23 and 35, 2978 x 848 x 7070 in 2 62 and 48, 9000 x 1999 x 1501 in 3 68 and 79)
      const int64_t pairs = tiles_of(T, 128, 256) * groups, last = pairs % 512;
      const double few = (double)((n + 255) / 256) * (0.4 * nk + 4);
      const double two = (double)(pairs / 512) * (1.25 * nk + 16) + (last == 0 ? 0 : last <= 256 ? 0.68 * nk + 11 : 1.25 * nk + 16);
      if (two < few) cols = 256;
    } else slices = (int)std::min<int64_t>({MAX_WEIGHT_SLICES, nk / 8, 256 / n});
  } else if (out == QFLOAT_BF16 && cols == 64 && groups == 1) {
    slices = nk < 32 ? 1 : (int)std::min<int64_t>({MAX_SLICES, nk / 10, (nk < 64 ? 240 : 256) / tiles(rows, cols)});
  }
  while (slices > 1 && slices * rows * cols * 4 * (out == QFLOAT_F32 ? tiles_of(T, 128, 128) * groups : tiles(rows, cols)) > ws_bytes) --slices;
  while (slices > 1 && (nk + slices - 1) / slices * (slices - 1) >= nk) --slices;   // every slice has a part of K
  if (slices < 1) slices = 1;
  route[0] = rows; route[1] = cols; route[2] = slices;
}

hipError_t stem_qfloat_gemm_launch(stem_ctx* ctx, int kid, QfloatOut out, const QfloatGemmArgs& p, hipStream_t s) {
  ProfScope prof(ctx, kid, s);
  QfloatGemmArgs a = p;
  int32_t route[3];
  const int nk = out == QFLOAT_F32 ? (int)(((int64_t)a.groups.T / a.groups.n + 63) / 64) : a.K / 128;
  stem_route_qfloat(a.M, a.groups.n, a.N, nk * 128, out, a.ws_bytes, route);
  a.ksplit = a.groups.offsets && out != QFLOAT_F32 ? 1 : route[2];
  if (out == QFLOAT_F32 && route[1] == 256) pair_kernel<QFLOAT_F32><<<grid_of<QFLOAT_F32>(a, 128, 256), 256, 0, s>>>(a);
  else if (out == QFLOAT_F32) return launch<QFLOAT_F32, Tile128>(a, s);
  else if (route[0] == 256) ring_kernel<<<grid_of<QFLOAT_BF16>(a, 256, 256), 256, 0, s>>>(a);
  else if (route[1] == 256 && out == QFLOAT_HIDDEN) pair_kernel<QFLOAT_HIDDEN><<<grid_of<QFLOAT_HIDDEN>(a, 128, 256), 256, 0, s>>>(a);
  else if (route[1] == 256) pair_kernel<QFLOAT_BF16><<<grid_of<QFLOAT_BF16>(a, 128, 256), 256, 0, s>>>(a);
  else if (out == QFLOAT_HIDDEN) return route[0] == 64 ? launch<QFLOAT_HIDDEN, Hidden64>(a, s) : launch<QFLOAT_HIDDEN, Hidden128>(a, s);
  else return route[1] == 64 ? launch<QFLOAT_BF16, Tile128x64>(a, s) : launch<QFLOAT_BF16, Tile128>(a, s);
  return hipGetLastError();
}
