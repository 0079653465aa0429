// 8-bit MFMA products for gfx950: y[m,n] = s_m t_n sum_k a_mk b_nk, tokens a and weights b in blocks of 32 rows x 32 k (quant.h).
//
// A block is one operand of v_mfma_i32_32x32x32_i8 as it lies in memory, so a tile of an operand is 4 KB for each 32 rows and 128 k, in
// a row; it goes to LDS as it is (buffer_load ... lds), and a fragment is the 16 bytes at 16 x lane of a block: no swizzle, no bank
// conflict, one address register for an operand.  The sums are integers, so neither the order of K nor its cuts change a result.
//
// The instruction multiplies twice as many k as the bf16 one of the same shape in the same 32 clocks on operands of the same bytes, so
// the large tile is that product's (gemm_bf16.hip): 256 x 256, 4 wavefronts of 4 x 4 accumulators, a ring of five 32 KB slots.
// Measured: 16384 x 8192 x 8192 and 16384 x 2048 x 8192 at 2.5 10^15 operations a second, the matrix units busy 3/4 of the workgroups' clocks;
// what holds it there is the clock that the card keeps under this load.
#include <algorithm>

#include "quant.h"

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4_t;
typedef __attribute__((ext_vector_type(4))) int i32x4_t;
typedef __attribute__((ext_vector_type(16))) int i32x16_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
typedef __attribute__((address_space(3))) void* lds_ptr_t;
typedef __amdgpu_buffer_rsrc_t rsrc_t;

namespace {

constexpr uint32_t OOB = 0x80000000u;   // a buffer offset beyond any operand: reads as zero, is not stored
constexpr int SC1 = 16;                 // cache policy bit of the buffer instructions: device scope
constexpr int MAX_SLICES = 4;

__device__ __forceinline__ float sigmoidf_fast(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
__device__ __forceinline__ void lds_dma_16(rsrc_t rs, char* lds_dst, uint32_t off, int soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr_t)lds_dst, 16, off, soff, 0, 0);
}
__device__ __forceinline__ rsrc_t resource(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}
// 16 bytes to a buffer, all of the address in the vector offset.  With a scalar register as the other offset the compiler has been seen to let the
// next vector instruction write one of the data's registers (it keeps two apart only where that offset is a constant), and the last 4 lanes of
// each 16 stored what that had written: hidden values of zero in the gate product's second workgroup of a compute unit.
template <int POLICY = 0>
__device__ __forceinline__ void store_16(u32x4_t v, rsrc_t r, uint32_t off) {
  __builtin_amdgcn_raw_buffer_store_b128(v, r, off, 0, POLICY);
}

// Workgroup -> tile, as the bf16 products do it: the workgroups of an XCD take a contiguous run of tiles, walked in bands of 4 token tiles.
__device__ __forceinline__ void tile_of(int b, int nb, int ntm, int ntn, int& tm, int& tn) {
  const int q = nb >> 3, r = nb & 7, xcd = b & 7;
  const int L = xcd * q + (xcd < r ? xcd : r) + (b >> 3);
  const int per = 4 * ntn, group = L / per, first = group * 4, rows = ntm - first < 4 ? ntm - first : 4, in = L - group * per;
  tm = first + in % rows;
  tn = in / rows;
}

// The operand tiles of a workgroup: EDGE rows x 128 k, LOADS loads of 1 KB for each of LOADERS wavefronts
template <int EDGE, int LOADERS>
struct Loader {
  static constexpr int LOADS = EDGE * 128 / 1024 / LOADERS;
  rsrc_t r;
  uint32_t off[(LOADS + 3) / 4];   // of the 32-row groups this wavefront loads from
  const void* base;
  int bytes;
  __device__ __forceinline__ void init(const int8_t* p, int rows, int K, int row0, int wave, int lane) {
    base = p;
    bytes = (rows + 31) / 32 * 32 * K;
    r = resource(p, bytes);
#pragma unroll
    for (int i = 0; i < (LOADS + 3) / 4; ++i) {
      const int group = row0 / 32 + (wave * LOADS + i * 4) / 4;
      off[i] = group * 32 < rows ? (uint32_t)(group * 32 * K + lane * 16) : OOB;
    }
  }
  // load i of the K tile at byte `k` of a group
  __device__ __forceinline__ void issue(int i, char* tile, int wave, int k) const {
    const int piece = wave * LOADS + i;
    lds_dma_16(r, tile + piece * 1024, off[LOADS < 4 ? 0 : i / 4], k + (piece & 3) * 1024);
  }
};

// ---- epilogue of a product: a wavefront's 32 MI x 32 NJ results, 32 rows at a time through LDS ---------------------------------
// acc[i][j]: token block i, channel block j; a lane holds token lane & 31 and channels 8 g + 4 (lane >> 5) + 0..3 of each.  They are scaled
// on their way into LDS.
template <int MI, int NJ>
struct Output {
  static constexpr int COLS = 32 * NJ, PITCH = COLS + 4;       // of a staged row, in words
  static constexpr int BYTES = (32 * PITCH + COLS) * 4;        // of LDS, for each wavefront: the rows, and the channels' scales
  static constexpr int LPR = COLS / 8, RPP = 64 / LPR, PASSES = 32 / RPP;   // 8 columns a lane

  static __device__ __forceinline__ void run(const QuantGemmArgs& p, const i32x16_t (&acc)[MI][NJ], char* stg, int m0, int n0, int lane) {
    float* const st = reinterpret_cast<float*>(stg);
    if (m0 >= p.M || n0 >= p.N) return;
    float* const scales = st + 32 * PITCH;
#pragma unroll
    for (int c = lane; c < COLS; c += 64) scales[c] = p.scale_b[n0 + c < p.N ? n0 + c : 0];
    float sa[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) sa[i] = p.scale_a[min(m0 + i * 32 + (lane & 31), p.M - 1)];
    // A lane outside the matrix is given an offset beyond the buffer: its loads read zero and its stores are dropped.  The buffers begin at the
    // 16-byte boundary in front of row m0.
    const bool whole = p.N % 8 == 0;                           // all rows begin at one
    const int rows = p.M - m0 < 32 * MI ? p.M - m0 : 32 * MI, lim = p.N - n0 < COLS ? p.N - n0 : COLS;
    const size_t first = (size_t)m0 * p.N & ~(size_t)7;
    const int skip = (int)((size_t)m0 * p.N & 7), size = (skip + rows * p.N) * 2;
    const rsrc_t ry = resource(p.y + first, size), rr = resource(p.residual ? p.residual + first : nullptr, p.residual ? size : 0);
    auto at = [&](int r, int col, bool ok) __attribute__((always_inline)) { return ok ? (uint32_t)(skip + r * p.N + n0 + col) * 2u : OOB; };
    auto to_lds = [&](int i) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int col = j * 32 + g * 8 + (lane >> 5) * 4;
          const f32x4_t sb = *reinterpret_cast<const f32x4_t*>(scales + col);
          f32x4_t w;
#pragma unroll
          for (int q = 0; q < 4; ++q) w[q] = (float)acc[i][j][4 * g + q] * (sa[i] * sb[q]);
          *reinterpret_cast<f32x4_t*>(st + (lane & 31) * PITCH + col) = w;
        }
      in_order();
    };
    auto add_and_store = [&](const float* from, uint32_t off, u32x4_t res) __attribute__((always_inline)) {
      float z[8];
      __builtin_memcpy(z, from, 32);
      bf16x8_t o;
#pragma unroll
      for (int q = 0; q < 8; ++q) o[q] = (__bf16)(z[q] + __uint_as_float(q & 1 ? res[q >> 1] & 0xffff0000u : res[q >> 1] << 16));
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, o), ry, off, 0, 0);
    };
    // what the rows of a block are added to: requested for all blocks at once where registers allow
    constexpr int AHEAD = MI * NJ <= 4 ? MI : 1;
    if (whole) {
      const int srow = lane / LPR, scol = (lane % LPR) * 8;
      uint32_t off[AHEAD][PASSES];
      u32x4_t res[AHEAD][PASSES];
      auto fetch = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int pass = 0; pass < PASSES; ++pass) {
          const int r = i * 32 + pass * RPP + srow;
          off[i % AHEAD][pass] = at(r, scol, scol < lim && r < rows);
          res[i % AHEAD][pass] = u32x4_t{};
          if (p.residual) res[i % AHEAD][pass] = __builtin_amdgcn_raw_buffer_load_b128(rr, off[i % AHEAD][pass], 0, 0);
        }
      };
      if (AHEAD > 1)
#pragma unroll
        for (int i = 0; i < MI; ++i) fetch(i);
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        if (AHEAD == 1) fetch(i);
        to_lds(i);
#pragma unroll
        for (int pass = 0; pass < PASSES; ++pass) add_and_store(st + (pass * RPP + srow) * PITCH + scol, off[i % AHEAD][pass], res[i % AHEAD][pass]);
        in_order();   // all have read the rows before they are staged over
        __builtin_amdgcn_sched_barrier(0);   // (all blocks' reads at once would not fit the registers)
      }
      return;
    }
    // Rows of y at any 2-byte address: the same lanes store the same 8 columns, as global stores, which take any address; the last ones of the
    // matrix's rows that are fewer go one by one, eight rows at a time.  (4000 x 5001, K 1999, with residual: 62 us, against 56 at 5000 columns; 191 with
    // all columns one by one, 77 with 16-byte boundaries sought in each row.)
    const int srow = lane / LPR, scol = (lane % LPR) * 8, left = lim - scol;
    const bool edge = lim % 8 != 0;                            // of the matrix, in this tile
    bf16_t* const y = p.y + (size_t)m0 * p.N + n0 + scol;
    const bf16_t* const res = p.residual ? p.residual + (size_t)m0 * p.N + n0 + scol : nullptr;
    u32x4_t rz[AHEAD][PASSES];
    uint32_t end_at[AHEAD][4];
    uint16_t re[AHEAD][4];
    const int end_col = (lim & ~7) + (lane & 7);
    auto fetch = [&](int i) __attribute__((always_inline)) {
#pragma unroll
      for (int pass = 0; pass < PASSES; ++pass) {
        const int r = i * 32 + pass * RPP + srow;
        u32x4_t& v = rz[i % AHEAD][pass];
        v = u32x4_t{};
        if (res && left >= 8 && r < rows) __builtin_memcpy(&v, res + (size_t)r * p.N, 16);
      }
      if (edge)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int r = i * 32 + u * 8 + (lane >> 3);
          end_at[i % AHEAD][u] = at(r, end_col, end_col < lim && r < rows);
          re[i % AHEAD][u] = p.residual ? __builtin_amdgcn_raw_buffer_load_b16(rr, end_at[i % AHEAD][u], 0, 0) : 0;
        }
    };
    if (AHEAD > 1)
#pragma unroll
      for (int i = 0; i < MI; ++i) fetch(i);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      if (AHEAD == 1) fetch(i);
      to_lds(i);
#pragma unroll
      for (int pass = 0; pass < PASSES; ++pass) {
        const int r = i * 32 + pass * RPP + srow;
        float z[8];
        __builtin_memcpy(z, st + (pass * RPP + srow) * PITCH + scol, 32);
        if (left >= 8 && r < rows) {
          const u32x4_t v = rz[i % AHEAD][pass];
          bf16x8_t o;
#pragma unroll
          for (int q = 0; q < 8; ++q) o[q] = (__bf16)(z[q] + __uint_as_float(q & 1 ? v[q >> 1] & 0xffff0000u : v[q >> 1] << 16));
          __builtin_memcpy(y + (size_t)r * p.N, &o, 16);
        }
      }
      if (edge)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float z = st[(u * 8 + (lane >> 3)) * PITCH + end_col];
          __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (__bf16)(z + __uint_as_float((uint32_t)re[i % AHEAD][u] << 16))), ry,
                                                end_at[i % AHEAD][u], 0, 0);
        }
      in_order();
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  static __device__ __forceinline__ void in_order() {   // of LDS, within the wavefront
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
};

// ---- epilogue of the gate product: hidden values SiLU(z) * E[ids] ---------------------------------------------------------------------
// A token's scale is the largest of all its hidden values, which lie in as many workgroups as there are tiles of d_ff.  So the values are
// kept in fp32 (rounded to bf16 on the way, one integer in a hundred would be another), in the lanes' own layout, 4 KB a block, and the maxima
// of the tokens are taken on the way (a maximum of integers, whose order does not matter); quant_hidden_kernel makes integers of them.
// (Workgroups that wait for the others' maxima and quantise what they hold in registers save that traffic, and wait: 16384 tokens of 2048 x
// 8192, 520 us, 34 thousand of a workgroup's 114 thousand clocks in the wait; the two kernels take 333 and 109.)
//
// The lanes' layout is kept throughout: a lane has one token, so its maximum is over its registers and one other lane's.  The table rows
// are what moves: they go to LDS as they are gathered, 16 bytes a lane, chunk c of row r at chunk c ^ f(r) so that 16 rows' reads fall into
// 16 chunk columns.
template <int MI, int NJ>
struct Hidden {
  static constexpr int CH = 4 * NJ;                            // 16-byte chunks of a row of the table, of this wavefront's columns
  static constexpr int ROWS = 32 * MI * CH * 16;               // of LDS, for each wavefront, and 128 NJ for the channels' scales
  static constexpr int BYTES = ROWS + 128 * NJ;
  static __device__ __forceinline__ int swz(int r) { return NJ == 4 ? r & 15 : NJ == 2 ? r >> 1 & 7 : r >> 2 & 3; }

  static __device__ __forceinline__ void run(const QuantGemmArgs& p, const i32x16_t (&acc)[MI][NJ], const float (&sa)[MI],
                                             const int (&row_id)[(MI + 1) / 2], char* lds, int m0, int n0, int lane) {
    if (m0 >= p.M || n0 >= p.N) return;
#pragma unroll
    for (int q = 0; q < MI * CH / 2; ++q) {
      const int r = q * (64 / CH) + lane / CH, col = n0 + ((lane % CH) ^ swz(r)) * 8;
      const int id = __builtin_amdgcn_ds_bpermute((r & 63) * 4, row_id[(q * (64 / CH)) >> 6]);
      const bf16_t* const at = p.E + (size_t)id * p.N + (col < p.N ? col : 0);
      __builtin_amdgcn_global_load_lds(const_cast<bf16_t*>(at), (lds_ptr_t)(lds + q * 1024), 16, 0, 0);
    }
    float* const scales = reinterpret_cast<float*>(lds + ROWS);
#pragma unroll
    for (int c = lane; c < 32 * NJ; c += 64) scales[c] = p.scale_b[n0 + c < p.N ? n0 + c : 0];
    // Columns past d_ff that a wavefront has have sums of zero, and a row's first columns of the table: they become zeros, or NaN where the
    // row's own first columns are no numbers either.  Blocks past d_ff that no wavefront has are not written (quant.h).
    const int blocks = (p.N + 127) / 128 * 4, first = n0 >> 5;
    const rsrc_t rh = resource(p.h, (p.M + 31) / 32 * blocks * 4096);
    // largest positive value as an integer, and as an unsigned one the largest negative: NaN are above all numbers in both
    int top_pos[MI];
    uint32_t top_neg[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) { top_pos[i] = 0; top_neg[i] = 0; }
    struct Step { f32x4_t sb; u32x2_t e[MI]; };
    auto load = [&](int t) __attribute__((always_inline)) {
      Step s;
      s.sb = *reinterpret_cast<const f32x4_t*>(scales + 8 * t + 4 * (lane >> 5));
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int m = i * 32 + (lane & 31);
        s.e[i] = *reinterpret_cast<const u32x2_t*>(lds + m * (CH * 16) + ((t ^ swz(m)) << 4) + (lane >> 5) * 8);
      }
      return s;
    };
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    Step cur = load(0);
#pragma unroll
    for (int t = 0; t < 4 * NJ; ++t) {                         // 8 channels a step
      const int j = t >> 2, g = t & 3;
      const Step nxt = t + 1 < 4 * NJ ? load(t + 1) : cur;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const float u[4] = {__uint_as_float(cur.e[i][0] << 16), __uint_as_float(cur.e[i][0] & 0xffff0000u),
                            __uint_as_float(cur.e[i][1] << 16), __uint_as_float(cur.e[i][1] & 0xffff0000u)};
        u32x4_t h;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float z = (float)acc[i][j][4 * g + q] * (sa[i] * cur.sb[q]);
          h[q] = __float_as_uint(z * sigmoidf_fast(z) * u[q]);
        }
        top_pos[i] = max(max(top_pos[i], (int)h[0]), (int)h[1]);
        top_pos[i] = max(max(top_pos[i], (int)h[2]), (int)h[3]);
        top_neg[i] = max(max(top_neg[i], h[0]), h[1]);
        top_neg[i] = max(max(top_neg[i], h[2]), h[3]);
        const bool out = first + j >= blocks || m0 + 32 * i >= p.M;
        store_16(h, rh, (out ? OOB : (uint32_t)(((m0 >> 5) + i) * blocks + first + j) * 4096u + lane * 16u) + g * 1024u);
      }
      __builtin_amdgcn_sched_barrier(0);                       // (all steps' reads at once would not fit the registers)
      cur = nxt;
    }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      uint32_t v = max((uint32_t)top_pos[i], top_neg[i] & 0x7fffffffu);
      v = max(v, (uint32_t)__shfl_xor((int)v, 32));
      const int m = m0 + i * 32 + lane;
      if (lane < 32 && m < p.M) __hip_atomic_fetch_max(p.amax + m, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
};

// Scales of a wavefront's tokens, lane & 31 of each block of 32, and the ids of their table rows, lane l having rows l and 64 + l
template <int MI, bool GATE>
struct Rows {
  float scale[MI];
  int id[(MI + 1) / 2];
  __device__ __forceinline__ void init(const QuantGemmArgs& p, int m0, int lane) {
#pragma unroll
    for (int i = 0; i < MI; ++i) scale[i] = p.scale_a[min(m0 + i * 32 + (lane & 31), p.M - 1)];
#pragma unroll
    for (int h = 0; h < (MI + 1) / 2; ++h) {
      int v = p.ids[min(m0 + h * 64 + lane, p.M - 1)];
      if ((unsigned)v >= (unsigned)p.E_rows) {   // reported to the host, clamped so no access leaves the table
        *p.flag = 1;
        v = v < 0 ? 0 : p.E_rows - 1;
      }
      id[h] = v;
    }
  }
};

// ---- 256 x 256 ----------------------------------------------------------------------------------------------------------------
constexpr int SLOT = 32768;   // an operand tile: 256 rows x 128 k

__global__ __launch_bounds__(256) void gemm_int8_256_kernel(QuantGemmArgs p) {
  __shared__ __attribute__((aligned(16))) char smem[5 * SLOT];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  int tm, tn;
  tile_of(blockIdx.x, gridDim.x, (p.M + 255) / 256, (p.N + 255) / 256, tm, tn);
  const int m0 = tm * 256, n0 = tn * 256;
  Loader<256, 4> la, lb;
  la.init(p.A, p.M, p.K, m0, wave, lane);
  lb.init(p.B, p.N, p.K, n0, wave, lane);
  const int nk = p.K / 128, kbytes = nk * 4096;
  // every XCD starts at another eighth of K: the rows' groups are a power of two apart where K is, and so their blocks at one k in the
  // same few memory channels
  int ka = nk >= 16 ? (int)(blockIdx.x & 7) * nk / 8 * 4096 : 0, kb = ka;
  int left_a = nk, left_b = nk;   // tiles still to be requested; requests beyond the last one read nothing
  auto next = [&](int& k, int& left, auto& l) __attribute__((always_inline)) {
    k += 4096;
    if (k >= kbytes) k = 0;
    if (--left <= 0) l.r = resource(l.base, 0);
  };
  i32x16_t acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = i32x16_t{};

  i32x4_t xa[4], xb[4], ya[4], yb[4];
  const uint32_t fa = wm * 16384 + lane * 16, fb = wn * 16384 + lane * 16;
  auto frag = [&](int slot, uint32_t f, int ks, int i) __attribute__((always_inline)) {
    return *reinterpret_cast<const i32x4_t*>(smem + slot * SLOT + f + i * 4096 + ks * 1024);
  };
  // order of a k-step's fragments and of the products that use them, two a fragment
  auto mma2 = [&](int q, i32x4_t(&a)[4], i32x4_t(&b)[4]) __attribute__((always_inline)) {
    constexpr int ii[16] = {0, 0, 1, 1, 0, 1, 0, 1, 2, 2, 2, 2, 3, 3, 3, 3};
    constexpr int jj[16] = {0, 1, 0, 1, 2, 2, 3, 3, 0, 1, 2, 3, 0, 1, 2, 3};
#pragma unroll
    for (int h = 2 * q; h < 2 * q + 2; ++h)
      acc[ii[h]][jj[h]] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[jj[h]], a[ii[h]], acc[ii[h]][jj[h]], 0, 0, 0);
  };
  auto read = [&](int sa, int sb, int ks, int q, i32x4_t(&a)[4], i32x4_t(&b)[4]) __attribute__((always_inline)) {
    constexpr int isA[8] = {1, 0, 0, 1, 0, 0, 1, 1};
    constexpr int idx[8] = {0, 0, 1, 1, 2, 3, 2, 3};
    if (isA[q]) a[idx[q]] = frag(sa, fa, ks, idx[q]);
    else b[idx[q]] = frag(sb, fb, ks, idx[q]);
  };
  // Operand tiles alternate through the slots: A of K tile t in slot 2t mod 5, B in 2t+1 mod 5.  A(t+2) is requested during the first two
  // k-steps of tile t, B(t+2) behind the barrier before its last: whole K tiles before they are needed, and the wait in front of the
  // barrier leaves the youngest 8 loads in flight.
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
    const int sa = (2 * tmod) % 5, sb = (2 * tmod + 1) % 5, na = (2 * tmod + 2) % 5, nb = (2 * tmod + 3) % 5, ia = (2 * tmod + 4) % 5;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      read(sa, sb, 1, q, ya, yb);
      if (q < 4) la.issue(q, smem + ia * SLOT, wave, ka);
      mma2(q, xa, xb);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      read(sa, sb, 2, q, xa, xb);
      if (q < 4) la.issue(4 + q, smem + ia * SLOT, wave, ka);
      mma2(q, ya, yb);
      __builtin_amdgcn_sched_barrier(0);
    }
    next(ka, left_a, la);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      read(sa, sb, 3, q, ya, yb);
      mma2(q, xa, xb);
      __builtin_amdgcn_sched_barrier(0);
    }
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(8) : "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      read(na, nb, 0, q, xa, xb);
      lb.issue(q, smem + sa * SLOT, wave, kb);
      mma2(q, ya, yb);
      __builtin_amdgcn_sched_barrier(0);
    }
    next(kb, left_b, lb);
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
  typedef Output<4, 4> Out;
  static_assert(4 * Out::BYTES <= 5 * SLOT, "staging");
  Out::run(p, acc, smem + wave * Out::BYTES, m0 + wm * 128, n0 + wn * 128, lane);
}

// ---- 128 x 256, two workgroups a compute unit -----------------------------------------------------------------------------------------
// 4 wavefronts of 2 x 4 accumulators, K tiles of 64 in a ring of three 24 KB slots: one workgroup's epilogue, which the gate product has a long one of,
// runs beside the other's products.  Measured, 4096 tokens of N 8192, K 2048 with SiLU * gather: 83 us, 55 of them the products' at the rate of
// the 256 x 256 tile; it writes 134 MB of hidden values.
constexpr int PAIR_A = 8192, PAIR_SLOT = 24576;

template <bool GATE>
__global__ __launch_bounds__(256, 2) void gemm_int8_pair_kernel(QuantGemmArgs p) {
  typedef Hidden<2, 4> Hid;
  typedef Output<2, 4> Out;
  static_assert(4 * Hid::BYTES <= 3 * PAIR_SLOT && 4 * Out::BYTES <= 3 * PAIR_SLOT, "room for the epilogue");
  __shared__ __attribute__((aligned(16))) char smem[3 * PAIR_SLOT];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  int tm, tn;
  tile_of(blockIdx.x, gridDim.x, (p.M + 127) / 128, (p.N + 255) / 256, tm, tn);
  const int m0 = tm * 128, n0 = tn * 256;
  Rows<2, GATE> rows;
  if (GATE) rows.init(p, m0 + wm * 64, lane);
  const int nk = p.K / 64, kbytes = p.K * 32;
  const rsrc_t none = resource(p.A, 0);
  rsrc_t ra = resource(p.A, (p.M + 31) / 32 * 32 * p.K), rb = resource(p.B, (p.N + 31) / 32 * 32 * p.K);
  // a wavefront loads one 32-row group of the tokens and two of the weights: 2 KB of each and K tile
  uint32_t oa, ob[2];
  oa = m0 + wave * 32 < p.M ? (uint32_t)((m0 + wave * 32) * p.K + lane * 16) : OOB;
#pragma unroll
  for (int h = 0; h < 2; ++h) ob[h] = n0 + wave * 64 + h * 32 < p.N ? (uint32_t)((n0 + wave * 64 + h * 32) * p.K + lane * 16) : OOB;
  int k = nk >= 32 ? (int)(blockIdx.x & 7) * (nk >> 4) * 4096 : 0, left = nk;
  auto issue = [&](int q, char* slot) __attribute__((always_inline)) {   // load q of 6
    if (q < 2) lds_dma_16(ra, slot + (wave * 2 + q) * 1024, oa, k + q * 1024);
    else lds_dma_16(rb, slot + PAIR_A + (wave * 4 + q - 2) * 1024, ob[(q - 2) >> 1], k + (q & 1) * 1024);
  };
  auto next = [&]() __attribute__((always_inline)) {
    k += 2048;
    if (k >= kbytes) k = 0;
    if (--left <= 0) ra = rb = none;
  };
  i32x16_t acc[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = i32x16_t{};
  i32x4_t xa[2], xb[4], ya[2], yb[4];
  const char* const fa = smem + wm * 4096 + lane * 16;
  const char* const fb = smem + PAIR_A + wn * 8192 + lane * 16;
  auto read = [&](int slot, int ks, int q, i32x4_t(&a)[2], i32x4_t(&b)[4]) __attribute__((always_inline)) {   // a0 b0 b1 a1 b2 b3
    constexpr int isA[6] = {1, 0, 0, 1, 0, 0}, idx[6] = {0, 0, 1, 1, 2, 3};
    if (isA[q]) a[idx[q]] = *reinterpret_cast<const i32x4_t*>(fa + slot * PAIR_SLOT + idx[q] * 2048 + ks * 1024);
    else b[idx[q]] = *reinterpret_cast<const i32x4_t*>(fb + slot * PAIR_SLOT + idx[q] * 2048 + ks * 1024);
  };
  auto mma = [&](int u, i32x4_t(&a)[2], i32x4_t(&b)[4]) __attribute__((always_inline)) {
    constexpr int ii[8] = {0, 0, 1, 1, 0, 1, 0, 1}, jj[8] = {0, 1, 0, 1, 2, 2, 3, 3};
    acc[ii[u]][jj[u]] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[jj[u]], a[ii[u]], acc[ii[u]][jj[u]], 0, 0, 0);
  };
#pragma unroll
  for (int st = 0; st < 2; ++st) {
#pragma unroll
    for (int q = 0; q < 6; ++q) issue(q, smem + st * PAIR_SLOT);
    next();
  }
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(6) : "memory");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int q = 0; q < 6; ++q) read(0, 0, q, xa, xb);
  // K tile t in slot t mod 3; tile t + 2 is requested while t is multiplied, into the slot that t - 1 has left
  auto iteration = [&](const int st) __attribute__((always_inline)) {
    const int nx = (st + 1) % 3, in = (st + 2) % 3;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (u < 6) read(st, 1, u, ya, yb);
      if (u >= 2) issue(u - 2, smem + in * PAIR_SLOT);
      mma(u, xa, xb);
      __builtin_amdgcn_sched_barrier(0);
    }
    next();
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(6) : "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (u < 6) read(nx, 0, u, xa, xb);
      mma(u, ya, yb);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  int kt = 0;
  for (; kt + 3 <= nk; kt += 3) {
    iteration(0);
    iteration(1);
    iteration(2);
  }
  if (kt < nk) iteration(0);
  if (kt + 1 < nk) iteration(1);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if constexpr (GATE) Hid::run(p, acc, rows.scale, rows.id, smem + wave * Hid::BYTES, m0 + wm * 64, n0 + wn * 128, lane);
  else Out::run(p, acc, smem + wave * Out::BYTES, m0 + wm * 64, n0 + wn * 128, lane);
}

// ---- smaller tiles: STAGES whole K tiles in LDS, filled by LW wavefronts of their own ---------------------------------------------
template <int MI_, int NJ_, int WM_, int WN_, int STAGES_, int LW_>
struct Tiling {
  static constexpr int MI = MI_, NJ = NJ_, WM = WM_, WN = WN_, STAGES = STAGES_, LW = LW_, WAVES = WM * WN;
  static constexpr int TM = 32 * MI * WM, TN = 32 * NJ * WN;
  static constexpr int A_BYTES = TM * 128, STAGE = (TM + TN) * 128;
};

// Split K (few tiles): every slice writes its sums in the lanes' layout and takes a ticket of its tile; the workgroup that takes the last one
// adds the others' to its own, in any order: they are integers.  Nobody waits for anybody.  The slices run on different XCDs, whose L2s don't
// see each other's lines: stores and loads carry the device scope bit, and a wavefront's stores are there for the device when they
// leave its counter, which is before the workgroup's ticket is taken.  `at`: this wavefront's place among all of a slice's, `stride` apart.
template <int MI, int NJ>
__device__ __forceinline__ bool last_slice(const QuantGemmArgs& p, i32x16_t (&acc)[MI][NJ], char* smem, int at, int stride, int slice, int tile, int lane) {
  constexpr int BYTES = MI * NJ * 4096;
  const rsrc_t rw = resource(p.ws, p.ksplit * stride * BYTES);
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const i32x4_t v = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
        store_16<SC1>(__builtin_bit_cast(u32x4_t, v), rw, (uint32_t)(at * BYTES + lane * 16) + ((i * NJ + j) * 4 + g) * 1024u);
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
  // the others' sums, all in flight together; what is beyond the last slice reads as zero
  constexpr int N = MI * NJ * 4;
  i32x4_t v[MAX_SLICES - 1][N];
#pragma unroll
  for (int o = 0; o < MAX_SLICES - 1; ++o) {
    const int s = o + (o >= slice);
#pragma unroll
    for (int k = 0; k < N; ++k)
      v[o][k] = __builtin_bit_cast(i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rw, s < p.ksplit ? lane * 16 : OOB, (at + (s - slice) * stride) * BYTES + k * 1024, SC1));
  }
#pragma unroll
  for (int o = 0; o < MAX_SLICES - 1; ++o)
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int q = 0; q < 4; ++q) acc[i][j][4 * g + q] += v[o][(i * NJ + j) * 4 + g][q];
  __syncthreads();   // the ticket has been read: LDS may be used again
  return true;
}

template <bool GATE, class C>
__global__ __launch_bounds__((C::WAVES + C::LW) * 64) void gemm_int8_kernel(QuantGemmArgs p) {
  constexpr int MI = C::MI, NJ = C::NJ, S = C::STAGES, STAGE = C::STAGE;
  typedef Output<MI, NJ> Out;
  typedef Hidden<MI, NJ> Hid;
  constexpr int EPI = C::WAVES * (GATE ? Hid::BYTES : Out::BYTES);
  constexpr int LDS = S * STAGE > EPI ? S * STAGE : EPI;
  __shared__ __attribute__((aligned(16))) char smem[LDS];
  const int lane = threadIdx.x & 63, wave_id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool load_wave = wave_id >= C::WAVES;
  const int wave = load_wave ? wave_id - C::WAVES : wave_id, wm = wave / C::WN, wn = wave % C::WN;
  int tm, tn;
  const int ntm = (p.M + C::TM - 1) / C::TM, ntn = (p.N + C::TN - 1) / C::TN, tiles = ntm * ntn;
  const int slice = blockIdx.x / tiles;
  tile_of(blockIdx.x - slice * tiles, tiles, ntm, ntn, tm, tn);
  const int m0 = tm * C::TM, n0 = tn * C::TN;
  const int nk_all = p.K / 128, per = (nk_all + p.ksplit - 1) / p.ksplit, k0 = slice * per, nk = nk_all - k0 < per ? nk_all - k0 : per;
  Rows<MI, GATE> rows;
  if (GATE && !load_wave) rows.init(p, m0 + wm * MI * 32, lane);
  if (load_wave) {
    Loader<C::TM, C::LW> la;
    Loader<C::TN, C::LW> lb;
    constexpr int LOADS = la.LOADS + lb.LOADS;
    la.init(p.A, p.M, p.K, m0, wave, lane);
    lb.init(p.B, p.N, p.K, n0, wave, lane);
    int k = (k0 + (nk >= 16 ? (int)(blockIdx.x & 7) * nk / 8 : 0)) * 4096, left = nk;
    auto request = [&](const int st) __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < la.LOADS; ++q) la.issue(q, smem + st * STAGE, wave, k);
#pragma unroll
      for (int q = 0; q < lb.LOADS; ++q) lb.issue(q, smem + st * STAGE + C::A_BYTES, wave, k);
      k += 4096;
      if (k >= (k0 + nk) * 4096) k = k0 * 4096;
      if (--left <= 0) { la.r = resource(p.A, 0); lb.r = resource(p.B, 0); }
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
    return;
  }
  i32x16_t acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = i32x16_t{};
  i32x4_t xa[MI], xb[NJ], ya[MI], yb[NJ];
  const char* const fa = smem + wm * MI * 4096 + lane * 16;
  const char* const fb = smem + C::A_BYTES + wn * NJ * 4096 + lane * 16;
  constexpr int NFRAG = MI + NJ, NMMA = MI * NJ;
  auto read = [&](int st, int ks, int q, i32x4_t(&a)[MI], i32x4_t(&b)[NJ]) __attribute__((always_inline)) {   // order a0, b0, b1, .., a1, ..
    if (q == 0) a[0] = *reinterpret_cast<const i32x4_t*>(fa + st * STAGE + ks * 1024);
    else if (q <= NJ) b[q - 1] = *reinterpret_cast<const i32x4_t*>(fb + st * STAGE + (q - 1) * 4096 + ks * 1024);
    else a[q - NJ] = *reinterpret_cast<const i32x4_t*>(fa + st * STAGE + (q - NJ) * 4096 + ks * 1024);
  };
  auto kstep = [&](int st, int ks_next, i32x4_t(&a)[MI], i32x4_t(&b)[NJ], i32x4_t(&na)[MI], i32x4_t(&nb)[NJ]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < NMMA; ++u) {
#pragma unroll
      for (int q = u * NFRAG / NMMA; q < (u + 1) * NFRAG / NMMA; ++q) read(st, ks_next, q, na, nb);
      acc[u / NJ][u % NJ] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[u % NJ], a[u / NJ], acc[u / NJ][u % NJ], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int q = 0; q < NFRAG; ++q) read(0, 0, q, xa, xb);
  // One barrier a K tile, before its last k-step: the load wavefronts have seen the next tile land, the others have read the last of this.
  auto stage_iteration = [&](const int st) __attribute__((always_inline)) {
    kstep(st, 1, xa, xb, ya, yb);
    kstep(st, 2, ya, yb, xa, xb);
    kstep(st, 3, xa, xb, ya, yb);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    kstep((st + 1) % S, 0, ya, yb, xa, xb);
  };
  int kt = 0;
  for (; kt + S <= nk; kt += S) {
#pragma unroll
    for (int st = 0; st < S; ++st) stage_iteration(st);
  }
#pragma unroll
  for (int st = 0; st < S - 1; ++st)
    if (kt + st < nk) stage_iteration(st);
  __syncthreads();
  if constexpr (!GATE && C::TN == 64)   // (only these are cut)
    if (p.ksplit > 1 && !last_slice<MI, NJ>(p, acc, smem, (slice * tiles + tn * ntm + tm) * C::WAVES + wave, tiles * C::WAVES, slice, tn * ntm + tm, lane)) return;
  if constexpr (GATE) Hid::run(p, acc, rows.scale, rows.id, smem + wave * Hid::BYTES, m0 + wm * MI * 32, n0 + wn * NJ * 32, lane);
  else Out::run(p, acc, smem + wave * Out::BYTES, m0 + wm * MI * 32, n0 + wn * NJ * 32, lane);
}

typedef Tiling<2, 2, 2, 2, 4, 4> Tile128;       // 128 x 128, 128 KB of LDS
typedef Tiling<2, 1, 2, 2, 6, 4> Tile128x64;    // 144 KB

template <class C>
hipError_t launch(const QuantGemmArgs& a, hipStream_t s) {
  const int grid = ((a.M + C::TM - 1) / C::TM) * ((a.N + C::TN - 1) / C::TN) * a.ksplit;
  if (a.y) gemm_int8_kernel<false, C><<<grid, (C::WAVES + C::LW) * 64, 0, s>>>(a);
  else gemm_int8_kernel<true, C><<<grid, (C::WAVES + C::LW) * 64, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

// ---- choice of the tile and of the K slices ----------------------------------------------------------------------------------------
// One round of workgroups with as many bytes in flight as may be: the smallest tile whose grid is at most one workgroup a compute unit, and
// beyond 256 tiles of 128 x 128 the large ones.  us, products without / with SiLU * gather, 128 x 64 / 128 x 128 / 128 x 256 / 256 x 256:
//   N 8192, K 2048, gate: 80 tokens 15.4 / 14.9 / 20, 256 17.6 / 16.1 / 21, 400 23 / 18 / 22, 700 32 / 27 / 24.5, 4096 155 / 121 / 83
//   N 4096, K 1024, gate: 256 tokens 11.7 / 11.7 / 15, 700 17 / 14 / 17, 1500 24 / 23 / 18
//   N 2048, K 8192: 700 tokens 24 / 28 / 47 / 73, 1500 44 / 31 / 50 / 76, 4096 94 / 72 / 66 / 89, 16384 - / - / 241 / 218
// K is cut where tiles are few and slices long, in up to 4 (from 32 K tiles on, a slice of 10 or more, 240 workgroups or fewer; in two slices 256, from 48
// K tiles): K 2048, 1 / 2 / 3 slices of 128 x 64 tiles: 700 tokens of N 1000 13.1 / 14.6 / -, 256 of N 1024 11.2 / 12.0 / 11.7; K 4096, 1024 of N 512 20.5 / 19.7 / 19.2; N 2048, K 8192, 1 / 2 / 3 / 4 slices of 128 x 64 tiles: 80 tokens 19 / 15.5 / 14.1 / 14.2, 256 20.6 / 17.1 / 15.6 / 16.6, 400 21.5 / 18.2 / 24 / 23;
// N 1024, K 4096: 128 tokens 13.3 / 12.5 / 12.0 / 12.1, 1024 14.6 / 15.5.
// Cut gate products were slower throughout (256 tokens of N 8192, K 2048 17.6 / 23.1).
extern "C" void stem_route_quant(int M, int N, int K, int gate, int64_t ws_bytes, int32_t* route) {
  auto tiles = [&](int tm, int tn) { return (int64_t)((M + tm - 1) / tm) * ((N + tn - 1) / tn); };
  const int64_t t64 = tiles(128, 64), t128 = tiles(128, 128), pair = tiles(128, 256), t256 = tiles(256, 256);
  const int nk = K / 128;
  int rows = 128, cols = 64, slices = 1;
  if (t64 > 256 || (gate && nk > 8 && t128 >= 64)) cols = 128;
  if (cols == 128 && t128 > 256) {
    cols = 256;
    // rounds of 256 x 256, and of 128 x 256 in their terms: two of these a compute unit, and the last round's alone are faster
    const int64_t last = pair % 512;
    const double few = 1.1 * (double)(pair / 512) + (last == 0 ? 0 : last <= 256 ? 0.72 : 1.1);
    if (!gate && (double)((t256 + 255) / 256) <= few) rows = 256;
  }
  if (!gate && cols == 64) {
    slices = nk < 32 ? 1 : (int)std::min<int64_t>({MAX_SLICES, nk / 10, 240 / t64});
    if (slices < 2 && t64 <= 128 && nk >= 48) slices = 2;
    while (slices > 1 && (int64_t)slices * t64 * 128 * 64 * 4 > ws_bytes) --slices;
    while (slices > 1 && (nk + slices - 1) / slices * (slices - 1) >= nk) --slices;   // every slice has a part of K
    if (slices < 1) slices = 1;
  }
  route[0] = rows; route[1] = cols; route[2] = slices;
}

hipError_t stem_quant_gemm_launch(stem_ctx* ctx, int kid, const QuantGemmArgs& p, hipStream_t s) {
  ProfScope prof(ctx, kid, s);
  QuantGemmArgs a = p;
  int32_t route[3];
  stem_route_quant(a.M, a.N, a.K, !a.y, (int64_t)a.ws_bytes, route);
  a.ksplit = route[2];
  const int grid = ((a.M + route[0] - 1) / route[0]) * ((a.N + route[1] - 1) / route[1]);
  if (route[0] == 256) gemm_int8_256_kernel<<<grid, 256, 0, s>>>(a);
  else if (route[1] == 256 && a.y) gemm_int8_pair_kernel<false><<<grid, 256, 0, s>>>(a);
  else if (route[1] == 256) gemm_int8_pair_kernel<true><<<grid, 256, 0, s>>>(a);
  else return route[1] == 128 ? launch<Tile128>(a, s) : launch<Tile128x64>(a, s);
  return hipGetLastError();
}
