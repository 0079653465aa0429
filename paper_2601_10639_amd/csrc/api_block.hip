// Entry points of what stands around the layer: argument checks and launch sequences of the block's norms, gate, dropout and residual
// (block.hip), and of the layer in 8-bit integers (quant.hip).
#include <math.h>

#include <algorithm>

#include "block.h"
#include "quant.h"

namespace {

#define HIP_TRY(c, expr)                                                                                                       \
  do {                                                                                                                         \
    hipError_t e_ = (expr);                                                                                                    \
    if (e_ != hipSuccess)                                                                                                      \
      return stem_fail((c), STEM_ERR_HIP, "%s failed: %s (%s:%d)", #expr, hipGetErrorString(e_), __FILE__, __LINE__);          \
  } while (0)
#define STEM_TRY(expr)                                   \
  do {                                                   \
    const stem_status st_ = (expr);                      \
    if (st_ != STEM_OK) return st_;                      \
  } while (0)

constexpr int64_t QUANT_MAX_CHANNELS = 1 << 22;   // 256 rows of an output are addressed with 32 bits
constexpr int64_t QUANT_MAX_K = 131072;           // up to here a sum of products of two bytes, 127 x 127 at most, fits 32 bits

struct Buffer { const void* p; size_t bytes; };

bool overlap(const Buffer& a, const Buffer& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && x < y + b.bytes && y < x + a.bytes;
}

// Alignment of all buffers; no output over another, nor over an input unless `in_place` and it is that input.
stem_status check_buffers(stem_ctx* c, const char* who, std::initializer_list<Buffer> in, std::initializer_list<Buffer> out, bool in_place) {
  for (auto& list : {in, out})
    for (const Buffer& b : list)
      if (reinterpret_cast<uintptr_t>(b.p) & 15u) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", who);
  for (const Buffer* o = out.begin(); o != out.end(); ++o) {
    for (const Buffer& i : in)
      if (overlap(*o, i) && !(in_place && o->p == i.p && o->bytes == i.bytes))
        return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: an output lies over an input", who);
    for (const Buffer* other = out.begin(); other != o; ++other)
      if (overlap(*o, *other)) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: an output lies over another", who);
  }
  return STEM_OK;
}

stem_status check_norm(stem_ctx* c, const char* who, const stem_norm& n) {
  if (n.kind != STEM_NORM_NONE && n.kind != STEM_NORM_RMS && n.kind != STEM_NORM_LAYER)
    return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: %d is not a stem_norm_kind", who, n.kind);
  if (n.kind != STEM_NORM_NONE && !(n.eps >= 0.f && n.eps < INFINITY))
    return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: eps = %g", who, (double)n.eps);
  return STEM_OK;
}

// (every workgroup reads the step, also when others have stored their part of an output)
stem_status check_drop(stem_ctx* c, const char* who, const stem_drop& d, std::initializer_list<Buffer> outputs, DropArgs* out) {
  if (!(d.p >= 0.f && d.p <= 1.f)) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: p = %g is not in [0, 1]", who, (double)d.p);
  if (reinterpret_cast<uintptr_t>(d.step) & 7u) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: step must be 8-byte aligned", who);
  for (const Buffer& o : outputs)
    if (overlap(o, {d.step, sizeof *d.step})) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: an output lies over step", who);
  out->threshold = (uint32_t)lrint((double)d.p * 65536.0);
  out->scale = out->threshold < 65536 ? (float)(65536.0 / (65536 - out->threshold)) : 0.f;
  out->seed = d.seed; out->offset = d.offset; out->step = d.step;
  return STEM_OK;
}

size_t type_bytes(const stem_ctx* c) { return c->desc.dtype == STEM_BF16 ? 2 : 4; }

stem_status check_width(stem_ctx* c, const char* who) {
  if (c->desc.d_model > STEM_BLOCK_MAX_WIDTH)
    return stem_fail(c, STEM_ERR_UNSUPPORTED, "%s: d_model = %d is over %d", who, c->desc.d_model, STEM_BLOCK_MAX_WIDTH);
  return STEM_OK;
}

BlockArgs block_args(const stem_ctx* c, int64_t T) {
  BlockArgs a = {};
  a.T = T;
  a.d = c->desc.d_model;
  a.inv_d = 1.0f / (float)a.d;
  a.residual_scale = a.branch_scale = 1.f;
  a.part[0] = c->block_part;
  return a;
}

stem_status check_leave(stem_ctx* c, const char* who, const stem_leave& L, std::initializer_list<Buffer> outputs, BlockArgs* a) {
  STEM_TRY(check_norm(c, who, L.out));
  STEM_TRY(check_norm(c, who, L.next));
  STEM_TRY(check_drop(c, who, L.drop, outputs, &a->drop));
  if (L.gate_kind < STEM_GATE_NONE || L.gate_kind > STEM_GATE_FULL)
    return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: %d is not a stem_gate_kind", who, L.gate_kind);
  if ((L.gate_kind != STEM_GATE_NONE) != (L.gate != nullptr))
    return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: a gate and its kind go together", who);
  a->out = L.out; a->next = L.next;
  a->residual_scale = L.residual_scale; a->branch_scale = L.branch_scale;
  a->gate_kind = L.gate_kind; a->gate = L.gate;
  return STEM_OK;
}

// Sums over no tokens: zero, unless they are added to what is there.
stem_status no_tokens(stem_ctx* c, const char* who, std::initializer_list<float*> sums, int accumulate, void* stream) {
  const size_t sum = (size_t)c->desc.d_model * 4;
  for (float* p : sums) {
    STEM_TRY(check_buffers(c, who, {}, {{p, sum}}, false));
    if (p && !accumulate) HIP_TRY(c, stem_fill_zero(p, sum, static_cast<hipStream_t>(stream)));
  }
  return STEM_OK;
}

size_t gate_bytes(const stem_ctx* c, int kind, int64_t T, size_t es) {
  const size_t d = c->desc.d_model;
  return kind == STEM_GATE_CHANNEL ? d * es : kind == STEM_GATE_TOKEN ? T * es : kind == STEM_GATE_FULL ? T * d * es : 0;
}

stem_status check_quant(stem_ctx* c, const char* who) {
  if (c->desc.dtype != STEM_BF16) return stem_fail(c, STEM_ERR_UNSUPPORTED, "%s: needs a bf16 context", who);
  if (!c->quant_hidden) return stem_fail(c, STEM_ERR_WORKSPACE, "%s: needs stem_reserve(ctx, STEM_RESERVE_QUANT)", who);
  return STEM_OK;
}

hipError_t quant_rows(stem_ctx* c, int kid, const void* x, int64_t rows, int64_t K, const stem_norm* norm, bool pad, int8_t* q, float* scale,
                      uint32_t* clear, int64_t words, hipStream_t s) {
  const QuantRowsArgs a = {static_cast<const bf16_t*>(x), rows, (int)K, pad, norm ? *norm : stem_norm{STEM_NORM_NONE, 0.f, nullptr}, q, scale, clear, words, 0};
  return stem_quant_rows_launch(c, kid, a, s);
}

QuantGemmArgs gemm_args(const stem_ctx* c) {
  QuantGemmArgs a = {};
  a.ws = c->quant_ws; a.ws_bytes = QUANT_WS; a.tickets = c->tickets;
  return a;
}

QuantDecodeArgs decode_args(const stem_ctx* c, int64_t T, int64_t N, int64_t K, const void* q, const float* scale) {
  QuantDecodeArgs a = {};
  a.B = static_cast<const int8_t*>(q); a.scale_b = scale;
  a.M = (int)T; a.N = (int)N; a.K = (int)K;
  a.ksplit = stem_quant_decode_slices((int)N, (int)K, QUANT_WS, (int)T);
  a.ws = c->quant_ws; a.tickets = c->tickets;
  return a;
}

// The tokens of a decode product from rows x: in place, or quantised by a kernel before it (which clears `words` words too)
hipError_t decode_tokens(stem_ctx* c, const void* x, int64_t K, const stem_norm* norm, bool in_place, uint32_t* clear, int64_t words,
                         QuantDecodeArgs& a, hipStream_t s) {
  if (in_place && stem_quant_decode_inline(a.M, K)) {
    a.x = static_cast<const bf16_t*>(x);
    a.row_K = (int)K;
    a.norm = norm ? *norm : stem_norm{STEM_NORM_NONE, 0.f, nullptr};
    return hipSuccess;
  }
  a.A = c->quant_x; a.scale_a = c->quant_sx;
  return quant_rows(c, K_QUANT_ROWS, x, a.M, K, norm, false, c->quant_x, c->quant_sx, clear, words, s);
}

}  // namespace

extern "C" {

stem_status stem_block_enter_forward(stem_ctx* c, const void* x, int64_t T, const stem_norm* norm, void* n, void* stream) {
  static const char who[] = "stem_block_enter_forward";
  STEM_TRY(stem_enter(c, T));
  if (T == 0) return STEM_OK;
  if (!x || !norm || !n) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  STEM_TRY(check_width(c, who));
  STEM_TRY(check_norm(c, who, *norm));
  if (norm->kind == STEM_NORM_NONE) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: no norm", who);
  const size_t es = type_bytes(c), row = c->desc.d_model * es;
  STEM_TRY(check_buffers(c, who, {{x, T * row}}, {{n, T * row}}, true));
  STEM_TRY(check_buffers(c, who, {{norm->weight, row}}, {{n, T * row}}, false));
  BlockArgs a = block_args(c, T);
  a.x = x; a.n = n; a.next = *norm;
  HIP_TRY(c, stem_block_forward_launch(c, c->desc.dtype == STEM_BF16, false, a, static_cast<hipStream_t>(stream)));
  return STEM_OK;
}

stem_status stem_block_enter_backward(stem_ctx* c, const void* dn, const void* x, int64_t T, const stem_norm* norm, const void* dres, void* dx,
                                      float* dw, int accumulate, void* stream) {
  static const char who[] = "stem_block_enter_backward";
  STEM_TRY(stem_enter(c, T));
  if (T == 0) return no_tokens(c, who, {dw}, accumulate, stream);
  if (!dn || !x || !norm || !dx) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  STEM_TRY(check_width(c, who));
  STEM_TRY(check_norm(c, who, *norm));
  if (norm->kind == STEM_NORM_NONE) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: no norm", who);
  const size_t es = type_bytes(c), row = c->desc.d_model * es, sum = c->desc.d_model * 4;
  STEM_TRY(check_buffers(c, who, {{dn, T * row}, {x, T * row}, {dres, T * row}}, {{dx, T * row}}, true));
  STEM_TRY(check_buffers(c, who, {{dn, T * row}, {x, T * row}, {dres, T * row}}, {{dw, sum}}, false));
  STEM_TRY(check_buffers(c, who, {{norm->weight, row}}, {{dx, T * row}, {dw, sum}}, false));
  BlockArgs a = block_args(c, T);
  a.dy = dres; a.dn = dn; a.x = x; a.dx = dx; a.next = *norm;
  a.part_of[0] = dw; a.accumulate = accumulate;
  HIP_TRY(c, stem_block_backward_launch(c, c->desc.dtype == STEM_BF16, false, a, static_cast<hipStream_t>(stream)));
  return STEM_OK;
}

stem_status stem_block_leave_forward(stem_ctx* c, const void* f, const void* x, int64_t T, const stem_leave* L, void* y, void* n, void* stream) {
  static const char who[] = "stem_block_leave_forward";
  STEM_TRY(stem_enter(c, T));
  if (T == 0) return STEM_OK;
  if (!f || !x || !L || !y) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  STEM_TRY(check_width(c, who));
  BlockArgs a = block_args(c, T);
  const size_t es = type_bytes(c), row = c->desc.d_model * es;
  STEM_TRY(check_leave(c, who, *L, {{y, T * row}, {n, T * row}}, &a));
  if ((L->next.kind != STEM_NORM_NONE) != (n != nullptr)) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: n and the next norm go together", who);
  const Buffer gate = {L->gate, gate_bytes(c, L->gate_kind, T, es)};
  // (a gate of another kind than [T,d] is read for every row: no output lies over it, though it may be as long as one)
  STEM_TRY(check_buffers(c, who, {{f, T * row}, {x, T * row}, L->gate_kind == STEM_GATE_FULL ? gate : Buffer{}}, {{y, T * row}, {n, T * row}}, true));
  STEM_TRY(check_buffers(c, who, {{L->out.weight, row}, {L->next.weight, row}, L->gate_kind == STEM_GATE_FULL ? Buffer{} : gate},
                         {{y, T * row}, {n, T * row}}, false));
  a.f = f; a.x = x; a.y = y; a.n = n;
  HIP_TRY(c, stem_block_forward_launch(c, c->desc.dtype == STEM_BF16, true, a, static_cast<hipStream_t>(stream)));
  return STEM_OK;
}

stem_status stem_block_leave_backward(stem_ctx* c, const void* dy, const void* dn, const void* f, const void* y, int64_t T, const stem_leave* L,
                                      void* dx, void* df, void* dgate, float* dw_out, float* dw_next, int accumulate, void* stream) {
  static const char who[] = "stem_block_leave_backward";
  STEM_TRY(stem_enter(c, T));
  if (T == 0)
    return no_tokens(c, who, {dw_out, dw_next, L && L->gate_kind == STEM_GATE_CHANNEL ? static_cast<float*>(dgate) : nullptr}, accumulate, stream);
  if (!L || (!dy && !dn)) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  STEM_TRY(check_width(c, who));
  BlockArgs a = block_args(c, T);
  const size_t es = type_bytes(c), row = c->desc.d_model * es, sum = c->desc.d_model * 4;
  const bool full = L->gate_kind == STEM_GATE_FULL;
  const size_t gate_size = gate_bytes(c, L->gate_kind, T, es);
  const Buffer gate = {L->gate, gate_size}, of_gate = {dgate, L->gate_kind == STEM_GATE_CHANNEL ? sum : gate_size};
  STEM_TRY(check_leave(c, who, *L, {{dx, T * row}, {df, T * row}, of_gate, {dw_out, sum}, {dw_next, sum}}, &a));
  if (dn && L->next.kind == STEM_NORM_NONE) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: dn without a next norm", who);
  if ((dn && !y) || (dw_next && !dn)) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: the next norm's gradients need dn and y", who);
  if (dgate && L->gate_kind == STEM_GATE_NONE) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: dgate without a gate", who);
  // dw_out is asked for: of N_out(f), also where that is f
  const bool need_f = (df && L->out.kind != STEM_NORM_NONE) || dgate || dw_out;
  if (need_f && !f) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: these gradients need f", who);
  const Buffer in_f = {need_f ? f : nullptr, T * row}, in_y = {dn ? y : nullptr, T * row}, in_dy = {dy, T * row}, in_dn = {dn, T * row};
  STEM_TRY(check_buffers(c, who, {in_dy, in_dn, in_f, in_y, full ? gate : Buffer{}}, {{dx, T * row}, {df, T * row}, full ? of_gate : Buffer{}}, true));
  STEM_TRY(check_buffers(c, who, {{L->out.weight, row}, {L->next.weight, row}, full ? Buffer{} : gate},
                         {{dx, T * row}, {df, T * row}, of_gate, {dw_out, sum}, {dw_next, sum}}, false));
  STEM_TRY(check_buffers(c, who, {in_dy, in_dn, in_f, in_y, full ? gate : Buffer{}}, {full ? Buffer{} : of_gate, {dw_out, sum}, {dw_next, sum}}, false));
  a.dy = dy; a.dn = dn; a.f = in_f.p; a.x = y; a.dx = dx; a.df = df;
  if (L->gate_kind != STEM_GATE_CHANNEL) a.dgate = dgate;
  a.part_of[0] = dw_next; a.part_of[1] = dw_out;
  a.part_of[2] = L->gate_kind == STEM_GATE_CHANNEL ? static_cast<float*>(dgate) : nullptr;
  a.accumulate = accumulate;
  HIP_TRY(c, stem_block_backward_launch(c, c->desc.dtype == STEM_BF16, true, a, static_cast<hipStream_t>(stream)));
  return STEM_OK;
}

stem_status stem_dropout(stem_ctx* c, const void* x, int64_t T, int64_t width, const stem_drop* drop, void* y, void* stream) {
  static const char who[] = "stem_dropout";
  STEM_TRY(stem_enter(c, T));
  if (width < 0 || width > INT32_MAX || (width > 0 && T > (1ll << 40) / width))
    return stem_fail(c, STEM_ERR_SHAPE, "%s: rows of %lld elements", who, (long long)width);
  if (T == 0 || width == 0) return STEM_OK;
  if (!x || !drop || !y) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  DropArgs d;
  const size_t bytes = (size_t)T * width * type_bytes(c);
  STEM_TRY(check_drop(c, who, *drop, {{y, bytes}}, &d));
  STEM_TRY(check_buffers(c, who, {{x, bytes}}, {{y, bytes}}, true));
  HIP_TRY(c, stem_dropout_launch(c, c->desc.dtype == STEM_BF16, x, T, width, d, y, static_cast<hipStream_t>(stream)));
  return STEM_OK;
}

int64_t stem_quant_bytes(int64_t N, int64_t K) { return N < 1 || K < 1 ? 0 : stem_quant_size(N, K); }

stem_status stem_quant_weights(stem_ctx* c, const void* W, int64_t N, int64_t K, void* q, float* scale, void* stream) {
  static const char who[] = "stem_quant_weights";
  STEM_TRY(stem_enter(c, 0));
  if (c->desc.dtype != STEM_BF16) return stem_fail(c, STEM_ERR_UNSUPPORTED, "%s: needs a bf16 context", who);
  if (N < 1 || K < 1 || K > QUANT_MAX_K || stem_quant_size(N, K) > INT32_MAX)
    return stem_fail(c, STEM_ERR_SHAPE, "%s: a matrix [%lld, %lld]; K is up to %lld and the 8-bit form below 2^31 bytes", who, (long long)N, (long long)K,
                     (long long)QUANT_MAX_K);
  if (!W || !q || !scale) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  STEM_TRY(check_buffers(c, who, {{W, (size_t)(N * K * 2)}}, {{q, (size_t)stem_quant_size(N, K)}, {scale, (size_t)N * 4}}, false));
  HIP_TRY(c, quant_rows(c, K_QUANT_WEIGHTS, W, N, K, nullptr, true, static_cast<int8_t*>(q), scale, nullptr, 0, static_cast<hipStream_t>(stream)));
  return STEM_OK;
}

stem_status stem_quant_linear(stem_ctx* c, const void* x, int64_t T, int64_t K, const stem_norm* norm, const void* q, const float* scale, int64_t N,
                              const void* residual, void* y, void* stream) {
  static const char who[] = "stem_quant_linear";
  STEM_TRY(stem_enter(c, T));
  STEM_TRY(check_quant(c, who));
  const int64_t most = std::min<int64_t>(std::max(c->desc.d_model, c->desc.d_ff), QUANT_MAX_K);
  if (N < 1 || N > QUANT_MAX_CHANNELS || K < 1 || K > most || stem_quant_size(N, K) > INT32_MAX || stem_quant_size(std::max<int64_t>(T, 1), K) > INT32_MAX)
    return stem_fail(c, STEM_ERR_SHAPE, "%s: a product [%lld, %lld] x [%lld, %lld]^T; K is up to %lld here, N up to 2^22 and each "
                     "operand's 8-bit form below 2^31 bytes", who, (long long)T, (long long)K, (long long)N, (long long)K, (long long)most);
  if (T == 0) return STEM_OK;
  if (!x || !q || !scale || !y) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  if (norm) STEM_TRY(check_norm(c, who, *norm));
  const size_t xb = (size_t)T * K * 2, yb = (size_t)T * N * 2;
  STEM_TRY(check_buffers(c, who, {{residual, yb}}, {{y, yb}}, true));
  STEM_TRY(check_buffers(c, who, {{q, (size_t)stem_quant_size(N, K)}, {scale, (size_t)N * 4}, {norm ? norm->weight : nullptr, (size_t)K * 2}},
                         {{y, yb}}, false));
  STEM_TRY(check_buffers(c, who, {{x, xb}}, {}, false));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (T <= STEM_QUANT_DECODE_TOKENS) {
    QuantDecodeArgs a = decode_args(c, T, N, stem_quant_pitch(K), q, scale);
    a.y = static_cast<bf16_t*>(y); a.residual = static_cast<const bf16_t*>(residual);
    // (in place every workgroup reads x, also when others have written their part of y)
    HIP_TRY(c, decode_tokens(c, x, K, norm, !overlap({x, xb}, {y, yb}), nullptr, 0, a, s));
    HIP_TRY(c, stem_quant_decode_launch(c, K_QUANT_DOWN, a, s));
    return STEM_OK;
  }
  HIP_TRY(c, quant_rows(c, K_QUANT_ROWS, x, T, K, norm, false, c->quant_x, c->quant_sx, nullptr, 0, s));
  QuantGemmArgs g = gemm_args(c);
  g.A = c->quant_x; g.scale_a = c->quant_sx;
  g.B = static_cast<const int8_t*>(q); g.scale_b = scale;
  g.M = (int)T; g.N = (int)N; g.K = (int)stem_quant_pitch(K);
  g.y = static_cast<bf16_t*>(y); g.residual = static_cast<const bf16_t*>(residual);
  HIP_TRY(c, stem_quant_gemm_launch(c, K_QUANT_DOWN, g, s));
  return STEM_OK;
}

stem_status stem_quant_ffn_forward(stem_ctx* c, const void* x, const int32_t* ids, int64_t T, const stem_norm* norm, const void* gate_q,
                                   const float* gate_scale, const void* down_q, const float* down_scale, const void* E, int64_t E_rows,
                                   const void* residual, void* y, void* stream) {
  static const char who[] = "stem_quant_ffn_forward";
  STEM_TRY(stem_enter(c, T));
  STEM_TRY(check_quant(c, who));
  if (T == 0) return STEM_OK;
  if (!x || !ids || !gate_q || !gate_scale || !down_q || !down_scale || !E || !y)
    return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  if (E_rows < 1 || E_rows > INT32_MAX) return stem_fail(c, STEM_ERR_SHAPE, "%s: E_rows = %lld", who, (long long)E_rows);
  if (norm) STEM_TRY(check_norm(c, who, *norm));
  const int64_t d = c->desc.d_model, F = c->desc.d_ff;
  if (std::max(d, F) > QUANT_MAX_K) return stem_fail(c, STEM_ERR_SHAPE, "%s: d_model or d_ff is over %lld", who, (long long)QUANT_MAX_K);
  for (int64_t bytes : {stem_quant_size(T, d), stem_quant_size(T, F), stem_quant_size(F, d), stem_quant_size(d, F)})
    if (bytes > INT32_MAX) return stem_fail(c, STEM_ERR_SHAPE, "%s: %lld tokens or the weights are %lld bytes in 8 bits, 2^31 or more", who, (long long)T, (long long)bytes);
  const size_t xb = (size_t)(T * d) * 2;
  STEM_TRY(check_buffers(c, who, {{x, xb}, {residual, xb}}, {{y, xb}}, true));
  STEM_TRY(check_buffers(c, who, {{gate_q, (size_t)stem_quant_size(F, d)}, {gate_scale, (size_t)F * 4}, {down_q, (size_t)stem_quant_size(d, F)},
                                  {down_scale, (size_t)d * 4}, {norm ? norm->weight : nullptr, (size_t)d * 2}, {E, (size_t)(E_rows * F) * 2}},
                         {{y, xb}}, false));
  if (reinterpret_cast<uintptr_t>(ids) & 3u) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: ids must be 4-byte aligned", who);
  if (overlap({ids, (size_t)T * 4}, {y, xb})) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: an output lies over an input", who);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t chunk = stem_quant_chunk(F), pitch = stem_quant_pitch(F);
  if (T <= STEM_QUANT_DECODE_TOKENS) {
    QuantDecodeArgs g = decode_args(c, T, F, stem_quant_pitch(d), gate_q, gate_scale);
    g.h_out = c->quant_hidden;
    g.ids = ids; g.E = static_cast<const bf16_t*>(E); g.E_rows = (int)E_rows; g.flag = c->flag;
    QuantDecodeArgs b = decode_args(c, T, d, pitch, down_q, down_scale);
    b.y = static_cast<bf16_t*>(y); b.residual = static_cast<const bf16_t*>(residual);
    // (a slice of the hidden values is quantised in place, by what all of them come to)
    const bool hidden = T <= 8 && stem_quant_decode_inline(T, (pitch / 128 + b.ksplit - 1) / b.ksplit * 128);
    if (hidden) g.max_out = c->quant_max; else g.amax = c->quant_amax;
    HIP_TRY(c, decode_tokens(c, x, d, norm, true, hidden ? nullptr : c->quant_amax, T * QUANT_AMAX_STRIDE, g, s));
    if (!hidden && g.x) HIP_TRY(c, stem_fill_zero(c->quant_amax, T * QUANT_AMAX_STRIDE * 4, s));
    HIP_TRY(c, stem_quant_decode_launch(c, K_QUANT_GATE, g, s));
    if (hidden) {
      b.h = c->quant_hidden; b.max_in = c->quant_max; b.maxima = (int)(F / 32);
    } else {
      const QuantHiddenArgs q = {c->quant_hidden, c->quant_amax, QUANT_AMAX_STRIDE, (int)T, (int)(pitch / 32), c->quant_h, c->quant_sh};
      HIP_TRY(c, stem_quant_hidden_launch(c, q, s));
      b.A = c->quant_h; b.scale_a = c->quant_sh;
    }
    HIP_TRY(c, stem_quant_decode_launch(c, K_QUANT_DOWN, b, s));
    return STEM_OK;
  }
  HIP_TRY(c, quant_rows(c, K_QUANT_ROWS, x, T, d, norm, false, c->quant_x, c->quant_sx, c->quant_amax, T, s));
  for (int64_t t0 = 0; t0 < T; t0 += chunk) {
    const int64_t n = std::min<int64_t>(chunk, T - t0);
    QuantGemmArgs g = gemm_args(c);
    g.A = c->quant_x + t0 * stem_quant_pitch(d); g.scale_a = c->quant_sx + t0;
    g.B = static_cast<const int8_t*>(gate_q); g.scale_b = gate_scale;
    g.M = (int)n; g.N = (int)F; g.K = (int)stem_quant_pitch(d);
    g.h = c->quant_hidden; g.amax = c->quant_amax + t0;
    g.ids = ids + t0; g.E = static_cast<const bf16_t*>(E); g.E_rows = (int)E_rows; g.flag = c->flag;
    HIP_TRY(c, stem_quant_gemm_launch(c, K_QUANT_GATE, g, s));
    const QuantHiddenArgs q = {c->quant_hidden, c->quant_amax + t0, 1, (int)n, (int)(pitch / 32), c->quant_h + t0 * pitch, c->quant_sh + t0};
    HIP_TRY(c, stem_quant_hidden_launch(c, q, s));
  }
  QuantGemmArgs b = gemm_args(c);
  b.A = c->quant_h; b.scale_a = c->quant_sh;
  b.B = static_cast<const int8_t*>(down_q); b.scale_b = down_scale;
  b.M = (int)T; b.N = (int)d; b.K = (int)stem_quant_pitch(F);
  b.y = static_cast<bf16_t*>(y); b.residual = static_cast<const bf16_t*>(residual);
  HIP_TRY(c, stem_quant_gemm_launch(c, K_QUANT_DOWN, b, s));
  return STEM_OK;
}

}  // extern "C"
