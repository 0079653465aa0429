// Entry points of the products in 8-bit floating point: argument checks and launch sequences (qfloat.hip, gemm_qfloat.hip).
#include <algorithm>

#include "checks.h"
#include "qfloat.h"

namespace {

constexpr stem_norm no_norm = {STEM_NORM_NONE, 0.f, nullptr};
constexpr int64_t MAX_CHANNELS = 1 << 22;
// The layer of up to 16 rows, 8 by groups: its gate product leaves fp32 hidden values, of which every workgroup of the down product makes its operands where they are few,
// else a kernel between the two.  More rows: tiles of the gate product leave 8 bits.  us, the whole layer, hidden values inline / by a kernel: 2048 x 8192, 1, 4, 8 rows
// 13.5 / 17.4, 16.7 / 18.1, 20.1 / 18.1; 1024 x 4096 8.4 / 11.8 at one row, 11.5 / 12.3 at 8, 16.6 / 14.3 at 16.  In a graph of 16 layers, by tiles / by fp32 hidden values:
// 512 x 1536 9 rows 13.3 / 10.7, 16 rows 13.4 / 11.6; 1024 x 4096 15.4 / 14.4 and 15.5 / 14.7; 2048 x 8192 24.0 / 22.7 and 24.2 / 23.4.
constexpr int64_t GATE_ROWS = 16, GATE_ROWS_GROUPS = 8, HIDDEN_INLINE = 32768;
constexpr int64_t MAX_FORM = INT32_MAX;   // elements of a form, which kernels address with 32 bits

int64_t widest(const stem_ctx* c) { return std::max(c->desc.d_model, c->desc.d_ff); }

stem_status check_context(stem_ctx* c, const char* who, int groups, bool backward) {
  if (c->desc.dtype != STEM_BF16) return stem_fail(c, STEM_ERR_UNSUPPORTED, "%s: needs a bf16 context", who);
  if (groups < 1 || groups > STEM_EXPERTS_MAX) return stem_fail(c, STEM_ERR_SHAPE, "%s: %d groups; 1 to %d", who, groups, STEM_EXPERTS_MAX);
  if (groups > c->qfloat_groups || (backward && !c->qfloat_backward))
    return stem_fail(c, STEM_ERR_WORKSPACE, "%s: needs stem_qfloat_reserve(ctx, %d or more, %d)", who, groups, backward ? 1 : 0);
  return STEM_OK;
}

stem_status check_form(stem_ctx* c, const char* who, int64_t rows, int64_t K) {
  if (stem_qfloat_size(rows, K) > MAX_FORM)
    return stem_fail(c, STEM_ERR_SHAPE, "%s: an operand of %lld rows (padded) by %lld is 2^31 bytes or more in 8 bits", who, (long long)rows, (long long)K);
  return STEM_OK;
}

stem_status check_groups(stem_ctx* c, const char* who, const int32_t* offsets, int groups) {
  if (!offsets && groups != 1) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: %d groups without offsets", who, groups);
  return check_words(c, who, {offsets});
}

struct Form { uint8_t *q, *scale; int64_t bytes; };
Form form(const void* p, int64_t rows, int64_t K) {
  uint8_t* const q = static_cast<uint8_t*>(const_cast<void*>(p));
  const int64_t bytes = stem_qfloat_size(rows, K);
  return {q, q + bytes, bytes};
}

QfloatGemmArgs gemm_args(const stem_ctx* c, const Form& a, const Form& b, int64_t stride_b, int64_t M, int64_t N, int64_t K, const QfloatGroups& g) {
  QfloatGemmArgs r = {};
  r.A = a.q; r.sa = a.scale; r.a_bytes = a.bytes;
  r.B = b.q; r.sb = b.scale; r.stride_b = stride_b;
  r.M = (int)M; r.N = (int)N; r.K = (int)stem_qfloat_pitch(K);
  r.groups = g;
  r.ws = c->qfloat_ws; r.ws_bytes = QFLOAT_WS; r.tickets = c->tickets;
  return r;
}

hipError_t rows_form(stem_ctx* c, const void* x, const QfloatGroups& g, int64_t K, const stem_norm* norm, const Form& f, hipStream_t s) {
  const QfloatRowsArgs a = {static_cast<const bf16_t*>(x), nullptr, g, (int)K, norm ? *norm : no_norm, f.q, f.scale};
  return stem_qfloat_rows_launch(c, a, s);
}

QfloatDecodeArgs decode_args(const Form& b, int64_t stride_b, int64_t N, int64_t K, const QfloatGroups& g) {
  QfloatDecodeArgs r = {};
  r.B = b.q; r.sb = b.scale; r.stride_b = stride_b;
  r.N = (int)N; r.K = (int)stem_qfloat_pitch(K); r.row_K = (int)K;
  r.groups = g;
  return r;
}

// The rows of a decode product: in place, or their form, which a kernel makes before it
hipError_t decode_rows(stem_ctx* c, const void* x, int64_t K, const stem_norm* norm, bool in_place, const Form& f, QfloatDecodeArgs& a, hipStream_t s) {
  if (in_place && stem_qfloat_decode_inline(a.groups.T, K)) {
    a.x = static_cast<const bf16_t*>(x);
    a.norm = norm ? *norm : no_norm;
    return hipSuccess;
  }
  a.A = f.q; a.sa = f.scale; a.a_bytes = f.bytes;
  return rows_form(c, x, a.groups, K, norm, f, s);
}

// Both forms of the gradients.  rounded: dW is of values in 8 bits
stem_status linear_backward(stem_ctx* c, const char* who, bool rounded, const void* dy, const void* x, int64_t T, int64_t K, const void* qt, int64_t N,
                            int groups, const int32_t* offsets, void* dx, float* dW, int accumulate, void* stream) {
  STEM_TRY(stem_enter(c, T));
  STEM_TRY(check_context(c, who, groups, true));
  if (N < 1 || N > widest(c) || K < 1 || K > widest(c))
    return stem_fail(c, STEM_ERR_SHAPE, "%s: gradients of [%lld, %lld] x [%lld, %lld]^T; K and N are up to %lld here", who, (long long)T, (long long)K,
                     (long long)N, (long long)K, (long long)widest(c));
  const int64_t rows = stem_qfloat_rows(T, groups);
  if (dx) STEM_TRY(check_form(c, who, rows, N));
  STEM_TRY(check_form(c, who, N, K));
  if (dW && stem_qfloat_size(rows, std::max(N, K)) > MAX_FORM / 2)   // (its product addresses dy and x, or their transposes, with 32 bits)
    return stem_fail(c, STEM_ERR_SHAPE, "%s: dy or x of %lld rows (padded) by %lld is 2^31 bytes or more in bf16", who, (long long)rows, (long long)std::max(N, K));
  const size_t xb = (size_t)T * K * 2, yb = (size_t)T * N * 2, wb = (size_t)groups * N * K * 4;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (T == 0) {
    STEM_TRY(check_buffers(c, who, {}, {{dW, wb}}, false));
    if (dW && !accumulate) HIP_TRY(c, stem_fill_zero(dW, wb, s));
    return STEM_OK;
  }
  if (!dy || (dx && !qt) || (dW && !x)) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  if (!dx && !dW) return STEM_OK;
  STEM_TRY(check_groups(c, who, offsets, groups));
  const Buffer in_x = {dW ? x : nullptr, xb}, in_q = {dx ? qt : nullptr, (size_t)groups * stem_qfloat_form(K, N)};
  STEM_TRY(check_buffers(c, who, {{dy, yb}, in_x, in_q}, {{dW, wb}}, false));
  STEM_TRY(check_buffers(c, who, {in_q}, {{dx, xb}, {dW, wb}}, false));
  STEM_TRY(check_apart(c, who, {{offsets, (size_t)(groups + 1) * 4}}, {{dx, xb}, {dW, wb}}));
  const QfloatGroups g = {offsets, groups, (int)T};
  const Form f = form(c->qfloat_x, rows, N);
  const auto *g_in = static_cast<const bf16_t*>(dy), *x_in = static_cast<const bf16_t*>(x);
  // Whole matrices of aligned rows are read as they lie; others are transposed first (of dy, together with its 8-bit form)
  const bool as_stored = !rounded && groups == 1 && !offsets && N % 64 == 0 && K % 64 == 0 && wb <= INT32_MAX;
  if (dW && !as_stored) {
    HIP_TRY(c, stem_qfloat_turn_launch(c, {g_in, g, (int)N, c->qfloat_dyt, (int)rows * 2, dx ? f.q : nullptr, f.scale},
                                       {x_in, g, (int)K, c->qfloat_xt, (int)rows * 2, nullptr, nullptr}, rounded, s));
  } else if (dx) {
    HIP_TRY(c, rows_form(c, dy, g, N, nullptr, f, s));
  }
  if (dW && as_stored) {
    GemmArgs a = {};
    a.A = g_in; a.lda = (int)N;
    a.B = x_in; a.ldb = (int)K;
    a.M = (int)N; a.N = (int)K; a.K = (int)T;
    a.C = dW; a.accumulate = accumulate;
    a.ws = c->splitk_ws; a.ws_bytes = c->splitk_bytes; a.tickets = c->tickets;
    HIP_TRY(c, stem_gemm_bf16(c, K_QFLOAT_DW, OP_MC, OP_MC, EPI_F32, a, s));
  } else if (dW) {
    QfloatGemmArgs a = gemm_args(c, {c->qfloat_dyt, nullptr, stem_qfloat_pitch(N) * rows * 2}, {c->qfloat_xt, nullptr, 0}, 0, N, K, rows * 2, g);
    a.c = dW; a.accumulate = accumulate;
    HIP_TRY(c, stem_qfloat_gemm_launch(c, K_QFLOAT_DW, QFLOAT_F32, a, s));
  }
  if (dx) {
    QfloatGemmArgs a = gemm_args(c, f, form(qt, K, N), stem_qfloat_form(K, N), T, K, N, g);
    a.y = static_cast<bf16_t*>(dx);
    HIP_TRY(c, stem_qfloat_gemm_launch(c, K_QFLOAT_DX, QFLOAT_BF16, a, s));
  }
  return STEM_OK;
}

}  // namespace

extern "C" {

// All buffers that are still to be had, or none: one that was left of a call that failed would have that call's size, for a later one of more groups.
int stem_qfloat_room_take(stem_qfloat_room* r, int64_t tokens, int64_t wide, int64_t F, int groups, int backward, int (*take)(void**, int64_t), void (*give)(void*)) {
  const int most = r->groups ? r->groups : groups;
  const int64_t rows = stem_qfloat_rows(std::max<int64_t>(tokens, 1), most), turned = stem_qfloat_size(wide, rows) * 2;
  const int64_t bytes[5] = {stem_qfloat_form(rows, wide), stem_qfloat_form(rows, F), QFLOAT_WS, turned, turned};
  void* got[5] = {};
  for (int i = 0; i < (backward ? 5 : 3); ++i) {
    if (r->p[i]) continue;
    const int failed = take(&got[i], bytes[i]);
    if (!failed) continue;
    while (i--)
      if (got[i]) give(got[i]);
    return failed;
  }
  for (int i = 0; i < 5; ++i)
    if (got[i]) r->p[i] = got[i];
  r->groups = most;
  if (backward) r->backward = 1;
  return 0;
}

int64_t stem_qfloat_bytes(int64_t N, int64_t K) { return N < 1 || K < 1 ? 0 : stem_qfloat_form(N, K); }

stem_status stem_qfloat_reserve(stem_ctx* c, int groups, int backward) {
  static const char who[] = "stem_qfloat_reserve";
  STEM_TRY(stem_enter(c, 0));
  if (c->desc.dtype != STEM_BF16) return stem_fail(c, STEM_ERR_UNSUPPORTED, "%s: needs a bf16 context", who);
  if (groups < 1 || groups > STEM_EXPERTS_MAX) return stem_fail(c, STEM_ERR_SHAPE, "%s: %d groups; 1 to %d", who, groups, STEM_EXPERTS_MAX);
  if (c->qfloat_groups && groups > c->qfloat_groups)
    return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: reserved for %d groups before; the first call names the most", who, c->qfloat_groups);
  HIP_TRY(c, hipSetDevice(c->device));
  stem_qfloat_room room = {c->qfloat_groups, c->qfloat_backward, {c->qfloat_x, c->qfloat_h, c->qfloat_ws, c->qfloat_dyt, c->qfloat_xt}};
  HIP_TRY(c, static_cast<hipError_t>(stem_qfloat_room_take(
                 &room, c->max_tokens, widest(c), c->desc.d_ff, groups, backward, [](void** p, int64_t bytes) { return (int)hipMalloc(p, (size_t)bytes); },
                 [](void* p) { (void)hipFree(p); })));
  c->qfloat_x = static_cast<uint8_t*>(room.p[0]);
  c->qfloat_h = static_cast<uint8_t*>(room.p[1]);
  c->qfloat_ws = static_cast<float*>(room.p[2]);
  c->qfloat_dyt = static_cast<uint8_t*>(room.p[3]);
  c->qfloat_xt = static_cast<uint8_t*>(room.p[4]);
  c->qfloat_groups = room.groups;
  c->qfloat_backward = room.backward;
  return STEM_OK;
}

stem_status stem_qfloat_weights(stem_ctx* c, const void* W, int groups, int64_t N, int64_t K, void* q, void* qt, void* stream) {
  static const char who[] = "stem_qfloat_weights";
  STEM_TRY(stem_enter(c, 0));
  if (c->desc.dtype != STEM_BF16) return stem_fail(c, STEM_ERR_UNSUPPORTED, "%s: needs a bf16 context", who);
  if (groups < 1 || groups > STEM_EXPERTS_MAX) return stem_fail(c, STEM_ERR_SHAPE, "%s: %d groups; 1 to %d", who, groups, STEM_EXPERTS_MAX);
  if (N < 1 || K < 1 || N > MAX_CHANNELS || K > MAX_CHANNELS) return stem_fail(c, STEM_ERR_SHAPE, "%s: matrices [%lld, %lld]", who, (long long)N, (long long)K);
  STEM_TRY(check_form(c, who, N, K));
  if (!W || (!q && !qt)) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  const size_t bytes = (size_t)groups * stem_qfloat_form(N, K);
  STEM_TRY(check_buffers(c, who, {{W, (size_t)groups * N * K * 2}}, {{q, bytes}, {qt, bytes}}, false));
  const QfloatTilesArgs a = {static_cast<const bf16_t*>(W), (int)N, (int)K, groups, static_cast<uint8_t*>(q), static_cast<uint8_t*>(qt)};
  HIP_TRY(c, stem_qfloat_weights_launch(c, a, static_cast<hipStream_t>(stream)));
  return STEM_OK;
}

stem_status stem_qfloat_linear(stem_ctx* c, const void* x, int64_t T, int64_t K, const stem_norm* norm, const void* q, int64_t N, int groups,
                               const int32_t* offsets, const void* residual, void* y, void* stream) {
  static const char who[] = "stem_qfloat_linear";
  STEM_TRY(stem_enter(c, T));
  STEM_TRY(check_context(c, who, groups, false));
  if (N < 1 || N > MAX_CHANNELS || K < 1 || K > widest(c))
    return stem_fail(c, STEM_ERR_SHAPE, "%s: a product [%lld, %lld] x [%lld, %lld]^T; K is up to %lld here, N up to 2^22", who, (long long)T, (long long)K,
                     (long long)N, (long long)K, (long long)widest(c));
  const int64_t rows = stem_qfloat_rows(T, groups);
  STEM_TRY(check_form(c, who, rows, K));
  STEM_TRY(check_form(c, who, N, K));
  if (T == 0) return STEM_OK;
  if (!x || !q || !y) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  STEM_TRY(check_groups(c, who, offsets, groups));
  if (norm) STEM_TRY(check_norm(c, who, *norm));
  const size_t xb = (size_t)T * K * 2, yb = (size_t)T * N * 2;
  STEM_TRY(check_buffers(c, who, {{residual, yb}}, {{y, yb}}, true));
  STEM_TRY(check_buffers(c, who, {{q, (size_t)groups * stem_qfloat_form(N, K)}, {norm ? norm->weight : nullptr, (size_t)K * 2}}, {{y, yb}}, false));
  STEM_TRY(check_buffers(c, who, {{x, xb}}, {}, false));
  STEM_TRY(check_apart(c, who, {{offsets, (size_t)(groups + 1) * 4}}, {{y, yb}}));
  hipStream_t s = static_cast<hipStream_t>(stream);
  const QfloatGroups g = {offsets, groups, (int)T};
  const Form f = form(c->qfloat_x, rows, K);
  if (stem_route_qfloat_few(T, offsets != nullptr, (int)N, (int)K)) {
    QfloatDecodeArgs a = decode_args(form(q, N, K), stem_qfloat_form(N, K), N, K, g);
    a.y = static_cast<bf16_t*>(y); a.residual = static_cast<const bf16_t*>(residual);
    // (in place every workgroup reads x, also when others have written their part of y)
    HIP_TRY(c, decode_rows(c, x, K, norm, !overlap({x, xb}, {y, yb}), f, a, s));
    HIP_TRY(c, stem_qfloat_decode_launch(c, K_QFLOAT_LINEAR, a, s));
    return STEM_OK;
  }
  HIP_TRY(c, rows_form(c, x, g, K, norm, f, s));
  QfloatGemmArgs a = gemm_args(c, f, form(q, N, K), stem_qfloat_form(N, K), T, N, K, g);
  a.y = static_cast<bf16_t*>(y); a.residual = static_cast<const bf16_t*>(residual);
  HIP_TRY(c, stem_qfloat_gemm_launch(c, K_QFLOAT_LINEAR, QFLOAT_BF16, a, s));
  return STEM_OK;
}

stem_status stem_qfloat_linear_backward(stem_ctx* c, const void* dy, const void* x, int64_t T, int64_t K, const void* qt, int64_t N, int groups,
                                        const int32_t* offsets, void* dx, float* dW, int accumulate, void* stream) {
  return linear_backward(c, "stem_qfloat_linear_backward", false, dy, x, T, K, qt, N, groups, offsets, dx, dW, accumulate, stream);
}

stem_status stem_qfloat_linear_backward_quantised(stem_ctx* c, const void* dy, const void* x, int64_t T, int64_t K, const void* qt, int64_t N, int groups,
                                                  const int32_t* offsets, void* dx, float* dW, int accumulate, void* stream) {
  return linear_backward(c, "stem_qfloat_linear_backward_quantised", true, dy, x, T, K, qt, N, groups, offsets, dx, dW, accumulate, stream);
}

stem_status stem_qfloat_ffn_forward(stem_ctx* c, const void* x, const int32_t* ids, int64_t T, const stem_norm* norm, const void* gate_q,
                                    const void* down_q, int groups, const int32_t* offsets, const void* E, int64_t E_rows, const void* residual,
                                    void* y, void* stream) {
  static const char who[] = "stem_qfloat_ffn_forward";
  STEM_TRY(stem_enter(c, T));
  STEM_TRY(check_context(c, who, groups, false));
  if (T == 0) return STEM_OK;
  if (!x || !ids || !gate_q || !down_q || !E || !y) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: null pointer argument", who);
  if (E_rows < 1 || E_rows > INT32_MAX) return stem_fail(c, STEM_ERR_SHAPE, "%s: E_rows = %lld", who, (long long)E_rows);
  if (norm) STEM_TRY(check_norm(c, who, *norm));
  const int64_t d = c->desc.d_model, F = c->desc.d_ff, rows = stem_qfloat_rows(T, groups);
  STEM_TRY(check_form(c, who, rows, std::max(d, F)));
  STEM_TRY(check_form(c, who, F, d));
  STEM_TRY(check_form(c, who, d, F));
  STEM_TRY(check_groups(c, who, offsets, groups));
  const size_t xb = (size_t)(T * d) * 2;
  STEM_TRY(check_buffers(c, who, {{x, xb}, {residual, xb}}, {{y, xb}}, true));
  STEM_TRY(check_buffers(c, who, {{gate_q, (size_t)groups * stem_qfloat_form(F, d)}, {down_q, (size_t)groups * stem_qfloat_form(d, F)},
                                  {norm ? norm->weight : nullptr, (size_t)d * 2}, {E, (size_t)(E_rows * F) * 2}}, {{y, xb}}, false));
  STEM_TRY(check_words(c, who, {ids}));
  STEM_TRY(check_apart(c, who, {{ids, (size_t)T * 4}, {offsets, (size_t)(groups + 1) * 4}}, {{y, xb}}));
  hipStream_t s = static_cast<hipStream_t>(stream);
  const QfloatGroups g = {offsets, groups, (int)T};
  const Form f = form(c->qfloat_x, rows, d), h = form(c->qfloat_h, rows, F);
  QfloatDecodeArgs b = decode_args(form(down_q, d, F), stem_qfloat_form(d, F), d, F, g);
  b.y = static_cast<bf16_t*>(y); b.residual = static_cast<const bf16_t*>(residual);
  b.A = h.q; b.sa = h.scale; b.a_bytes = h.bytes;
  if (T <= (offsets ? GATE_ROWS_GROUPS : GATE_ROWS) && stem_qfloat_decode_inline(T, d) && T * F * 4 <= QFLOAT_WS) {
    QfloatDecodeArgs a = decode_args(form(gate_q, F, d), stem_qfloat_form(F, d), F, d, g);
    a.h_out = c->qfloat_ws;
    a.ids = ids; a.E = static_cast<const bf16_t*>(E); a.E_rows = (int)E_rows; a.flag = c->flag;
    a.x = static_cast<const bf16_t*>(x);
    a.norm = norm ? *norm : no_norm;
    HIP_TRY(c, stem_qfloat_decode_launch(c, K_QFLOAT_GATE, a, s));
    if (T * F <= HIDDEN_INLINE && stem_qfloat_decode_inline(T, F)) b.h = c->qfloat_ws;
    else HIP_TRY(c, stem_qfloat_rows_launch(c, {nullptr, c->qfloat_ws, g, (int)F, no_norm, h.q, h.scale}, s));
    HIP_TRY(c, stem_qfloat_decode_launch(c, K_QFLOAT_LINEAR, b, s));
    return STEM_OK;
  }
  HIP_TRY(c, rows_form(c, x, g, d, norm, f, s));
  QfloatGemmArgs a = gemm_args(c, f, form(gate_q, F, d), stem_qfloat_form(F, d), T, F, d, g);
  a.hq = h.q; a.hs = h.scale;
  a.ids = ids; a.E = static_cast<const bf16_t*>(E); a.E_rows = (int)E_rows; a.flag = c->flag;
  HIP_TRY(c, stem_qfloat_gemm_launch(c, K_QFLOAT_GATE, QFLOAT_HIDDEN, a, s));
  if (stem_route_qfloat_few(T, offsets != nullptr, (int)d, (int)F)) {
    HIP_TRY(c, stem_qfloat_decode_launch(c, K_QFLOAT_LINEAR, b, s));
    return STEM_OK;
  }
  a = gemm_args(c, h, form(down_q, d, F), stem_qfloat_form(d, F), T, d, F, g);
  a.y = static_cast<bf16_t*>(y); a.residual = static_cast<const bf16_t*>(residual);
  HIP_TRY(c, stem_qfloat_gemm_launch(c, K_QFLOAT_LINEAR, QFLOAT_BF16, a, s));
  return STEM_OK;
}

}  // extern "C"
