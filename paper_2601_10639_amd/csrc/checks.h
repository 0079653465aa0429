// What entry points check their arguments with (api_block.hip, api_qfloat.hip, api_experts.hip).
#pragma once
#include <math.h>

#include <initializer_list>

#include "stem_internal.h"

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

struct Buffer { const void* p; size_t bytes; };

inline bool overlap(const Buffer& a, const Buffer& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && x < y + b.bytes && y < x + a.bytes;
}

// Alignment of all buffers; no output over another, nor over an input unless `in_place` and it is that input.
inline stem_status check_buffers(stem_ctx* c, const char* who, std::initializer_list<Buffer> in, std::initializer_list<Buffer> out, bool in_place) {
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

inline stem_status check_norm(stem_ctx* c, const char* who, const stem_norm& n) {
  if (n.kind != STEM_NORM_NONE && n.kind != STEM_NORM_RMS && n.kind != STEM_NORM_LAYER)
    return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: %d is not a stem_norm_kind", who, n.kind);
  if (n.kind != STEM_NORM_NONE && !(n.eps >= 0.f && n.eps < INFINITY))
    return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: eps = %g", who, (double)n.eps);
  return STEM_OK;
}

// Arrays of 4-byte elements may begin at any of them.
inline stem_status check_words(stem_ctx* c, const char* who, std::initializer_list<const void*> list) {
  for (const void* p : list)
    if (reinterpret_cast<uintptr_t>(p) & 3u) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: integers, offsets and weights must be 4-byte aligned", who);
  return STEM_OK;
}
// No output over anything
inline stem_status check_apart(stem_ctx* c, const char* who, std::initializer_list<Buffer> in, std::initializer_list<Buffer> out) {
  for (const Buffer* o = out.begin(); o != out.end(); ++o) {
    for (const Buffer& i : in)
      if (overlap(*o, i)) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: an output lies over an input", who);
    for (const Buffer* other = out.begin(); other != o; ++other)
      if (overlap(*o, *other)) return stem_fail(c, STEM_ERR_INVALID_ARG, "%s: an output lies over another", who);
  }
  return STEM_OK;
}
