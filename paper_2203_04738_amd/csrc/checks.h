// Checks of arguments that the entry points of mgrit_ops.h and mgrit_tokens.h share; host only.
#pragma once
#include <cmath>

#include "ops.h"

namespace mg {

inline bool off16(const void* p) { return ((uintptr_t)p & 15) != 0; }
inline bool off(const void* p, size_t n) { return (uintptr_t)p % n != 0; }
inline bool is_dtype(int d) { return d == MGRIT_F32 || d == MGRIT_BF16 || d == MGRIT_F16; }
inline size_t elem_bytes(int d) { return d == MGRIT_F32 ? 4 : 2; }
inline size_t up(size_t v, size_t n) { return (v + n - 1) / n * n; }
inline int code_of(hipError_t e) {
  return e == hipSuccess ? MGRIT_OK : e == TOO_LARGE ? MGRIT_E_SIZE : MGRIT_E_LAUNCH;
}

// A sequence of c.T steps, c.B rows and `width` channels (those of glr_cfg) of the dtype.
template <typename CFG>
inline int seq_check(const CFG& c, const glr_seq* q, bool out, int width) {
  if (!q || !q->data) return MGRIT_E_NULL;
  if (off(q->data, elem_bytes(c.dtype))) return MGRIT_E_ALIGN;
  if (q->stride_t < 0 || q->stride_b < 0) return MGRIT_E_SIZE;
  // the last element's offset has to be a number of bytes
  const long double last = (long double)(c.T - 1) * q->stride_t + (long double)(c.B - 1) * q->stride_b + width;
  if (last > 1e18L) return MGRIT_E_SIZE;
  if (!out) return MGRIT_OK;
  long long lo = q->stride_t, hi = q->stride_b, n = c.T;      // smaller stride and its extent
  if (c.T == 1 && c.B == 1) return MGRIT_OK;
  if (c.T == 1) return q->stride_b < width ? MGRIT_E_SIZE : MGRIT_OK;
  if (c.B == 1) return q->stride_t < width ? MGRIT_E_SIZE : MGRIT_OK;
  if (lo > hi) {
    const long long t = lo;
    lo = hi;
    hi = t;
    n = c.B;
  }
  return lo < width || hi / n < lo ? MGRIT_E_SIZE : MGRIT_OK;
}
template <typename CFG>
inline int seq_check(const CFG& c, const glr_seq* q, bool out) {
  return seq_check(c, q, out, c.H);
}

// Rows of logits.
inline int logits_check(const logits_cfg* c) {
  if (!c) return MGRIT_E_NULL;
  if (c->N < 1 || c->V < 1 || c->V > (1 << 20) || c->K < 0) return MGRIT_E_SIZE;
  if ((long long)c->N * 33 > 0x7fffffffLL) return MGRIT_E_SIZE;                 // segments of all rows
  if (c->ld < c->V || c->ld > (1LL << 40)) return MGRIT_E_SIZE;
  if (!is_dtype(c->dtype)) return MGRIT_E_ENUM;
  // (the exponents' factor log2(e) / t has to be a float)
  if (!std::isfinite(c->temperature) || c->temperature <= 0.f || !std::isfinite(LOG2E * (1.0f / c->temperature)))
    return MGRIT_E_SIZE;
  return MGRIT_OK;
}
inline int logits_space(const logits_cfg& c, const void* ws, size_t n) {
  const size_t need = logits_workspace(c);
  if (n < need) return MGRIT_E_WORKSPACE;
  if (need && !ws) return MGRIT_E_NULL;
  return need && off16(ws) ? MGRIT_E_ALIGN : MGRIT_OK;
}

}  // namespace mg
