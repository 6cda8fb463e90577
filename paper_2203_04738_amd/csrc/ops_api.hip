// C ABI of the operators around a gated linear recurrent layer (include/mgrit_ops.h): arguments are checked on the
// host before anything is launched.
#include <cmath>

#include "ops.h"

namespace mg {

static bool off16(const void* p) { return ((uintptr_t)p & 15) != 0; }
static bool off(const void* p, size_t n) { return (uintptr_t)p % n != 0; }
static bool is_dtype(int d) { return d == MGRIT_F32 || d == MGRIT_BF16 || d == MGRIT_F16; }
static size_t elem_bytes(int d) { return d == MGRIT_F32 ? 4 : 2; }
static size_t up(size_t v, size_t n) { return (v + n - 1) / n * n; }
static int code_of(hipError_t e) {
  return e == hipSuccess ? MGRIT_OK : e == TOO_LARGE ? MGRIT_E_SIZE : MGRIT_E_LAUNCH;
}

// ---- gated linear recurrence
static int glr_sizes(const glr_cfg* c) {
  if (!c) return MGRIT_E_NULL;
  if (c->T < 1 || c->B < 1 || c->H < 1) return MGRIT_E_SIZE;
  if ((long long)c->T * c->B > (1LL << 30) || (long long)c->B * c->H > (1LL << 30)) return MGRIT_E_SIZE;
  if (c->form != GLR_MIX && c->form != GLR_DECAY) return MGRIT_E_ENUM;
  return is_dtype(c->dtype) ? MGRIT_OK : MGRIT_E_ENUM;
}
// Sequences: the tiles, and the threads that clear their words, are one launch each.
static int glr_check(const glr_cfg* c) {
  const int rc = glr_sizes(c);
  if (rc) return rc;
  for (int backward = 0; backward < 2; ++backward) {
    const GlrShape s = glr_shape(*c, backward);
    if (!launchable((long long)s.chunks * s.cols * c->B, GLR_WAVES * 64) || !launchable((s.words + 511) / 512, 256))
      return MGRIT_E_SIZE;
  }
  return MGRIT_OK;
}
static int seq_check(const glr_cfg& c, const glr_seq* q, bool out) {
  if (!q || !q->data) return MGRIT_E_NULL;
  if (off(q->data, elem_bytes(c.dtype))) return MGRIT_E_ALIGN;
  if (q->stride_t < 0 || q->stride_b < 0) return MGRIT_E_SIZE;
  // the last element's offset has to be a number of bytes
  const long double last = (long double)(c.T - 1) * q->stride_t + (long double)(c.B - 1) * q->stride_b + c.H;
  if (last > 1e18L) return MGRIT_E_SIZE;
  if (!out) return MGRIT_OK;
  long long lo = q->stride_t, hi = q->stride_b, n = c.T;      // smaller stride and its extent
  if (c.T == 1 && c.B == 1) return MGRIT_OK;
  if (c.T == 1) return q->stride_b < c.H ? MGRIT_E_SIZE : MGRIT_OK;
  if (c.B == 1) return q->stride_t < c.H ? MGRIT_E_SIZE : MGRIT_OK;
  if (lo > hi) {
    const long long t = lo;
    lo = hi;
    hi = t;
    n = c.B;
  }
  return lo < c.H || hi / n < lo ? MGRIT_E_SIZE : MGRIT_OK;
}
static size_t glr_ws(const GlrShape& s) { return s.words ? 256 + 8 * (size_t)s.words : 0; }
static size_t glr_save(const glr_cfg& c) { return 4 * (size_t)glr_shape(c, true).chunks * c.B * c.H; }
static size_t glr_ws(const glr_cfg& c) {
  const size_t f = glr_ws(glr_shape(c, false)), b = glr_ws(glr_shape(c, true));
  return f > b ? f : b;
}
static bool glr_past(const glr_cfg& c, bool backward) {
  return results_past_caches((backward ? 2.0 : 1.0) * elem_bytes(c.dtype) * c.T * c.B * c.H, backward ? 95e6 : 45e6,
                             c.dtype == MGRIT_F32 ? 150e6 : 1e300);
}
static int glr_space(const glr_cfg& c, const GlrShape& s, void* ws, size_t n, GlrArgs* a) {
  const size_t need = glr_ws(c);
  if (n < need) return MGRIT_E_WORKSPACE;
  if (need && !ws) return MGRIT_E_NULL;
  if (need && off16(ws)) return MGRIT_E_ALIGN;
  a->c = c;
  a->s = s;
  a->save = glr_shape(c, true).steps;
  a->past = false;
  a->ticket = (int*)ws;
  a->words = need ? (unsigned long long*)((char*)ws + 256) : nullptr;
  return MGRIT_OK;
}

// ---- rows of logits
static int logits_check(const logits_cfg* c) {
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
static int logits_space(const logits_cfg& c, const void* ws, size_t n) {
  const size_t need = logits_workspace(c);
  if (n < need) return MGRIT_E_WORKSPACE;
  if (need && !ws) return MGRIT_E_NULL;
  return need && off16(ws) ? MGRIT_E_ALIGN : MGRIT_OK;
}
static int distill_check(const logits_cfg* c, const void* logits, const int64_t* ids, const float* teacher,
                         const float* weight, const void* dlogits) {
  const int rc = logits_check(c);
  if (rc) return rc;
  if (c->K < 1 || c->K > DISTILL_MAX_K) return MGRIT_E_SIZE;
  if (!logits || !ids || !teacher) return MGRIT_E_NULL;
  if (dlogits && (c->ld_grad < c->V || c->ld_grad > (1LL << 40))) return MGRIT_E_SIZE;
  if (dlogits == logits && c->ld_grad != c->ld) return MGRIT_E_SIZE;
  const size_t e = elem_bytes(c->dtype);
  if (off(logits, e) || off(dlogits, e) || off(ids, 8) || off(teacher, 4) || off(weight, 4)) return MGRIT_E_ALIGN;
  return MGRIT_OK;
}

// ---- product in 8-bit integers
static int q8_check(const q8_cfg* c, bool product) {
  if (!c) return MGRIT_E_NULL;
  if (c->M < 1 || c->K < 1 || c->K > 131072) return MGRIT_E_SIZE;
  if (c->ldx < c->K || c->ldx > (1LL << 40)) return MGRIT_E_SIZE;
  if (!is_dtype(c->dtype)) return MGRIT_E_ENUM;
  if (!product) return MGRIT_OK;
  if (c->N < 1 || c->ldy < c->N || c->ldy > (1LL << 40)) return MGRIT_E_SIZE;
  if ((((long long)c->M + 15) / 16) * (((long long)c->N + 15) / 16) > 0x7fffffffLL) return MGRIT_E_SIZE;
  return MGRIT_OK;
}
static size_t q8_scales(const q8_cfg& c) { return up(4 * (size_t)c.M, 256); }

}  // namespace mg

using namespace mg;

extern "C" {

int glr_workspace_bytes(const glr_cfg* cfg, size_t* bytes) {
  const int rc = glr_check(cfg);
  if (rc) return rc;
  if (!bytes) return MGRIT_E_NULL;
  *bytes = glr_ws(*cfg);
  return MGRIT_OK;
}
int glr_saved_bytes(const glr_cfg* cfg, size_t* bytes) {
  const int rc = glr_check(cfg);
  if (rc) return rc;
  if (!bytes) return MGRIT_E_NULL;
  *bytes = glr_save(*cfg);
  return MGRIT_OK;
}

int glr_forward(const glr_cfg* cfg, const glr_seq* gate, const glr_seq* value, const float* h0,
                const uint8_t* reset, const glr_seq* h, float* h_last, void* saved, size_t saved_bytes,
                void* workspace, size_t workspace_bytes, void* stream) {
  int rc = glr_check(cfg);
  if (rc) return rc;
  const glr_seq* in[2] = {gate, value};
  for (const glr_seq* q : in)
    if ((rc = seq_check(*cfg, q, false))) return rc;
  if ((rc = seq_check(*cfg, h, true))) return rc;
  if (off(h0, 4) || off(h_last, 4) || off16(saved)) return MGRIT_E_ALIGN;
  GlrArgs a{};
  const GlrShape s = glr_shape(*cfg, false);
  if ((rc = glr_space(*cfg, s, workspace, workspace_bytes, &a))) return rc;
  if (saved && saved_bytes < glr_save(*cfg)) return MGRIT_E_WORKSPACE;
  a.gate = *gate;
  a.value = *value;
  a.h = *h;
  a.h0 = h0;
  a.reset = reset;
  a.h_last = h_last;
  a.saved = (float*)saved;
  a.past = glr_past(*cfg, false);
  (void)hipGetLastError();   // an error left by earlier, unrelated work is not this call's
  return code_of(launch_glr_forward(a, (hipStream_t)stream));
}

int glr_backward(const glr_cfg* cfg, const glr_seq* gate, const glr_seq* value, const uint8_t* reset,
                 const void* saved, size_t saved_bytes, const glr_seq* dh, const float* dh_last,
                 const glr_seq* dgate, const glr_seq* dvalue, float* dh0, void* workspace,
                 size_t workspace_bytes, void* stream) {
  int rc = glr_check(cfg);
  if (rc) return rc;
  const glr_seq* in[3] = {gate, value, dh};
  for (const glr_seq* q : in)
    if ((rc = seq_check(*cfg, q, false))) return rc;
  if ((rc = seq_check(*cfg, dgate, true)) || (rc = seq_check(*cfg, dvalue, true))) return rc;
  if (!saved) return MGRIT_E_NULL;
  if (off16(saved) || off(dh_last, 4) || off(dh0, 4)) return MGRIT_E_ALIGN;
  GlrArgs a{};
  const GlrShape s = glr_shape(*cfg, true);
  if ((rc = glr_space(*cfg, s, workspace, workspace_bytes, &a))) return rc;
  if (saved_bytes < glr_save(*cfg)) return MGRIT_E_WORKSPACE;
  a.gate = *gate;
  a.value = *value;
  a.dh = *dh;
  a.dgate = *dgate;
  a.dvalue = *dvalue;
  a.reset = reset;
  a.saved = (float*)const_cast<void*>(saved);
  a.dh_last = dh_last;
  a.dh0 = dh0;
  a.past = glr_past(*cfg, true);
  (void)hipGetLastError();
  return code_of(launch_glr_backward(a, (hipStream_t)stream));
}

int glr_step(const glr_cfg* cfg, const glr_seq* gate, const glr_seq* value, const int32_t* slots,
             int32_t n_slots, const uint8_t* reset, const float* state_in, float* state_out, const glr_seq* h,
             void* stream) {
  int rc = glr_sizes(cfg);
  if (rc) return rc;
  if (cfg->T != 1 || n_slots < 1 || (!slots && n_slots < cfg->B)) return MGRIT_E_SIZE;
  glr_seq rows[3] = {};                               // gate, value, h
  const glr_seq* given[3] = {gate, value, h};
  for (int i = 0; i < 3; ++i) {
    if (given[i]) rows[i] = *given[i];
    rows[i].stride_t = 0;
    if ((rc = seq_check(*cfg, &rows[i], i == 2))) return rc;
  }
  if (!state_in || !state_out) return MGRIT_E_NULL;
  if (off(state_in, 4) || off(state_out, 4) || off(slots, 4)) return MGRIT_E_ALIGN;
  GlrStepArgs a{*cfg, rows[0], rows[1], rows[2], slots, n_slots, reset, state_in, state_out};
  (void)hipGetLastError();
  return code_of(launch_glr_step(a, (hipStream_t)stream));
}

int logits_workspace_bytes(const logits_cfg* cfg, size_t* bytes) {
  const int rc = logits_check(cfg);
  if (rc) return rc;
  if (!bytes) return MGRIT_E_NULL;
  *bytes = logits_workspace(*cfg);
  return MGRIT_OK;
}

int token_logprobs(const logits_cfg* cfg, const void* logits, const int64_t* tokens, float* logp,
                   float* entropy, float* top_logp, int64_t* top_ids, void* workspace, size_t workspace_bytes,
                   void* stream) {
  int rc = logits_check(cfg);
  if (rc) return rc;
  if (cfg->K > LOGPROBS_MAX_K || cfg->K > cfg->V) return MGRIT_E_SIZE;
  if (!logits || !tokens != !logp) return MGRIT_E_NULL;
  if ((cfg->K > 0) != (top_logp != nullptr) || (cfg->K > 0) != (top_ids != nullptr)) return MGRIT_E_NULL;
  if (off(logits, elem_bytes(cfg->dtype)) || off(tokens, 8) || off(logp, 4) || off(entropy, 4) ||
      off(top_logp, 4) || off(top_ids, 8))
    return MGRIT_E_ALIGN;
  if ((rc = logits_space(*cfg, workspace, workspace_bytes))) return rc;
  LogitsArgs a{};
  a.c = *cfg;
  a.logits = logits;
  a.ids = tokens;
  a.logp = logp;
  a.entropy = entropy;
  a.top_logp = top_logp;
  a.top_ids = top_ids;
  a.workspace = (char*)workspace;
  (void)hipGetLastError();
  return code_of(launch_token_logprobs(a, (hipStream_t)stream));
}

int distill_topk(const logits_cfg* cfg, const void* logits, const int64_t* ids, const float* teacher,
                 const float* weight, float* loss, float* stats, void* dlogits, void* workspace,
                 size_t workspace_bytes, void* stream) {
  int rc = distill_check(cfg, logits, ids, teacher, weight, dlogits);
  if (rc) return rc;
  if (!loss) return MGRIT_E_NULL;
  if (off(loss, 4) || off(stats, 4)) return MGRIT_E_ALIGN;
  if ((rc = logits_space(*cfg, workspace, workspace_bytes))) return rc;
  LogitsArgs a{};
  a.c = *cfg;
  a.logits = logits;
  a.ids = ids;
  a.teacher = teacher;
  a.weight = weight;
  a.loss = loss;
  a.stats = stats;
  a.dlogits = dlogits;
  a.workspace = (char*)workspace;
  (void)hipGetLastError();
  return code_of(launch_distill(a, (hipStream_t)stream));
}

int distill_topk_backward(const logits_cfg* cfg, const void* logits, const int64_t* ids, const float* teacher,
                          const float* stats, const float* dloss, void* dlogits, void* stream) {
  const int rc = distill_check(cfg, logits, ids, teacher, dloss, dlogits);
  if (rc) return rc;
  if (!stats || !dlogits) return MGRIT_E_NULL;
  if (off(stats, 4)) return MGRIT_E_ALIGN;
  LogitsArgs a{};
  a.c = *cfg;
  a.logits = logits;
  a.ids = ids;
  a.teacher = teacher;
  a.weight = dloss;
  a.stats_in = stats;
  a.dlogits = dlogits;
  (void)hipGetLastError();
  return code_of(launch_distill_grad(a, (hipStream_t)stream));
}

int64_t q8_row_bytes(int32_t K) { return ((int64_t)K + 127) / 128 * 128; }

int q8_workspace_bytes(const q8_cfg* cfg, size_t* bytes) {
  const int rc = q8_check(cfg, true);
  if (rc) return rc;
  if (!bytes) return MGRIT_E_NULL;
  *bytes = q8_scales(*cfg) + (size_t)cfg->M * q8_row_bytes(cfg->K);
  return MGRIT_OK;
}

int q8_quantize(const q8_cfg* cfg, const void* x, int8_t* q, float* scale, void* stream) {
  const int rc = q8_check(cfg, false);
  if (rc) return rc;
  if (!x || !q || !scale) return MGRIT_E_NULL;
  if (off(x, elem_bytes(cfg->dtype)) || off16(q) || off(scale, 4)) return MGRIT_E_ALIGN;
  Q8Args a{};
  a.c = *cfg;
  a.x = x;
  a.q = q;
  a.scale = scale;
  (void)hipGetLastError();
  return code_of(launch_q8_quantize(a, (hipStream_t)stream));
}

int q8_linear(const q8_cfg* cfg, const void* x, const int8_t* w_q, const float* w_scale, const float* bias,
              void* y, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = q8_check(cfg, true);
  if (rc) return rc;
  if (!x || !w_q || !w_scale || !y || !workspace) return MGRIT_E_NULL;
  const size_t e = elem_bytes(cfg->dtype);
  if (off(x, e) || off(y, e) || off16(w_q) || off(w_scale, 4) || off(bias, 4) || off16(workspace))
    return MGRIT_E_ALIGN;
  if (workspace_bytes < q8_scales(*cfg) + (size_t)cfg->M * q8_row_bytes(cfg->K)) return MGRIT_E_WORKSPACE;
  Q8Args a{};
  a.c = *cfg;
  a.x = x;
  a.w = w_q;
  a.w_scale = w_scale;
  a.bias = bias;
  a.y = y;
  a.scale = (float*)workspace;
  a.q = (int8_t*)workspace + q8_scales(*cfg);
  a.past = results_past_caches((double)e * cfg->M * cfg->N, 95e6);
  (void)hipGetLastError();
  return code_of(launch_q8_linear(a, (hipStream_t)stream));
}

}  // extern "C"
