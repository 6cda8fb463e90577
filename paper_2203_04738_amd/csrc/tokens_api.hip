// C ABI of the operators of a recurrent student over tokens (include/mgrit_tokens.h): arguments are checked on the host
// before anything is launched.
#include <cmath>
#include <initializer_list>

#include "checks.h"
#include "tokens.h"

namespace mg {

// Whether a buffer that is written begins where another of the call does.
static bool begins_as(const void* out, std::initializer_list<const void*> others) {
  for (const void* p : others)
    if (out && out == p) return true;
  return false;
}

// ---- embedding
static int embed_check(const embed_cfg* c) {
  if (!c) return MGRIT_E_NULL;
  if (c->N < 1 || c->N > (1 << 26) || c->V < 1 || c->V > (1 << 20) || c->D < 1 || c->D > (1 << 20)) return MGRIT_E_SIZE;
  if (c->ld_table < c->D || c->ld_table > (1LL << 40) || c->ld_out < c->D || c->ld_out > (1LL << 40)) return MGRIT_E_SIZE;
  if (!is_dtype(c->dtype)) return MGRIT_E_ENUM;
  return std::isfinite(c->scale) ? MGRIT_OK : MGRIT_E_SIZE;
}

// ---- causal convolution
static int conv_sizes(const conv_cfg* c) {
  if (!c) return MGRIT_E_NULL;
  if (c->T < 1 || c->B < 1 || c->H < 1 || c->W < 1 || c->W > CONV_MAX_W) return MGRIT_E_SIZE;
  if ((long long)c->T * c->B > (1LL << 30) || (long long)c->B * c->H > (1LL << 30)) return MGRIT_E_SIZE;
  if (c->act != CONV_LINEAR && c->act != CONV_SILU) return MGRIT_E_ENUM;
  return is_dtype(c->dtype) ? MGRIT_OK : MGRIT_E_ENUM;
}
static int conv_check(const conv_cfg* c) {
  const int rc = conv_sizes(c);
  return rc ? rc : conv_launchable(*c) ? MGRIT_OK : MGRIT_E_SIZE;
}
static bool conv_past(const conv_cfg& c) { return results_past_caches((double)elem_bytes(c.dtype) * c.T * c.B * c.H, 95e6); }

// ---- selective state space scan
static int ssm_sizes(const ssm_cfg* c) {
  if (!c) return MGRIT_E_NULL;
  if (c->T < 1 || c->B < 1 || c->H < 1 || c->S < 1 || c->S > SSM_MAX_S) return MGRIT_E_SIZE;
  if ((long long)c->T * c->B > (1LL << 30) || (long long)c->B * c->H > (1LL << 30)) return MGRIT_E_SIZE;
  if ((long long)c->B * c->H * c->S > (1LL << 32)) return MGRIT_E_SIZE;
  return is_dtype(c->dtype) ? MGRIT_OK : MGRIT_E_ENUM;
}
static int ssm_check(const ssm_cfg* c) {
  const int rc = ssm_sizes(c);
  return rc ? rc : ssm_launchable(*c) ? MGRIT_OK : MGRIT_E_SIZE;
}
static int ssm_inputs_check(const ssm_cfg& c, const ssm_inputs* in) {
  if (!in || !in->a) return MGRIT_E_NULL;
  int rc;
  if ((rc = seq_check(c, &in->x, false)) || (rc = seq_check(c, &in->dt, false))) return rc;
  if ((rc = seq_check(c, &in->b, false, c.S)) || (rc = seq_check(c, &in->c, false, c.S))) return rc;
  if (in->z.data && (rc = seq_check(c, &in->z, false))) return rc;
  return off(in->a, 4) || off(in->skip, 4) || off(in->bias, 4) ? MGRIT_E_ALIGN : MGRIT_OK;
}
static int ssm_space(const ssm_cfg& c, const void* ws, size_t n) {
  const size_t need = ssm_workspace(c);
  if (n < need) return MGRIT_E_WORKSPACE;
  if (need && !ws) return MGRIT_E_NULL;
  return need && off16(ws) ? MGRIT_E_ALIGN : MGRIT_OK;
}
static SsmArgs ssm_args(const ssm_cfg& c, const ssm_inputs& in, const uint8_t* reset) {
  SsmArgs a{};
  a.c = c;
  a.x = in.x;
  a.dt = in.dt;
  a.b = in.b;
  a.cc = in.c;
  a.z = in.z;
  a.a = in.a;
  a.skip = in.skip;
  a.bias = in.bias;
  a.reset = reset;
  return a;
}

// ---- policy loss
static int policy_check(const logits_cfg* c, const policy_cfg* rule, const void* logits, const int64_t* tokens,
                        const float* old_logp, const float* ref_logp, const float* advantage, const float* weight,
                        const void* dlogits) {
  const int rc = logits_check(c);
  if (rc) return rc;
  if (!rule || !logits || !tokens || !old_logp || !advantage) return MGRIT_E_NULL;
  if (!(rule->clip_low >= 0.f && rule->clip_low <= 1.f) || !(rule->clip_high >= 0.f && std::isfinite(rule->clip_high)) ||
      !(rule->kl >= 0.f && std::isfinite(rule->kl)))
    return MGRIT_E_SIZE;
  if (dlogits && (c->ld_grad < c->V || c->ld_grad > (1LL << 40))) return MGRIT_E_SIZE;
  if (dlogits == logits && c->ld_grad != c->ld) return MGRIT_E_SIZE;
  const size_t e = elem_bytes(c->dtype);
  if (off(logits, e) || off(dlogits, e) || off(tokens, 8) || off(old_logp, 4) || off(ref_logp, 4) || off(advantage, 4) ||
      off(weight, 4))
    return MGRIT_E_ALIGN;
  return begins_as(dlogits, {tokens, old_logp, ref_logp, advantage, weight}) ? MGRIT_E_SIZE : MGRIT_OK;
}
static logits_cfg policy_space_cfg(const logits_cfg& c) {
  logits_cfg one = c;
  one.K = 1;
  return one;
}

}  // namespace mg

using namespace mg;

extern "C" {

int embed_lookup(const embed_cfg* cfg, const int64_t* tokens, const void* table, void* out, void* stream) {
  const int rc = embed_check(cfg);
  if (rc) return rc;
  if (!tokens || !table || !out) return MGRIT_E_NULL;
  if (off(tokens, 8) || off(table, elem_bytes(cfg->dtype)) || off(out, elem_bytes(cfg->dtype))) return MGRIT_E_ALIGN;
  if (begins_as(out, {table, tokens})) return MGRIT_E_SIZE;
  EmbedArgs a{};
  a.c = *cfg;
  a.tokens = tokens;
  a.in = table;
  a.out = out;
  (void)hipGetLastError();   // an error left by earlier, unrelated work is not this call's
  return code_of(launch_embed_lookup(a, (hipStream_t)stream));
}

int embed_workspace_bytes(const embed_cfg* cfg, size_t* bytes) {
  const int rc = embed_check(cfg);
  if (rc) return rc;
  if (!bytes) return MGRIT_E_NULL;
  *bytes = embed_workspace(*cfg);
  return MGRIT_OK;
}

int embed_backward(const embed_cfg* cfg, const int64_t* tokens, const void* dout, void* dtable, void* workspace,
                   size_t workspace_bytes, void* stream) {
  const int rc = embed_check(cfg);
  if (rc) return rc;
  if (!tokens || !dout || !dtable || !workspace) return MGRIT_E_NULL;
  if (off(tokens, 8) || off(dout, elem_bytes(cfg->dtype)) || off(dtable, elem_bytes(cfg->dtype)) || off16(workspace))
    return MGRIT_E_ALIGN;
  if (workspace_bytes < embed_workspace(*cfg)) return MGRIT_E_WORKSPACE;
  if (begins_as(dtable, {dout, tokens, workspace})) return MGRIT_E_SIZE;
  EmbedArgs a{};
  a.c = *cfg;
  a.tokens = tokens;
  a.in = dout;
  a.out = dtable;
  (void)hipGetLastError();
  return code_of(launch_embed_backward(a, (char*)workspace, (hipStream_t)stream));
}

int causal_conv_forward(const conv_cfg* cfg, const glr_seq* x, const float* weight, const float* bias,
                        const float* past, const uint8_t* reset, const glr_seq* y, float* last, void* stream) {
  int rc = conv_check(cfg);
  if (rc) return rc;
  if ((rc = seq_check(*cfg, x, false)) || (rc = seq_check(*cfg, y, true))) return rc;
  if (!weight) return MGRIT_E_NULL;
  if (off(weight, 4) || off(bias, 4) || off(past, 4) || off(last, 4)) return MGRIT_E_ALIGN;
  if (begins_as(y->data, {x->data}) || (cfg->W > 1 && begins_as(last, {past}))) return MGRIT_E_SIZE;
  ConvArgs a{};
  a.c = *cfg;
  a.x = *x;
  a.y = *y;
  a.weight = weight;
  a.bias = bias;
  a.past = past;
  a.reset = reset;
  a.last = last;
  a.past_caches = conv_past(*cfg);
  (void)hipGetLastError();
  return code_of(launch_conv_forward(a, (hipStream_t)stream));
}

int causal_conv_workspace_bytes(const conv_cfg* cfg, size_t* bytes) {
  const int rc = conv_check(cfg);
  if (rc) return rc;
  if (!bytes) return MGRIT_E_NULL;
  *bytes = conv_workspace(*cfg);
  return MGRIT_OK;
}

int causal_conv_backward(const conv_cfg* cfg, const glr_seq* x, const float* weight, const float* bias,
                         const float* past, const uint8_t* reset, const glr_seq* dy, const float* dlast,
                         const glr_seq* dx, float* dweight, float* dbias, float* dpast, void* workspace,
                         size_t workspace_bytes, void* stream) {
  int rc = conv_check(cfg);
  if (rc) return rc;
  if ((rc = seq_check(*cfg, x, false)) || (rc = seq_check(*cfg, dy, false)) || (rc = seq_check(*cfg, dx, true))) return rc;
  if (!weight || !workspace) return MGRIT_E_NULL;
  if (off(weight, 4) || off(bias, 4) || off(past, 4) || off(dlast, 4) || off(dweight, 4) || off(dbias, 4) ||
      off(dpast, 4) || off16(workspace))
    return MGRIT_E_ALIGN;
  if (workspace_bytes < conv_workspace(*cfg)) return MGRIT_E_WORKSPACE;
  if (begins_as(dx->data, {x->data, dy->data}) || (cfg->W > 1 && begins_as(dpast, {dlast, past}))) return MGRIT_E_SIZE;
  ConvArgs a{};
  a.c = *cfg;
  a.x = *x;
  a.dy = *dy;
  a.dx = *dx;
  a.weight = weight;
  a.bias = bias;
  a.past = past;
  a.reset = reset;
  a.dlast = dlast;
  a.dweight = dweight;
  a.dbias = dbias;
  a.dpast = dpast;
  a.part = (float*)workspace;
  a.past_caches = conv_past(*cfg);
  (void)hipGetLastError();
  return code_of(launch_conv_backward(a, (hipStream_t)stream));
}

int causal_conv_step(const conv_cfg* cfg, const glr_seq* x, const float* weight, const float* bias, const int32_t* slots,
                     int32_t n_slots, const uint8_t* reset, const float* past_in, float* past_out, const glr_seq* y,
                     void* stream) {
  int rc = conv_sizes(cfg);
  if (rc) return rc;
  if (cfg->T != 1 || n_slots < 1 || (!slots && n_slots < cfg->B)) return MGRIT_E_SIZE;
  glr_seq rows[2] = {};                               // x, y
  const glr_seq* given[2] = {x, y};
  for (int i = 0; i < 2; ++i) {
    if (given[i]) rows[i] = *given[i];
    rows[i].stride_t = 0;
    if ((rc = seq_check(*cfg, &rows[i], i == 1))) return rc;
  }
  if (!weight || (cfg->W > 1 && (!past_in || !past_out))) return MGRIT_E_NULL;
  if (off(weight, 4) || off(bias, 4) || off(slots, 4)) return MGRIT_E_ALIGN;
  if (cfg->W > 1 && (off(past_in, 4) || off(past_out, 4))) return MGRIT_E_ALIGN;
  if (begins_as(y->data, {x->data})) return MGRIT_E_SIZE;
  ConvStepArgs a{*cfg, rows[0], rows[1], weight, bias, slots, n_slots, reset, past_in, past_out};
  (void)hipGetLastError();
  return code_of(launch_conv_step(a, (hipStream_t)stream));
}

int ssm_workspace_bytes(const ssm_cfg* cfg, size_t* bytes) {
  const int rc = ssm_check(cfg);
  if (rc) return rc;
  if (!bytes) return MGRIT_E_NULL;
  *bytes = ssm_workspace(*cfg);
  return MGRIT_OK;
}
int ssm_saved_bytes(const ssm_cfg* cfg, size_t* bytes) {
  const int rc = ssm_check(cfg);
  if (rc) return rc;
  if (!bytes) return MGRIT_E_NULL;
  *bytes = ssm_saved(*cfg);
  return MGRIT_OK;
}

int ssm_forward(const ssm_cfg* cfg, const ssm_inputs* in, const float* h0, const uint8_t* reset, const glr_seq* y,
                float* h_last, void* saved, size_t saved_bytes, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = ssm_check(cfg);
  if (rc) return rc;
  if ((rc = ssm_inputs_check(*cfg, in)) || (rc = seq_check(*cfg, y, true))) return rc;
  if (off(h0, 4) || off(h_last, 4) || off16(saved)) return MGRIT_E_ALIGN;
  if ((rc = ssm_space(*cfg, workspace, workspace_bytes))) return rc;
  if (saved && saved_bytes < ssm_saved(*cfg)) return MGRIT_E_WORKSPACE;
  if (begins_as(y->data, {in->x.data, in->dt.data, in->b.data, in->c.data, in->z.data}) || begins_as(h_last, {h0}))
    return MGRIT_E_SIZE;
  SsmArgs a = ssm_args(*cfg, *in, reset);
  a.h0 = h0;
  a.y = *y;
  a.h_last = h_last;
  a.saved = (float*)saved;
  (void)hipGetLastError();
  return code_of(launch_ssm_forward(a, (char*)workspace, (hipStream_t)stream));
}

int ssm_backward(const ssm_cfg* cfg, const ssm_inputs* in, const uint8_t* reset, const void* saved, size_t saved_bytes,
                 const glr_seq* dy, const float* dh_last, const ssm_grads* out, void* workspace, size_t workspace_bytes,
                 void* stream) {
  int rc = ssm_check(cfg);
  if (rc) return rc;
  if ((rc = ssm_inputs_check(*cfg, in)) || (rc = seq_check(*cfg, dy, false))) return rc;
  if (!saved || !out || !out->da || !in->z.data != !out->dz.data) return MGRIT_E_NULL;
  if ((rc = seq_check(*cfg, &out->dx, true)) || (rc = seq_check(*cfg, &out->ddt, true))) return rc;
  if ((rc = seq_check(*cfg, &out->db, true, cfg->S)) || (rc = seq_check(*cfg, &out->dc, true, cfg->S))) return rc;
  if (out->dz.data && (rc = seq_check(*cfg, &out->dz, true))) return rc;
  if (off16(saved) || off(dh_last, 4) || off(out->da, 4) || off(out->dskip, 4) || off(out->dbias, 4) || off(out->dh0, 4))
    return MGRIT_E_ALIGN;
  if ((rc = ssm_space(*cfg, workspace, workspace_bytes))) return rc;
  if (saved_bytes < ssm_saved(*cfg)) return MGRIT_E_WORKSPACE;
  const void* read[] = {in->x.data, in->dt.data, in->b.data, in->c.data, in->z.data, dy->data};
  const void* written[] = {out->dx.data, out->ddt.data, out->db.data, out->dc.data, out->dz.data};
  for (int i = 0; i < 5; ++i) {
    for (const void* p : read)
      if (begins_as(written[i], {p})) return MGRIT_E_SIZE;
    for (int j = 0; j < i; ++j)
      if (begins_as(written[i], {written[j]})) return MGRIT_E_SIZE;
  }
  if (begins_as(out->dh0, {dh_last})) return MGRIT_E_SIZE;
  SsmArgs a = ssm_args(*cfg, *in, reset);
  a.saved = (float*)const_cast<void*>(saved);
  a.dy = *dy;
  a.dh_last = dh_last;
  a.dx = out->dx;
  a.ddt = out->ddt;
  a.db = out->db;
  a.dc = out->dc;
  a.dz = out->dz;
  a.da = out->da;
  a.dskip = out->dskip;
  a.dbias = out->dbias;
  a.dh0 = out->dh0;
  (void)hipGetLastError();
  return code_of(launch_ssm_backward(a, (char*)workspace, (hipStream_t)stream));
}

int ssm_step(const ssm_cfg* cfg, const ssm_inputs* in, const int32_t* slots, int32_t n_slots, const uint8_t* reset,
             const float* state_in, float* state_out, const glr_seq* y, void* stream) {
  int rc = ssm_sizes(cfg);
  if (rc) return rc;
  if (cfg->T != 1 || n_slots < 1 || (!slots && n_slots < cfg->B)) return MGRIT_E_SIZE;
  if (!in || !y) return MGRIT_E_NULL;
  ssm_inputs i = *in;
  glr_seq out = *y;
  i.x.stride_t = i.dt.stride_t = i.b.stride_t = i.c.stride_t = i.z.stride_t = out.stride_t = 0;
  if ((rc = ssm_inputs_check(*cfg, &i)) || (rc = seq_check(*cfg, &out, true))) return rc;
  if (!state_in || !state_out) return MGRIT_E_NULL;
  if (off(state_in, 4) || off(state_out, 4) || off(slots, 4)) return MGRIT_E_ALIGN;
  if (begins_as(y->data, {i.x.data, i.dt.data, i.b.data, i.c.data, i.z.data})) return MGRIT_E_SIZE;
  SsmStepArgs a{*cfg, i.x, i.dt, i.b, i.c, i.z, out, i.a, i.skip, i.bias, slots, n_slots, reset, state_in, state_out};
  (void)hipGetLastError();
  return code_of(launch_ssm_step(a, (hipStream_t)stream));
}

int policy_workspace_bytes(const logits_cfg* cfg, size_t* bytes) {
  const int rc = logits_check(cfg);
  if (rc) return rc;
  if (!bytes) return MGRIT_E_NULL;
  *bytes = logits_workspace(policy_space_cfg(*cfg));
  return MGRIT_OK;
}

int policy_loss(const logits_cfg* cfg, const policy_cfg* rule, const void* logits, const int64_t* tokens,
                const float* old_logp, const float* ref_logp, const float* advantage, const float* weight, float* loss,
                float* logp, float* ratio, float* kl, float* stats, void* dlogits, void* workspace,
                size_t workspace_bytes, void* stream) {
  int rc = policy_check(cfg, rule, logits, tokens, old_logp, ref_logp, advantage, weight, dlogits);
  if (rc) return rc;
  if (!loss) return MGRIT_E_NULL;
  if (off(loss, 4) || off(logp, 4) || off(ratio, 4) || off(kl, 4) || off(stats, 4)) return MGRIT_E_ALIGN;
  if ((rc = logits_space(policy_space_cfg(*cfg), workspace, workspace_bytes))) return rc;
  const void* rows[] = {loss, logp, ratio, kl, stats};
  for (int i = 0; i < 5; ++i) {
    if (begins_as(rows[i], {logits, tokens, old_logp, ref_logp, advantage, weight, dlogits})) return MGRIT_E_SIZE;
    for (int j = 0; j < i; ++j)
      if (begins_as(rows[i], {rows[j]})) return MGRIT_E_SIZE;
  }
  PolicyArgs a{*cfg, *rule, logits, tokens, old_logp, ref_logp, advantage, weight, loss, logp, ratio, kl, stats, nullptr,
               dlogits, (char*)workspace};
  (void)hipGetLastError();
  return code_of(launch_policy(a, (hipStream_t)stream));
}

int policy_loss_backward(const logits_cfg* cfg, const policy_cfg* rule, const void* logits, const int64_t* tokens,
                         const float* old_logp, const float* ref_logp, const float* advantage, const float* stats,
                         const float* dloss, void* dlogits, void* stream) {
  const int rc = policy_check(cfg, rule, logits, tokens, old_logp, ref_logp, advantage, dloss, dlogits);
  if (rc) return rc;
  if (!stats || !dlogits) return MGRIT_E_NULL;
  if (off(stats, 4)) return MGRIT_E_ALIGN;
  if (begins_as(dlogits, {stats})) return MGRIT_E_SIZE;
  PolicyArgs a{};
  a.c = *cfg;
  a.rule = *rule;
  a.logits = logits;
  a.tokens = tokens;
  a.old_logp = old_logp;
  a.ref_logp = ref_logp;
  a.advantage = advantage;
  a.weight = dloss;
  a.stats_in = stats;
  a.dlogits = dlogits;
  (void)hipGetLastError();
  return code_of(launch_policy_grad(a, (hipStream_t)stream));
}

}  // extern "C"
