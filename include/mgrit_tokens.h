/*
 * mgrit_tokens.h -- C ABI of the operators of a recurrent student over tokens.
 *
 * mgrit_ops.h has the recurrence of one state per channel, the loss against a teacher and the product in 8 bits.
 * The entry points here give such a student tokens to read, a recurrence with several states per channel whose steps
 * the input chooses, and rewards to learn from:
 *
 *   embed_lookup, embed_backward                               rows of a table, scaled, and the table's gradient
 *   causal_conv_forward, causal_conv_backward, causal_conv_step   short convolution of every channel
 *   ssm_forward, ssm_backward, ssm_step                        selective state space scan, its adjoint, one token
 *   policy_loss, policy_loss_backward                          clipped policy loss with a KL term, gradient
 *
 * Conventions are those of mgrit_ops.h: device pointers, everything enqueued on `stream`, no allocation, no
 * synchronisation, arguments checked on the host before anything is launched, MGRIT_E_* codes, outputs overwritten,
 * never accumulated, no exception crosses the ABI, every output bitwise reproducible, buffers that a call writes
 * overlap no other buffer of the call unless its comment says so, nothing kept in a workspace from call to call, a
 * workspace of 0 bytes may be NULL, others are 16-byte aligned, calls that share one are ordered on one stream.
 * Sums, states and statistics are float (a row's loss double); a result is rounded once, to nearest, when it is stored.
 * A call whose launches would take 2^32 threads or more is refused with MGRIT_E_SIZE, and so is one over sequences or rows
 * of which one that is written begins where another begins (but for a gradient of logits in their place).
 */
#ifndef MGRIT_TOKENS_H
#define MGRIT_TOKENS_H

#include "mgrit_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------
 * Embedding of tokens:  out[n,:] = scale table[tokens[n],:].
 * A negative token is padding: its row is zero.  A token >= V makes its row NaN.  Neither has a gradient.
 */
typedef struct {
  int32_t N, V, D;            /* tokens 1 .. 2^26, rows of the table 1 .. 2^20, width 1 .. 2^20 */
  int32_t dtype;              /* of table, out and their gradients */
  float scale;                /* finite */
  int64_t ld_table, ld_out;   /* row strides (>= D, elements) of table / dtable and out / dout */
} embed_cfg;

MGRIT_API int embed_lookup(const embed_cfg* cfg, const int64_t* tokens, const void* table, void* out, void* stream);
/* dtable[v,:] = scale sum_{n: tokens[n] = v} dout[n,:], the sum over n in an order that N and the tokens decide; rows that
 * no token names are zero.  The tokens are sorted on the way. */
MGRIT_API int embed_workspace_bytes(const embed_cfg* cfg, size_t* bytes);
MGRIT_API int embed_backward(const embed_cfg* cfg, const int64_t* tokens, const void* dout, void* dtable,
                             void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Causal convolution of every channel over its last W inputs:
 *     p_t = bias + sum_{k<W} weight[k] x_{t-W+1+k},   y_t = p_t (CONV_LINEAR) or p_t sigmoid(p_t) (CONV_SILU).
 * Inputs before the first are `past`.  A step whose `reset` byte is not zero forgets the past: the inputs before it
 * count as zeros, whatever they are, for it and for all steps behind it, and no gradient passes to them.
 */
enum { CONV_LINEAR = 0, CONV_SILU = 1 };
#define CONV_MAX_W 8

typedef struct {
  int32_t T, B, H;      /* steps, batch rows, channels; each >= 1, T * B <= 2^30, B * H <= 2^30 */
  int32_t W;            /* inputs that a step sees, 1 .. CONV_MAX_W */
  int32_t act;          /* CONV_* */
  int32_t dtype;        /* of x, y, dy, dx */
} conv_cfg;

/* Sequences are as in mgrit_ops.h ([T,B,H], any strides).  weight[H,W] float, bias[H] float or NULL (zeros).
 *   past[B,W-1,H] float or NULL (zeros): the W - 1 inputs before the first, oldest first; reset[T,B] bytes or NULL;
 *   last[B,W-1,H] float out or NULL: the same behind the last step, zeros for what was forgotten: the past of a call
 *   that goes on with the sequence (not `past` itself: MGRIT_E_SIZE).  (W = 1: neither is looked at.) */
MGRIT_API int causal_conv_forward(const conv_cfg* cfg, const glr_seq* x, const float* weight, const float* bias,
                                  const float* past, const uint8_t* reset, const glr_seq* y, float* last, void* stream);

/* Backward, from the same inputs.  dlast[B,W-1,H] float or NULL (zeros).  Out: dx; dweight[H,W], dbias[H] float, each or
 * NULL; dpast[B,W-1,H] float or NULL (not dlast itself: MGRIT_E_SIZE). */
MGRIT_API int causal_conv_workspace_bytes(const conv_cfg* cfg, size_t* bytes);
MGRIT_API int causal_conv_backward(const conv_cfg* cfg, const glr_seq* x, const float* weight, const float* bias,
                                   const float* past, const uint8_t* reset, const glr_seq* dy, const float* dlast,
                                   const glr_seq* dx, float* dweight, float* dbias, float* dpast, void* workspace,
                                   size_t workspace_bytes, void* stream);

/* One step of B running sequences whose pasts live in a pool of n_slots rows (cfg->T is 1).
 *   x, y: [1,B,H] (stride_t is not read); slots[B] int32 or NULL (row b is slot b; then n_slots >= B): a row whose slot is
 *   outside 0..n_slots-1 is idle: its y is zero and no past is touched.  Two rows must not name the same slot.
 *   reset[B] or NULL.  past_in, past_out[n_slots,W-1,H] float; they may be the same array, and slots that no row
 *   names are left alone.  (W = 1: neither is looked at.) */
MGRIT_API int causal_conv_step(const conv_cfg* cfg, const glr_seq* x, const float* weight, const float* bias,
                               const int32_t* slots, int32_t n_slots, const uint8_t* reset, const float* past_in,
                               float* past_out, const glr_seq* y, void* stream);

/* ------------------------------------------------------------------------
 * Selective state space scan, S states n per batch row and channel:
 *     d_t = softplus(dt_t + bias),   h_t[n] = exp(d_t a[n]) h_{t-1}[n] + d_t b_t[n] x_t,
 *     y_t = (sum_n c_t[n] h_t[n] + skip x_t) z_t sigmoid(z_t),
 * b_t and c_t the same for all channels of a batch row, a, bias and skip of each channel.
 * a <= 0 is a decay; it is not enforced.  a > 0 can carry exp(d a) beyond the floats, where a state becomes infinite or
 * NaN (one of zero too), or its product over some steps, where one that is not zero does.  An infinite state may be NaN later.
 * a = -infinity forgets at every step; ssm_backward needs finite ones (others leave NaN).
 * A step whose `reset` byte is not zero forgets the past: h_t = d_t b_t x_t, whatever h_{t-1} was, and no gradient
 * passes to the steps before it.
 */
#define SSM_MAX_S 64

typedef struct {
  int32_t T, B, H;      /* steps, batch rows, channels; each >= 1, T * B <= 2^30, B * H <= 2^30 */
  int32_t S;            /* states per channel, 1 .. SSM_MAX_S; B * H * S <= 2^32 */
  int32_t dtype;        /* of all sequences */
} ssm_cfg;

/* What a layer's scan reads.  Sequences have any strides; b, c: [T,B,S], the others [T,B,H]. */
typedef struct {
  glr_seq x, dt, b, c;
  glr_seq z;            /* data NULL: no gate, y_t = sum_n c_t[n] h_t[n] + skip x_t */
  const float* a;       /* [H,S] */
  const float* skip;    /* [H] or NULL: zeros */
  const float* bias;    /* [H] or NULL: zeros */
} ssm_inputs;

/* Gradients; sequences may be parts of the same rows but must not overlap, themselves included. */
typedef struct {
  glr_seq dx, ddt, db, dc;
  glr_seq dz;           /* data NULL if and only if z's is */
  float* da;            /* [H,S] */
  float* dskip;         /* [H] or NULL */
  float* dbias;         /* [H] or NULL */
  float* dh0;           /* [B,H,S] or NULL */
} ssm_grads;

/* Host only: bytes of the workspace of both directions, and of `saved`. */
MGRIT_API int ssm_workspace_bytes(const ssm_cfg* cfg, size_t* bytes);
MGRIT_API int ssm_saved_bytes(const ssm_cfg* cfg, size_t* bytes);

/* Forward.  h0[B,H,S] float or NULL (zeros); reset[T,B] bytes or NULL; y out; h_last[B,H,S] float out or NULL: h_T, the h0
 * of a call that goes on with the sequence (not h0 itself: MGRIT_E_SIZE).  saved: out or NULL: the states (float) that
 * ssm_backward starts from, 16-byte aligned. */
MGRIT_API int ssm_forward(const ssm_cfg* cfg, const ssm_inputs* in, const float* h0, const uint8_t* reset,
                          const glr_seq* y, float* h_last, void* saved, size_t saved_bytes, void* workspace,
                          size_t workspace_bytes, void* stream);

/* Backward, from the same inputs and what the forward call left in `saved`.  dh_last[B,H,S] float or NULL (zeros);
 * not dh0 itself: MGRIT_E_SIZE. */
MGRIT_API int ssm_backward(const ssm_cfg* cfg, const ssm_inputs* in, const uint8_t* reset, const void* saved,
                           size_t saved_bytes, const glr_seq* dy, const float* dh_last, const ssm_grads* out,
                           void* workspace, size_t workspace_bytes, void* stream);

/* One step of B running sequences whose states live in a pool of n_slots rows (cfg->T is 1; no stride_t is read); slots,
 * n_slots, reset, idle rows (y is zero) and pools state_in, state_out[n_slots,H,S] as in causal_conv_step. */
MGRIT_API int ssm_step(const ssm_cfg* cfg, const ssm_inputs* in, const int32_t* slots, int32_t n_slots,
                       const uint8_t* reset, const float* state_in, float* state_out, const glr_seq* y, void* stream);

/* ------------------------------------------------------------------------
 * Clipped policy loss with a KL term, on rows of logits x[N,V] (logits_cfg; K is not looked at), per row
 *     lp = log softmax(x / t)[token],   r = exp(lp - old),
 *     loss = - min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl k,   k = exp(ref - lp) - (ref - lp) - 1,
 *     dlogits = weight / t  dloss/dlp  (e[token] - softmax(x / t)),
 * the gradient of the minimum that of r A where the two are equal.
 *   tokens[N] int64: a negative one is a position that was not sampled: loss, logp, ratio, kl and gradient 0, whatever
 *   else the row holds.  One >= V makes its row NaN.
 *   old_logp[N], advantage[N] float; ref_logp[N] float or NULL: no KL term (k = 0; rule->kl is not looked at).
 *   weight[N] float or NULL (ones): dL/dloss of each row; a row of weight 0 has gradient 0 whatever it holds.
 *   loss[N] float (not multiplied by the weight); logp, ratio, kl[N] float out or NULL: lp, r and k.
 *   stats[N,2] float out or NULL: max_j x_j and sum_j exp((x_j - max) / t), for policy_loss_backward.
 *   dlogits[N,V] of the dtype, row stride ld_grad, or NULL: the gradient in the same pass; it may be
 *   logits itself (then ld_grad == ld).
 * A token that the mask (-inf) leaves out has lp = -inf: r = 0, and with a KL term an infinite loss, also where
 * old or ref is -inf.  A ratio or KL term beyond the floats is infinite.  The row of dlogits of an infinite loss is not
 * finite.
 */
typedef struct {
  float clip_low, clip_high;   /* 0 <= clip_low <= 1, 0 <= clip_high, finite */
  float kl;                    /* finite, >= 0 */
} policy_cfg;

MGRIT_API int policy_workspace_bytes(const logits_cfg* cfg, size_t* bytes);
MGRIT_API int policy_loss(const logits_cfg* cfg, const policy_cfg* rule, const void* logits, const int64_t* tokens,
                          const float* old_logp, const float* ref_logp, const float* advantage, const float* weight,
                          float* loss, float* logp, float* ratio, float* kl, float* stats, void* dlogits,
                          void* workspace, size_t workspace_bytes, void* stream);
/* The gradient alone, where dL/dloss (dloss[N], or NULL: ones) is known later; stats from policy_loss, dlogits as there. */
MGRIT_API int policy_loss_backward(const logits_cfg* cfg, const policy_cfg* rule, const void* logits,
                                   const int64_t* tokens, const float* old_logp, const float* ref_logp,
                                   const float* advantage, const float* stats, const float* dloss, void* dlogits,
                                   void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MGRIT_TOKENS_H */
