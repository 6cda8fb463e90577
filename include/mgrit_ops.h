/*
 * mgrit_ops.h -- C ABI of the operators around a gated linear recurrent layer.
 *
 * A GRU's gates read the state, which is why its solve over time needs MGRIT's
 * cycles (mgrit_gru.h).  A layer whose gates read the input alone is linear in
 * its state and is solved exactly, in one pass over the sequence.  The entry
 * points here train such a layer, as a student of a GRU or by itself, serve it
 * and score what it says:
 *
 *   glr_forward, glr_backward, glr_step       the recurrence and its adjoint, and one token
 *   distill_topk, distill_topk_backward       loss against a teacher's top logits, gradient
 *   token_logprobs                            log probabilities, entropy, top alternatives
 *   q8_quantize, q8_linear                    product in 8-bit integers, scales per token / channel
 *
 * Conventions are those of mgrit_gru.h: device pointers, everything enqueued on
 * `stream`, no allocation, no synchronisation, arguments checked on the host before
 * anything is launched, MGRIT_E_* codes, outputs overwritten, never accumulated, no
 * exception crosses the ABI.  Every output is bitwise reproducible.  Buffers that a
 * call writes must not overlap any other buffer of the call unless its comment says so.
 * A workspace of 0 bytes may be NULL; other workspaces are 16-byte aligned; calls that
 * share one are ordered on one stream.
 * A call whose launches would take 2^32 threads or more is refused with MGRIT_E_SIZE:
 * from 2^23 tiles on for a sequence (128 to 512 steps of 32 to 128 channels of one batch
 * row each), from 2^22 on for rows of logits (of up to 2^15 entries; longer ones count
 * as several) or tokens to quantise, more where they are short.
 * Nothing is kept in a workspace from call to call.
 */
#ifndef MGRIT_OPS_H
#define MGRIT_OPS_H

#include "mgrit_gru.h"

#ifdef __cplusplus
extern "C" {
#endif

/* dtype of the arrays that a comment calls "of the dtype": MGRIT_F32, MGRIT_BF16 or MGRIT_F16.
 * All sums, states and statistics are float; a result is rounded once, to nearest, when it is stored. */
enum { MGRIT_F16 = 4 };

/* ------------------------------------------------------------------------
 * Gated linear recurrence, per batch row and channel
 *     h_t = a_t h_{t-1} + b_t,   t = 1..T,
 * GLR_MIX:   a = sigmoid(gate), b = (1 - a) value    (a GRU's update whose gates do not read the state)
 * GLR_DECAY: a = exp(gate),     b = value            (gate <= 0 is a decay; it is not enforced)
 * A sequence is composed from runs of steps, h -> A h + S with A the product of the run's a.  Gates above 0
 * can carry A beyond the floats within some steps, where a state that is not zero becomes infinite or NaN; one
 * of zero stays what its inputs make it.  An infinite state, which nothing but a reset ends, may be NaN once A
 * is below the floats.
 * A step whose `reset` byte is not zero forgets the past: h_t = b_t, whatever h_{t-1} was (infinities
 * and NaN included), and no gradient passes to the steps before it: sequences packed one behind the other.
 */
enum { GLR_MIX = 0, GLR_DECAY = 1 };

typedef struct {
  int32_t T, B, H;      /* steps, batch rows, channels; each >= 1, T * B <= 2^30, B * H <= 2^30 */
  int32_t form;         /* GLR_* */
  int32_t dtype;        /* of gate, value, h, dh, dgate, dvalue */
} glr_cfg;

/* An array [T,B,H] of the dtype: element (t,b,c) is data[t * stride_t + b * stride_b + c], strides in
 * elements and not negative.  Any strides serve (gate and value as halves of one product's rows, batch-first
 * storage); an array that is written must not overlap itself: of the two strides that are used
 * (that of T where T > 1, of B where B > 1) the smaller is at least H, and the larger at least
 * the smaller times its extent. */
typedef struct {
  void* data;
  int64_t stride_t, stride_b;
} glr_seq;

/* Host only: bytes of the workspace of both directions, and of `saved`. */
MGRIT_API int glr_workspace_bytes(const glr_cfg* cfg, size_t* bytes);
MGRIT_API int glr_saved_bytes(const glr_cfg* cfg, size_t* bytes);

/* Forward.
 *   h0[B,H] float or NULL (zeros); reset[T,B] bytes or NULL; h out; h_last[B,H] float out or NULL: h_T
 *   unrounded, the h0 of a call that goes on with the sequence (it may be h0 itself).  It is formed from
 *   the tiles' maps as the states between tiles are; a float h_T may differ from it in the last bits.
 *   saved: out or NULL: the states (float) that glr_backward starts from, 16-byte aligned. */
MGRIT_API int glr_forward(const glr_cfg* cfg, const glr_seq* gate, const glr_seq* value, const float* h0,
                          const uint8_t* reset, const glr_seq* h, float* h_last, void* saved,
                          size_t saved_bytes, void* workspace, size_t workspace_bytes, void* stream);

/* Backward, from the same gate, value and reset and what the forward call left in `saved`:
 *     l_t = dh_t + a_{t+1} l_{t+1}  (l_T = dh_T + dh_last),
 *     dgate_t = l_t da_t (h_{t-1} - value_t) (mix) or l_t a_t h_{t-1} (decay),  dvalue_t = l_t db/dvalue,
 *     dh0 = a_1 l_1.
 * The states between the saved ones are computed again, unrounded; h is not read.
 *   dh_last[B,H] float or NULL (zeros); dgate, dvalue out; dh0[B,H] float out or NULL. */
MGRIT_API int glr_backward(const glr_cfg* cfg, const glr_seq* gate, const glr_seq* value,
                           const uint8_t* reset, const void* saved, size_t saved_bytes, const glr_seq* dh,
                           const float* dh_last, const glr_seq* dgate, const glr_seq* dvalue, float* dh0,
                           void* workspace, size_t workspace_bytes, void* stream);

/* One step of B running sequences whose states live in a pool of n_slots rows (cfg->T is 1).
 *   gate, value, h: arrays [1,B,H] as above (stride_t is not read); slots[B] int32 or NULL (row b is
 *   slot b; then n_slots >= B): a row whose slot is outside 0..n_slots-1 is idle: its h is zero and no
 *   state is touched.  Two rows must not name the same slot.  reset[B] or NULL.  state_in,
 *   state_out[n_slots,H] float; they may be the same array, and slots that no row names are left alone. */
MGRIT_API int glr_step(const glr_cfg* cfg, const glr_seq* gate, const glr_seq* value, const int32_t* slots,
                       int32_t n_slots, const uint8_t* reset, const float* state_in, float* state_out,
                       const glr_seq* h, void* stream);

/* ------------------------------------------------------------------------
 * Rows of logits x[N,V] of the dtype, row stride ld >= V elements, at a temperature t:
 *     p = softmax(x / t).
 * Entries of -inf are what a mask leaves out: p = 0.  A row with a NaN or +inf has NaN results.
 */
typedef struct {
  int32_t N, V;         /* rows >= 1; entries 1 .. 2^20 */
  int32_t K;            /* entries per row of the top / teacher arrays */
  int32_t dtype;
  float temperature;    /* finite, > 0, log2(e) / temperature finite (from 4.3e-39 on) */
  int64_t ld, ld_grad;  /* row strides of logits and dlogits */
} logits_cfg;

/* Host only: workspace of token_logprobs and distill_topk. */
MGRIT_API int logits_workspace_bytes(const logits_cfg* cfg, size_t* bytes);

/* Log probabilities of given tokens and of the top alternatives, entropy (nats), in one pass.
 *   tokens[N] int64 or NULL; logp[N] float, NULL if and only if tokens is: log p of the token; 0 for a negative
 *   token (a position without one), NaN for one >= V.  entropy[N] float or NULL.
 *   top_logp[N,K] float, top_ids[N,K] int64: the K largest entries in falling order, equal ones
 *   by rising index; both NULL if and only if K is 0.  K <= 64 and K <= V.
 *   A row of nothing but -inf: log probabilities -inf, entropy 0, the first K indices. */
#define LOGPROBS_MAX_K 64
MGRIT_API int token_logprobs(const logits_cfg* cfg, const void* logits, const int64_t* tokens, float* logp,
                             float* entropy, float* top_logp, int64_t* top_ids, void* workspace,
                             size_t workspace_bytes, void* stream);

/* Distillation from the K logits that a teacher gives for every row:
 *     q = softmax over the row's entries of teacher / t,   loss = sum_k q_k (log q_k - log p[ids_k]),
 *     dlogits = weight / t (p - sum_k q_k e[ids_k]).
 *   ids[N,K] int64 (negative: padding, no entry; the same id twice: both count), teacher[N,K] float (-inf: no
 *   weight; nor has an entry whose q is below the smallest normal float).  A row without any entry of weight
 *   has loss 0 and gradient 0.  K = 1 is cross entropy.
 *   An id >= V makes its row NaN.  K <= 256.
 *   weight[N] float or NULL (ones): dL/dloss of each row; a row of weight 0 has gradient 0 whatever it holds.
 *   loss[N] float (not multiplied by the weight).
 *   stats[N,2] float out or NULL: max_j x_j and sum_j exp((x_j - max) / t), for distill_topk_backward
 *   (0 and 1 where the row has no teacher).
 *   dlogits[N,V] of the dtype, row stride ld_grad, or NULL: the gradient in the same pass; it may be
 *   logits itself (then ld_grad == ld). */
#define DISTILL_MAX_K 256
MGRIT_API int distill_topk(const logits_cfg* cfg, const void* logits, const int64_t* ids,
                           const float* teacher, const float* weight, float* loss, float* stats,
                           void* dlogits, void* workspace, size_t workspace_bytes, void* stream);
/* The gradient alone, where dL/dloss (dloss[N], or NULL: ones) is known later; stats from distill_topk. */
MGRIT_API int distill_topk_backward(const logits_cfg* cfg, const void* logits, const int64_t* ids,
                                    const float* teacher, const float* stats, const float* dloss,
                                    void* dlogits, void* stream);

/* ------------------------------------------------------------------------
 * Product in 8-bit integers:  y[m,n] = xs_m ws_n sum_k xq[m,k] wq[n,k] + bias_n,
 * the sum exact (32-bit integers), then multiplied by ws, by xs, and the bias added, in floats.
 * A row is quantised by
 *     scale = max(max|x| / 127, 2^-126),   q = x / scale rounded to nearest (ties to even),
 * both quotients rounded to float.  A row with an infinity or a NaN has scale NaN and q 0: its results are NaN.
 * Rows of q are q8_row_bytes(K) bytes apart, K rounded up to 128.
 */
typedef struct {
  int32_t M, N, K;      /* tokens, output channels, input channels; each >= 1, K <= 131072 */
  int32_t dtype;        /* of x and y */
  int64_t ldx, ldy;     /* row strides of x (>= K) and y (>= N), elements */
} q8_cfg;

MGRIT_API int64_t q8_row_bytes(int32_t K);
/* Host only: workspace of q8_linear. */
MGRIT_API int q8_workspace_bytes(const q8_cfg* cfg, size_t* bytes);
/* Quantises rows x[M,K] of the dtype (tokens, or the output channels of a weight matrix); cfg->N and
 * ldy are not read.
 *   q[M, q8_row_bytes(K)] int8, 16-byte aligned, zeros beyond K; scale[M] float. */
MGRIT_API int q8_quantize(const q8_cfg* cfg, const void* x, int8_t* q, float* scale, void* stream);
/* w_q[N, q8_row_bytes(K)] int8 (16-byte aligned; what lies beyond K does not matter), w_scale[N] float,
 * bias[N] float or NULL; y[M,N] of the dtype. */
MGRIT_API int q8_linear(const q8_cfg* cfg, const void* x, const int8_t* w_q, const float* w_scale,
                        const float* bias, void* y, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MGRIT_OPS_H */
