// Internal declarations of the operators around a gated linear recurrent layer (include/mgrit_ops.h).
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/mgrit_ops.h"

namespace mg {

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

// Whether a call's results are stored past the caches.  That leaves the caches (256 MB behind the L2s) to what the
// call reads, and it makes the next kernel read the results from memory, so what counts is the call with a product
// that reads its results behind it; past : through the caches, us, in turn, the call alone in brackets.
//  - recurrence: states of 45 MB on, gradients of 95 MB on, floats up to 150 MB of either.  Forward, product,
//    adjoint, product: bf16 T x 4 x 1024, T = 3200 (52 MB of gradients) 116 : 114, 6000 170 : 176, 8000 213 : 217,
//    16384 392 : 391 (260 : 274), 32768 750 : 763; floats T x 100 x 1000, T = 128 (102 MB) 274 : 276 (86 : 95), 160
//    334 : 332, 200 410 : 395, 256 529 : 499, 400 851 : 813;
//  - gradients of the distillation, of 180 MB on: bf16 rows of 32768, 1024 rows (67 MB) 178 : 167, 2048 219 : 203,
//    3000 264 : 272, 8192 444 : 455 (218 : 230), 16384 748 : 772; 1003 x 50048 bf16 265 : 253; 1003 x 50021 floats
//    (201 MB) 672 : 682 (108 : 124);
//  - 8-bit product, results of 95 MB on: M x 2048 x 2048 bf16, M = 16384 (67 MB) 144 : 143, 24576 187 : 195, 32768
//    253 : 256 (201 : 209), 49152 374 : 392; floats 8192 (67 MB) 140 : 139, 16384 239 : 242 (116 : 127).
inline bool results_past_caches(double bytes, double from, double to = 1e300) { return bytes >= from && bytes <= to; }

// What a launch can be: fewer than 2^32 threads in all.
inline bool launchable(long long groups, int threads) { return groups * threads <= 0xffffffffLL; }
// What a launch function returns, before it has launched anything, for a call whose launches would be larger.
constexpr hipError_t TOO_LARGE = hipErrorInvalidConfiguration;

// ---- gated linear recurrence (kernels_glr.hip)
// A workgroup of GLR_WAVES waves covers one row of the batch, 2 * lanes channels (two per lane) and
// GLR_WAVES * (64 / lanes) * run steps: a wave's lanes hold 64 / lanes runs.  Forward: runs of 16 steps over up to
// 128 channels; the adjoint, which keeps three arrays where the forward sweep keeps two: runs of 8 steps over up to
// 64 channels.
constexpr int GLR_WAVES = 8, GLR_RUN_FWD = 16, GLR_RUN_BWD = 8;
struct GlrShape {
  int lanes;                // lanes across the channels: 16, 32 or (forward) 64
  int steps;                // of a tile
  int chunks;               // tiles along the sequence
  int cols;                 // tiles along the channels
  long long words;          // tiles' words in the workspace (none where a sequence is one tile)
};
inline GlrShape glr_shape(const glr_cfg& c, bool backward) {
  GlrShape s;
  s.lanes = c.H > 64 && !backward ? 64 : c.H > 32 ? 32 : 16;
  s.steps = GLR_WAVES * (64 / s.lanes) * (backward ? GLR_RUN_BWD : GLR_RUN_FWD);
  s.chunks = (int)(((long long)c.T + s.steps - 1) / s.steps);
  s.cols = (c.H + 2 * s.lanes - 1) / (2 * s.lanes);
  s.words = s.chunks > 1 ? (long long)s.chunks * c.B * s.cols * 2 * s.lanes : 0;
  return s;
}
struct GlrArgs {
  glr_cfg c;
  GlrShape s;
  glr_seq gate, value, h, dh, dgate, dvalue;
  const float* h0;
  const uint8_t* reset;
  float* h_last;
  float* saved;             // [.,B,H]: the state before every `save`-th step (the tiles of the adjoint)
  int save;
  const float* dh_last;
  float* dh0;
  unsigned long long* words;
  int* ticket;
  bool past;                // results past the caches
};
hipError_t launch_glr_forward(const GlrArgs& a, hipStream_t s);
hipError_t launch_glr_backward(const GlrArgs& a, hipStream_t s);

struct GlrStepArgs {
  glr_cfg c;
  glr_seq gate, value, h;   // (stride_t 0)
  const int32_t* slots;
  int n_slots;
  const uint8_t* reset;
  const float* state_in;
  float* state_out;
};
hipError_t launch_glr_step(const GlrStepArgs& a, hipStream_t s);

// ---- rows of logits (kernels_logits.hip)
struct LogitsArgs {
  logits_cfg c;
  const void* logits;
  const int64_t* ids;       // tokens[N] / the teacher's ids[N,K]
  float *logp, *entropy, *top_logp;
  int64_t* top_ids;
  const float *teacher, *weight;
  float* loss;
  float* stats;             // [N,2]
  const float* stats_in;
  void* dlogits;
  char* workspace;
};
size_t logits_workspace(const logits_cfg& c);
hipError_t launch_token_logprobs(const LogitsArgs& a, hipStream_t s);
hipError_t launch_distill(const LogitsArgs& a, hipStream_t s);
hipError_t launch_distill_grad(const LogitsArgs& a, hipStream_t s);

// ---- product in 8-bit integers (kernels_q8.hip)
struct Q8Args {
  q8_cfg c;
  const void* x;
  const int8_t* w;
  const float *w_scale, *bias;
  void* y;
  int8_t* q;                // [M, q8_row_bytes(K)]
  float* scale;             // [M]
  bool past;                // results past the caches
};
hipError_t launch_q8_quantize(const Q8Args& a, hipStream_t s);
hipError_t launch_q8_linear(const Q8Args& a, hipStream_t s);

}  // namespace mg
