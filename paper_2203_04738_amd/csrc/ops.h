// Internal declarations of the operators around a gated linear recurrent layer (include/mgrit_ops.h).
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/mgrit_ops.h"

namespace mg {

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

// Whether a call moves so much that what it writes would not stay in the last-level cache (256 MB) for the next kernel
// anyway: it is then stored past the caches, which leaves them to what the call reads.  Plain : past them, us:
// recurrence 128 x 100 x 1000 floats 93 : 88 (forward 154 MB, backward 256 MB), 16384 x 4 x 1024 bf16 282 : 272; gradient of 1003 x
// 50021 floats behind the forward pass 130 : 103; 8-bit product of 32768 x 2048 x 2048 224 : 216.
inline bool stores_past_caches(double bytes) { return bytes >= 128e6; }

// What a launch can be: fewer than 2^32 threads in all.
inline bool launchable(long long groups, int threads) { return groups * threads <= 0xffffffffLL; }
// What a launch function returns, before it has launched anything, for a call whose launches would be larger.
constexpr hipError_t TOO_LARGE = hipErrorInvalidConfiguration;

// ---- gated linear recurrence (kernels_glr.hip)
// A workgroup of GLR_WAVES waves covers one row of the batch, 2 * lanes channels (two per lane) and GLR_WAVES * (64 / lanes) *
// run steps: a wave's lanes hold 64 / lanes runs.  Forward: runs of 16 steps over up to 128 channels; the adjoint, which
// keeps three arrays where the forward sweep keeps two: runs of 8 steps over up to 64 channels.
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
