// Internal declarations of the operators of a recurrent student over tokens (include/mgrit_tokens.h).
#pragma once
#include "../../include/mgrit_tokens.h"
#include "ops.h"

namespace mg {

// ---- embedding (kernels_embed.hip)
struct EmbedArgs {
  embed_cfg c;
  const int64_t* tokens;
  const void* in;           // table, or dout
  void* out;                // out, or dtable
  int run;                  // sorted places that a wave adds up: a block
  int* total;               // tokens that name a row
  int* place;               // [N]: places of the tokens in order of token and place
  int* token;               // [N]: their tokens
  int* crosses;             // [ceil(N / run)]: the token of a run that begins in the block and goes on, or -1
  float* part;              // [ceil(N / run)][2][D]: sums of runs that go on beyond their block
};
size_t embed_workspace(const embed_cfg& c);
hipError_t launch_embed_lookup(const EmbedArgs& a, hipStream_t s);
hipError_t launch_embed_backward(EmbedArgs a, char* workspace, hipStream_t s);

// ---- causal convolution (kernels_conv.hip)
struct ConvArgs {
  conv_cfg c;
  glr_seq x, y, dy, dx;
  const float *weight, *bias, *past, *dlast;
  const uint8_t* reset;
  float *last, *dweight, *dbias, *dpast;
  float* part;              // [groups][H][W + 1]
  int groups, seg;          // backward: of workgroups along the sequences; steps of a thread's segment
  bool past_caches;
};
size_t conv_workspace(const conv_cfg& c);
bool conv_launchable(const conv_cfg& c);
hipError_t launch_conv_forward(const ConvArgs& a, hipStream_t s);
hipError_t launch_conv_backward(const ConvArgs& a, hipStream_t s);

struct ConvStepArgs {
  conv_cfg c;
  glr_seq x, y;             // (stride_t 0)
  const float *weight, *bias;
  const int32_t* slots;
  int n_slots;
  const uint8_t* reset;
  const float* past_in;
  float* past_out;
};
hipError_t launch_conv_step(const ConvStepArgs& a, hipStream_t s);

// ---- selective state space scan (kernels_ssm.hip)
// A wave covers 16 channels, four lanes a channel, `per` states a lane; a workgroup 64 channels of one batch row and a
// chunk of steps.
// Steps between saved states, which are the tile of the adjoint, for lanes of `per` states.
constexpr int ssm_save(int per) { return per <= 8 ? 8 : 4; }
struct SsmShape {
  int per;                  // states of a lane: 1, 2, 4, 8, 16
  int save;                 // steps between saved states
  int cols;                 // workgroups across the channels
  int chunks, len;          // chunks of a sequence, their steps (a multiple of 16)
};
// Whether every workgroup goes through the chunks before its own itself.
__host__ __device__ inline bool few_chunks(const SsmShape& s) { return s.chunks <= 64; }
SsmShape ssm_shape(const ssm_cfg& c, bool backward);
struct SsmArgs {
  ssm_cfg c;
  SsmShape s;
  glr_seq x, dt, b, cc, z;  // cc: the c of the formulas
  const float *a, *skip, *bias, *h0;
  const uint8_t* reset;
  glr_seq y;
  float* h_last;
  float* saved;             // [ceil(T / save)][B,H,S]: the state before every save-th step
  float* ends;              // [chunks][B,H,S]
  float* sums;              // [chunks][B,H]: sum of the chunk's d; negative: it forgets
  // backward
  glr_seq dy, dx, ddt, db, dc, dz;
  const float* dh_last;
  float *da, *dskip, *dbias, *dh0;
  float* part_bc;           // [cols][T,B,2S]
  float* part_a;            // [chunks * B][H,S]
  float* part_h;            // [chunks * B][H][2]
};
size_t ssm_workspace(const ssm_cfg& c);
size_t ssm_saved(const ssm_cfg& c);
bool ssm_launchable(const ssm_cfg& c);
hipError_t launch_ssm_forward(SsmArgs a, char* workspace, hipStream_t s);
hipError_t launch_ssm_backward(SsmArgs a, char* workspace, hipStream_t s);

struct SsmStepArgs {
  ssm_cfg c;
  glr_seq x, dt, b, cc, z, y;
  const float *a, *skip, *bias;
  const int32_t* slots;
  int n_slots;
  const uint8_t* reset;
  const float* state_in;
  float* state_out;
};
hipError_t launch_ssm_step(const SsmStepArgs& a, hipStream_t s);

// ---- policy loss (kernels_logits.hip)
struct PolicyArgs {
  logits_cfg c;
  policy_cfg rule;
  const void* logits;
  const int64_t* tokens;
  const float *old_logp, *ref_logp, *advantage, *weight;
  float *loss, *logp, *ratio, *kl, *stats;
  const float* stats_in;
  void* dlogits;
  char* workspace;
};
hipError_t launch_policy(const PolicyArgs& a, hipStream_t s);
hipError_t launch_policy_grad(const PolicyArgs& a, hipStream_t s);

}  // namespace mg
