// Gated linear recurrence h_t = a_t h_{t-1} + b_t (include/mgrit_ops.h), its adjoint, and one step of it.
//
// A run of steps is the map h -> A h + S with A = prod a, S its result from a zero state, and two runs behind each
// other compose to (A2 A1, A2 S1 + S2): that is all a sequence needs to be cut up.  A workgroup reads its
// tile once, into registers; every lane goes through its run of 16 steps from a zero state; the runs of the tile meet in
// LDS; the tiles of a sequence meet in the workspace, where each leaves its (A, S) as soon as it has read its
// tile and, once it knows the state before it, the state behind it.  The bytes are those of the arrays, each read or written once.
//
// The word of a tile and channel is A in the low half and S in the high one, stored by one 64-bit store, so that a reader that
// sees one sees the other.  All bits set: not written yet (no A is stored so).  A = -0: S does not depend on what was
// before (a reset, or the state itself: what a tile knows once it knows the state before it).  No other A is -0:
// no a is negative, so that a product that underflows is +0: a NaN or an infinity in the state stays in it for as
// long as no reset stands in between.  The state before a tile is always computed as S + A h
// tile by tile, whether the states between were there to be read or not: the result does not depend on timing.
//
// Tiles are taken by a ticket, first tiles first (the adjoint: last tiles first), so that those a workgroup waits for
// have been started, wait for none behind it, and every wait ends.
#include "elem.h"
#include "ops.h"

namespace mg {

constexpr int GLR_THREADS = GLR_WAVES * 64;
constexpr int GLR_RUNS_X_CH = GLR_WAVES * 128;      // runs of a tile x its channels
constexpr int GLR_WINDOW = 32;                      // tiles looked at at a time
constexpr unsigned GLR_NONE = 0xffffffffu, GLR_FREE = 0x80000000u;

struct Pair {
  float x, y;
};

// Raw words of two neighbouring channels of one step.
template <typename E>
struct RawPair {
  unsigned w[sizeof(E) / 2];
  __device__ inline float at(int i) const {
    if constexpr (sizeof(E) == 4) return __uint_as_float(w[i]);
    else return word_elem<E>(w[0], i);
  }
};
// Channels c and c + 1 of a step at p; ALIGNED: as one word, with c + 1 < H.  Otherwise `second` says whether
// there is a channel c + 1.
template <typename E, bool ALIGNED>
__device__ inline RawPair<E> load_pair(const E* p, bool second) {
  RawPair<E> r;
  if constexpr (ALIGNED) {
    if constexpr (sizeof(E) == 4) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      r.w[0] = v.x;
      r.w[1] = v.y;
    } else {
      r.w[0] = *reinterpret_cast<const unsigned*>(p);
    }
  } else {
    const E a = p[0], b = p[second ? 1 : 0];
    if constexpr (sizeof(E) == 4) {
      r.w[0] = __float_as_uint(a);
      r.w[1] = __float_as_uint(b);
    } else {
      r.w[0] = (unsigned)a.bits | ((unsigned)b.bits << 16);
    }
  }
  return r;
}
template <typename E, bool ALIGNED>
__device__ inline void store_pair(E* p, float a, float b, bool second) {
  if constexpr (ALIGNED) {
    if constexpr (sizeof(E) == 4) *reinterpret_cast<float2*>(p) = make_float2(a, b);
    else *reinterpret_cast<unsigned*>(p) = pack2<E>(a, b);
  } else {
    p[0] = elem_of<E>(a);
    if (second) p[1] = elem_of<E>(b);
  }
}

// a and, for GLR_MIX, 1 - a of a gate.  sigmoid: with e = exp(-|g|), the smaller of the two is e / (1 + e), to
// full precision at any g, and the larger one minus that.
template <int FORM>
struct Gate {
  float a, na;
  __device__ inline explicit Gate(float g) {
    if constexpr (FORM == GLR_MIX) {
      const float e = __builtin_amdgcn_exp2f(-1.44269504088896341f * fabsf(g));
      const float s = e * __builtin_amdgcn_rcpf(1.0f + e), l = 1.0f - s;
      a = g < 0.0f ? s : l;
      na = g < 0.0f ? l : s;
    } else {
      a = __builtin_amdgcn_exp2f(1.44269504088896341f * g);
      na = 1.0f;
    }
  }
};

__device__ inline bool is_free(float A) { return __float_as_uint(A) == GLR_FREE; }
// A of a run behind another run.
__device__ inline float both(float A, float before) {
  return is_free(A) || is_free(before) ? -0.0f : A * before;
}
// The state behind a run (A, S) from the state h before it.
__device__ inline float behind(float A, float S, float h) { return is_free(A) ? S : fmaf(A, h, S); }

__device__ inline unsigned long long make_word(float A, float S) {
  unsigned a = __float_as_uint(A);
  if (a == GLR_NONE) a = 0x7fc00000u;               // a NaN of another kind
  return (unsigned long long)a | ((unsigned long long)__float_as_uint(S) << 32);
}
__device__ inline void store_word(unsigned long long* p, unsigned long long v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline unsigned long long load_word(const unsigned long long* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__global__ __launch_bounds__(256) void glr_clear_kernel(unsigned long long* words, long long n, int* ticket) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i < n) words[i] = ~0ull;
  if (i == 0) *ticket = 0;
}

// Where a thread stands.
struct GlrPlace {
  int lane_c, run, chunk, b, ch;       // lane across the channels, run of the tile, tile, batch row, channel
  int t0;                              // first step of the run
  bool has, second;                    // whether channels ch and ch + 1 exist
  __device__ inline GlrPlace(const GlrArgs& a, int tile, bool backward) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per_wave = 64 / a.s.lanes;
    lane_c = lane & (a.s.lanes - 1);
    run = wave * per_wave + lane / a.s.lanes;
    const int across = a.s.cols * a.c.B;
    const int k = tile / across, rest = tile - k * across;
    chunk = backward ? a.s.chunks - 1 - k : k;
    b = rest / a.s.cols;
    ch = (rest - b * a.s.cols) * 2 * a.s.lanes + 2 * lane_c;
    t0 = chunk * a.s.steps + run * GLR_STEPS;
    has = ch < a.c.H;
    second = ch + 1 < a.c.H;
  }
};

// Bits of the steps of the thread's run that reset (lanes >= 16 across the channels: each of the first 16
// lanes of a run looks at one step).
__device__ inline unsigned reset_bits(const GlrArgs& a, const GlrPlace& p) {
  const int t = p.t0 + p.lane_c;
  bool r = false;
  if (p.lane_c < GLR_STEPS && t < a.c.T) r = a.reset[(long long)t * a.c.B + p.b] != 0;
  const unsigned long long all = __ballot(r);
  return (unsigned)(all >> ((threadIdx.x & 63) / a.s.lanes * a.s.lanes)) & ((1u << GLR_STEPS) - 1);
}

// The 16 steps of a run of an input array; steps and channels that do not exist are read at the last one that does.
template <typename E, bool ALIGNED>
__device__ inline void load_run(const glr_seq& q, const GlrArgs& a, const GlrPlace& p,
                                RawPair<E> (&v)[GLR_STEPS]) {
  const int ch = p.has ? p.ch : 0;
  const E* base = (const E*)q.data + p.b * q.stride_b + ch;
  const bool second = ch + 1 < a.c.H;
#pragma unroll
  for (int r = 0; r < GLR_STEPS; ++r) {
    const int t = min(p.t0 + r, a.c.T - 1);
    v[r] = load_pair<E, ALIGNED>(base + t * q.stride_t, second);
  }
}

struct GlrShared {
  float2 run[GLR_RUNS_X_CH];                        // (A, S) of every run and channel
  unsigned long long window[GLR_WINDOW * 128];
  float carry[128];                                 // state before the tile
  int tile;
};

// The state before tile `chunk` of the thread's two channels (in sh.carry, for the lanes of run 0), from the words of
// the tiles before it (backward: behind it), whose distance is 1, 2, ...  All threads of the workgroup call it.
__device__ inline void glr_look_back(const GlrArgs& a, const GlrPlace& p, bool backward, GlrShared& sh) {
  const int before = backward ? a.s.chunks - 1 - p.chunk : p.chunk;
  const int n = min(before, GLR_WINDOW), runs = GLR_THREADS / a.s.lanes, chans = 2 * a.s.lanes;
  const long long per_tile = (long long)a.c.B * a.s.cols * chans;
  const int col = p.ch / chans;
  const long long at = ((long long)p.b * a.s.cols + col) * chans + 2 * p.lane_c;
  for (;;) {
    for (int i = p.run; i < n; i += runs) {
      const int other = backward ? p.chunk + 1 + i : p.chunk - 1 - i;
      const unsigned long long* w = a.words + other * per_tile + at;
      sh.window[i * chans + 2 * p.lane_c] = load_word(w);
      sh.window[i * chans + 2 * p.lane_c + 1] = load_word(w + 1);
    }
    __syncthreads();
    int ok = 1;
    if (p.run == 0) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        int i = 0;
        bool found = false;
        for (; i < n; ++i) {
          const unsigned A = (unsigned)sh.window[i * chans + 2 * p.lane_c + k];
          if (A == GLR_NONE) break;
          if (A == GLR_FREE) {
            found = true;
            break;
          }
        }
        if (found) {
          float h = __uint_as_float((unsigned)(sh.window[i * chans + 2 * p.lane_c + k] >> 32));
          while (--i >= 0) {
            const unsigned long long w = sh.window[i * chans + 2 * p.lane_c + k];
            h = fmaf(__uint_as_float((unsigned)w), h, __uint_as_float((unsigned)(w >> 32)));
          }
          sh.carry[2 * p.lane_c + k] = h;
        }
        ok &= found;
      }
    }
    if (__syncthreads_and(ok)) return;
    __builtin_amdgcn_s_sleep(1);
  }
}

// What both directions do between their sweeps: from (A, S) of the thread's run, per channel, the state before
// the run.  first: the state before the sequence's first tile (backward: behind its last one).  Returns in
// `out` (run 0's threads) the state behind the tile.
template <bool BACKWARD>
__device__ inline Pair glr_join(const GlrArgs& a, const GlrPlace& p, Pair A, Pair S, Pair first, Pair& out,
                                GlrShared& sh) {
  const int chans = 2 * a.s.lanes, runs = GLR_THREADS / a.s.lanes, c = 2 * p.lane_c;
  sh.run[p.run * chans + c] = make_float2(A.x, S.x);
  sh.run[p.run * chans + c + 1] = make_float2(A.y, S.y);
  __syncthreads();
  const bool at_start = BACKWARD ? p.chunk == a.s.chunks - 1 : p.chunk == 0;
  const bool chain = a.s.chunks > 1;
  unsigned long long* word =
      a.words + (((long long)p.chunk * a.c.B + p.b) * a.s.cols) * chans + p.ch;
  Pair tA = {1.f, 1.f}, tS = {0.f, 0.f};            // of the whole tile
  if (p.run == 0) {
    for (int i = 0; i < runs; ++i) {
      const int r = BACKWARD ? runs - 1 - i : i;
      const float2 x = sh.run[r * chans + c], y = sh.run[r * chans + c + 1];
      tS.x = behind(x.x, x.y, tS.x);
      tS.y = behind(y.x, y.y, tS.y);
      tA.x = both(x.x, tA.x);
      tA.y = both(y.x, tA.y);
    }
    if (chain && !at_start) {
      store_word(word, make_word(tA.x, tS.x));
      store_word(word + 1, make_word(tA.y, tS.y));
    }
  }
  if (at_start) {
    if (p.run == 0) {
      sh.carry[c] = first.x;
      sh.carry[c + 1] = first.y;
    }
    __syncthreads();
  } else {
    glr_look_back(a, p, BACKWARD, sh);
  }
  Pair h = {sh.carry[c], sh.carry[c + 1]};
  if (p.run == 0) {
    out.x = behind(tA.x, tS.x, h.x);
    out.y = behind(tA.y, tS.y, h.y);
    if (chain) {
      store_word(word, make_word(-0.0f, out.x));
      store_word(word + 1, make_word(-0.0f, out.y));
    }
  }
  for (int i = 0; i < (BACKWARD ? runs - 1 - p.run : p.run); ++i) {
    const int r = BACKWARD ? runs - 1 - i : i;
    const float2 x = sh.run[r * chans + c], y = sh.run[r * chans + c + 1];
    h.x = behind(x.x, x.y, h.x);
    h.y = behind(y.x, y.y, h.y);
  }
  return h;
}

__device__ inline int glr_tile(const GlrArgs& a, GlrShared& sh) {
  if (a.s.chunks == 1) return blockIdx.x;
  if (threadIdx.x == 0) sh.tile = atomicAdd(a.ticket, 1);
  __syncthreads();
  return sh.tile;
}

template <typename E, bool ALIGNED, int FORM, bool RESET>
__global__ __launch_bounds__(GLR_THREADS) void glr_forward_kernel(GlrArgs a) {
  __shared__ GlrShared sh;
  const GlrPlace p(a, glr_tile(a, sh), false);
  RawPair<E> g[GLR_STEPS], v[GLR_STEPS];
  load_run<E, ALIGNED>(a.gate, a, p, g);
  load_run<E, ALIGNED>(a.value, a, p, v);
  const unsigned resets = RESET ? reset_bits(a, p) : 0u;
  Pair first = {0.f, 0.f};
  if (p.chunk == 0 && a.h0 && p.run == 0) {
    const long long at = (long long)p.b * a.c.H + p.ch;
    if (p.has) first.x = a.h0[at];
    if (p.second) first.y = a.h0[at + 1];
  }
  // from a zero state: S[r], and A[r] of the steps up to r
  float A[GLR_STEPS][2], S[GLR_STEPS][2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float pa = 1.f, ps = 0.f;
#pragma unroll
    for (int r = 0; r < GLR_STEPS; ++r) {
      const Gate<FORM> gt(g[r].at(k));
      const float b = FORM == GLR_MIX ? gt.na * v[r].at(k) : v[r].at(k);
      if (p.t0 + r < a.c.T) {
        if (RESET && (resets >> r & 1)) {
          pa = -0.0f;
          ps = b;
        } else {
          pa = RESET && is_free(pa) ? pa : pa * gt.a;
          ps = fmaf(gt.a, ps, b);
        }
      }
      A[r][k] = pa;
      S[r][k] = ps;
    }
  }
  constexpr int L = GLR_STEPS - 1;
  Pair end;
  const Pair h = glr_join<false>(a, p, {A[L][0], A[L][1]}, {S[L][0], S[L][1]}, first, end, sh);
  if (p.run == 0) {
    const long long at = (long long)p.b * a.c.H + p.ch;
    if (a.saved) {
      float* s = a.saved + (long long)p.chunk * a.c.B * a.c.H + at;
      if (p.has) s[0] = h.x;
      if (p.second) s[1] = h.y;
    }
    if (a.h_last && p.chunk == a.s.chunks - 1) {
      if (p.has) a.h_last[at] = end.x;
      if (p.second) a.h_last[at + 1] = end.y;
    }
  }
  if (!p.has) return;
  E* out = (E*)a.h.data + p.b * a.h.stride_b + p.ch;
#pragma unroll
  for (int r = 0; r < GLR_STEPS; ++r) {
    const int t = p.t0 + r;
    if (t >= a.c.T) break;
    const float x = RESET ? behind(A[r][0], S[r][0], h.x) : fmaf(A[r][0], h.x, S[r][0]);
    const float y = RESET ? behind(A[r][1], S[r][1], h.y) : fmaf(A[r][1], h.y, S[r][1]);
    store_pair<E, ALIGNED>(out + t * a.h.stride_t, x, y, p.second);
  }
}

// mu_t = a_t l_t is what step t hands on to step t - 1: mu -> a (dh + mu), the same composition from the other end.
template <typename E, bool ALIGNED, int FORM, bool RESET>
__global__ __launch_bounds__(GLR_THREADS) void glr_backward_kernel(GlrArgs a) {
  __shared__ GlrShared sh;
  __shared__ float2 fwd[GLR_RUNS_X_CH];             // (A, S) of every run forward
  const GlrPlace p(a, glr_tile(a, sh), true);
  const int chans = 2 * a.s.lanes, c = 2 * p.lane_c;
  RawPair<E> g[GLR_STEPS], v[GLR_STEPS], d[GLR_STEPS];
  load_run<E, ALIGNED>(a.gate, a, p, g);
  load_run<E, ALIGNED>(a.value, a, p, v);
  load_run<E, ALIGNED>(a.dh, a, p, d);
  const unsigned resets = RESET ? reset_bits(a, p) : 0u;
  const long long at = (long long)p.b * a.c.H + p.ch;
  Pair first = {0.f, 0.f}, h = {0.f, 0.f};
  if (p.chunk == a.s.chunks - 1 && a.dh_last && p.run == 0) {
    if (p.has) first.x = a.dh_last[at];
    if (p.second) first.y = a.dh_last[at + 1];
  }
  {
    const float* s = a.saved + (long long)p.chunk * a.c.B * a.c.H + at;
    if (p.has) h.x = s[0];
    if (p.second) h.y = s[1];
  }
  float pA[2], pS[2], qS[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    pA[k] = 1.f;
    pS[k] = qS[k] = 0.f;
    float as[GLR_STEPS];
#pragma unroll
    for (int r = 0; r < GLR_STEPS; ++r) {
      const Gate<FORM> gt(g[r].at(k));
      as[r] = gt.a;
      if (p.t0 + r < a.c.T) {
        const float b = FORM == GLR_MIX ? gt.na * v[r].at(k) : v[r].at(k);
        if (RESET && (resets >> r & 1)) {
          pA[k] = -0.0f;
          pS[k] = b;
        } else {
          pA[k] = RESET && is_free(pA[k]) ? pA[k] : pA[k] * gt.a;
          pS[k] = fmaf(gt.a, pS[k], b);
        }
      }
    }
#pragma unroll
    for (int r = GLR_STEPS - 1; r >= 0; --r) {
      if (p.t0 + r >= a.c.T) continue;
      qS[k] = RESET && (resets >> r & 1) ? 0.f : as[r] * (d[r].at(k) + qS[k]);
    }
  }
  fwd[p.run * chans + c] = make_float2(pA[0], pS[0]);
  fwd[p.run * chans + c + 1] = make_float2(pA[1], pS[1]);
  Pair end;
  const Pair mu = glr_join<true>(a, p, {pA[0], pA[1]}, {qS[0], qS[1]}, first, end, sh);
  if (p.run == 0 && p.chunk == 0 && a.dh0) {
    if (p.has) a.dh0[at] = end.x;
    if (p.second) a.dh0[at + 1] = end.y;
  }
  if (!p.has) return;
  for (int i = 0; i < p.run; ++i) {
    const float2 x = fwd[i * chans + c], y = fwd[i * chans + c + 1];
    h.x = behind(x.x, x.y, h.x);
    h.y = behind(y.x, y.y, h.y);
  }
  float l[GLR_STEPS][2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float m = k ? mu.y : mu.x;
#pragma unroll
    for (int r = GLR_STEPS - 1; r >= 0; --r) {
      l[r][k] = 0.f;
      if (p.t0 + r >= a.c.T) continue;
      l[r][k] = d[r].at(k) + m;
      m = RESET && (resets >> r & 1) ? 0.f : Gate<FORM>(g[r].at(k)).a * l[r][k];
    }
  }
  E* dg = (E*)a.dgate.data + p.b * a.dgate.stride_b + p.ch;
  E* dv = (E*)a.dvalue.data + p.b * a.dvalue.stride_b + p.ch;
#pragma unroll
  for (int r = 0; r < GLR_STEPS; ++r) {
    const int t = p.t0 + r;
    if (t >= a.c.T) break;
    float og[2], ov[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const Gate<FORM> gt(g[r].at(k));
      const float val = v[r].at(k), cur = k ? h.y : h.x;
      const bool cut = RESET && (resets >> r & 1);
      const float past = cut ? 0.f : cur;
      float next;
      if constexpr (FORM == GLR_MIX) {
        ov[k] = l[r][k] * gt.na;
        og[k] = ov[k] * gt.a * (past - val);
        next = gt.na * val;
      } else {
        ov[k] = l[r][k];
        og[k] = cut ? 0.f : l[r][k] * gt.a * past;
        next = val;
      }
      next = cut ? next : fmaf(gt.a, past, next);
      (k ? h.y : h.x) = next;
    }
    store_pair<E, ALIGNED>(dg + t * a.dgate.stride_t, og[0], og[1], p.second);
    store_pair<E, ALIGNED>(dv + t * a.dvalue.stride_t, ov[0], ov[1], p.second);
  }
}

// Whether two channels of every step of the array are one aligned word.
template <typename E>
static bool pairs(const glr_seq& q, int H) {
  return H % 2 == 0 && q.stride_t % 2 == 0 && q.stride_b % 2 == 0 && (uintptr_t)q.data % (2 * sizeof(E)) == 0;
}

template <typename E, int FORM, bool RESET>
static void glr_start(const GlrArgs& a, bool backward, unsigned grid, hipStream_t s) {
  const int H = a.c.H;
  bool al = pairs<E>(a.gate, H) && pairs<E>(a.value, H);
  al = al && (backward ? pairs<E>(a.dh, H) && pairs<E>(a.dgate, H) && pairs<E>(a.dvalue, H) : pairs<E>(a.h, H));
  const dim3 g(grid), t(GLR_THREADS);
  if (backward) {
    if (al) hipLaunchKernelGGL((glr_backward_kernel<E, true, FORM, RESET>), g, t, 0, s, a);
    else hipLaunchKernelGGL((glr_backward_kernel<E, false, FORM, RESET>), g, t, 0, s, a);
  } else {
    if (al) hipLaunchKernelGGL((glr_forward_kernel<E, true, FORM, RESET>), g, t, 0, s, a);
    else hipLaunchKernelGGL((glr_forward_kernel<E, false, FORM, RESET>), g, t, 0, s, a);
  }
}
template <typename E>
static void glr_form(const GlrArgs& a, bool backward, unsigned grid, hipStream_t s) {
  if (a.c.form == GLR_MIX) {
    if (a.reset) glr_start<E, GLR_MIX, true>(a, backward, grid, s);
    else glr_start<E, GLR_MIX, false>(a, backward, grid, s);
  } else {
    if (a.reset) glr_start<E, GLR_DECAY, true>(a, backward, grid, s);
    else glr_start<E, GLR_DECAY, false>(a, backward, grid, s);
  }
}
static hipError_t glr_launch(const GlrArgs& a, bool backward, hipStream_t s) {
  if (a.s.words) {
    const long long n = a.s.words;
    hipLaunchKernelGGL(glr_clear_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a.words, n,
                       a.ticket);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const unsigned grid = (unsigned)((long long)a.s.chunks * a.s.cols * a.c.B);
  if (a.c.dtype == MGRIT_F32) glr_form<float>(a, backward, grid, s);
  else if (a.c.dtype == MGRIT_BF16) glr_form<Bf16>(a, backward, grid, s);
  else glr_form<F16>(a, backward, grid, s);
  return hipGetLastError();
}
hipError_t launch_glr_forward(const GlrArgs& a, hipStream_t s) { return glr_launch(a, false, s); }
hipError_t launch_glr_backward(const GlrArgs& a, hipStream_t s) { return glr_launch(a, true, s); }

// One step: two channels per thread.
template <typename E, bool ALIGNED, int FORM>
__global__ __launch_bounds__(256) void glr_step_kernel(GlrStepArgs a) {
  const int pairs = (a.c.H + 1) / 2;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const int b = (int)(i / pairs), ch = 2 * (int)(i - (long long)b * pairs);
  if (b >= a.c.B) return;
  const bool second = ch + 1 < a.c.H;
  E* out = (E*)a.h.data + b * a.h.stride_b + ch;
  const int slot = a.slots ? a.slots[b] : b;
  if (slot < 0 || slot >= a.n_slots) {
    store_pair<E, ALIGNED>(out, 0.f, 0.f, second);
    return;
  }
  const RawPair<E> g = load_pair<E, ALIGNED>((const E*)a.gate.data + b * a.gate.stride_b + ch, second);
  const RawPair<E> v = load_pair<E, ALIGNED>((const E*)a.value.data + b * a.value.stride_b + ch, second);
  const bool cut = a.reset && a.reset[b];
  const long long at = (long long)slot * a.c.H + ch;
  float h[2] = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (k && !second) break;
    const Gate<FORM> gt(g.at(k));
    const float in = FORM == GLR_MIX ? gt.na * v.at(k) : v.at(k);
    h[k] = cut ? in : fmaf(gt.a, a.state_in[at + k], in);
    a.state_out[at + k] = h[k];
  }
  store_pair<E, ALIGNED>(out, h[0], h[1], second);
}

template <typename E>
static void glr_step_start(const GlrStepArgs& a, hipStream_t s) {
  auto one = [&](glr_seq q) {
    q.stride_t = 0;
    return pairs<E>(q, a.c.H);
  };
  const bool al = one(a.gate) && one(a.value) && one(a.h);
  const dim3 g((unsigned)(((long long)a.c.B * ((a.c.H + 1) / 2) + 255) / 256)), t(256);
  if (a.c.form == GLR_MIX) {
    if (al) hipLaunchKernelGGL((glr_step_kernel<E, true, GLR_MIX>), g, t, 0, s, a);
    else hipLaunchKernelGGL((glr_step_kernel<E, false, GLR_MIX>), g, t, 0, s, a);
  } else {
    if (al) hipLaunchKernelGGL((glr_step_kernel<E, true, GLR_DECAY>), g, t, 0, s, a);
    else hipLaunchKernelGGL((glr_step_kernel<E, false, GLR_DECAY>), g, t, 0, s, a);
  }
}
hipError_t launch_glr_step(const GlrStepArgs& a, hipStream_t s) {
  if (a.c.dtype == MGRIT_F32) glr_step_start<float>(a, s);
  else if (a.c.dtype == MGRIT_BF16) glr_step_start<Bf16>(a, s);
  else glr_step_start<F16>(a, s);
  return hipGetLastError();
}

}  // namespace mg
