// Gated linear recurrence h_t = a_t h_{t-1} + b_t (include/mgrit_ops.h), its adjoint, and one step of it.
//
// A run of steps is the map h -> A h + S with A = prod a, S its result from a zero state, and two runs behind each
// other compose to (A2 A1, A2 S1 + S2): that is all a sequence needs to be cut up.  A workgroup reads its tile once,
// into registers; every lane goes through its run of 8 or 16 steps from a zero state; the runs of the tile meet in
// LDS; the tiles of a sequence meet in the workspace, where each leaves its (A, S) as soon as it has read its tile
// and, once it knows the state before it, the state behind it.  The bytes are those of the arrays, each read or
// written once.
//
// The word of a tile and channel is A in the low half and S in the high one, stored by one 64-bit store, so that a
// reader that sees one sees the other.  All bits set: not written yet (no A is stored so).  A = -0: S does not depend
// on what was before (a reset, or the state itself: what a tile knows once it knows the state before it).  No other A
// is -0: no a is negative, so that a product that underflows is +0, and a state that is not finite does not become
// finite again (0 times it is NaN) as long as no reset stands in between.  The state before a tile is always computed
// as S + A h tile by tile, by the tile itself (glr_join) as by those behind it that find the map and not yet the
// state (window_state): the two round alike, and the result does not depend on timing.
//
// Tiles are taken by a ticket, first tiles first (the adjoint: last tiles first), so that those a workgroup waits for
// have been started, wait for none behind it, and every wait ends.
#include <type_traits>

#include "elem.h"
#include "ops.h"
#include "pairs.h"

namespace mg {

constexpr int GLR_THREADS = GLR_WAVES * 64;
constexpr int GLR_CHANNELS = 128;                   // channels of a tile at most
constexpr int GLR_WORDS = 2048;                     // words looked at at a time: 16 tiles of 128 channels, 32 of 64
constexpr unsigned GLR_NONE = 0xffffffffu, GLR_FREE = 0x80000000u;

struct Pair {
  float x, y;
};

// a and, for GLR_MIX, 1 - a of a gate, both to a few units of their own last place: with e = exp(-|g|), the smaller
// of the two is e / (1 + e) at any g, and the larger one 1 minus that.
template <int FORM>
struct Gate {
  float a, na;
  __device__ inline explicit Gate(float g) {
    if constexpr (FORM == GLR_MIX) {
      const float e = exp_of(-fabsf(g));
      const float s = e * __builtin_amdgcn_rcpf(1.0f + e), l = 1.0f - s;
      a = g < 0.0f ? s : l;
      na = g < 0.0f ? l : s;
    } else {
      a = exp_of(g);
      na = 1.0f;
    }
  }
};
// The same as the adjoint keeps it between its sweeps.  BOTH: a and 1 - a (16-bit arrays leave the registers for it,
// and it saves instructions).  Otherwise one float, the smaller of the two under the sign of g, which
// says which it is.
template <int FORM, bool BOTH>
struct KeptGate {
  float v, w;
  __device__ inline void set(float g) {
    if constexpr (FORM == GLR_MIX && !BOTH) {
      const float e = exp_of(-fabsf(g));
      v = copysignf(e * __builtin_amdgcn_rcpf(1.0f + e), g);
    } else {
      const Gate<FORM> gt(g);
      v = gt.a;
      w = gt.na;
    }
  }
  // What was computed from it is computed again from here on rather than kept: registers are what the adjoint lacks.
  __device__ inline void anew() {
    if constexpr (!BOTH) asm volatile("" : "+v"(v));
  }
  __device__ inline bool small_a() const { return (int)__float_as_uint(v) < 0; }
  __device__ inline float a() const {
    return FORM == GLR_DECAY || BOTH ? v : small_a() ? fabsf(v) : 1.0f - fabsf(v);
  }
  __device__ inline float na() const {
    return FORM == GLR_DECAY ? 1.0f : BOTH ? w : small_a() ? 1.0f - fabsf(v) : fabsf(v);
  }
};

__device__ inline bool is_free(float A) { return __float_as_uint(A) == GLR_FREE; }
// GLR_DECAY: gates above 0 are allowed, and the product of a run's a can be beyond the floats.  A state of zero stays
// what it is then, and what a run has forgotten stays forgotten (infinity times 0 would be NaN).

// A of a run behind another run.
template <int FORM>
__device__ inline float both(float A, float before) {
  if (is_free(A) || is_free(before)) return -0.0f;
  return FORM == GLR_DECAY && before == 0.f ? 0.f : A * before;
}
// The state behind a run (A, S) that knows no reset, and behind any run, from the state h before it.
template <int FORM>
__device__ inline float behind_whole(float A, float S, float h) {
  return FORM == GLR_DECAY && h == 0.f ? S : fmaf(A, h, S);
}
template <int FORM>
__device__ inline float behind(float A, float S, float h) {
  return is_free(A) ? S : behind_whole<FORM>(A, S, h);
}

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

// (an even number of words)
__global__ __launch_bounds__(256) void glr_clear_kernel(unsigned long long* words, long long n, int* ticket) {
  const long long i = 2 * ((long long)blockIdx.x * 256 + threadIdx.x);
  if (i < n) *reinterpret_cast<ulonglong2*>(words + i) = make_ulonglong2(~0ull, ~0ull);
  if (i == 0) *ticket = 0;
}

// Where a thread stands.  LANES > 0: that many lanes across the channels, and strides that allow 32-bit offsets
// within a wave: tile, channels and steps are the wave's (in scalar registers), and a lane has an offset in it.  0:
// as the shape says, any strides.  STEPS: of a run.
template <int LANES, int STEPS>
struct GlrPlace {
  int lanes, lane_c;                   // lanes across the channels, this one's place
  int run, chunk, b;                   // run of the tile, tile, batch row
  int ch0, ch;                         // first channel of the tile, of the lane
  int t0, wave_t0;                     // first step of the run, of the wave
  bool has, second;                    // whether channels ch and ch + 1 exist
  __device__ inline GlrPlace(const GlrArgs& a, int tile, bool backward) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lanes = LANES ? LANES : a.s.lanes;
    lane_c = lane & (lanes - 1);
    run = wave * (64 / lanes) + (LANES == 64 ? 0 : lane / lanes);
    tile = __builtin_amdgcn_readfirstlane(tile);
    const int across = a.s.cols * a.c.B;
    const int k = tile / across, rest = tile - k * across;
    chunk = backward ? a.s.chunks - 1 - k : k;
    b = rest / a.s.cols;
    ch0 = (rest - b * a.s.cols) * 2 * lanes;
    ch = ch0 + 2 * lane_c;
    wave_t0 = chunk * a.s.steps + wave * (64 / lanes) * STEPS;
    t0 = wave_t0 + (LANES == 64 ? 0 : lane / lanes * STEPS);
    has = ch < a.c.H;
    second = ch + 1 < a.c.H;
  }
  __device__ inline int runs() const { return GLR_THREADS / lanes; }
  // the wave's steps all lie within the sequence
  __device__ inline bool inside(const GlrArgs& a) const { return wave_t0 + 64 / lanes * STEPS <= a.c.T; }
};

// Bits of the steps of the thread's run that reset (each of the first lanes of a run looks at one step).
template <int LANES, int STEPS>
__device__ inline unsigned reset_bits(const GlrArgs& a, const GlrPlace<LANES, STEPS>& p) {
  if (!a.reset) return 0;
  const int t = p.t0 + p.lane_c;
  bool r = false;
  if (p.lane_c < STEPS && t < a.c.T) r = a.reset[(long long)t * a.c.B + p.b] != 0;
  const unsigned long long all = __ballot(r);
  return (unsigned)(LANES == 64 ? all : all >> ((threadIdx.x & 63) / p.lanes * p.lanes)) & ((1u << STEPS) - 1);
}
// Whether no step of the wave's runs resets or lies behind the sequence's end: the same answer in all lanes of the
// wave, whose sweeps then look at neither.
template <int LANES, int STEPS>
__device__ inline bool glr_whole(const GlrArgs& a, const GlrPlace<LANES, STEPS>& p, unsigned resets) {
  return p.inside(a) && !__any(resets != 0);
}

// The steps of a thread's run in an array, from step t on.  LANES > 0: the wave's place and a 32-bit offset (the host
// has looked at the strides).
template <typename E, int LANES, int STEPS>
struct RunOf {
  char* base;
  long long far, stride;                // bytes; far: LANES == 0
  unsigned off;
  __device__ inline RunOf(const glr_seq& q, const GlrArgs& a, const GlrPlace<LANES, STEPS>& p, int t, int lane_c) {
    const int from = LANES ? min(p.wave_t0, a.c.T - 1) : 0;
    stride = q.stride_t * (long long)sizeof(E);
    base = (char*)q.data + (p.b * q.stride_b + p.ch0) * (long long)sizeof(E) + from * stride;
    off = 2 * lane_c * sizeof(E);
    far = 0;
    if (LANES) off += (unsigned)(t - from) * (unsigned)stride;
    else far = t * stride;
  }
  __device__ inline E* at() const { return (E*)(LANES ? base + off : base + far + off); }
  __device__ inline void next() {
    if (LANES) off += (unsigned)stride;
    else far += stride;
  }
};

// The steps of a run of an input array; steps and channels that do not exist are read at one that does.
template <typename E, bool ALIGNED, int LANES, int STEPS>
__device__ inline void load_run(const glr_seq& q, const GlrArgs& a, const GlrPlace<LANES, STEPS>& p,
                                RawPair<E> (&v)[STEPS]) {
  const int lane_c = p.has ? p.lane_c : 0;
  const bool second = p.ch0 + 2 * lane_c + 1 < a.c.H;
  RunOf<E, LANES, STEPS> run(q, a, p, min(p.t0, a.c.T - 1), lane_c);
  if (p.inside(a)) {
#pragma unroll
    for (int r = 0; r < STEPS; ++r, run.next()) v[r] = load_pair<E, ALIGNED>(run.at(), second);
  } else {
#pragma unroll
    for (int r = 0; r < STEPS; ++r) {
      v[r] = load_pair<E, ALIGNED>(run.at(), second);
      if (p.t0 + r + 1 < a.c.T) run.next();
    }
  }
}

// Steps behind the sequence's end change nothing: a = 1, b = 0.
template <int FORM, typename E, int LANES, int STEPS>
__device__ inline void clear_tail(const GlrArgs& a, const GlrPlace<LANES, STEPS>& p, RawPair<E> (&g)[STEPS],
                                  RawPair<E> (&v)[STEPS]) {
#pragma unroll
  for (int r = 0; r < STEPS; ++r)
    if (p.t0 + r >= a.c.T) {
      g[r].set(FORM == GLR_MIX ? __builtin_inff() : 0.f);
      v[r].set(0.f);
    }
}

// x, or 0 (whatever x is) at a step that resets
__device__ inline float unless(unsigned resets, int r, float x) { return resets >> r & 1 ? 0.f : x; }

struct GlrShared {
  float4 run[GLR_THREADS];                          // (A, S) of runs and channels
  unsigned long long window[GLR_WORDS];
  float carry[GLR_CHANNELS];                        // state before the tile
  int tile;
};

// The state before a tile from the n words of the tiles before it that the window holds for a channel (word 0 the
// nearest): false where a word that is needed is not there yet.  The words are read four at a time.
template <int FORM>
__device__ inline bool window_state(const unsigned long long* w, int n, int stride, float& h) {
  int at = -1;
  bool stop = false;
  for (int i0 = 0; i0 < n && !stop; i0 += 4) {
    unsigned A[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) A[k] = (unsigned)w[min(i0 + k, n - 1) * stride];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (stop || i0 + k >= n) continue;
      stop = A[k] == GLR_NONE || A[k] == GLR_FREE;
      if (A[k] == GLR_FREE) at = i0 + k;
    }
  }
  if (at < 0) return false;
  h = __uint_as_float((unsigned)(w[at * stride] >> 32));
  for (int i0 = (at - 1) & ~3; i0 >= 0; i0 -= 4) {
    unsigned long long v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = w[min(i0 + k, at) * stride];
#pragma unroll
    for (int k = 3; k >= 0; --k)
      if (i0 + k < at)
        h = behind_whole<FORM>(__uint_as_float((unsigned)v[k]), __uint_as_float((unsigned)(v[k] >> 32)), h);
  }
  return true;
}

// The state before tile `chunk` of the thread's two channels, in sh.carry, from the words of
// the tiles before it (backward: behind it), whose distance is 1, 2, ...  All threads of the workgroup call it.
template <int FORM, int LANES, int STEPS>
__device__ inline void glr_look_back(const GlrArgs& a, const GlrPlace<LANES, STEPS>& p, bool backward,
                                     GlrShared& sh) {
  const int before = backward ? a.s.chunks - 1 - p.chunk : p.chunk;
  const int runs = p.runs(), chans = 2 * p.lanes, n = min(before, GLR_WORDS / chans);
  const long long per_tile = (long long)a.c.B * a.s.cols * chans;
  const long long at = (long long)p.b * a.s.cols * chans + p.ch;
  for (;;) {
    for (int i = p.run; i < n; i += runs) {
      const int other = backward ? p.chunk + 1 + i : p.chunk - 1 - i;
      const unsigned long long* w = a.words + other * per_tile + at;
      sh.window[i * chans + 2 * p.lane_c] = load_word(w);
      sh.window[i * chans + 2 * p.lane_c + 1] = load_word(w + 1);
    }
    __syncthreads();
    int ok = 1;
    if (p.run < 2) {                                  // run 0: channel ch, run 1: ch + 1
      float h = 0.f;
      ok = window_state<FORM>(&sh.window[2 * p.lane_c + p.run], n, chans, h);
      sh.carry[2 * p.lane_c + p.run] = h;
    }
    if (__syncthreads_and(ok)) return;
    __builtin_amdgcn_s_sleep(1);
  }
}

// (A, S) per channel of the runs before the thread's own in its tile, from the own one, through LDS (`all`).  32
// lanes: the halves of a wave meet by exchange, the waves in LDS.  before_barrier() is called in front of the
// barrier.
template <bool BACKWARD, int FORM, int LANES, int STEPS, typename FN>
__device__ inline void runs_before(const GlrPlace<LANES, STEPS>& p, Pair A, Pair S, float4* all, Pair& pA, Pair& pS,
                                   FN before_barrier) {
  auto behind_it = [&](const float4& x) {             // one more run: (A, S) of either channel
    pS.x = behind<FORM>(x.x, x.y, pS.x);
    pS.y = behind<FORM>(x.z, x.w, pS.y);
    pA.x = both<FORM>(x.x, pA.x);
    pA.y = both<FORM>(x.z, pA.y);
  };
  pA = {1.f, 1.f};
  pS = {0.f, 0.f};
  if constexpr (LANES > 0) {
    const int wave = p.run / (64 / LANES);
    // the other half's run, and whether it lies before the own one
    const bool later = LANES == 64 || ((threadIdx.x & 32) ? !BACKWARD : BACKWARD);
    float4 other = {1.f, 0.f, 1.f, 0.f};
    if constexpr (LANES == 32)
      other = make_float4(__shfl_xor(A.x, 32, 64), __shfl_xor(S.x, 32, 64), __shfl_xor(A.y, 32, 64),
                          __shfl_xor(S.y, 32, 64));
    float4 mine = {A.x, S.x, A.y, S.y};
    if constexpr (LANES == 32)
      mine = make_float4(both<FORM>(A.x, other.x), behind<FORM>(A.x, S.x, other.y), both<FORM>(A.y, other.z),
                         behind<FORM>(A.y, S.y, other.w));
    if (later) all[wave * LANES + p.lane_c] = mine;
    before_barrier();
    __syncthreads();
    const int n = BACKWARD ? GLR_WAVES - 1 - wave : wave;
#pragma unroll
    for (int i = 0; i < GLR_WAVES - 1; i += 2) {     // (two at a time: the sweeps' results hold the registers)
      if (i >= n) break;
      const float4 x = all[(BACKWARD ? GLR_WAVES - 1 - i : i) * LANES + p.lane_c];
      const float4 y = all[(BACKWARD ? GLR_WAVES - 2 - i : i + 1) * LANES + p.lane_c];
      behind_it(x);
      if (i + 1 < n) behind_it(y);
    }
    if (LANES == 32 && later) behind_it(other);
  } else {
    const int runs = p.runs();
    all[p.run * p.lanes + p.lane_c] = make_float4(A.x, S.x, A.y, S.y);
    before_barrier();
    __syncthreads();
    for (int i = 0; i < (BACKWARD ? runs - 1 - p.run : p.run); ++i)
      behind_it(all[(BACKWARD ? runs - 1 - i : i) * p.lanes + p.lane_c]);
  }
}

// What both directions do between their sweeps: from (A, S) of the thread's run, per channel, the state before
// the run.  first: the state before the sequence's first tile (backward: behind its last one).  The threads of the
// tile's last run (backward: its first) get in `out` the state behind the tile.
template <bool BACKWARD, int FORM, int LANES, int STEPS>
__device__ inline Pair glr_join(const GlrArgs& a, const GlrPlace<LANES, STEPS>& p, Pair A, Pair S, Pair first,
                                Pair& out, GlrShared& sh) {
  const int chans = 2 * p.lanes, runs = p.runs(), c = 2 * p.lane_c;
  const bool at_start = BACKWARD ? p.chunk == a.s.chunks - 1 : p.chunk == 0;
  const bool chain = a.s.chunks > 1;
  const int place = BACKWARD ? runs - 1 - p.run : p.run;      // runs of the tile before this one
  Pair pA, pS;
  runs_before<BACKWARD, FORM, LANES, STEPS>(p, A, S, sh.run, pA, pS, [&]() {
    if (at_start && place == 0) {
      sh.carry[c] = first.x;
      sh.carry[c + 1] = first.y;
    }
  });
  unsigned long long* word =
      a.words + (((long long)p.chunk * a.c.B + p.b) * a.s.cols) * chans + p.ch;
  const bool last = place == runs - 1;
  // the tile's own map (in the last run): what a reader composes and the state behind it are formed from the same A
  // and S
  const Pair tA = {both<FORM>(A.x, pA.x), both<FORM>(A.y, pA.y)};
  const Pair tS = {behind<FORM>(A.x, S.x, pS.x), behind<FORM>(A.y, S.y, pS.y)};
  if (last && chain && !at_start) {
    store_word(word, make_word(tA.x, tS.x));
    store_word(word + 1, make_word(tA.y, tS.y));
  }
  if (!at_start) glr_look_back<FORM>(a, p, BACKWARD, sh);
  const Pair carry = {sh.carry[c], sh.carry[c + 1]};
  if (last) {
    out.x = behind<FORM>(tA.x, tS.x, carry.x);
    out.y = behind<FORM>(tA.y, tS.y, carry.y);
    if (chain) {
      store_word(word, make_word(-0.0f, out.x));
      store_word(word + 1, make_word(-0.0f, out.y));
    }
  }
  const Pair h = {behind<FORM>(pA.x, pS.x, carry.x), behind<FORM>(pA.y, pS.y, carry.y)};
  return h;
}

__device__ inline int glr_tile(const GlrArgs& a, GlrShared& sh) {
  if (a.s.chunks == 1) return blockIdx.x;
  if (threadIdx.x == 0) sh.tile = atomicAdd(a.ticket, 1);
  __syncthreads();
  return sh.tile;
}

// Memory bounds it where a sequence is one tile (128 x 100 x 1000 floats: 154 MB in 30 us, 5.2 TB/s); over several
// tiles it is the wait for those before (16384 x 4 x 1024 bf16: 403 MB in 102 us; copies whose tiles did not wait
// took 78).  Runs of 16 steps halve the tiles against runs of 8 (143 us), and 128 channels make a row's piece 256
// bytes.
template <typename E, bool ALIGNED, int FORM, int LANES>
__global__ __launch_bounds__(GLR_THREADS, 4) void glr_forward_kernel(GlrArgs a) {
  constexpr int STEPS = GLR_RUN_FWD;
  __shared__ GlrShared sh;
  const GlrPlace<LANES, STEPS> p(a, glr_tile(a, sh), false);
  RawPair<E> g[STEPS], v[STEPS];
  load_run<E, ALIGNED, LANES, STEPS>(a.gate, a, p, g);
  load_run<E, ALIGNED, LANES, STEPS>(a.value, a, p, v);
  const unsigned resets = reset_bits(a, p);
  const int runs = p.runs();
  Pair first = {0.f, 0.f};
  if (p.chunk == 0 && a.h0 && p.run == 0) {
    const long long at = (long long)p.b * a.c.H + p.ch;
    if (p.has) first.x = a.h0[at];
    if (p.second) first.y = a.h0[at + 1];
  }
  // (floats: one form of the sweep for all, which memory bounds; two would take more registers than there are)
  const bool whole = sizeof(E) == 2 && glr_whole(a, p, resets);
  // from a zero state: S[r], and A[r] of the steps up to r
  float A[STEPS][2], S[STEPS][2];
  auto sweep = [&](auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    float pa[2] = {1.f, 1.f}, ps[2] = {0.f, 0.f};
#pragma unroll
    for (int r = 0; r < STEPS; ++r) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const Gate<FORM> gt(g[r].at(k));
        const float b = FORM == GLR_MIX ? gt.na * v[r].at(k) : v[r].at(k);
        pa[k] *= gt.a;
        ps[k] = MASKED && (resets >> r & 1) ? b : fmaf(gt.a, ps[k], b);
        A[r][k] = MASKED && (resets & ((2u << r) - 1)) ? -0.0f : pa[k];
        S[r][k] = ps[k];
      }
    }
  };
  if (whole) {
    sweep(std::false_type{});
  } else {
    clear_tail<FORM>(a, p, g, v);
    sweep(std::true_type{});
  }
  constexpr int L = STEPS - 1;
  Pair end = {0.f, 0.f};
  const Pair h = glr_join<false, FORM, LANES, STEPS>(a, p, {A[L][0], A[L][1]}, {S[L][0], S[L][1]}, first, end, sh);
  const long long at = (long long)p.b * a.c.H + p.ch;
  if (a.saved && p.t0 % a.save == 0 && p.t0 < a.c.T) {
    float* s = a.saved + (long long)(p.t0 / a.save) * a.c.B * a.c.H + at;
    if (p.has) s[0] = h.x;
    if (p.second) s[1] = h.y;
  }
  if (p.run == runs - 1 && a.h_last && p.chunk == a.s.chunks - 1) {
    // h_last may be h0 itself, and behind a reset nothing so far has waited for the first tile, whose word says that
    // it has read h0 (that tile waits for none)
    if (a.h_last == a.h0 && p.chunk > 0) {
      const unsigned long long* w = a.words + (long long)p.b * a.s.cols * 2 * p.lanes + p.ch;
      while ((unsigned)load_word(w) == GLR_NONE) __builtin_amdgcn_s_sleep(1);
    }
    if (p.has) a.h_last[at] = end.x;
    if (p.second) a.h_last[at + 1] = end.y;
  }
  if (!p.has) return;
  RunOf<E, LANES, STEPS> out(a.h, a, p, min(p.t0, a.c.T - 1), p.lane_c);
  auto write = [&](auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
#pragma unroll
    for (int r = 0; r < STEPS; ++r, out.next()) {
      const float x = MASKED ? behind<FORM>(A[r][0], S[r][0], h.x) : behind_whole<FORM>(A[r][0], S[r][0], h.x);
      const float y = MASKED ? behind<FORM>(A[r][1], S[r][1], h.y) : behind_whole<FORM>(A[r][1], S[r][1], h.y);
      if (!MASKED || p.t0 + r < a.c.T) store_pair<E, ALIGNED>(out.at(), x, y, p.second, a.past);
    }
  };
  if (whole) write(std::false_type{});
  else write(std::true_type{});
}

// mu_t = a_t l_t is what step t hands on to step t - 1: mu -> a (dh + mu), the same composition from the other end.
// 128 x 100 x 1000 floats: 256 MB in 58 us (4.4 TB/s); 16384 x 4 x 1024 bf16: 671 MB in 174 us (3.9 TB/s), where its
// waves wait for 57 % of their cycles, for the tiles behind and for memory, two workgroups a CU; arithmetic, 54
// vector instructions a value, is next.  Runs of 8 steps: with 16 the three arrays, the gates and the adjoints do not
// fit 128 registers (267 us).
template <typename E, bool ALIGNED, int FORM, int LANES>
__global__ __launch_bounds__(GLR_THREADS, 4) void glr_backward_kernel(GlrArgs a) {
  constexpr int STEPS = GLR_RUN_BWD;
  __shared__ GlrShared sh;
  __shared__ float4 fwd[GLR_THREADS];               // (A, S) of runs and channels, forward
  const GlrPlace<LANES, STEPS> p(a, glr_tile(a, sh), true);
  RawPair<E> g[STEPS], v[STEPS], d[STEPS];
  load_run<E, ALIGNED, LANES, STEPS>(a.gate, a, p, g);
  load_run<E, ALIGNED, LANES, STEPS>(a.value, a, p, v);
  load_run<E, ALIGNED, LANES, STEPS>(a.dh, a, p, d);
  const unsigned resets = reset_bits(a, p);
  const long long at = (long long)p.b * a.c.H + p.ch;
  const int runs = p.runs();
  Pair first = {0.f, 0.f}, h = {0.f, 0.f};
  if (p.chunk == a.s.chunks - 1 && a.dh_last && p.run == runs - 1) {
    if (p.has) first.x = a.dh_last[at];
    if (p.second) first.y = a.dh_last[at + 1];
  }
  {
    const float* s = a.saved + (long long)p.chunk * a.c.B * a.c.H + at;
    if (p.has) h.x = s[0];
    if (p.second) h.y = s[1];
  }
  const bool whole = glr_whole(a, p, resets);
  KeptGate<FORM, sizeof(E) == 2> gk[STEPS][2];
  auto anew = [&]() {
#pragma unroll
    for (int r = 0; r < STEPS; ++r) {
      gk[r][0].anew();
      gk[r][1].anew();
      v[r].anew();
    }
  };
  float pA[2], pS[2], qS[2];
  auto sums = [&](auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    pA[0] = pA[1] = 1.f;
    pS[0] = pS[1] = qS[0] = qS[1] = 0.f;
#pragma unroll
    for (int r = 0; r < STEPS; ++r)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        gk[r][k].set(g[r].at(k));
        const float ga = gk[r][k].a();
        const float b = FORM == GLR_MIX ? gk[r][k].na() * v[r].at(k) : v[r].at(k);
        pA[k] *= ga;
        pS[k] = MASKED && (resets >> r & 1) ? b : fmaf(ga, pS[k], b);
      }
    anew();
#pragma unroll
    for (int r = STEPS - 1; r >= 0; --r)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        qS[k] = gk[r][k].a() * (d[r].at(k) + qS[k]);
        if (MASKED) qS[k] = unless(resets, r, qS[k]);
      }
    if (MASKED && resets) pA[0] = pA[1] = -0.0f;
  };
  if (whole) {
    sums(std::false_type{});
  } else {
    clear_tail<FORM>(a, p, g, v);
#pragma unroll
    for (int r = 0; r < STEPS; ++r)
      if (p.t0 + r >= a.c.T) d[r].set(0.f);
    sums(std::true_type{});
  }
  anew();
  Pair fA, fS;
  runs_before<false, FORM, LANES, STEPS>(p, {pA[0], pA[1]}, {pS[0], pS[1]}, fwd, fA, fS, []() {});
  h.x = behind<FORM>(fA.x, fS.x, h.x);
  h.y = behind<FORM>(fA.y, fS.y, h.y);
  Pair end = {0.f, 0.f};
  const Pair mu = glr_join<true, FORM, LANES, STEPS>(a, p, {pA[0], pA[1]}, {qS[0], qS[1]}, first, end, sh);
  if (p.run == 0 && p.chunk == 0 && a.dh0) {
    if (p.has) a.dh0[at] = end.x;
    if (p.second) a.dh0[at + 1] = end.y;
  }
  if (!p.has) return;
  const int from = min(p.t0, a.c.T - 1);
  RunOf<E, LANES, STEPS> dg(a.dgate, a, p, from, p.lane_c), dv(a.dvalue, a, p, from, p.lane_c);
  auto write = [&](auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    float l[STEPS][2], m[2] = {mu.x, mu.y};
#pragma unroll
    for (int r = STEPS - 1; r >= 0; --r)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        l[r][k] = d[r].at(k) + m[k];
        m[k] = gk[r][k].a() * l[r][k];
        if (MASKED) m[k] = unless(resets, r, m[k]);
      }
    anew();
#pragma unroll
    for (int r = 0; r < STEPS; ++r) {
      float og[2], ov[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float ga = gk[r][k].a(), val = v[r].at(k);
        float past = k ? h.y : h.x, in = val;
        if (MASKED) past = unless(resets, r, past);
        if constexpr (FORM == GLR_MIX) {
          const float na = gk[r][k].na();
          ov[k] = l[r][k] * na;
          og[k] = ov[k] * ga * (past - val);
          in = na * val;
        } else {
          ov[k] = l[r][k];
          og[k] = l[r][k] * ga * past;
          if (MASKED) og[k] = unless(resets, r, og[k]);
        }
        (k ? h.y : h.x) = MASKED && (resets >> r & 1) ? in : fmaf(ga, past, in);
      }
      if (!MASKED || p.t0 + r < a.c.T) {
        store_pair<E, ALIGNED>(dg.at(), og[0], og[1], p.second, a.past);
        store_pair<E, ALIGNED>(dv.at(), ov[0], ov[1], p.second, a.past);
      }
      dg.next();
      dv.next();
    }
  };
  if (whole) write(std::false_type{});
  else write(std::true_type{});
}

// Whether the steps of a wave lie within 32-bit offsets.
static bool near(const glr_seq& q, int size) { return !q.data || q.stride_t * size < (1LL << 27); }

template <typename E, int FORM>
static void glr_start(const GlrArgs& a, bool backward, unsigned grid, hipStream_t s) {
  const int H = a.c.H, e = sizeof(E);
  bool al = pairs<E>(a.gate, H) && pairs<E>(a.value, H);
  al = al && (backward ? pairs<E>(a.dh, H) && pairs<E>(a.dgate, H) && pairs<E>(a.dvalue, H) : pairs<E>(a.h, H));
  const bool wide = a.s.lanes == (backward ? 32 : 64) && near(a.gate, e) && near(a.value, e) && near(a.h, e) &&
                    near(a.dh, e) && near(a.dgate, e) && near(a.dvalue, e);
  const dim3 g(grid), t(GLR_THREADS);
  if (backward) {
    if (al && wide) hipLaunchKernelGGL((glr_backward_kernel<E, true, FORM, 32>), g, t, 0, s, a);
    else if (al) hipLaunchKernelGGL((glr_backward_kernel<E, true, FORM, 0>), g, t, 0, s, a);
    else if (wide) hipLaunchKernelGGL((glr_backward_kernel<E, false, FORM, 32>), g, t, 0, s, a);
    else hipLaunchKernelGGL((glr_backward_kernel<E, false, FORM, 0>), g, t, 0, s, a);
  } else {
    if (al && wide) hipLaunchKernelGGL((glr_forward_kernel<E, true, FORM, 64>), g, t, 0, s, a);
    else if (al) hipLaunchKernelGGL((glr_forward_kernel<E, true, FORM, 0>), g, t, 0, s, a);
    else if (wide) hipLaunchKernelGGL((glr_forward_kernel<E, false, FORM, 64>), g, t, 0, s, a);
    else hipLaunchKernelGGL((glr_forward_kernel<E, false, FORM, 0>), g, t, 0, s, a);
  }
}
template <typename E>
static void glr_form(const GlrArgs& a, bool backward, unsigned grid, hipStream_t s) {
  if (a.c.form == GLR_MIX) glr_start<E, GLR_MIX>(a, backward, grid, s);
  else glr_start<E, GLR_DECAY>(a, backward, grid, s);
}
static hipError_t glr_launch(const GlrArgs& a, bool backward, hipStream_t s) {
  if (a.s.words) {
    const long long n = a.s.words;
    hipLaunchKernelGGL(glr_clear_kernel, dim3((unsigned)((n + 511) / 512)), dim3(256), 0, s, a.words, n,
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

// One step: two channels per thread.  100 rows of 1024 bf16: 3.0 us, the latency of slot, gates and state one after
// the other.
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
  const bool al = pairs<E>(a.gate, a.c.H) && pairs<E>(a.value, a.c.H) && pairs<E>(a.h, a.c.H);
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
