// Selective state space scan (include/mgrit_tokens.h), its adjoint, and one step of it.
//
// Four lanes are a channel, each with a quarter of its states; 16 channels are a wave.  What a channel has per step
// (d, x, gates) is computed for four steps at a time, one by each of its lanes, and handed round by quad permutations;
// sums over the states are exchanges between the four lanes.  b and c, the same for all channels, are staged in LDS a
// tile of steps at a time.
//
// Where there are too few channels and batch rows to fill the card, a sequence is cut into chunks.  A chunk is the map
// h -> P h + S with S its result from a zero state and P = exp(a sum d): first every chunk's S and sum of d, then the
// states between chunks, one chunk after the other, then the chunks from their true states.
#include <type_traits>

#include "elem.h"
#include "pairs.h"
#include "row_sums.h"
#include "tokens.h"

namespace mg {

// (arrays that a call takes by reference would be in memory)
#define SSM_INLINE __attribute__((always_inline))

constexpr int SSM_THREADS = 256, SSM_COLS = 64, SSM_TILE = 16;

// ---- lanes of a channel
template <int J>
__device__ inline float quad_of(float v) {                // lane J of the four
  return __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), J * 0x55, 0xf, 0xf, true));
}
__device__ inline float quad_xor1(float v) {
  return __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0xb1, 0xf, 0xf, true));
}
__device__ inline float quad_xor2(float v) {
  return __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x4e, 0xf, 0xf, true));
}
// p[j] of every lane: the sum over the four lanes of p[q] in lane q.
__device__ inline float quad_sums(const float (&p)[4], int q) {
  const bool odd = q & 1, high = q & 2;
  const float a = (odd ? p[1] : p[0]) + quad_xor1(odd ? p[0] : p[1]);
  const float b = (odd ? p[3] : p[2]) + quad_xor1(odd ? p[2] : p[3]);
  return (high ? b : a) + quad_xor2(high ? a : b);
}
__device__ inline float quad_sum(float v) {
  v += quad_xor1(v);
  return v + quad_xor2(v);
}

// ---- elementwise
// softplus(v) and its derivative sigmoid(v).  With e = exp(-|v|): softplus = max(v, 0) + log(1 + e), and log(1 + e) is
// log u + c for u = 1 + e as rounded and c = e - (u - 1) what the rounding left (exact; c / u would be nearer by c e / u, at
// most 2^-24 of the result).
struct Softplus {
  float d, e;
  __device__ inline explicit Softplus(float v) {
    e = exp_of(-fabsf(v));
    const float u = 1.0f + e, c = e - (u - 1.0f);
    d = fmaxf(v, 0.f) + fmaf(__builtin_amdgcn_logf(u), LN2, c);
  }
  __device__ inline float slope(float v) const {
    const float r = __builtin_amdgcn_rcpf(1.0f + e);
    return v < 0.f ? e * r : r;
  }
};
// ---- states of a lane
typedef float Quad __attribute__((ext_vector_type(4), aligned(4)));
template <int SP>
__device__ inline void load_states(const float* p, int S, int n0, float (&v)[SP]) {
  if constexpr (SP >= 4) {
    if (S == 4 * SP) {
#pragma unroll
      for (int i = 0; i < SP; i += 4) {
        const Quad w = *reinterpret_cast<const Quad*>(p + n0 + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[i + k] = w[k];
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < SP; ++i) v[i] = n0 + i < S ? p[n0 + i] : 0.f;
}
template <int SP>
__device__ inline void store_states(float* p, int S, int n0, const float (&v)[SP]) {
  if constexpr (SP >= 4) {
    if (S == 4 * SP) {
#pragma unroll
      for (int i = 0; i < SP; i += 4) *reinterpret_cast<Quad*>(p + n0 + i) = Quad{v[i], v[i + 1], v[i + 2], v[i + 3]};
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < SP; ++i)
    if (n0 + i < S) p[n0 + i] = v[i];
}

// Where a thread stands.
struct SsmPlace {
  int q, wave, b, chunk, ch, n0;                     // ch: channel (one that exists)
  bool has;                                          // whether it is the thread's own
  long long at;                                      // of (b, ch) in [B,H]
  int t0, t1;                                        // steps of the chunk
  template <int SP>
  __device__ inline void set(const SsmArgs& a, int first_chunk, std::integral_constant<int, SP>) {
    const int tid = threadIdx.x;
    q = tid & 3;
    wave = tid >> 6;
    n0 = q * SP;
    const unsigned across = (unsigned)a.s.cols * a.c.B;
    const unsigned k = blockIdx.x / across, rest = blockIdx.x - k * across;
    chunk = first_chunk + (int)k;
    b = (int)(rest / a.s.cols);
    const int col = (int)(rest - (unsigned)b * a.s.cols);
    ch = col * SSM_COLS + (tid >> 2);
    has = ch < a.c.H;
    if (!has) ch = a.c.H - 1;
    at = (long long)b * a.c.H + ch;
    t0 = chunk * a.s.len;
    t1 = min(a.c.T, t0 + a.s.len);
  }
};

// (field by field: a choice between structures would go through memory)
__device__ inline glr_seq one_of(bool first, const glr_seq& x, const glr_seq& y) {
  return {first ? x.data : y.data, first ? x.stride_t : y.stride_t, first ? x.stride_b : y.stride_b};
}

// A channel's elements of a sequence, one step for each of its four lanes, at a tile that starts at step t and moves on by
// whole tiles: a lane's own address and scalar distances, without products.  FULL: the tile's steps all exist; otherwise
// the last one is read for those behind it.
template <typename E>
struct Steps {
  char* p;                                           // of step t + q
  long long stride;                                  // bytes
  __device__ inline Steps(const glr_seq& s, const SsmPlace& at, int t) : stride(s.stride_t * (long long)sizeof(E)) {
    p = (char*)s.data + (at.b * s.stride_b + at.ch) * (long long)sizeof(E) + (t + at.q) * stride;
  }
  __device__ inline void move(int steps) { p += steps * stride; }
  template <bool FULL, int G>
  __device__ inline void load(E (&v)[G], int left) const {      // left: steps behind t + q
#pragma unroll
    for (int g = 0; g < G; ++g) v[g] = *(const E*)(p + (FULL ? 4 * g : min(4 * g, left)) * stride);
  }
  __device__ inline void put(int g, float v) const { *(E*)(p + 4 * g * stride) = elem_of<E>(v); }
};

// b and c of a tile of TB steps in LDS, as floats: [step][lane of four][b SP | c SP]; zeros where there is no state.  Half of
// the waves read b, half c.
template <typename E, int SP, int TB>
struct BcTile {
  static constexpr int row = 8 * SP, n = TB * row;
  static constexpr int steps = SSM_THREADS / row;    // of the tile between a thread's elements
  static constexpr int per = (TB + steps - 1) / steps;
  E raw[per];
  const char* p;                                     // the thread's element of the tile that starts at step t
  long long stride;
  int step, to;
  bool has;
  __device__ inline BcTile(const SsmArgs& a, int b, int t) {
    const int which = __builtin_amdgcn_readfirstlane(threadIdx.x / (SSM_THREADS / 2)), r = threadIdx.x % (SSM_THREADS / 2);
    const int s = r % (4 * SP);
    const glr_seq& q = which ? a.cc : a.b;
    step = r / (4 * SP);
    has = s < a.c.S;
    stride = q.stride_t * (long long)sizeof(E);
    p = (const char*)q.data + (b * q.stride_b + (t + step) * q.stride_t + (has ? s : 0)) * (long long)sizeof(E);
    to = step * row + s / SP * (2 * SP) + which * SP + s % SP;
  }
  __device__ inline bool mine(int k) const { return TB % steps == 0 || step + k * steps < TB; }
  __device__ inline void move(int n) { p += n * stride; }
  __device__ inline void load(int t, int last) {
    const bool full = t + TB - 1 <= last;
#pragma unroll
    for (int k = 0; k < per; ++k) {
      if (!mine(k)) continue;
      if (full) raw[k] = *(const E*)(p + k * steps * stride);
      else raw[k] = *(const E*)(p + min(k * steps, last - t - step) * stride);
    }
  }
  __device__ inline void store(float* lds) const {
#pragma unroll
    for (int k = 0; k < per; ++k)
      if (mine(k)) lds[to + k * steps * row] = has ? elem_f32(raw[k]) : 0.f;
  }
};
template <int SP>
__device__ inline void read_bc(const float* lds, int step, int q, int which, float (&v)[SP]) {
  const float* p = lds + step * 8 * SP + q * 2 * SP + which * SP;
#pragma unroll
  for (int i = 0; i < SP; ++i) v[i] = p[i];
}

// Which steps reset, 64 of a chunk looked at together, a lane each: a look for every tile would be a wait for every tile.
struct Resets {
  unsigned long long bits = 0;
  // Bits of the n steps of the tile at t, tiles one after the other, forward or backward (n divides 64); first: the first one.
  __device__ inline unsigned of(const SsmArgs& a, const SsmPlace& p, int t, int n, bool first, bool backward) {
    if (!a.reset) return 0;
    const int in = (t - p.t0) & 63;
    if (first || in == (backward ? 64 - n : 0)) {
      const int at = t - in + (int)(threadIdx.x & 63);
      bits = __ballot(at < a.c.T && a.reset[(long long)at * a.c.B + p.b] != 0);
    }
    return (unsigned)(bits >> in) & ((1u << n) - 1);
  }
};

// d as the decays take it.  A softplus is above 0: where it is below the floats, an infinite a still forgets, and for any other
// the smallest float is as little of a decay as 0 is (to 2^-20 for the lowest float).  (A NaN reaches the state through d b x.)
__device__ inline float above_zero(float d) { return fmaxf(d, 0x1p-149f); }
__device__ inline float decay(float d, float a2) { return __builtin_amdgcn_exp2f(d * a2); }

// The state behind a chunk from the one before it: S + P v, P = exp(a sum d); a sum below 0: the chunk forgets.
__device__ inline float behind_chunk(float v, float S, float sum, float a2) {
  return sum < 0.f || v == 0.f ? S : fmaf(decay(sum, a2), v, S);
}
// v, the state at the sequence's end, taken through the chunks that lie between it and the thread's own: 0, 1, .. (backward:
// the last, the one before it, ..).  Where there are few chunks every workgroup does that itself, as ssm_between_kernel does
// it for many.  With the launch : without, us a pass: 777 x 3 x 500 floats, 25 chunks, 33.4 : 30.4; forward and backward of
// 8192 x 4 x 1024 bf16, 16 chunks each, 1001 : 998; a launch for 63 chunks of 2000 x 512 takes 11.5.
template <int SP, bool BACKWARD>
__device__ inline void through_chunks(const SsmArgs& a, const SsmPlace& p, const float (&A2)[SP], float (&v)[SP]) {
  const long long per = (long long)a.c.B * a.c.H;
  const int n = BACKWARD ? a.s.chunks - 1 - p.chunk : p.chunk;
  constexpr int AHEAD = 8;
  for (int s0 = 0; s0 < n; s0 += AHEAD) {
    float e[AHEAD][SP], d[AHEAD];
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      const int step = min(s0 + s, n - 1);
      const long long k = (BACKWARD ? a.s.chunks - 1 - step : step) * per + p.at;
      load_states<SP>(a.ends + k * a.c.S, a.c.S, p.n0, e[s]);
      d[s] = a.sums[k];
    }
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
      if (s0 + s >= n) break;
#pragma unroll
      for (int i = 0; i < SP; ++i) v[i] = behind_chunk(v[i], e[s][i], d[s], A2[i]);
    }
  }
}

// ---- forward
// MAIN: results of a chunk from its state; otherwise its end state from zero and the sum of its d.
// Per step and state: d a, an exponential, b d x and two multiply-adds; around them, for every 16 states, softplus, the gate
// and the loads of a channel's step.  Instructions bound it: 8192 x 4 x 1024 bf16, 16 states, takes 191 us as traced (163
// without states to save, which are 268 of its 600 MB), 120 for the chunks' ends; four waves a SIMD hold 80 to 90 % of its
// issue.  128 x 100 x 1000 floats, one chunk: 94 us.  Four lanes a channel rather than one: a quarter of the chunks' second
// sweep for as many waves, and softplus and gate still once for each step.
template <typename E, int SP, bool MAIN>
__global__ __launch_bounds__(SSM_THREADS) void ssm_forward_kernel(SsmArgs a) {
  constexpr int TB = SSM_TILE, G = TB / 4;
  using Tile = BcTile<E, SP, TB>;
  __shared__ float bc[2][Tile::n];
  SsmPlace p;
  p.set(a, 0, std::integral_constant<int, SP>());
  const int S = a.c.S, last = a.c.T - 1, q = p.q;
  float A2[SP], h[SP];
  load_states<SP>(a.a + (long long)p.ch * S, S, p.n0, A2);
#pragma unroll
  for (int i = 0; i < SP; ++i) {
    A2[i] *= LOG2E;
    h[i] = 0.f;
  }
  if (MAIN && p.has) {
    const long long at = p.at * S;
    if (p.chunk > 0 && !few_chunks(a.s)) load_states<SP>(a.ends + (long long)p.chunk * a.c.B * a.c.H * S + at, S, p.n0, h);
    else if (a.h0) load_states<SP>(a.h0 + at, S, p.n0, h);
    if (few_chunks(a.s)) through_chunks<SP, false>(a, p, A2, h);
  }
  const float bias = a.bias ? a.bias[p.ch] : 0.f, skip = MAIN && a.skip ? a.skip[p.ch] : 0.f;
  const bool gated = MAIN && a.z.data;
  Steps<E> xs(a.x, p, p.t0), ds(a.dt, p, p.t0), zs(one_of(gated, a.z, a.x), p, p.t0), ys(one_of(MAIN, a.y, a.x), p, p.t0);
  constexpr int SAVE = ssm_save(SP);
  const long long states = (long long)a.c.B * a.c.H * S;
  float* saved = a.saved + p.t0 / SAVE * states + p.at * S;
  const bool save = a.saved && p.has;
  Tile next(a, p.b, p.t0);
  E xn[G], dn[G], zn[G];
  auto load = [&](int t) SSM_INLINE {
    auto steps = [&](auto full) SSM_INLINE {
      constexpr bool FULL = decltype(full)::value;
      xs.template load<FULL>(xn, last - t - q);
      ds.template load<FULL>(dn, last - t - q);
      if (gated) zs.template load<FULL>(zn, last - t - q);
    };
    if (t + TB <= a.c.T) steps(std::true_type{});
    else steps(std::false_type{});
    next.load(t, last);
    xs.move(TB);
    ds.move(TB);
    zs.move(TB);
    next.move(TB);
  };
  load(p.t0);
  float sum = 0.f;
  bool forgets = false;
  Resets looked;
  int buf = 0;
  for (int t = p.t0; t < p.t1; t += TB, buf ^= 1) {
    float x[G], d[G], z[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      x[g] = elem_f32(xn[g]);
      d[g] = elem_f32(dn[g]) + bias;
      z[g] = gated ? elem_f32(zn[g]) : 0.f;
    }
    next.store(bc[buf]);
    const unsigned resets = looked.of(a, p, t, TB, t == p.t0, false);
    __syncthreads();
    if (t + TB < p.t1) load(t + TB);
    forgets |= resets != 0;
    // PLAIN: every step exists and none resets.  (Lanes without a channel go through another one's and store nothing.)
    auto tile = [&](auto plain) SSM_INLINE {
      constexpr bool PLAIN = decltype(plain)::value;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const int ts = t + 4 * g;
        if (MAIN && 4 * g % SAVE == 0 && save && (PLAIN || ts < a.c.T))
          store_states<SP>(saved + 4 * g / SAVE * states, S, p.n0, h);
        const bool in = PLAIN || ts + q < a.c.T;
        const float delta = in ? Softplus(d[g]).d : 0.f;
        const float xv = in ? x[g] : 0.f, dx = delta * xv, dd = above_zero(delta);
        if (!MAIN) sum += dd;
        float part[4];
        auto step = [&](auto j_) SSM_INLINE {
          constexpr int j = decltype(j_)::value;
          part[j] = 0.f;
          if (!PLAIN && ts + j >= a.c.T) return;
          const float dj = quad_of<j>(dd), xj = quad_of<j>(dx);
          const bool cut = !PLAIN && (resets >> (4 * g + j) & 1);
          float b[SP], c[SP];
          read_bc<SP>(bc[buf], 4 * g + j, q, 0, b);
          if (MAIN) read_bc<SP>(bc[buf], 4 * g + j, q, 1, c);
          float y = 0.f;
#pragma unroll
          for (int i = 0; i < SP; ++i) {
            h[i] = cut ? xj * b[i] : fmaf(decay(dj, A2[i]), h[i], xj * b[i]);
            if (MAIN) y = fmaf(h[i], c[i], y);
          }
          part[j] = y;
        };
        step(std::integral_constant<int, 0>());
        step(std::integral_constant<int, 1>());
        step(std::integral_constant<int, 2>());
        step(std::integral_constant<int, 3>());
        if constexpr (MAIN) {
          float y = quad_sums(part, q);
          y = fmaf(skip, xv, y);
          if (gated) y *= silu(z[g]);
          if (in && p.has) ys.put(g, y);
        }
      }
    };
    if (!resets && t + TB <= a.c.T) tile(std::true_type{});
    else tile(std::false_type{});
    if (MAIN) {
      ys.move(TB);
      saved += TB / SAVE * states;
    }
  }
  if (!p.has) return;
  if (MAIN) {
    if (a.h_last && p.chunk == a.s.chunks - 1) store_states<SP>(a.h_last + p.at * S, S, p.n0, h);
  } else {
    const long long k = (long long)p.chunk * a.c.B * a.c.H + p.at;
    store_states<SP>(a.ends + k * S, S, p.n0, h);
    sum = quad_sum(sum);
    if (q == 0) a.sums[k] = forgets ? -1.f : sum;
  }
}

// Many chunks: the states between them, in place of the chunks' own: forward before, backward behind each chunk.  A thread per
// state.
__global__ __launch_bounds__(256) void ssm_between_kernel(SsmArgs a, const float* first, bool backward) {
  const long long n = (long long)a.c.B * a.c.H * a.c.S, i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const long long bh = i / a.c.S, per = (long long)a.c.B * a.c.H;
  const float a2 = LOG2E * a.a[bh % a.c.H * a.c.S + (i - bh * a.c.S)];
  float v = first ? first[i] : 0.f;
  const int K = a.s.chunks;
  for (int s0 = 0; s0 < K; s0 += 8) {
    float e[8], d[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const int step = min(s0 + s, K - 1), k = backward ? K - 1 - step : step;
      // (the last chunk of the way has no map, and needs none)
      e[s] = step < K - 1 ? a.ends[k * n + i] : 0.f;
      d[s] = step < K - 1 ? a.sums[k * per + bh] : -1.f;
    }
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      if (s0 + s >= K) break;
      const int k = backward ? K - 1 - (s0 + s) : s0 + s;
      a.ends[k * n + i] = v;
      v = behind_chunk(v, e[s], d[s], a2);
    }
  }
}

// ---- backward
// mu_t = exp(d_t a) lambda_t is what step t hands on to step t - 1.  What a chunk hands on from nothing, and the sum of
// its d.  (Chunk 0 hands on to nobody.)  142 us at the sizes above.
template <typename E, int SP>
__global__ __launch_bounds__(SSM_THREADS) void ssm_adjoint_ends_kernel(SsmArgs a) {
  constexpr int TB = SSM_TILE, G = TB / 4;
  using Tile = BcTile<E, SP, TB>;
  __shared__ float bc[2][Tile::n];
  SsmPlace p;
  p.set(a, 1, std::integral_constant<int, SP>());
  const int S = a.c.S, last = a.c.T - 1, q = p.q;
  float A2[SP], mu[SP];
  load_states<SP>(a.a + (long long)p.ch * S, S, p.n0, A2);
#pragma unroll
  for (int i = 0; i < SP; ++i) {
    A2[i] *= LOG2E;
    mu[i] = 0.f;
  }
  const float bias = a.bias ? a.bias[p.ch] : 0.f;
  const bool gated = a.z.data;
  const int tiles = (p.t1 - p.t0 + TB - 1) / TB, end = p.t0 + (tiles - 1) * TB;
  Steps<E> ys(a.dy, p, end), ds(a.dt, p, end), zs(one_of(gated, a.z, a.dy), p, end);
  Tile next(a, p.b, end);
  E yn[G], dn[G], zn[G];
  auto load = [&](int t) SSM_INLINE {
    auto steps = [&](auto full) SSM_INLINE {
      constexpr bool FULL = decltype(full)::value;
      ys.template load<FULL>(yn, last - t - q);
      ds.template load<FULL>(dn, last - t - q);
      if (gated) zs.template load<FULL>(zn, last - t - q);
    };
    if (t + TB <= a.c.T) steps(std::true_type{});
    else steps(std::false_type{});
    next.load(t, last);
    ys.move(-TB);
    ds.move(-TB);
    zs.move(-TB);
    next.move(-TB);
  };
  load(end);
  float sum = 0.f;
  bool forgets = false;
  Resets looked;
  int buf = 0;
  for (int k = tiles - 1; k >= 0; --k, buf ^= 1) {
    const int t = p.t0 + k * TB;
    float y[G], d[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const bool in = t + 4 * g + q < a.c.T;
      const float z = gated ? elem_f32(zn[g]) : 0.f, dy = elem_f32(yn[g]);
      y[g] = !in ? 0.f : gated ? dy * silu(z) : dy;
      d[g] = in ? Softplus(elem_f32(dn[g]) + bias).d : 0.f;
      sum += d[g];
    }
    next.store(bc[buf]);
    const unsigned resets = looked.of(a, p, t, TB, k == tiles - 1, true);
    __syncthreads();
    if (k > 0) load(t - TB);
    forgets |= resets != 0;
#pragma unroll
    for (int g = G - 1; g >= 0; --g) {
      auto step = [&](auto j_) SSM_INLINE {
        constexpr int j = decltype(j_)::value;
        const float dj = quad_of<j>(d[g]), yj = quad_of<j>(y[g]);
        const bool cut = resets >> (4 * g + j) & 1;
        float c[SP];
        read_bc<SP>(bc[buf], 4 * g + j, q, 1, c);
#pragma unroll
        for (int i = 0; i < SP; ++i) {
          const float m = decay(dj, A2[i]) * fmaf(c[i], yj, mu[i]);
          mu[i] = cut ? 0.f : m;
        }
      };
      step(std::integral_constant<int, 3>());
      step(std::integral_constant<int, 2>());
      step(std::integral_constant<int, 1>());
      step(std::integral_constant<int, 0>());
    }
  }
  if (!p.has) return;
  const long long k = (long long)p.chunk * a.c.B * a.c.H + p.at;
  store_states<SP>(a.ends + k * S, S, p.n0, mu);
  sum = quad_sum(sum);
  if (q == 0) a.sums[k] = forgets ? -1.f : sum;
}

// Sums of b's and c's gradients over the 16 channels of a wave: v = (of b, of c) of a lane's states, to
// out[which * 4 SP + n].
template <int SP>
__device__ inline void channel_sums(const float (&v)[2 * SP], float* out, int lane) {
  float w[SP], u[(SP + 1) / 2];
#pragma unroll
  for (int i = 0; i < SP; ++i) {               // lower half of the wave: of b, upper half: of c
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i + SP]), false, false);
    w[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  constexpr int H2 = (SP + 1) / 2;
#pragma unroll
  for (int i = 0; i < H2; ++i) {               // even rows of 16 lanes: the lower half of the states
    const unsigned other = SP > 1 ? __float_as_uint(w[(i + H2) % SP]) : __float_as_uint(w[i]);
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(w[i]), other, false, false);
    u[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    // the four channels of a row
    u[i] += __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(u[i]), 0x124, 0xf, 0xf, true));
    u[i] += __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(u[i]), 0x128, 0xf, 0xf, true));
  }
  if ((lane & 12) == 0 && (SP > 1 || (lane & 16) == 0)) {
    const int n0 = (lane >> 5) * 4 * SP + (lane & 3) * SP + (SP > 1 && (lane & 16) ? H2 : 0);
#pragma unroll
    for (int i = 0; i < H2; ++i) out[n0 + i] = u[i];
  }
}

// A tile of R steps goes forward again from its saved state, keeping the decays and the states before each step in registers,
// and then back.  Instructions bound it (105 a wave and step, two waves a SIMD, a vector instruction in execution 94 % of
// the time): 8192 x 4 x 1024 bf16, 16 states, 504 us as traced, 128 x 100 x 1000 floats 240 to 260.  Tiles of 8 steps: 16 leave
// room for one wave a SIMD (755 us).  Of a step's instructions the states take 60 %, the sums over the channels 15 %: through LDS
// those took 576 against 549 us, on the matrix pipe (products with ones) the registers of the second wave (840).
template <typename E, int SP, int R>
__global__ __launch_bounds__(SSM_THREADS) void ssm_backward_kernel(SsmArgs a) {
  constexpr int G = R / 4;
  using Tile = BcTile<E, SP, R>;
  __shared__ float bc[2][Tile::n];
  __shared__ float red[4][R][8 * SP];
  SsmPlace p;
  p.set(a, 0, std::integral_constant<int, SP>());
  const int S = a.c.S, last = a.c.T - 1, q = p.q, lane = threadIdx.x & 63;
  const long long states = (long long)a.c.B * a.c.H * S;
  float A2[SP], mu[SP], dA[SP];
  load_states<SP>(a.a + (long long)p.ch * S, S, p.n0, A2);
#pragma unroll
  for (int i = 0; i < SP; ++i) {
    A2[i] *= LOG2E;
    mu[i] = dA[i] = 0.f;
  }
  if (p.has) {
    if (p.chunk < a.s.chunks - 1 && !few_chunks(a.s)) load_states<SP>(a.ends + p.chunk * states + p.at * S, S, p.n0, mu);
    else if (a.dh_last) load_states<SP>(a.dh_last + p.at * S, S, p.n0, mu);
    if (few_chunks(a.s)) through_chunks<SP, true>(a, p, A2, mu);
  }
  const float bias = a.bias ? a.bias[p.ch] : 0.f, skip = a.skip ? a.skip[p.ch] : 0.f;
  const bool gated = a.z.data;
  const int tiles = (p.t1 - p.t0 + R - 1) / R, end = p.t0 + (tiles - 1) * R;
  Steps<E> xs(a.x, p, end), ds(a.dt, p, end), ys(a.dy, p, end), zs(one_of(gated, a.z, a.x), p, end);
  Steps<E> xo(a.dx, p, end), dto(a.ddt, p, end), zo(one_of(gated, a.dz, a.dx), p, end);
  Tile next(a, p.b, end);
  const float* saved = a.saved + end / R * states + p.at * S;
  E xn[G], dn[G], yn[G], zn[G];
  float hn[SP];
  auto load = [&](int t) SSM_INLINE {
    auto steps = [&](auto full) SSM_INLINE {
      constexpr bool FULL = decltype(full)::value;
      xs.template load<FULL>(xn, last - t - q);
      ds.template load<FULL>(dn, last - t - q);
      ys.template load<FULL>(yn, last - t - q);
      if (gated) zs.template load<FULL>(zn, last - t - q);
    };
    if (t + R <= a.c.T) steps(std::true_type{});
    else steps(std::false_type{});
    next.load(t, last);
    load_states<SP>(saved, S, p.n0, hn);
    xs.move(-R);
    ds.move(-R);
    ys.move(-R);
    zs.move(-R);
    next.move(-R);
    saved -= states;
  };
  load(end);
  // the thread's place in the tile's sums (those i * SSM_THREADS behind it are of the same state): [col][T,B,2S]
  const int own = threadIdx.x % (8 * SP), own_n = own % (4 * SP) < S ? own / (4 * SP) * S + own % (4 * SP) : -1;
  const long long own_row = (long long)(blockIdx.x % (unsigned)a.s.cols) * a.c.T + end + threadIdx.x / (8 * SP);
  float* part_bc = a.part_bc + (own_row * a.c.B + p.b) * (2 * S) + own_n;
  const long long row = 2LL * a.c.B * S;                // of a step
  float dskip = 0.f, dbias = 0.f;
  Resets looked;
  int buf = 0;
  for (int k = tiles - 1; k >= 0; --k, buf ^= 1) {
    const int t = p.t0 + k * R;
    E xr[G], dr[G], yr[G], zr[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      xr[g] = xn[g];
      dr[g] = dn[g];
      yr[g] = yn[g];
      if (gated) zr[g] = zn[g];
    }
    float h[SP];
#pragma unroll
    for (int i = 0; i < SP; ++i) h[i] = p.has ? hn[i] : 0.f;
    next.store(bc[buf]);
    const unsigned resets = looked.of(a, p, t, R, k == tiles - 1, true);
    __syncthreads();                               // (and red has been read)
    if (k > 0) load(t - R);
    auto tile = [&](auto plain) SSM_INLINE {
      constexpr bool PLAIN = decltype(plain)::value;
      // (Lanes without a channel go through another one's, with dy = 0: they add nothing to the sums over channels.)
      float x[G], delta[G], slope[G], dy[G], z[G], sz[G];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const bool in = PLAIN || t + 4 * g + q < a.c.T;
        const float v = elem_f32(dr[g]) + bias;
        const Softplus sp(v);
        x[g] = in ? elem_f32(xr[g]) : 0.f;
        delta[g] = in ? sp.d : 0.f;
        slope[g] = sp.slope(v);
        dy[g] = in && p.has ? elem_f32(yr[g]) : 0.f;
        z[g] = in && gated ? gate_factor(elem_f32(zr[g])) : 1.f;
        sz[g] = gated ? Sigmoid(z[g]).s : 1.f;
      }
      float keep[R][SP], past[R][SP], sum[G];
      // forward, again
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const float dx = delta[g] * x[g];
        float part[4];
        auto step = [&](auto j_) SSM_INLINE {
          constexpr int j = decltype(j_)::value;
          const int r = 4 * g + j;
          part[j] = 0.f;
          if (!PLAIN && t + r >= a.c.T) return;       // (0 times an infinite state or b would be NaN)
          const float dj = quad_of<j>(delta[g]), xj = quad_of<j>(dx);
          const bool cut = !PLAIN && (resets >> r & 1);
          float b[SP], c[SP];
          read_bc<SP>(bc[buf], r, q, 0, b);
          read_bc<SP>(bc[buf], r, q, 1, c);
          float y = 0.f;
#pragma unroll
          for (int i = 0; i < SP; ++i) {
            past[r][i] = h[i];
            keep[r][i] = decay(dj, A2[i]);
            h[i] = cut ? xj * b[i] : fmaf(keep[r][i], h[i], xj * b[i]);
            y = fmaf(h[i], c[i], y);
          }
          part[j] = y;
        };
        step(std::integral_constant<int, 0>());
        step(std::integral_constant<int, 1>());
        step(std::integral_constant<int, 2>());
        step(std::integral_constant<int, 3>());
        sum[g] = quad_sums(part, q);
      }
      // back
#pragma unroll
      for (int g = G - 1; g >= 0; --g) {
        // dL/d(sum c h + skip x)
        const float dx = delta[g] * x[g], out = dy[g] * (z[g] * sz[g]);
        float of_x[4], of_d[4];
        auto step = [&](auto j_) SSM_INLINE {
          constexpr int j = decltype(j_)::value;
          const int r = 4 * g + j;
          of_x[j] = of_d[j] = 0.f;
          if (!PLAIN && t + r >= a.c.T) return;
          const float dj = quad_of<j>(delta[g]), xj = quad_of<j>(dx), oj = quad_of<j>(out);
          const bool cut = !PLAIN && (resets >> r & 1);
          float b[SP], c[SP], v[2 * SP];
          read_bc<SP>(bc[buf], r, q, 0, b);
          read_bc<SP>(bc[buf], r, q, 1, c);
          float lb = 0.f, ld = 0.f;
#pragma unroll
          for (int i = 0; i < SP; ++i) {
            const float lam = fmaf(c[i], oj, mu[i]);
            v[i] = lam * xj;
            v[SP + i] = oj * h[i];
            lb = fmaf(lam, b[i], lb);
            mu[i] = cut ? 0.f : keep[r][i] * lam;
            const float m = cut ? 0.f : mu[i] * past[r][i];
            ld = fmaf(m, A2[i], ld);
            dA[i] = fmaf(m, dj, dA[i]);
            h[i] = past[r][i];
          }
          of_x[j] = lb;
          of_d[j] = ld;
          channel_sums<SP>(v, red[p.wave][r], lane);
        };
        step(std::integral_constant<int, 3>());
        step(std::integral_constant<int, 2>());
        step(std::integral_constant<int, 1>());
        step(std::integral_constant<int, 0>());
        const float lb = quad_sums(of_x, q), ld = quad_sums(of_d, q);
        const float ddt = fmaf(lb, x[g], ld * LN2) * slope[g];
        if (p.has && (PLAIN || t + 4 * g + q < a.c.T)) {
          xo.put(g, fmaf(lb, delta[g], out * skip));
          dto.put(g, ddt);
          if (gated) zo.put(g, dy[g] * fmaf(skip, x[g], sum[g]) * (sz[g] * fmaf(z[g], 1.f - sz[g], 1.f)));
          dskip = fmaf(out, x[g], dskip);
          dbias += ddt;
        }
      }
    };
    if (!resets && t + R <= a.c.T) tile(std::true_type{});
    else tile(std::false_type{});
    __syncthreads();
    // the waves' sums of the tile
    constexpr int W = R * 8 * SP;                  // of a wave
#pragma unroll
    for (int i = 0; i < (W + SSM_THREADS - 1) / SSM_THREADS; ++i) {
      const int e = threadIdx.x + i * SSM_THREADS, r = e / (8 * SP);
      if (own_n < 0 || (W % SSM_THREADS != 0 && e >= W) || t + r >= a.c.T) continue;
      const float* f = &red[0][0][0] + e;
      part_bc[i * (SSM_THREADS / (8 * SP)) * row] = (f[0] + f[W]) + (f[2 * W] + f[3 * W]);
    }
    part_bc -= R * row;
    xo.move(-R);
    dto.move(-R);
    zo.move(-R);
  }
  if (!p.has) return;
  const long long k = (long long)p.chunk * a.c.B * a.c.H + p.at;
  store_states<SP>(a.part_a + k * S, S, p.n0, dA);
  dskip = quad_sum(dskip);
  dbias = quad_sum(dbias);
  if (q == 0) {
    a.part_h[2 * k] = dskip;
    a.part_h[2 * k + 1] = dbias;
  }
  if (a.dh0 && p.chunk == 0) store_states<SP>(a.dh0 + p.at * S, S, p.n0, mu);
}

// Gradients of b and c: the workgroups' sums across the channels (16 us for 67 MB).
template <typename E>
__global__ __launch_bounds__(256) void ssm_bc_kernel(SsmArgs a) {
  const int S2 = 2 * a.c.S;
  const long long n = (long long)a.c.T * a.c.B * S2, i = 2 * ((long long)blockIdx.x * 256 + threadIdx.x);
  if (i >= n) return;                                // (n is even)
  float x = 0.f, y = 0.f;
  const float* f = a.part_bc + i;
#pragma unroll 8
  for (int c = 0; c < a.s.cols; ++c, f += n) {
    const float2 v = *reinterpret_cast<const float2*>(f);
    x += v.x;
    y += v.y;
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const long long row = (i + k) / S2;
    const int s = (int)(i + k - row * S2), t = (int)(row / a.c.B), b = (int)(row - (long long)t * a.c.B);
    const glr_seq& o = s < a.c.S ? a.db : a.dc;
    ((E*)o.data)[t * o.stride_t + b * o.stride_b + (s < a.c.S ? s : s - a.c.S)] = elem_of<E>(k ? y : x);
  }
}

// Gradients of a, skip and bias: sums over the chunks and batch rows.
__global__ __launch_bounds__(SUM_THREADS) void ssm_params_kernel(SsmArgs a) {
  const long long HS = (long long)a.c.H * a.c.S, H2 = 2LL * a.c.H, i = sum_column();
  const bool of_a = i < HS;
  float v;
  if (!sum_rows(of_a ? a.part_a + i : a.part_h + (i - HS), of_a ? HS : H2, (long long)a.s.chunks * a.c.B, i < HS + H2, v))
    return;
  if (of_a) {
    a.da[i] = v;
  } else {
    float* o = (i - HS) & 1 ? a.dbias : a.dskip;
    if (o) o[(i - HS) >> 1] = v;
  }
}

// ---- one step: 100 rows x 1024 x 16 states 7.2 us, 13 MB of states behind the slot's latency
template <typename E, int SP>
__global__ __launch_bounds__(SSM_THREADS) void ssm_step_kernel(SsmStepArgs a) {
  const long long i = ((long long)blockIdx.x * SSM_THREADS + threadIdx.x) >> 2;
  const int q = threadIdx.x & 3, H = a.c.H, S = a.c.S, b = (int)(i / H), ch = (int)(i - (long long)b * H);
  if (b >= a.c.B) return;                             // (four lanes together)
  E* y = (E*)a.y.data + b * a.y.stride_b + ch;
  const int slot = a.slots ? a.slots[b] : b;
  if (slot < 0 || slot >= a.n_slots) {
    if (q == 0) *y = elem_of<E>(0.f);
    return;
  }
  auto one = [&](const glr_seq& s) { return elem_f32(((const E*)s.data)[b * s.stride_b + ch]); };
  const float x = one(a.x), d = Softplus(one(a.dt) + (a.bias ? a.bias[ch] : 0.f)).d;
  const bool cut = a.reset && a.reset[b];
  float A[SP], h[SP], sum = 0.f;
  const long long at = ((long long)slot * H + ch) * S;
  load_states<SP>(a.a + (long long)ch * S, S, q * SP, A);
  load_states<SP>(a.state_in + at, S, q * SP, h);
  const E *bs = (const E*)a.b.data + b * a.b.stride_b, *cs = (const E*)a.cc.data + b * a.cc.stride_b;
#pragma unroll
  for (int k = 0; k < SP; ++k) {
    const int n = min(q * SP + k, S - 1);
    const float keep = decay(above_zero(d), A[k] * LOG2E), in = d * x * elem_f32(bs[n]);
    h[k] = cut ? in : fmaf(keep, h[k], in);
    if (q * SP + k < S) sum = fmaf(h[k], elem_f32(cs[n]), sum);
  }
  store_states<SP>(a.state_out + at, S, q * SP, h);
  sum = quad_sum(sum);
  if (q) return;
  float v = fmaf(a.skip ? a.skip[ch] : 0.f, x, sum);
  if (a.z.data) {
    const float z = one(a.z);
    v *= silu(z);
  }
  *y = elem_of<E>(v);
}

// ---- launches
SsmShape ssm_shape(const ssm_cfg& c, bool backward) {
  SsmShape s;
  s.per = c.S <= 4 ? 1 : c.S <= 8 ? 2 : c.S <= 16 ? 4 : c.S <= 32 ? 8 : 16;
  s.save = ssm_save(s.per);
  s.cols = (c.H + SSM_COLS - 1) / SSM_COLS;
  const long long across = (long long)s.cols * c.B, tiles = ((long long)c.T + SSM_TILE - 1) / SSM_TILE;
  long long chunks = 1;
  // Chunks cost a second sweep and fill the card: with : without, us, 1024 steps of bf16, 16 states, by workgroups across
  // - forward: 130 88 : 135, 250 135 : 135, 320 168 : 187, 380 206 : 190, 510 252 : 193, 640 307 : 272, 770 400 : 332;
  // - backward: 130 194 : 327, 250 295 : 327, 320 363 : 466, 380 452 : 471, 510 548 : 471, 640 683 : 722, 770 914 : 899.
  // Then about four a CU (8192 x 4 x 1024: 768 to 2048 workgroups within 3 % of each other), of two tiles at least.
  if (across < (backward ? 416 : 352)) {
    chunks = (1024 + across - 1) / across;
    chunks = chunks < (tiles + 1) / 2 ? chunks : (tiles + 1) / 2;
  }
  s.len = (int)((tiles + chunks - 1) / chunks) * SSM_TILE;
  s.chunks = (int)(((long long)c.T + s.len - 1) / s.len);
  return s;
}
static size_t piece(size_t n) { return (n + 255) / 256 * 256; }
namespace {
struct SsmSpace {
  size_t ends, sums, bc, pa, ph, total;
  SsmSpace(const ssm_cfg& c, bool backward) {
    const SsmShape s = ssm_shape(c, backward);
    const size_t bh = (size_t)c.B * c.H;
    total = 0;
    auto take = [&](size_t n) {
      const size_t at = total;
      total += piece(n);
      return at;
    };
    ends = take(s.chunks > 1 ? 4 * s.chunks * bh * c.S : 0);
    sums = take(s.chunks > 1 ? 4 * s.chunks * bh : 0);
    bc = take(backward ? 4 * (size_t)s.cols * c.T * c.B * 2 * c.S : 0);
    pa = take(backward ? 4 * s.chunks * bh * c.S : 0);
    ph = take(backward ? 8 * s.chunks * bh : 0);
  }
};
}  // namespace
size_t ssm_workspace(const ssm_cfg& c) {
  const size_t f = SsmSpace(c, false).total, b = SsmSpace(c, true).total;
  return f > b ? f : b;
}
size_t ssm_saved(const ssm_cfg& c) {
  const SsmShape s = ssm_shape(c, true);
  return 4 * (((size_t)c.T + s.save - 1) / s.save) * c.B * c.H * c.S;
}
static unsigned blocks(long long n) { return (unsigned)((n + 255) / 256); }
bool ssm_launchable(const ssm_cfg& c) {
  for (int backward = 0; backward < 2; ++backward) {
    const SsmShape s = ssm_shape(c, backward);
    if (!launchable((long long)s.chunks * s.cols * c.B, SSM_THREADS)) return false;
  }
  return launchable(((long long)c.B * c.H * c.S + 255) / 256, 256) &&
         launchable(((long long)c.T * c.B * c.S + 255) / 256, 256) &&
         launchable(sum_groups((long long)c.H * (c.S + 2)), SUM_THREADS);
}
static void ssm_place(SsmArgs& a, char* ws, bool backward) {
  const SsmSpace w(a.c, backward);
  a.s = ssm_shape(a.c, backward);
  a.ends = (float*)(ws + w.ends);
  a.sums = (float*)(ws + w.sums);
  a.part_bc = (float*)(ws + w.bc);
  a.part_a = (float*)(ws + w.pa);
  a.part_h = (float*)(ws + w.ph);
}
static hipError_t ssm_between(const SsmArgs& a, const float* first, bool backward, hipStream_t s) {
  hipLaunchKernelGGL(ssm_between_kernel, dim3(blocks((long long)a.c.B * a.c.H * a.c.S)), dim3(256), 0, s, a, first,
                     backward);
  return hipGetLastError();
}
template <typename E, int SP>
static hipError_t ssm_forward_start(const SsmArgs& a, hipStream_t s) {
  const long long across = (long long)a.s.cols * a.c.B;
  const dim3 t(SSM_THREADS);
  if (a.s.chunks > 1) {
    hipLaunchKernelGGL((ssm_forward_kernel<E, SP, false>), dim3((unsigned)(across * (a.s.chunks - 1))), t, 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!few_chunks(a.s) && (e = ssm_between(a, a.h0, false, s)) != hipSuccess)) return e;
  }
  hipLaunchKernelGGL((ssm_forward_kernel<E, SP, true>), dim3((unsigned)(across * a.s.chunks)), t, 0, s, a);
  return hipGetLastError();
}
template <typename E, int SP>
static hipError_t ssm_backward_start(const SsmArgs& a, hipStream_t s) {
  const long long across = (long long)a.s.cols * a.c.B;
  const dim3 t(SSM_THREADS);
  hipError_t e;
  if (a.s.chunks > 1) {
    hipLaunchKernelGGL((ssm_adjoint_ends_kernel<E, SP>), dim3((unsigned)(across * (a.s.chunks - 1))), t, 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess || (!few_chunks(a.s) && (e = ssm_between(a, a.dh_last, true, s)) != hipSuccess))
      return e;
  }
  hipLaunchKernelGGL((ssm_backward_kernel<E, SP, ssm_save(SP)>), dim3((unsigned)(across * a.s.chunks)), t, 0, s, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL((ssm_bc_kernel<E>), dim3(blocks((long long)a.c.T * a.c.B * a.c.S)), dim3(256), 0, s, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL(ssm_params_kernel, dim3(sum_groups((long long)a.c.H * (a.c.S + 2))), dim3(SUM_THREADS), 0, s, a);
  return hipGetLastError();
}
template <typename E, int SP>
static hipError_t ssm_run(const SsmArgs& a, bool backward, hipStream_t s) {
  return backward ? ssm_backward_start<E, SP>(a, s) : ssm_forward_start<E, SP>(a, s);
}
template <typename E, int SP>
static hipError_t ssm_step_start(const SsmStepArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((ssm_step_kernel<E, SP>), dim3((unsigned)(((long long)a.c.B * a.c.H * 4 + 255) / 256)), dim3(256), 0,
                     s, a);
  return hipGetLastError();
}
template <typename E>
static hipError_t ssm_by_states(const SsmArgs& a, bool backward, hipStream_t s) {
  switch (a.s.per) {
    case 1: return ssm_run<E, 1>(a, backward, s);
    case 2: return ssm_run<E, 2>(a, backward, s);
    case 4: return ssm_run<E, 4>(a, backward, s);
    case 8: return ssm_run<E, 8>(a, backward, s);
    default: return ssm_run<E, 16>(a, backward, s);
  }
}
static hipError_t ssm_typed(const SsmArgs& a, bool backward, hipStream_t s) {
  if (a.c.dtype == MGRIT_F32) return ssm_by_states<float>(a, backward, s);
  if (a.c.dtype == MGRIT_BF16) return ssm_by_states<Bf16>(a, backward, s);
  return ssm_by_states<F16>(a, backward, s);
}
template <typename E>
static hipError_t ssm_step_by_states(const SsmStepArgs& a, hipStream_t s) {
  switch (ssm_shape(a.c, false).per) {
    case 1: return ssm_step_start<E, 1>(a, s);
    case 2: return ssm_step_start<E, 2>(a, s);
    case 4: return ssm_step_start<E, 4>(a, s);
    case 8: return ssm_step_start<E, 8>(a, s);
    default: return ssm_step_start<E, 16>(a, s);
  }
}

hipError_t launch_ssm_forward(SsmArgs a, char* ws, hipStream_t s) {
  ssm_place(a, ws, false);
  return ssm_typed(a, false, s);
}
hipError_t launch_ssm_backward(SsmArgs a, char* ws, hipStream_t s) {
  ssm_place(a, ws, true);
  return ssm_typed(a, true, s);
}
hipError_t launch_ssm_step(const SsmStepArgs& a, hipStream_t s) {
  if (!launchable(((long long)a.c.B * a.c.H * 4 + 255) / 256, 256)) return TOO_LARGE;
  if (a.c.dtype == MGRIT_F32) return ssm_step_by_states<float>(a, s);
  if (a.c.dtype == MGRIT_BF16) return ssm_step_by_states<Bf16>(a, s);
  return ssm_step_by_states<F16>(a, s);
}

}  // namespace mg
