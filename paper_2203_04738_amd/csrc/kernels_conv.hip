// Causal convolution of every channel over its last few inputs (include/mgrit_tokens.h), its gradient, and one step.
//
// A thread has VEC neighbouring channels (two, as one word, where the arrays are aligned to that) and goes along time with
// the window of inputs that the next step sees in registers; a reset empties the window.  Every array is read or written
// once but for the few steps before (backward: behind) each thread's own, and what bounds it before memory does are vector
// instructions: 30 a step and channel forward, 47 backward, with one in execution 84 % and all of the time of each SIMD.
// 16384 x 4 x 1024 bf16, 4 taps: forward 268 MB in 62 to 69 us by box (4.3 TB/s at best; on that box runs of 8 steps 88 us,
// four channels a thread 65), backward 402 MB in 94 to 107 us (4.3; blocks of 8 steps 117).
#include <type_traits>

#include "elem.h"
#include "pairs.h"
#include "row_sums.h"
#include "tokens.h"

namespace mg {

constexpr int CONV_RUN = 16;                         // steps of a thread, forward
constexpr int CONV_BLOCK = 4;                        // steps of a block of a segment, backward

// One step of a thread's channels as it is stored.
template <typename E, int VEC>
struct ConvRaw {
  static constexpr int words = VEC * (int)sizeof(E) >= 4 ? VEC * (int)sizeof(E) / 4 : 1;
  typedef unsigned Word __attribute__((ext_vector_type(words)));
  unsigned w[words];
  __device__ inline void load(const E* p) {
    if constexpr (VEC == 1) {
      const E e = *p;
      if constexpr (sizeof(E) == 4) w[0] = __float_as_uint(e);
      else w[0] = e.bits;
    } else {
      const Word v = *reinterpret_cast<const Word*>(p);
#pragma unroll
      for (int i = 0; i < words; ++i) w[i] = v[i];
    }
  }
  __device__ inline float at(int c) const { return word_elem<E>(w[c / ELEMS_PER_WORD<E>], c % ELEMS_PER_WORD<E>); }
};
template <typename E, int VEC>
__device__ inline void conv_store(E* p, const float (&v)[VEC], bool past) {
  if constexpr (VEC == 1) {
    *p = elem_of<E>(v[0]);
  } else {
    typename ConvRaw<E, VEC>::Word w;
#pragma unroll
    for (int c = 0; c < VEC; c += ELEMS_PER_WORD<E>) {
      if constexpr (sizeof(E) == 4) w[c] = __float_as_uint(v[c]);
      else w[c / 2] = pack2<E>(v[c], v[c + 1]);
    }
    store_as(reinterpret_cast<typename ConvRaw<E, VEC>::Word*>(p), w, past);
  }
}

// The window of a thread's channels, oldest first; WT >= W taps, those before the last W never used.
template <int WT, int VEC>
struct Window {
  float v[WT - 1][VEC];
  __device__ inline void clear() {
#pragma unroll
    for (int i = 0; i < WT - 1; ++i)
#pragma unroll
      for (int c = 0; c < VEC; ++c) v[i][c] = 0.f;
  }
  template <typename FN>
  __device__ inline void push(FN x) {                // x(c): the newest input of channel c
#pragma unroll
    for (int i = 0; i + 1 < WT - 1; ++i)
#pragma unroll
      for (int c = 0; c < VEC; ++c) v[i][c] = v[i + 1][c];
#pragma unroll
    for (int c = 0; c < VEC; ++c) v[WT - 2][c] = x(c);
  }
};
template <int WT, int VEC>
struct Taps {
  float w[WT][VEC], bias[VEC];
  int skip;                                          // taps that do not exist
  __device__ inline Taps(const float* weight, const float* b, int W, int ch) : skip(WT - W) {
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
#pragma unroll
      for (int k = 0; k < WT; ++k) w[k][c] = k >= skip ? weight[(long long)(ch + c) * W + k - skip] : 0.f;
      bias[c] = b ? b[ch + c] : 0.f;
    }
  }
  __device__ inline bool exists(int k) const { return WT < 8 || k >= skip; }
  __device__ inline float apply(const Window<WT, VEC>& win, float x, int c) const {
    float p = bias[c];
#pragma unroll
    for (int k = 0; k < WT - 1; ++k)
      if (exists(k)) p = fmaf(w[k][c], win.v[k][c], p);
    return fmaf(w[WT - 1][c], x, p);
  }
};

// Where a thread stands: `lanes` threads side by side across the channels, 64 / lanes runs (segments) of steps in a wave.
struct ConvPlace {
  int lanes, lane_c, ch, row, rows;                  // row: the run of the workgroup's `rows`
  bool has;
  __device__ inline ConvPlace(int lanes_, int col, int H, int vec) : lanes(lanes_) {
    lane_c = threadIdx.x & (lanes - 1);
    row = threadIdx.x / lanes;
    rows = 256 / lanes;
    ch = (col * lanes + lane_c) * vec;
    has = ch < H;
    if (!has) ch = 0;
  }
  // Bits of the steps t .. t + n - 1 (n <= 24, at least 16 lanes a run) that reset; those outside the sequence do not.
  __device__ inline unsigned resets(const ConvArgs& a, int b, int t, int n) const {
    if (!a.reset) return 0;
    auto look = [&](int i) { return i < n && t + i >= 0 && t + i < a.c.T && a.reset[(long long)(t + i) * a.c.B + b] != 0; };
    unsigned bits = (unsigned)mine(__ballot(look(lane_c)));
    if (n > lanes) bits |= (unsigned)mine(__ballot(look(lane_c + lanes))) << lanes;
    return bits;
  }
  // What the run's lanes say of a ballot.
  __device__ inline unsigned long long mine(unsigned long long all) const {
    return lanes == 64 ? all : all >> ((threadIdx.x & 63) / lanes * lanes) & ((1ull << lanes) - 1);
  }
};

// Fills the window with the inputs before step t0; bit i of `resets`: step t0 - (WT - 1) + i resets.
template <typename E, int VEC, int WT>
__device__ inline void fill_window(const ConvArgs& a, int b, int ch, int t0, unsigned resets, Window<WT, VEC>& win) {
  win.clear();
  const E* x = (const E*)a.x.data + b * a.x.stride_b + ch;
#pragma unroll
  for (int i = 0; i < WT - 1; ++i) {
    const int s = t0 - (WT - 1) + i;
    if (s >= 0) {
      ConvRaw<E, VEC> r;
      r.load(x + s * a.x.stride_t);
      if (resets >> i & 1) win.clear();
      win.push([&](int c) { return r.at(c); });
    } else {
      const bool given = a.past && s >= 1 - a.c.W;
      const float* past = a.past + ((long long)b * (a.c.W - 1) + s + a.c.W - 1) * a.c.H + ch;
      win.push([&](int c) { return given ? past[c] : 0.f; });
    }
  }
}

template <typename E, int VEC, int WT>
__global__ __launch_bounds__(256) void conv_forward_kernel(ConvArgs a, int lanes, int cols) {
  const int T = a.c.T, runs = (T + CONV_RUN - 1) / CONV_RUN;
  const unsigned group = blockIdx.x / (unsigned)cols;
  const ConvPlace at(lanes, (int)(blockIdx.x - group * cols), a.c.H, VEC);
  const long long item = (long long)group * at.rows + at.row;
  // (all lanes of a run look at its resets)
  const bool run_exists = item < (long long)runs * a.c.B, has = at.has && run_exists;
  const int b = run_exists ? (int)(item / runs) : 0, t0 = run_exists ? (int)(item - (long long)b * runs) * CONV_RUN : 0;
  const int ch = at.ch;
  ConvRaw<E, VEC> raw[CONV_RUN];
  const E* x = (const E*)a.x.data + b * a.x.stride_b + ch;
#pragma unroll
  for (int r = 0; r < CONV_RUN; ++r) raw[r].load(x + min(t0 + r, T - 1) * a.x.stride_t);
  const Taps<WT, VEC> taps(a.weight, a.bias, a.c.W, ch);
  const unsigned resets = at.resets(a, b, t0 - (WT - 1), WT - 1 + CONV_RUN);
  Window<WT, VEC> win;
  fill_window<E, VEC, WT>(a, b, ch, t0, resets, win);
  if (!has) return;
  E* y = (E*)a.y.data + b * a.y.stride_b + ch;
  auto run = [&](auto plain) __attribute__((always_inline)) {     // plain: every step exists and none resets
    constexpr bool PLAIN = decltype(plain)::value;
#pragma unroll
    for (int r = 0; r < CONV_RUN; ++r) {
      const int t = t0 + r;
      if (!PLAIN && t >= T) break;
      if (!PLAIN && (resets >> (WT - 1 + r) & 1)) win.clear();
      float p[VEC];
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        p[c] = taps.apply(win, raw[r].at(c), c);
        if (a.c.act == CONV_SILU) p[c] = silu(p[c]);
      }
      conv_store<E, VEC>(y + t * a.y.stride_t, p, a.past_caches);
      win.push([&](int c) { return raw[r].at(c); });
    }
  };
  if (!resets && t0 + CONV_RUN <= T) run(std::true_type{});
  else run(std::false_type{});
  if (!a.last || t0 + CONV_RUN < T) return;
#pragma unroll
  for (int k = 0; k < WT - 1; ++k)
    if (k >= taps.skip) {
      float* o = a.last + ((long long)b * (a.c.W - 1) + k - taps.skip) * a.c.H + ch;
#pragma unroll
      for (int c = 0; c < VEC; ++c) o[c] = win.v[k][c];
    }
}

// What a thread carries along a segment: the window, and the gradients of the inputs t - WT + 1 .. t.
template <typename E, int VEC, int WT>
struct ConvBack {
  const ConvArgs& a;
  Window<WT, VEC> win;
  float g[WT][VEC], dw[WT][VEC], dbias[VEC];
  int b, ch, t0, t1, last_reset;                     // last_reset: the last step so far that resets

  __device__ inline ConvBack(const ConvArgs& a_) : a(a_) {
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
      dbias[c] = 0.f;
#pragma unroll
      for (int k = 0; k < WT; ++k) dw[k][c] = 0.f;
    }
  }
  // Step t's own output.  PLAIN: it exists, is the segment's and sees all of the window.
  template <bool PLAIN>
  __device__ inline void step(const Taps<WT, VEC>& taps, int t, const ConvRaw<E, VEC>& x, const ConvRaw<E, VEC>& dy) {
    const bool own = PLAIN || t < t1;
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
      const float xv = x.at(c);
      float dp = dy.at(c);
      if (a.c.act == CONV_SILU) {
        const float p = taps.apply(win, xv, c);
        const Sigmoid s(p);
        dp *= s.s * fmaf(gate_factor(p), s.n, 1.f);
      }
#pragma unroll
      for (int k = 0; k < WT; ++k) {
        if (!taps.exists(k) || (!PLAIN && t - (WT - 1) + k < last_reset)) continue;
        g[k][c] = fmaf(taps.w[k][c], dp, g[k][c]);
        if (own) dw[k][c] = fmaf(dp, k == WT - 1 ? xv : win.v[k < WT - 1 ? k : 0][c], dw[k][c]);
      }
      if (own) dbias[c] += dp;
    }
    win.push([&](int c) { return x.at(c); });
  }
  // The input t - (WT - 1), whose outputs are complete.
  template <bool PLAIN>
  __device__ inline void emit(int t) {
    const int s = t - (WT - 1), T = a.c.T, W = a.c.W, H = a.c.H;
    if (!PLAIN && a.dlast && s >= T - (W - 1) && s >= last_reset) {
      const float* d = a.dlast + ((long long)b * (W - 1) + s - (T - (W - 1))) * H + ch;
#pragma unroll
      for (int c = 0; c < VEC; ++c) g[0][c] += d[c];
    }
    if (s >= t0 && (PLAIN || s < t1)) {
      conv_store<E, VEC>((E*)a.dx.data + s * a.dx.stride_t + b * a.dx.stride_b + ch, g[0], a.past_caches);
    } else if (t0 == 0 && s < 0 && s >= 1 - W && a.dpast) {
      float* d = a.dpast + ((long long)b * (W - 1) + s + W - 1) * H + ch;
#pragma unroll
      for (int c = 0; c < VEC; ++c) d[c] = g[0][c];
    }
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
#pragma unroll
      for (int k = 0; k + 1 < WT; ++k) g[k][c] = g[k + 1][c];
      g[WT - 1][c] = 0.f;
    }
  }
};

// A thread goes through segments of a.seg steps, and the WT - 1 behind each, whose outputs its inputs reach.
template <typename E, int VEC, int WT>
__global__ __launch_bounds__(256) void conv_backward_kernel(ConvArgs a, int lanes, int cols) {
  const int T = a.c.T, W = a.c.W, H = a.c.H;
  const int group = blockIdx.x / cols, col = blockIdx.x - group * cols;
  const ConvPlace at(lanes, col, H, VEC);
  __shared__ float part[256][VEC];
  ConvBack<E, VEC, WT> v(a);
  v.ch = at.ch;
  const Taps<WT, VEC> taps(a.weight, a.bias, W, at.ch);
  const int segs = (T + a.seg - 1) / a.seg;
  const long long all = (long long)segs * a.c.B;
  // (the threads of a wave go through as many segments: they look at resets together)
  for (long long first = (long long)group * at.rows; first < all; first += (long long)a.groups * at.rows) {
    const long long item = first + at.row;
    const bool real = at.has && item < all;
    const int b = item < all ? (int)(item / segs) : 0;
    v.b = b;
    v.t0 = item < all ? (int)(item - (long long)b * segs) * a.seg : 0;
    v.t1 = min(v.t0 + a.seg, T);
    const E* x = (const E*)a.x.data + b * a.x.stride_b + at.ch;
    const E* dy = (const E*)a.dy.data + b * a.dy.stride_b + at.ch;
    const unsigned before = at.resets(a, b, v.t0 - (WT - 1), WT - 1);
    fill_window<E, VEC, WT>(a, b, at.ch, v.t0, before, v.win);
    v.last_reset = before ? v.t0 - (WT - 1) + 31 - __builtin_clz(before) : -(1 << 30);
#pragma unroll
    for (int k = 0; k < WT; ++k)
#pragma unroll
      for (int c = 0; c < VEC; ++c) v.g[k][c] = 0.f;
    ConvRaw<E, VEC> xn[CONV_BLOCK], dn[CONV_BLOCK];
    auto load = [&](int base) __attribute__((always_inline)) {
#pragma unroll
      for (int r = 0; r < CONV_BLOCK; ++r) {
        const long long t = min(base + r, T - 1);
        xn[r].load(x + t * a.x.stride_t);
        dn[r].load(dy + t * a.dy.stride_t);
      }
    };
    load(v.t0);
    unsigned long long ahead = 0;
    for (int off = 0; off < a.seg + WT - 1; off += CONV_BLOCK) {
      const int base = v.t0 + off;
      if (off % at.lanes == 0) {                     // (as many steps as a run has lanes to look at them)
        const int t = base + at.lane_c;
        ahead = a.reset ? at.mine(__ballot(t < T && a.reset[(long long)t * a.c.B + b] != 0)) : 0;
      }
      const unsigned resets = (unsigned)(ahead >> off % at.lanes) & ((1u << CONV_BLOCK) - 1);
      if (!real || base >= v.t1 + WT - 1) continue;
      ConvRaw<E, VEC> xr[CONV_BLOCK], dr[CONV_BLOCK];
#pragma unroll
      for (int r = 0; r < CONV_BLOCK; ++r) {
        xr[r] = xn[r];
        dr[r] = dn[r];
      }
      load(base + CONV_BLOCK);
      if (!resets && base - (WT - 1) >= v.last_reset && base + CONV_BLOCK <= v.t1) {
#pragma unroll
        for (int r = 0; r < CONV_BLOCK; ++r) {
          v.template step<true>(taps, base + r, xr[r], dr[r]);
          v.template emit<true>(base + r);
        }
      } else {
#pragma unroll
        for (int r = 0; r < CONV_BLOCK; ++r) {
          const int t = base + r;
          if (t >= v.t1 + WT - 1) break;
          if (resets >> r & 1) {
            v.win.clear();
            v.last_reset = t;
          }
          if (t < T) v.template step<false>(taps, t, xr[r], dr[r]);
          v.template emit<false>(t);
        }
      }
    }
  }
  // the rows' sums, one value after the other
  const int skip = WT - W;
#pragma unroll
  for (int k = 0; k <= WT; ++k) {
    if (k < skip) continue;
    __syncthreads();
#pragma unroll
    for (int c = 0; c < VEC; ++c) part[threadIdx.x][c] = k < WT ? v.dw[k < WT ? k : 0][c] : v.dbias[c];
    __syncthreads();
    for (int i = threadIdx.x; i < lanes * VEC; i += 256) {
      const int lane = i / VEC, c = i % VEC, ch = (col * lanes + lane) * VEC + c;
      if (ch >= H) continue;
      float sum = 0.f;
      for (int r = 0; r < at.rows; ++r) sum += part[r * lanes + lane][c];
      a.part[((long long)group * H + ch) * (W + 1) + k - skip] = sum;
    }
  }
}
// Gradients of the weights and biases from the groups' sums.
__global__ __launch_bounds__(SUM_THREADS) void conv_params_kernel(ConvArgs a) {
  const int W1 = a.c.W + 1;
  const long long n = (long long)a.c.H * W1, i = sum_column();
  float v;
  if (!sum_rows(a.part + i, n, a.groups, i < n, v)) return;
  const int ch = (int)(i / W1), k = (int)(i - (long long)ch * W1);
  if (k < a.c.W) {
    if (a.dweight) a.dweight[(long long)ch * a.c.W + k] = v;
  } else if (a.dbias) {
    a.dbias[ch] = v;
  }
}

// One step: a thread per channel.
template <typename E>
__global__ __launch_bounds__(256) void conv_step_kernel(ConvStepArgs a) {
  const int H = a.c.H, W = a.c.W;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  const int b = (int)(i / H), ch = (int)(i - (long long)b * H);
  if (b >= a.c.B) return;
  E* y = (E*)a.y.data + b * a.y.stride_b + ch;
  const int slot = a.slots ? a.slots[b] : b;
  if (slot < 0 || slot >= a.n_slots) {
    *y = elem_of<E>(0.f);
    return;
  }
  const float x = elem_f32(((const E*)a.x.data)[b * a.x.stride_b + ch]);
  const bool cut = a.reset && a.reset[b];
  const long long at = (long long)slot * (W - 1) * H + ch;
  const float* w = a.weight + (long long)ch * W;
  float past[CONV_MAX_W - 1], p = a.bias ? a.bias[ch] : 0.f;
#pragma unroll
  for (int k = 0; k < CONV_MAX_W - 1; ++k) past[k] = k < W - 1 && !cut ? a.past_in[at + (long long)k * H] : 0.f;
#pragma unroll
  for (int k = 0; k < CONV_MAX_W - 1; ++k)
    if (k < W - 1) {
      p = fmaf(w[k], past[k], p);
      a.past_out[at + (long long)k * H] = k + 1 < W - 1 ? past[k + 1 < CONV_MAX_W - 1 ? k + 1 : k] : x;
    }
  p = fmaf(w[W - 1], x, p);
  if (a.c.act == CONV_SILU) p = silu(p);
  *y = elem_of<E>(p);
}

// ---- launches
static int conv_taps(int W) { return W == 2 || W == 3 || W == 4 ? W : 8; }
// Threads of `vec` channels.  (The workspace and the limits hold for any.)
struct ConvShape {
  int lanes, cols, rows;                             // threads side by side, workgroups across, runs of a workgroup
  ConvShape(int H, int vec) {
    const long long n = ((long long)H + vec - 1) / vec;
    lanes = n > 32 ? 64 : n > 16 ? 32 : 16;
    cols = (int)((n + lanes - 1) / lanes);
    rows = 256 / lanes;
  }
};
static long long conv_runs(const conv_cfg& c, const ConvShape& s) {
  return ((c.T + CONV_RUN - 1LL) / CONV_RUN * c.B + s.rows - 1) / s.rows;
}
// Steps of a segment: as many as leave the card full, since each is followed by W - 1 that are looked at again.
static int conv_seg(const conv_cfg& c, const ConvShape& s) {
  int seg = 128;
  while (seg > 16 && (c.T + seg - 1LL) / seg * c.B * s.cols < 2048LL * s.rows / 4) seg /= 2;
  return seg;
}
static int conv_groups(const conv_cfg& c, const ConvShape& s) {
  const int seg = conv_seg(c, s);
  const long long all = ((c.T + seg - 1LL) / seg * c.B + s.rows - 1) / s.rows, most = (2047 + s.cols) / s.cols;
  return (int)(all < most ? all : most);
}
size_t conv_workspace(const conv_cfg& c) {
  const int two = conv_groups(c, ConvShape(c.H, 2)), one = conv_groups(c, ConvShape(c.H, 1));
  return 4 * (size_t)(two > one ? two : one) * c.H * (c.W + 1);
}
bool conv_launchable(const conv_cfg& c) {
  const ConvShape s(c.H, 1);
  return launchable(conv_runs(c, s) * s.cols, 256) && launchable((long long)conv_groups(c, s) * s.cols, 256) &&
         launchable(sum_groups((long long)c.H * (c.W + 1)), SUM_THREADS);
}
template <typename E, int VEC, int WT, bool BACKWARD>
static hipError_t conv_kernel(ConvArgs a, hipStream_t s) {
  const ConvShape c(a.c.H, VEC);
  const dim3 t(256);
  if constexpr (!BACKWARD) {
    hipLaunchKernelGGL((conv_forward_kernel<E, VEC, WT>), dim3((unsigned)(conv_runs(a.c, c) * c.cols)), t, 0, s, a, c.lanes,
                       c.cols);
    return hipGetLastError();
  } else {
    a.groups = conv_groups(a.c, c);
    a.seg = conv_seg(a.c, c);
    hipLaunchKernelGGL((conv_backward_kernel<E, VEC, WT>), dim3((unsigned)((long long)a.groups * c.cols)), t, 0, s, a, c.lanes,
                       c.cols);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!a.dweight && !a.dbias)) return e;
    hipLaunchKernelGGL(conv_params_kernel, dim3(sum_groups((long long)a.c.H * (a.c.W + 1))), dim3(SUM_THREADS), 0, s, a);
    return hipGetLastError();
  }
}
template <typename E, int VEC, bool BACKWARD>
static hipError_t conv_start(const ConvArgs& a, hipStream_t s) {
  switch (conv_taps(a.c.W)) {
    case 2: return conv_kernel<E, VEC, 2, BACKWARD>(a, s);
    case 3: return conv_kernel<E, VEC, 3, BACKWARD>(a, s);
    case 4: return conv_kernel<E, VEC, 4, BACKWARD>(a, s);
    default: return conv_kernel<E, VEC, 8, BACKWARD>(a, s);
  }
}
template <typename E>
static hipError_t conv_forward_start(const ConvArgs& a, hipStream_t s) {
  const bool words = pairs<E>(a.x, a.c.H) && pairs<E>(a.y, a.c.H);
  return words ? conv_start<E, 2, false>(a, s) : conv_start<E, 1, false>(a, s);
}
template <typename E>
static hipError_t conv_backward_start(const ConvArgs& a, hipStream_t s) {
  const bool words = pairs<E>(a.x, a.c.H) && pairs<E>(a.dy, a.c.H) && pairs<E>(a.dx, a.c.H);
  return words ? conv_start<E, 2, true>(a, s) : conv_start<E, 1, true>(a, s);
}
hipError_t launch_conv_forward(const ConvArgs& a, hipStream_t s) {
  if (a.c.dtype == MGRIT_F32) return conv_forward_start<float>(a, s);
  if (a.c.dtype == MGRIT_BF16) return conv_forward_start<Bf16>(a, s);
  return conv_forward_start<F16>(a, s);
}
hipError_t launch_conv_backward(const ConvArgs& a, hipStream_t s) {
  if (a.c.dtype == MGRIT_F32) return conv_backward_start<float>(a, s);
  if (a.c.dtype == MGRIT_BF16) return conv_backward_start<Bf16>(a, s);
  return conv_backward_start<F16>(a, s);
}
hipError_t launch_conv_step(const ConvStepArgs& a, hipStream_t s) {
  const long long n = ((long long)a.c.B * a.c.H + 255) / 256;
  if (!launchable(n, 256)) return TOO_LARGE;
  const dim3 g((unsigned)n), t(256);
  if (a.c.dtype == MGRIT_F32) hipLaunchKernelGGL((conv_step_kernel<float>), g, t, 0, s, a);
  else if (a.c.dtype == MGRIT_BF16) hipLaunchKernelGGL((conv_step_kernel<Bf16>), g, t, 0, s, a);
  else hipLaunchKernelGGL((conv_step_kernel<F16>), g, t, 0, s, a);
  return hipGetLastError();
}

}  // namespace mg
