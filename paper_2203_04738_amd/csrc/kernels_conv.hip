// Causal convolution of every channel over its last few inputs (include/mgrit_tokens.h), its gradient, and one step.
//
// A thread has two neighbouring channels and goes along time with the window of inputs that the next step sees in
// registers; a reset empties the window.  What bounds it is memory: every array is read or written once but for the
// few steps before (backward: around) each thread's own.
#include "elem.h"
#include "pairs.h"
#include "row_sums.h"
#include "tokens.h"

namespace mg {

constexpr int CONV_RUN = 16;                         // steps of a thread, forward
constexpr int CONV_SEG = 64;                         // steps that a thread looks at in a segment, backward

// The window of a thread's two channels, oldest first; WT >= W taps, those before the last W never used.
template <int WT>
struct Window {
  float v[WT - 1][2];
  __device__ inline void clear() {
#pragma unroll
    for (int i = 0; i < WT - 1; ++i) v[i][0] = v[i][1] = 0.f;
  }
  __device__ inline void push(float x, float y) {
#pragma unroll
    for (int i = 0; i + 1 < WT - 1; ++i) {
      v[i][0] = v[i + 1][0];
      v[i][1] = v[i + 1][1];
    }
    v[WT - 2][0] = x;
    v[WT - 2][1] = y;
  }
};
template <int WT>
struct Taps {
  float w[WT][2], bias[2];
  int skip;                                          // taps that do not exist
  __device__ inline Taps(const float* weight, const float* b, int W, int ch, bool second) : skip(WT - W) {
    const int c1 = second ? ch + 1 : ch;
#pragma unroll
    for (int k = 0; k < WT; ++k) {
      w[k][0] = k >= skip ? weight[(long long)ch * W + k - skip] : 0.f;
      w[k][1] = k >= skip ? weight[(long long)c1 * W + k - skip] : 0.f;
    }
    bias[0] = b ? b[ch] : 0.f;
    bias[1] = b ? b[c1] : 0.f;
  }
  __device__ inline float apply(const Window<WT>& win, float x, int c) const {
    float p = bias[c];
#pragma unroll
    for (int k = 0; k < WT - 1; ++k)
      if (WT < 8 || k >= skip) p = fmaf(w[k][c], win.v[k][c], p);
    return fmaf(w[WT - 1][c], x, p);
  }
};
__device__ inline float conv_sigmoid(float z) {
  const float e = exp_of(-fabsf(z));
  const float small = e * __builtin_amdgcn_rcpf(1.0f + e);
  return z != z ? z : z < 0.f ? small : 1.0f - small;
}

// Input s < 0 of a batch row's channel: from `past`, or zero.
__device__ inline float past_input(const float* past, int W, int H, int b, int s, int ch) {
  return past && s >= 1 - W ? past[((long long)b * (W - 1) + s + W - 1) * H + ch] : 0.f;
}

// Fills the window with the inputs before step t0.
template <typename E, bool ALIGNED, int WT>
__device__ inline void fill_window(const ConvArgs& a, int b, int ch, bool second, int t0, Window<WT>& win) {
  win.clear();
  const E* x = (const E*)a.x.data + b * a.x.stride_b + ch;
#pragma unroll
  for (int i = 0; i < WT - 1; ++i) {
    const int s = t0 - (WT - 1) + i;
    if (s >= 0) {
      const RawPair<E> r = load_pair<E, ALIGNED>(x + s * a.x.stride_t, second);
      if (a.reset && a.reset[(long long)s * a.c.B + b]) win.clear();
      win.push(r.at(0), r.at(1));
    } else {
      win.push(past_input(a.past, a.c.W, a.c.H, b, s, ch), past_input(a.past, a.c.W, a.c.H, b, s, second ? ch + 1 : ch));
    }
  }
}

template <typename E, bool ALIGNED, int WT>
__global__ __launch_bounds__(256) void conv_forward_kernel(ConvArgs a) {
  const int pairs = (a.c.H + 1) / 2, T = a.c.T;
  const int runs = (T + CONV_RUN - 1) / CONV_RUN;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, br = i / pairs;
  const int ch = 2 * (int)(i - br * pairs);
  const int b = (int)(br / runs), t0 = (int)(br - (long long)b * runs) * CONV_RUN;
  if (b >= a.c.B) return;
  const bool second = ch + 1 < a.c.H;
  RawPair<E> raw[CONV_RUN];
  const E* x = (const E*)a.x.data + b * a.x.stride_b + ch;
#pragma unroll
  for (int r = 0; r < CONV_RUN; ++r) raw[r] = load_pair<E, ALIGNED>(x + min(t0 + r, T - 1) * a.x.stride_t, second);
  const Taps<WT> taps(a.weight, a.bias, a.c.W, ch, second);
  Window<WT> win;
  fill_window<E, ALIGNED, WT>(a, b, ch, second, t0, win);
  E* y = (E*)a.y.data + b * a.y.stride_b + ch;
#pragma unroll
  for (int r = 0; r < CONV_RUN; ++r) {
    const int t = t0 + r;
    if (t >= T) break;
    if (a.reset && a.reset[(long long)t * a.c.B + b]) win.clear();
    float p[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      p[c] = taps.apply(win, raw[r].at(c), c);
      if (a.c.act == CONV_SILU) p[c] *= conv_sigmoid(p[c]);
    }
    store_pair<E, ALIGNED>(y + t * a.y.stride_t, p[0], p[1], second, a.past_caches);
    win.push(raw[r].at(0), raw[r].at(1));
  }
  if (!a.last || t0 + CONV_RUN < T) return;
#pragma unroll
  for (int k = 0; k < WT - 1; ++k)
    if (k >= taps.skip) {
      float* o = a.last + ((long long)b * (a.c.W - 1) + k - taps.skip) * a.c.H + ch;
      o[0] = win.v[k][0];
      if (second) o[1] = win.v[k][1];
    }
}

// A thread goes through segments of CONV_SEG - WT + 1 steps, and the WT - 1 behind each, whose outputs its inputs reach.
// LANES threads are side by side across the channels.
template <typename E, bool ALIGNED, int WT>
__global__ __launch_bounds__(256) void conv_backward_kernel(ConvArgs a, int lanes) {
  constexpr int OWN = CONV_SEG - (WT - 1), BLOCK = 8;
  const int T = a.c.T, B = a.c.B, H = a.c.H, W = a.c.W;
  const int cols = (H + 2 * lanes - 1) / (2 * lanes), rows = 256 / lanes;
  const int group = blockIdx.x / cols, col = blockIdx.x - group * cols;
  const int lane = threadIdx.x & (lanes - 1), row = threadIdx.x / lanes;
  const int ch = (col * lanes + lane) * 2;
  const bool has = ch < H, second = ch + 1 < H;
  __shared__ float part[256][2];
  float dw[WT][2], dbias[2] = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < WT; ++k) dw[k][0] = dw[k][1] = 0.f;
  const int segs = (T + OWN - 1) / OWN;
  const long long all = (long long)segs * B;
  if (has) {
    const Taps<WT> taps(a.weight, a.bias, W, ch, second);
    for (long long item = (long long)group * rows + row; item < all; item += (long long)a.groups * rows) {
      const int b = (int)(item / segs), t0 = (int)(item - (long long)b * segs) * OWN, t1 = min(t0 + OWN, T);
      const E* x = (const E*)a.x.data + b * a.x.stride_b + ch;
      const E* dy = (const E*)a.dy.data + b * a.dy.stride_b + ch;
      Window<WT> win;
      fill_window<E, ALIGNED, WT>(a, b, ch, second, t0, win);
      int last_reset = -(1 << 30);                   // the last step so far that resets
      if (a.reset)
        for (int s = max(0, t0 - (WT - 1)); s < t0; ++s)
          if (a.reset[(long long)s * B + b]) last_reset = s;
      float g[WT][2];                                // gradients of the inputs t - WT + 1 .. t
#pragma unroll
      for (int k = 0; k < WT; ++k) g[k][0] = g[k][1] = 0.f;
      for (int base = t0; base < t1 + WT - 1; base += BLOCK) {
        RawPair<E> xr[BLOCK], dr[BLOCK];
#pragma unroll
        for (int r = 0; r < BLOCK; ++r) {
          const long long t = min(base + r, T - 1);
          xr[r] = load_pair<E, ALIGNED>(x + t * a.x.stride_t, second);
          dr[r] = load_pair<E, ALIGNED>(dy + t * a.dy.stride_t, second);
        }
#pragma unroll
        for (int r = 0; r < BLOCK; ++r) {
          const int t = base + r;
          if (t >= t1 + WT - 1) break;
          if (t < T) {
            if (a.reset && a.reset[(long long)t * B + b]) {
              win.clear();
              last_reset = t;
            }
            const bool own = t < t1;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const float xv = xr[r].at(c);
              float dp = dr[r].at(c);
              if (a.c.act == CONV_SILU) {
                const float p = taps.apply(win, xv, c), s = conv_sigmoid(p);
                dp *= s * fmaf(p, 1.f - s, 1.f);
              }
#pragma unroll
              for (int k = 0; k < WT; ++k) {
                const bool seen = (WT < 8 || k >= taps.skip) && t - (WT - 1) + k >= last_reset;
                if (seen) {
                  g[k][c] = fmaf(taps.w[k][c], dp, g[k][c]);
                  if (own) dw[k][c] = fmaf(dp, k == WT - 1 ? xv : win.v[k < WT - 1 ? k : 0][c], dw[k][c]);
                }
              }
              if (own) dbias[c] += dp;
            }
            win.push(xr[r].at(0), xr[r].at(1));
          }
          // the input whose outputs are complete
          const int s = t - (WT - 1);
          if (a.dlast && s >= T - (W - 1) && s >= last_reset) {
            const float* d = a.dlast + ((long long)b * (W - 1) + s - (T - (W - 1))) * H + ch;
            g[0][0] += d[0];
            if (second) g[0][1] += d[1];
          }
          if (s >= t0 && s < t1) {
            store_pair<E, ALIGNED>((E*)a.dx.data + s * a.dx.stride_t + b * a.dx.stride_b + ch, g[0][0], g[0][1], second,
                                   a.past_caches);
          } else if (t0 == 0 && s < 0 && s >= 1 - W && a.dpast) {
            float* d = a.dpast + ((long long)b * (W - 1) + s + W - 1) * H + ch;
            d[0] = g[0][0];
            if (second) d[1] = g[0][1];
          }
#pragma unroll
          for (int k = 0; k + 1 < WT; ++k) {
            g[k][0] = g[k + 1][0];
            g[k][1] = g[k + 1][1];
          }
          g[WT - 1][0] = g[WT - 1][1] = 0.f;
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
    part[threadIdx.x][0] = k < WT ? dw[k < WT ? k : 0][0] : dbias[0];
    part[threadIdx.x][1] = k < WT ? dw[k < WT ? k : 0][1] : dbias[1];
    __syncthreads();
    if (row == 0 && has) {
      float u = 0.f, v = 0.f;
      for (int r = 0; r < rows; ++r) {
        u += part[r * lanes + lane][0];
        v += part[r * lanes + lane][1];
      }
      float* o = a.part + ((long long)group * H + ch) * (W + 1) + k - skip;
      o[0] = u;
      if (second) o[W + 1] = v;
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
  if (a.c.act == CONV_SILU) p *= conv_sigmoid(p);
  *y = elem_of<E>(p);
}

// ---- launches
static int conv_taps(int W) { return W == 2 || W == 3 || W == 4 ? W : 8; }
static int conv_lanes(int H) { return H > 64 ? 64 : H > 32 ? 32 : 16; }
static int conv_groups(const conv_cfg& c) {
  const int lanes = conv_lanes(c.H), own = CONV_SEG - (conv_taps(c.W) - 1);
  const long long cols = (c.H + 2LL * lanes - 1) / (2 * lanes), rows = 256 / lanes;
  const long long all = (((c.T + own - 1LL) / own) * c.B + rows - 1) / rows, most = (2047 + cols) / cols;
  return (int)(all < most ? all : most);
}
size_t conv_workspace(const conv_cfg& c) { return 4 * (size_t)conv_groups(c) * c.H * (c.W + 1); }
static long long conv_forward_groups(const conv_cfg& c) {
  return ((c.T + CONV_RUN - 1LL) / CONV_RUN * c.B * ((c.H + 1LL) / 2) + 255) / 256;
}
bool conv_launchable(const conv_cfg& c) {
  return launchable(conv_forward_groups(c), 256) && launchable(sum_groups((long long)c.H * (c.W + 1)), SUM_THREADS);
}
template <typename E, bool ALIGNED>
static void conv_forward_taps(const ConvArgs& a, hipStream_t s) {
  const dim3 g((unsigned)conv_forward_groups(a.c)), t(256);
  switch (conv_taps(a.c.W)) {
    case 2: hipLaunchKernelGGL((conv_forward_kernel<E, ALIGNED, 2>), g, t, 0, s, a); break;
    case 3: hipLaunchKernelGGL((conv_forward_kernel<E, ALIGNED, 3>), g, t, 0, s, a); break;
    case 4: hipLaunchKernelGGL((conv_forward_kernel<E, ALIGNED, 4>), g, t, 0, s, a); break;
    default: hipLaunchKernelGGL((conv_forward_kernel<E, ALIGNED, 8>), g, t, 0, s, a);
  }
}
template <typename E, bool ALIGNED>
static void conv_backward_taps(const ConvArgs& a, hipStream_t s) {
  const int lanes = conv_lanes(a.c.H);
  const dim3 g((unsigned)(a.groups * ((a.c.H + 2LL * lanes - 1) / (2 * lanes)))), t(256);
  switch (conv_taps(a.c.W)) {
    case 2: hipLaunchKernelGGL((conv_backward_kernel<E, ALIGNED, 2>), g, t, 0, s, a, lanes); break;
    case 3: hipLaunchKernelGGL((conv_backward_kernel<E, ALIGNED, 3>), g, t, 0, s, a, lanes); break;
    case 4: hipLaunchKernelGGL((conv_backward_kernel<E, ALIGNED, 4>), g, t, 0, s, a, lanes); break;
    default: hipLaunchKernelGGL((conv_backward_kernel<E, ALIGNED, 8>), g, t, 0, s, a, lanes);
  }
}
template <typename E>
static hipError_t conv_start(const ConvArgs& a, bool backward, hipStream_t s) {
  const int H = a.c.H;
  if (!backward) {
    if (pairs<E>(a.x, H) && pairs<E>(a.y, H)) conv_forward_taps<E, true>(a, s);
    else conv_forward_taps<E, false>(a, s);
    return hipGetLastError();
  }
  if (pairs<E>(a.x, H) && pairs<E>(a.dy, H) && pairs<E>(a.dx, H)) conv_backward_taps<E, true>(a, s);
  else conv_backward_taps<E, false>(a, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || (!a.dweight && !a.dbias)) return e;
  hipLaunchKernelGGL(conv_params_kernel, dim3(sum_groups((long long)H * (a.c.W + 1))), dim3(SUM_THREADS), 0, s, a);
  return hipGetLastError();
}
static hipError_t conv_typed(const ConvArgs& a, bool backward, hipStream_t s) {
  if (a.c.dtype == MGRIT_F32) return conv_start<float>(a, backward, s);
  if (a.c.dtype == MGRIT_BF16) return conv_start<Bf16>(a, backward, s);
  return conv_start<F16>(a, backward, s);
}
hipError_t launch_conv_forward(const ConvArgs& a, hipStream_t s) { return conv_typed(a, false, s); }
hipError_t launch_conv_backward(const ConvArgs& a_, hipStream_t s) {
  ConvArgs a = a_;
  a.groups = conv_groups(a.c);
  return conv_typed(a, true, s);
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
