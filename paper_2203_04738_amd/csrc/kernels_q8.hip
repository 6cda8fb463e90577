// Product in 8-bit integers with a scale for each token and channel (include/mgrit_ops.h).
#include "elem.h"
#include "ops.h"

namespace mg {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx16 __attribute__((ext_vector_type(16)));

__host__ __device__ inline long long q8_pad(int K) { return ((long long)K + 127) / 128 * 128; }

__device__ inline float quant_scale(float amax) { return fmaxf(amax * (1.0f / 127.0f), 0x1p-126f); }
__device__ inline int quant(float x, float scale) { return (int)rintf(x / scale); }

// One row per workgroup; the second pass reads the row from the caches.  A row that is not finite: scale NaN, zeros.
template <typename E>
__global__ __launch_bounds__(256) void q8_quantize_kernel(Q8Args a) {
  __shared__ float part[4];
  __shared__ int odd;
  const long long row = blockIdx.x;
  const E* x = (const E*)a.x + row * a.c.ldx;
  const int tid = threadIdx.x, K = a.c.K;
  if (tid == 0) odd = 0;
  __syncthreads();
  float m = 0.f;
  bool bad = false;
  for (int k = tid; k < K; k += 256) {
    const float v = fabsf(elem_f32(x[k]));
    bad |= !(v < __builtin_inff());
    m = fmaxf(m, v);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  if (__any(bad) && (tid & 63) == 0) odd = 1;
  if ((tid & 63) == 0) part[tid >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
  const bool finite = odd == 0;
  const float scale = quant_scale(finite ? m : 0.f);
  if (tid == 0) a.scale[row] = finite ? scale : __uint_as_float(0x7fc00000u);
  const int pad = (int)q8_pad(K);
  int* out = (int*)(a.q + row * pad);
  for (int k = 4 * tid; k < pad; k += 1024) {
    unsigned w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (finite && k + i < K) w |= ((unsigned)quant(elem_f32(x[k + i]), scale) & 255u) << (8 * i);
    out[k / 4] = (int)w;
  }
}

// Tile of TM tokens x TN channels, four waves of half of each.  The channels are the rows of the matrix
// instruction and the tokens its columns: a lane then holds four neighbouring channels of a token.
// Slices of 128 bytes of K go through LDS; a row's 16-byte pieces are stored in the order piece ^ (row & 7).
template <typename E, int TM, int TN>
__global__ __launch_bounds__(256) void q8_tile_kernel(Q8Args a) {
  constexpr int WM = TM / 64, WN = TN / 64;              // 32 x 32 blocks of a wave
  __shared__ intx4 sx[TM * 8], sw[TN * 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long pad = q8_pad(a.c.K);
  const int tiles_n = (a.c.N + TN - 1) / TN;
  const int tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
  const int m0 = tm * TM, n0 = tn * TN;
  const int wm = (wave & 1) * (TM / 2), wn = (wave >> 1) * (TN / 2);
  intx16 acc[WN][WM];
#pragma unroll
  for (int i = 0; i < WN; ++i)
#pragma unroll
    for (int j = 0; j < WM; ++j) acc[i][j] = intx16{};
  constexpr int LX = TM * 8 / 256, LW = TN * 8 / 256;
  intx4 rx[LX], rw[LW];
  auto load = [&](long long k) {
#pragma unroll
    for (int i = 0; i < LX; ++i) {
      const int e = tid + 256 * i, r = min(m0 + (e >> 3), a.c.M - 1);
      rx[i] = *reinterpret_cast<const intx4*>(a.q + r * pad + k + (e & 7) * 16);
    }
#pragma unroll
    for (int i = 0; i < LW; ++i) {
      const int e = tid + 256 * i, r = min(n0 + (e >> 3), a.c.N - 1);
      rw[i] = *reinterpret_cast<const intx4*>(a.w + r * pad + k + (e & 7) * 16);
    }
  };
  load(0);
  for (long long k = 0; k < pad; k += 128) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < LX; ++i) {
      const int e = tid + 256 * i;
      sx[(e & ~7) | ((e & 7) ^ ((e >> 3) & 7))] = rx[i];
    }
#pragma unroll
    for (int i = 0; i < LW; ++i) {
      const int e = tid + 256 * i;
      sw[(e & ~7) | ((e & 7) ^ ((e >> 3) & 7))] = rw[i];
    }
    __syncthreads();
    if (k + 128 < pad) load(k + 128);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      intx4 fx[WM], fw[WN];
      const int piece = kk * 2 + (lane >> 5);
#pragma unroll
      for (int j = 0; j < WM; ++j) {
        const int r = wm + 32 * j + (lane & 31);
        fx[j] = sx[r * 8 + (piece ^ (r & 7))];
      }
#pragma unroll
      for (int i = 0; i < WN; ++i) {
        const int r = wn + 32 * i + (lane & 31);
        fw[i] = sw[r * 8 + (piece ^ (r & 7))];
      }
#pragma unroll
      for (int i = 0; i < WN; ++i)
#pragma unroll
        for (int j = 0; j < WM; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[i], fx[j], acc[i][j], 0, 0, 0);
    }
  }
#pragma unroll
  for (int j = 0; j < WM; ++j) {
    const int m = m0 + wm + 32 * j + (lane & 31);
    if (m >= a.c.M) continue;
    const float sm = a.scale[m];
    E* y = (E*)a.y + (long long)m * a.c.ldy;
#pragma unroll
    for (int i = 0; i < WN; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int n = n0 + wn + 32 * i + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
        if (n >= a.c.N) continue;
        const float v = (float)acc[i][j][e] * sm * a.w_scale[n];
        y[n] = elem_of<E>(a.bias ? v + a.bias[n] : v);
      }
  }
}

hipError_t launch_q8_quantize(const Q8Args& a, hipStream_t s) {
  const dim3 g((unsigned)a.c.M), t(256);
  if (a.c.dtype == MGRIT_F32) hipLaunchKernelGGL(q8_quantize_kernel<float>, g, t, 0, s, a);
  else if (a.c.dtype == MGRIT_BF16) hipLaunchKernelGGL(q8_quantize_kernel<Bf16>, g, t, 0, s, a);
  else hipLaunchKernelGGL(q8_quantize_kernel<F16>, g, t, 0, s, a);
  return hipGetLastError();
}

template <typename E>
static void q8_start(const Q8Args& a, hipStream_t s) {
  const unsigned grid = (unsigned)((a.c.M + 127) / 128) * (unsigned)((a.c.N + 127) / 128);
  hipLaunchKernelGGL((q8_tile_kernel<E, 128, 128>), dim3(grid), dim3(256), 0, s, a);
}
hipError_t launch_q8_linear(const Q8Args& a, hipStream_t s) {
  const hipError_t e = launch_q8_quantize(a, s);
  if (e != hipSuccess) return e;
  if (a.c.dtype == MGRIT_F32) q8_start<float>(a, s);
  else if (a.c.dtype == MGRIT_BF16) q8_start<Bf16>(a, s);
  else q8_start<F16>(a, s);
  return hipGetLastError();
}

}  // namespace mg
