// Product in 8-bit integers with a scale for each token and channel (include/mgrit_ops.h).
//
// The tokens are quantised into the workspace by a kernel of their own (each row once; the product's tiles would do
// it once per column of tiles); rows are padded with zeros to 128 bytes, so that the products look at no tail of K.
// In the products the channels are the rows of the matrix instruction and the tokens its columns: a lane ends up with
// four neighbouring channels of one token.
#include <algorithm>
#include <cmath>

#include "elem.h"
#include "ops.h"

namespace mg {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx16 __attribute__((ext_vector_type(16)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

__host__ __device__ inline int q8_pad(int K) { return (K + 127) / 128 * 128; }

// ---------------------------------------------------------------------------
// quantisation
// ---------------------------------------------------------------------------
__device__ inline float quant_scale(float amax) { return fmaxf(amax / 127.0f, 0x1p-126f); }
__device__ inline unsigned quant(float x, float scale) { return (unsigned)(int)rintf(x / scale) & 255u; }
__device__ inline float wave_max(float v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// A row in the registers of a team of THREADS threads: LOADS pieces of 16 bytes per thread, zeros behind its end.
template <typename E, int THREADS, int LOADS>
struct QuantRow {
  static constexpr int PER = 16 / (int)sizeof(E);
  uintx4 raw[LOADS];
  __device__ inline void load(const E* x, int K, int tid) {
    if (((uintptr_t)x & 15) == 0 && K % PER == 0) {
#pragma unroll
      for (int j = 0; j < LOADS; ++j) {
        const int i = (j * THREADS + tid) * PER;
        raw[j] = uintx4{};
        if (i < K) raw[j] = *reinterpret_cast<const uintx4*>(x + i);
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int i = (j * THREADS + tid) * PER;
      E e[PER];
#pragma unroll
      for (int k = 0; k < PER; ++k) e[k] = i + k < K ? x[i + k] : elem_of<E>(0.f);
      raw[j] = __builtin_bit_cast(uintx4, e);
    }
  }
  __device__ inline float at(int j, int k) const {
    return word_elem<E>(raw[j][k / ELEMS_PER_WORD<E>], k % ELEMS_PER_WORD<E>);
  }
  // largest magnitude of what the wave holds; infinite where a value is not a number (the larger of a value and NaN
  // would be the value)
  __device__ inline float top() const {
    float m = 0.f;
#pragma unroll
    for (int j = 0; j < LOADS; ++j)
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const float v = fabsf(at(j, k));
        m = fmaxf(m, v == v ? v : __builtin_inff());
      }
    return wave_max(m);
  }
  // the quantised row (zeros where it is not finite); out 4-byte aligned
  __device__ inline void put(int8_t* out, int pad, int tid, bool finite, float scale) const {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int i = (j * THREADS + tid) * PER;
      if (i >= pad) continue;
#pragma unroll
      for (int k = 0; k < PER; k += 4) {
        unsigned w = 0;
        if (finite)
#pragma unroll
          for (int b = 0; b < 4; ++b) w |= quant(at(j, k + b), scale) << (8 * b);
        *reinterpret_cast<unsigned*>(out + i + k) = w;
      }
    }
  }
};

// A row per team of NW waves.  A row that is not finite: scale NaN, zeros.  32768 x 2048 bf16: 201 MB in 42 us (4.8
// TB/s).
template <typename E, int NW, int LOADS>
__global__ __launch_bounds__(NW == 1 ? 256 : NW * 64) void q8_quantize_kernel(Q8Args a) {
  __shared__ float part[NW];
  const int tid = NW == 1 ? threadIdx.x & 63 : threadIdx.x;
  const long long row = NW == 1 ? blockIdx.x * 4LL + (threadIdx.x >> 6) : blockIdx.x;
  if (row >= a.c.M) return;                          // (teams of one wave: whole waves)
  const int pad = q8_pad(a.c.K);
  QuantRow<E, NW * 64, LOADS> r;
  r.load((const E*)a.x + row * a.c.ldx, a.c.K, tid);
  float m = r.top();
  if constexpr (NW > 1) {
    if ((tid & 63) == 0) part[tid >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, part[w]);
  }
  const bool finite = m < __builtin_inff();
  const float scale = quant_scale(finite ? m : 0.f);
  if (tid == 0) a.scale[row] = finite ? scale : __uint_as_float(0x7fc00000u);
  r.put(a.q + row * pad, pad, tid, finite, scale);
}

// Rows longer than that, in two passes; the second reads the row from the caches.
template <typename E>
__global__ __launch_bounds__(1024) void q8_quantize_long_kernel(Q8Args a) {
  __shared__ float part[16];
  const long long row = blockIdx.x;
  const E* x = (const E*)a.x + row * a.c.ldx;
  const int tid = threadIdx.x, K = a.c.K, pad = q8_pad(K);
  float m = 0.f;
  for (int k = tid; k < K; k += 1024) {
    const float v = fabsf(elem_f32(x[k]));
    m = fmaxf(m, v == v ? v : __builtin_inff());
  }
  m = wave_max(m);
  if ((tid & 63) == 0) part[tid >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 16; ++w) m = fmaxf(m, part[w]);
  const bool finite = m < __builtin_inff();
  const float scale = quant_scale(finite ? m : 0.f);
  if (tid == 0) a.scale[row] = finite ? scale : __uint_as_float(0x7fc00000u);
  unsigned* out = (unsigned*)(a.q + row * pad);
  for (int k = 4 * tid; k < pad; k += 4096) {
    unsigned w = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b)
      if (finite && k + b < K) w |= quant(elem_f32(x[k + b]), scale) << (8 * b);
    out[k / 4] = w;
  }
}

// Teams that hold the row.  One wave per row : four, 2048 bf16, us: 512 rows 4.1 : 3.3, 2048 rows 5.6 : 5.9, 8192
// rows 14.2 : 16.6, 32768 rows 42.5 : 57; rows of 4096 take four (4096 rows 15.2 : 13.4).
struct QuantTeam {
  int waves, loads;                                  // of 16 bytes a thread; 0: the row is read twice
};
static QuantTeam quant_team(const q8_cfg& c) {
  const int per = c.dtype == MGRIT_F32 ? 4 : 8, pad = q8_pad(c.K);
  if (pad <= 2 * 64 * per) return {1, 2};
  if (pad <= 4 * 64 * per && c.M >= 2048) return {1, 4};
  if (pad <= 4 * 256 * per) return {4, 4};
  if (pad <= 4 * 1024 * per) return {16, 4};
  return {16, 0};
}
static bool quantize_launchable(const q8_cfg& c) {
  const int waves = quant_team(c).waves;
  return waves == 1 ? launchable(((long long)c.M + 3) / 4, 256) : launchable(c.M, waves * 64);
}
template <typename E>
static void quantize_start(const Q8Args& a, hipStream_t s) {
  const unsigned M = (unsigned)a.c.M;
  const QuantTeam t = quant_team(a.c);
  if (t.waves == 1 && t.loads == 2)
    hipLaunchKernelGGL((q8_quantize_kernel<E, 1, 2>), dim3((M + 3) / 4), dim3(256), 0, s, a);
  else if (t.waves == 1)
    hipLaunchKernelGGL((q8_quantize_kernel<E, 1, 4>), dim3((M + 3) / 4), dim3(256), 0, s, a);
  else if (t.waves == 4)
    hipLaunchKernelGGL((q8_quantize_kernel<E, 4, 4>), dim3(M), dim3(256), 0, s, a);
  else if (t.loads > 0)
    hipLaunchKernelGGL((q8_quantize_kernel<E, 16, 4>), dim3(M), dim3(1024), 0, s, a);
  else
    hipLaunchKernelGGL(q8_quantize_long_kernel<E>, dim3(M), dim3(1024), 0, s, a);
}
hipError_t launch_q8_quantize(const Q8Args& a, hipStream_t s) {
  if (!quantize_launchable(a.c)) return TOO_LARGE;
  if (a.c.dtype == MGRIT_F32) quantize_start<float>(a, s);
  else if (a.c.dtype == MGRIT_BF16) quantize_start<Bf16>(a, s);
  else quantize_start<F16>(a, s);
  return hipGetLastError();
}

// --------------------------------------------------------------------------- products
// --------------------------------------------------------------------------- Four neighbouring channels n .. n+3 of
// a token, from their sums and the scales and biases of the channels; wide: in one store (the row's place allows it).
//  The channel's scale comes first: a sum times the scale of a token near a float's largest value would be beyond it
// where the product of all three is not.
template <typename E>
__device__ inline void put4(const Q8Args& a, E* y, int n, const intx4& sum, float sm, const float4& ws,
                            const float4& bias, bool wide) {
  const float v[4] = {(float)sum[0] * ws.x * sm + bias.x, (float)sum[1] * ws.y * sm + bias.y,
                      (float)sum[2] * ws.z * sm + bias.z, (float)sum[3] * ws.w * sm + bias.w};
  if (wide && n + 3 < a.c.N) {
    if constexpr (sizeof(E) == 4)
      *reinterpret_cast<float4*>(y + n) = make_float4(v[0], v[1], v[2], v[3]);
    else
      *reinterpret_cast<uint2*>(y + n) = make_uint2(pack2<E>(v[0], v[1]), pack2<E>(v[2], v[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < a.c.N) y[n + i] = elem_of<E>(v[i]);
  }
}
// Scales (or biases: zeros where there are none) of channels n .. n+3
__device__ inline float4 channels4(const float* p, int n, int N) {
  if (!p) return make_float4(0.f, 0.f, 0.f, 0.f);
  return make_float4(p[min(n, N - 1)], p[min(n + 1, N - 1)], p[min(n + 2, N - 1)], p[min(n + 3, N - 1)]);
}
template <typename E>
__device__ inline bool wide_rows(const Q8Args& a) {
  return ((uintptr_t)a.y | (uintptr_t)(a.c.ldy * sizeof(E))) % (4 * sizeof(E)) == 0;
}

// Few tokens (up to 16 MB): the weights are read once, straight into the operands of the matrix instruction, and
// bound it.  A workgroup takes 16 channels; its four waves split K in turns of U slices of 64 bytes (two neighbouring
// slices are a line of memory) and add their sums up in LDS.  8 tokens x 2048 x 2048: 4.2 MB in 4.0 us, a trip to
// memory and the ends of a launch.
template <typename E, int MB>
__global__ __launch_bounds__(256) void q8_few_kernel(Q8Args a) {
  constexpr int U = MB == 1 ? 8 : 4;
  __shared__ intx4 sums[4][MB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int pad = q8_pad(a.c.K), slices = pad / 64, n0 = blockIdx.x * 16;
  const int8_t* w = a.w + (long long)min(n0 + (lane & 15), a.c.N - 1) * pad + (lane >> 4) * 16;
  const int8_t* x[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b)
    x[b] = a.q + (long long)min(16 * b + (lane & 15), a.c.M - 1) * pad + (lane >> 4) * 16;
  intx4 acc[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) acc[b] = intx4{};
  for (int s0 = wave * U; s0 < slices; s0 += 4 * U) {
    intx4 fw[U], fx[U][MB];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = 64 * min(s0 + u, slices - 1);
      fw[u] = *reinterpret_cast<const intx4*>(w + k);
#pragma unroll
      for (int b = 0; b < MB; ++b) fx[u][b] = *reinterpret_cast<const intx4*>(x[b] + k);
    }
    __builtin_amdgcn_sched_barrier(0);                 // (all of them in flight)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s0 + u >= slices) break;
#pragma unroll
      for (int b = 0; b < MB; ++b)
        acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u], fx[u][b], acc[b], 0, 0, 0);
    }
  }
#pragma unroll
  for (int b = 0; b < MB; ++b) sums[wave][b][lane] = acc[b];
  __syncthreads();
  const int n = n0 + 4 * (lane >> 4), m = 16 * wave + (lane & 15);
  if (wave >= MB || m >= a.c.M || n >= a.c.N) return;
  const float4 ws = channels4(a.w_scale, n, a.c.N), bias = channels4(a.bias, n, a.c.N);
  const intx4 sum = sums[0][wave][lane] + sums[1][wave][lane] + sums[2][wave][lane] + sums[3][wave][lane];
  put4<E>(a, (E*)a.y + (long long)m * a.c.ldy, n, sum, a.scale[m], ws, bias, wide_rows<E>(a));
}

// Up to 16 tokens of rows that a wave holds: one launch (8 tokens x 2048 x 2048: 7.8 us).  Every workgroup quantises
// all of them into LDS, from the L2 that they share, while its first weights are on their way.
constexpr int FUSED_LDS = 52 << 10, FUSED_WAVES = 8;
template <typename E>
__global__ __launch_bounds__(64 * FUSED_WAVES) void q8_fused_kernel(Q8Args a) {
  constexpr int U = 4;
  extern __shared__ intx4 dyn[];                       // [M][pad + 16] bytes: rows on different banks
  __shared__ intx4 sums[FUSED_WAVES][64];
  __shared__ float scales[16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int pad = q8_pad(a.c.K), slices = pad / 64, n0 = blockIdx.x * 16;
  const int8_t* w = a.w + (long long)min(n0 + (lane & 15), a.c.N - 1) * pad + (lane >> 4) * 16;
  char* xq = reinterpret_cast<char*>(dyn);
  const char* x = xq + min(lane & 15, a.c.M - 1) * (pad + 16) + (lane >> 4) * 16;
  intx4 fw[U], acc = {};
  auto load = [&](int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) fw[u] = *reinterpret_cast<const intx4*>(w + 64 * min(s0 + u, slices - 1));
  };
  load(wave * U);
  for (int r = wave; r < a.c.M; r += FUSED_WAVES) {
    QuantRow<E, 64, 8> row;
    row.load((const E*)a.x + (long long)r * a.c.ldx, a.c.K, lane);
    const float m = row.top();
    const bool finite = m < __builtin_inff();
    const float scale = quant_scale(finite ? m : 0.f);
    if (lane == 0) scales[r] = finite ? scale : __uint_as_float(0x7fc00000u);
    row.put(reinterpret_cast<int8_t*>(xq) + r * (pad + 16), pad, lane, finite, scale);
  }
  __syncthreads();
  for (int s0 = wave * U; s0 < slices; s0 += FUSED_WAVES * U) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s0 + u >= slices) break;
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(
          fw[u], *reinterpret_cast<const intx4*>(x + 64 * (s0 + u)), acc, 0, 0, 0);
    }
    if (s0 + FUSED_WAVES * U < slices) load(s0 + FUSED_WAVES * U);
  }
  sums[wave][lane] = acc;
  __syncthreads();
  const int n = n0 + 4 * (lane >> 4), m = lane & 15;
  if (wave != 0 || m >= a.c.M || n >= a.c.N) return;
  const float4 ws = channels4(a.w_scale, n, a.c.N), bias = channels4(a.bias, n, a.c.N);
  intx4 sum = sums[0][lane];
#pragma unroll
  for (int i = 1; i < FUSED_WAVES; ++i) sum += sums[i][lane];
  put4<E>(a, (E*)a.y + (long long)m * a.c.ldy, n, sum, scales[m], ws, bias, wide_rows<E>(a));
}

// A tile of TM tokens x TN channels: four waves, each half of either.  Slices of 128 bytes of K go through one of two
// LDS buffers; a row's 16-byte pieces lie in the order piece ^ (row & 7), which spreads a fragment's rows over the
// banks.  While the matrix instructions of slice s run, slice s + 1 goes from registers to the other buffer and slice
// s + 2 is loaded; the fragments of a quarter of a slice are read during the instructions of the quarter before, the
// first of the next slice behind the barrier in front of the last quarter.  32768 x 2048 x 2048: 186-200 us over
// traces, 1.4-1.5 POP/s; 135 us of them are the loop over K (2.0 POP/s; a library's 8192^3 reaches 2.1), the rest
// results, which a workgroup alone on its CU (all registers are taken) does not overlap with anything.
template <typename E, int TM, int TN>
__global__ __launch_bounds__(256) void q8_tile_kernel(Q8Args a, int tiles_m, int tiles_n) {
  constexpr int WM = TM / 64, WN = TN / 64;              // 32 x 32 blocks of a wave
  constexpr int LX = TM / 32, LW = TN / 32;              // pieces of a slice that a thread moves
  __shared__ intx4 lds[2][(TM + TN) * 8];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int pad = q8_pad(a.c.K), slices = pad / 128;
  // tiles of neighbouring tokens on one XCD (workgroups go to the eight in turn), channels first
  const int tiles = tiles_m * tiles_n, per = (tiles + 7) / 8;
  int tile = blockIdx.x;
  if (tiles % 8 == 0) tile = (tile & 7) * per + (tile >> 3);
  const int tm = tile / tiles_n, m0 = tm * TM, n0 = (tile - tm * tiles_n) * TN;
  const int wm = (wave & 1) * (TM / 2), wn = (wave >> 1) * (TN / 2);
  // what the thread moves: piece tid % 8 of rows tid / 8 + 32 i (rows that do not exist: the last one)
  const int8_t *gx = a.q + (long long)m0 * pad, *gw = a.w + (long long)n0 * pad;
  unsigned ox[LX], ow[LW];
#pragma unroll
  for (int i = 0; i < LX; ++i) ox[i] = min(tid / 8 + 32 * i, a.c.M - 1 - m0) * pad + (tid & 7) * 16;
#pragma unroll
  for (int i = 0; i < LW; ++i) ow[i] = min(tid / 8 + 32 * i, a.c.N - 1 - n0) * pad + (tid & 7) * 16;
  const int to = (tid & ~7) | ((tid & 7) ^ ((tid >> 3) & 7));
  intx4 rx[LX], rw[LW];
  auto load = [&](int s) {
#pragma unroll
    for (int i = 0; i < LX; ++i) rx[i] = *reinterpret_cast<const intx4*>(gx + s * 128 + ox[i]);
#pragma unroll
    for (int i = 0; i < LW; ++i) rw[i] = *reinterpret_cast<const intx4*>(gw + s * 128 + ow[i]);
  };
  auto store = [&](int buf) {
#pragma unroll
    for (int i = 0; i < LX; ++i) lds[buf][to + 256 * i] = rx[i];
#pragma unroll
    for (int i = 0; i < LW; ++i) lds[buf][TM * 8 + to + 256 * i] = rw[i];
  };
  intx4 fx[2][WM], fw[2][WN];
  auto read = [&](int buf, int kk, int set) {
    const int piece = (kk * 2 + (lane >> 5)) ^ (lane & 7);
#pragma unroll
    for (int j = 0; j < WM; ++j) fx[set][j] = lds[buf][(wm + 32 * j + (lane & 31)) * 8 + piece];
#pragma unroll
    for (int i = 0; i < WN; ++i) fw[set][i] = lds[buf][(TM + wn + 32 * i + (lane & 31)) * 8 + piece];
  };
  intx16 acc[WN][WM];
#pragma unroll
  for (int i = 0; i < WN; ++i)
#pragma unroll
    for (int j = 0; j < WM; ++j) acc[i][j] = intx16{};
  load(0);
  store(0);
  if (slices > 1) load(1);
  __syncthreads();
  read(0, 0, 0);
  for (int s = 0; s < slices; ++s) {
    const int buf = s & 1;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      if (kk == 0 && s + 1 < slices) {
        store(buf ^ 1);
        if (s + 2 < slices) load(s + 2);
      }
      if (kk < 3) {
        read(buf, kk + 1, (kk + 1) & 1);
      } else if (s + 1 < slices) {
        // every wave has read this buffer and written the other one
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        read(buf ^ 1, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < WN; ++i)
#pragma unroll
        for (int j = 0; j < WM; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[kk & 1][i], fx[kk & 1][j], acc[i][j], 0, 0, 0);
    }
  }
  // Scales and biases of the tile's channels through LDS; the results too, 32 tokens of a wave at a time, so that
  // rows are stored whole (from the lanes' own places a store would write 16 bytes each of 32 rows).
  __syncthreads();
  constexpr int CH = TN / 2, ROW = CH * (int)sizeof(E) + 16, PIECES = CH * (int)sizeof(E) / 16;
  constexpr int PER = 16 / (int)sizeof(E);
  char* mine = reinterpret_cast<char*>(lds) + wave * 32 * ROW;
  float4 *ws = reinterpret_cast<float4*>(reinterpret_cast<char*>(lds) + 4 * 32 * ROW), *bias = ws + TN / 4;
  static_assert(4 * 32 * ROW + TN * 8 <= (int)sizeof(lds), "the tile's results and scales fit its buffers");
  if (tid < TN / 4) {
    ws[tid] = channels4(a.w_scale, n0 + 4 * tid, a.c.N);
    bias[tid] = channels4(a.bias, n0 + 4 * tid, a.c.N);
  }
  float sm[WM];
#pragma unroll
  for (int j = 0; j < WM; ++j) sm[j] = a.scale[min(m0 + wm + 32 * j + (lane & 31), a.c.M - 1)];
  __syncthreads();
  const bool wide = (((uintptr_t)a.y | (uintptr_t)(a.c.ldy * (long long)sizeof(E))) & 15) == 0;
  auto own_lanes = [&]() {                                   // what the wave's own lanes wrote and read
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
  };
#pragma unroll
  for (int j = 0; j < WM; ++j) {
#pragma unroll
    for (int i = 0; i < WN; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = 32 * i + 8 * e + 4 * (lane >> 5);      // the wave's channel
        const float4 w4 = ws[(wn + c) / 4], b4 = bias[(wn + c) / 4];
        const float v0 = (float)acc[i][j][4 * e] * w4.x * sm[j] + b4.x;
        const float v1 = (float)acc[i][j][4 * e + 1] * w4.y * sm[j] + b4.y;
        const float v2 = (float)acc[i][j][4 * e + 2] * w4.z * sm[j] + b4.z;
        const float v3 = (float)acc[i][j][4 * e + 3] * w4.w * sm[j] + b4.w;
        char* to_row = mine + (lane & 31) * ROW + c * (int)sizeof(E);
        if constexpr (sizeof(E) == 4) *reinterpret_cast<float4*>(to_row) = make_float4(v0, v1, v2, v3);
        else *reinterpret_cast<uint2*>(to_row) = make_uint2(pack2<E>(v0, v1), pack2<E>(v2, v3));
      }
    own_lanes();
#pragma unroll
    for (int p = 0; p < PIECES / 2; ++p) {                   // 32 rows of PIECES pieces, 64 at a time
      const int k = p * 64 + lane, r = k / PIECES, q = k % PIECES;
      const int m = m0 + wm + 32 * j + r, n = n0 + wn + q * PER;
      const uintx4 v = *reinterpret_cast<const uintx4*>(mine + r * ROW + q * 16);
      if (m >= a.c.M || n >= a.c.N) continue;
      E* y = (E*)a.y + (long long)m * a.c.ldy + n;
      if (wide && n + PER <= a.c.N) {
        store_as(reinterpret_cast<uintx4*>(y), v, a.past);
      } else {
        E el[PER];
        __builtin_memcpy(el, &v, 16);
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (n + i < a.c.N) y[i] = el[i];
      }
    }
    own_lanes();
  }
}

template <typename E, int TM, int TN>
static void tile_start(const Q8Args& a, hipStream_t s) {
  const int tm = (int)(((long long)a.c.M + TM - 1) / TM), tn = (int)(((long long)a.c.N + TN - 1) / TN);
  hipLaunchKernelGGL((q8_tile_kernel<E, TM, TN>), dim3((unsigned)tm * (unsigned)tn), dim3(256), 0, s, a, tm, tn);
}
// Which product.  Measured with quantisation, K = 2048, bf16, us on the GPU:
//  - few tokens : tiles of 64 x 64.  17 x 2048 7.7 : 11.8, 64 x 2048 10.2 : 12.0, 64 x 8192 15.2 : 12.3 (every
//    workgroup of the former reads all tokens from the L2, and there are N / 16 of them), 48 x 8192 (K = 4096) 21.5 :
//    19.4;
//  - tiles of 64 : 128 : 256.  1024 x 2048 17 : 21 : 44, 2048 x 2048 26 : 25 : 48, 4096 x 2048 47 : 37 : 53, 6144 x
//    2048 69 : 52 : 57, 8192 x 2048 85 : 68 : 63, 1024 x 8192 49 : 33 : 48.  That is 20 us per 1024 tiles of 64 (four
//    of them share a CU), 27 per 512 of 128 (two) and 50 per round of 256 of 256 (one), 7 and 19 at least.
static double tiles_of(const q8_cfg& c, long long t) {
  return (double)((c.M + t - 1) / t) * (double)((c.N + t - 1) / t);
}
static int product_tile(const q8_cfg& c) {                   // 0: few tokens
  const long long blocks = ((long long)c.M + 15) / 16;
  if (blocks == 1 || (blocks <= 4 && blocks * c.N <= 16384)) return 0;
  const double c64 = std::max(7.0, tiles_of(c, 64) / 1024 * 20), c128 = std::max(19.0, tiles_of(c, 128) / 512 * 27);
  const double c256 = std::ceil(tiles_of(c, 256) / 256) * 50;
  return c256 <= c128 && c256 <= c64 ? 256 : c128 <= c64 ? 128 : 64;
}
static bool product_launchable(const q8_cfg& c) {
  const int tile = product_tile(c);
  return launchable(tile ? (long long)tiles_of(c, tile) : ((long long)c.N + 15) / 16, 256);
}
template <typename E>
static void q8_start(const Q8Args& a, hipStream_t s) {
  const int tile = product_tile(a.c);
  if (tile == 0) {
    const unsigned groups = ((unsigned)a.c.N + 15) / 16;
    switch ((a.c.M + 15) / 16) {
      case 1: hipLaunchKernelGGL((q8_few_kernel<E, 1>), dim3(groups), dim3(256), 0, s, a); break;
      case 2: hipLaunchKernelGGL((q8_few_kernel<E, 2>), dim3(groups), dim3(256), 0, s, a); break;
      case 3: hipLaunchKernelGGL((q8_few_kernel<E, 3>), dim3(groups), dim3(256), 0, s, a); break;
      default: hipLaunchKernelGGL((q8_few_kernel<E, 4>), dim3(groups), dim3(256), 0, s, a);
    }
  } else if (tile == 256) {
    tile_start<E, 256, 256>(a, s);
  } else if (tile == 128) {
    tile_start<E, 128, 128>(a, s);
  } else {
    tile_start<E, 64, 64>(a, s);
  }
}
// LDS of the product that quantises the tokens itself, 0 where that has a launch of its own.  One launch : two, K =
// 2048, us on the GPU: 1 x 2048 6.3 : 6.3, 8 x 2048 7.4 : 6.9, 16 x 2048 10.9 : 7.2, 1 x 8192 (K = 4096) 10.5 : 10.9,
// 8 x 8192 (K = 4096) 17.1 : 12.4; the second launch takes 2.5 us of the host.  So: as long as the workgroups
// together quantise at most 1024 rows.
static size_t fused_lds(const Q8Args& a) {
  const int pad = q8_pad(a.c.K), held = 8 * 64 * (a.c.dtype == MGRIT_F32 ? 4 : 8);
  const size_t need = (size_t)a.c.M * (pad + 16);
  const long long rows = a.c.M * (((long long)a.c.N + 15) / 16);
  return a.c.M <= 16 && rows <= 1024 && pad <= held && need <= FUSED_LDS ? need : 0;
}
hipError_t launch_q8_linear(const Q8Args& a, hipStream_t s) {
  if (const size_t lds = fused_lds(a)) {
    const dim3 g((unsigned)(a.c.N + 15) / 16), t(64 * FUSED_WAVES);
    if (a.c.dtype == MGRIT_F32) hipLaunchKernelGGL(q8_fused_kernel<float>, g, t, lds, s, a);
    else if (a.c.dtype == MGRIT_BF16) hipLaunchKernelGGL(q8_fused_kernel<Bf16>, g, t, lds, s, a);
    else hipLaunchKernelGGL(q8_fused_kernel<F16>, g, t, lds, s, a);
    return hipGetLastError();
  }
  if (!product_launchable(a.c)) return TOO_LARGE;
  const hipError_t e = launch_q8_quantize(a, s);
  if (e != hipSuccess) return e;
  if (a.c.dtype == MGRIT_F32) q8_start<float>(a, s);
  else if (a.c.dtype == MGRIT_BF16) q8_start<Bf16>(a, s);
  else q8_start<F16>(a, s);
  return hipGetLastError();
}

}  // namespace mg
