// Embedding of tokens and the gradient of its table (include/mgrit_tokens.h).
//
// The gradient sorts: a workgroup owns a range of the vocabulary and looks through all tokens of the call twice.  The
// first time it counts those below its range, which is where its own will stand, and, per wave, those of each of its
// own tokens; the second time every wave puts the places of its part behind those of the waves before it.  Places are
// therefore in order of token and place, whatever runs first.  The same workgroup clears the rows that no token names.
// Then a wave adds up a block of sorted places, however they fall into runs of one token, so that a token that is half
// of all is no longer than many; sums of runs that cross blocks meet in a third launch.
#include "elem.h"
#include "tokens.h"

namespace mg {

typedef unsigned Words __attribute__((ext_vector_type(4)));

// What a lane has of a row: 16 bytes, or one element where rows are not aligned to them.
template <typename E, bool WIDE>
struct Piece {
  static constexpr int n = WIDE ? 16 / (int)sizeof(E) : 1;
  float v[n];
  __device__ inline void load(const E* p) {
    if constexpr (WIDE) {
      const Words w = *reinterpret_cast<const Words*>(p);
#pragma unroll
      for (int k = 0; k < n; ++k) v[k] = word_elem<E>(w[k / ELEMS_PER_WORD<E>], k % ELEMS_PER_WORD<E>);
    } else {
      v[0] = elem_f32(*p);
    }
  }
  __device__ inline void store(E* p, float scale) const {
    if constexpr (WIDE) {
      Words w;
#pragma unroll
      for (int k = 0; k < n; k += ELEMS_PER_WORD<E>) {
        if constexpr (sizeof(E) == 4) w[k] = __float_as_uint(v[k] * scale);
        else w[k / 2] = pack2<E>(v[k] * scale, v[k + 1] * scale);
      }
      *reinterpret_cast<Words*>(p) = w;
    } else {
      *p = elem_of<E>(v[0] * scale);
    }
  }
};

template <typename E, bool WIDE>
__global__ __launch_bounds__(256) void embed_lookup_kernel(EmbedArgs a) {
  using P = Piece<E, WIDE>;
  const int pieces = (a.c.D + P::n - 1) / P::n;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, row = i / pieces;
  if (row >= a.c.N) return;
  const int col = (int)(i - row * pieces) * P::n;
  const long long tok = a.tokens[row];
  P v;
  if (tok >= 0 && tok < a.c.V) {
    v.load((const E*)a.in + tok * a.c.ld_table + col);
  } else {
#pragma unroll
    for (int k = 0; k < P::n; ++k) v.v[k] = tok < 0 ? 0.f : __uint_as_float(0x7fc00000u);
  }
  v.store((E*)a.out + row * a.c.ld_out + col, tok < 0 ? 1.f : a.c.scale);
}

// ---- gradient: places of the tokens of a range, in order; rows without a token
constexpr int PLAN_WAVES = 16, PLAN_THREADS = 64 * PLAN_WAVES;
template <typename E, bool WIDE, int RANGE>
__global__ __launch_bounds__(PLAN_THREADS) void embed_plan_kernel(EmbedArgs a) {
  __shared__ int count[PLAN_WAVES][RANGE];
  __shared__ int start[RANGE];
  __shared__ int part[PLAN_WAVES], below;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lo = blockIdx.x * RANGE, hi = min(lo + RANGE, a.c.V);
  for (int i = tid; i < PLAN_WAVES * RANGE; i += PLAN_THREADS) (&count[0][0])[i] = 0;
  if (tid == 0) below = 0;
  __syncthreads();
  const int per = ((a.c.N + PLAN_THREADS - 1) / PLAN_THREADS) * 64;      // places of a wave
  const int begin = (int)min((long long)a.c.N, (long long)wave * per), end = (int)min((long long)a.c.N, (long long)begin + per);
  int less = 0;
  for (int i0 = begin; i0 < end; i0 += 256) {
    long long k[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) k[j] = i0 + 64 * j + lane < end ? a.tokens[i0 + 64 * j + lane] : -1;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      less += k[j] >= 0 && k[j] < lo;
      if (k[j] >= lo && k[j] < hi) atomicAdd(&count[wave][(int)k[j] - lo], 1);
    }
  }
  atomicAdd(&below, less);
  __syncthreads();
  // where each token's places start: behind those of the smaller ones; then where each wave's do
  constexpr int PER = (RANGE + PLAN_THREADS - 1) / PLAN_THREADS;
  int own[PER], sum = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int r = tid * PER + j;
    own[j] = 0;
    if (r < RANGE)
      for (int w = 0; w < PLAN_WAVES; ++w) own[j] += count[w][r];
    sum += own[j];
  }
  int upto = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(upto, o, 64);
    if (lane >= o) upto += v;
  }
  if (lane == 63) part[wave] = upto;
  __syncthreads();
  int at = below + upto - sum;
  for (int w = 0; w < wave; ++w) at += part[w];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int r = tid * PER + j;
    if (r >= RANGE) break;
    start[r] = own[j];                               // (how many, from here on)
    int pos = at;
    for (int w = 0; w < PLAN_WAVES; ++w) {
      const int n = count[w][r];
      count[w][r] = pos;
      pos += n;
    }
    at = pos;
  }
  if (blockIdx.x == gridDim.x - 1 && tid == PLAN_THREADS - 1) *a.total = at;
  __syncthreads();
  for (int i0 = begin; i0 < end; i0 += 64) {
    const long long k = i0 + lane < end ? a.tokens[i0 + lane] : -1;
    const bool mine = k >= lo && k < hi;
    const int r = (int)k - lo;
    unsigned long long left = __ballot(mine);
    while (left) {                                   // (each pass takes one token's lanes)
      const int key = __builtin_amdgcn_readlane(r, __builtin_ctzll(left));
      const bool same = mine && r == key;
      const unsigned long long who = __ballot(same);
      const int pos = count[wave][key];
      if (same) {
        const int to = pos + __popcll(who & ((1ull << lane) - 1));
        a.place[to] = i0 + lane;
        a.token[to] = (int)k;
      }
      if (lane == 0) count[wave][key] = pos + __popcll(who);
      left &= ~who;
    }
  }
  using P = Piece<E, WIDE>;
  const int pieces = (a.c.D + P::n - 1) / P::n;
  P zero;
#pragma unroll
  for (int k = 0; k < P::n; ++k) zero.v[k] = 0.f;
  const long long all = (long long)(hi - lo) * pieces;
  for (long long i = tid; i < all; i += PLAN_THREADS) {
    const int r = (int)(i / pieces);
    if (start[r] == 0) zero.store((E*)a.out + (lo + r) * a.c.ld_table + (i - (long long)r * pieces) * P::n, 1.f);
  }
}

// ---- gradient: sums of a block of sorted places, in one wave per 64 pieces of the width
template <typename E, bool WIDE>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs a) {
  using P = Piece<E, WIDE>;
  constexpr int AHEAD = 8;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int pieces = (a.c.D + P::n - 1) / P::n, across = (pieces + 63) / 64;
  const long long item = (long long)blockIdx.x * 4 + wave;
  const int block = (int)(item / across), piece = (int)(item - (long long)block * across) * 64 + lane;
  const int M = *a.total;
  const int first = block * EMBED_RUN;
  if (first >= M) return;
  const int n = min(EMBED_RUN, M - first), col = min(piece, pieces - 1) * P::n;
  const bool has = piece < pieces;
  // a lane for each place: its token, and whether its run ends there
  const int i = first + min(lane, n - 1);
  const int tok = a.token[i], place = a.place[i];
  const bool ends = lane < n && (i + 1 >= M || a.token[i + 1] != tok);
  const unsigned long long breaks = __ballot(ends);
  const bool before = first > 0 && a.token[first - 1] == __builtin_amdgcn_readfirstlane(tok);
  P sum;
#pragma unroll
  for (int k = 0; k < P::n; ++k) sum.v[k] = 0.f;
  bool open = before;                                // the run began in an earlier block
  auto partial = [&](int slot) {
    float* p = a.part + (2LL * block + slot) * a.c.D + col;
#pragma unroll
    for (int k = 0; k < P::n; ++k) p[k] = sum.v[k];
  };
  const E* in = (const E*)a.in + col;
  for (int j0 = 0; j0 < n; j0 += AHEAD) {
    P v[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
      v[j].load(in + (long long)__builtin_amdgcn_readlane(place, min(j0 + j, n - 1)) * a.c.ld_out);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (j0 + j >= n) break;
#pragma unroll
      for (int k = 0; k < P::n; ++k) sum.v[k] += v[j].v[k];
      if (breaks >> (j0 + j) & 1) {
        if (has) {
          if (open) partial(0);
          else sum.store((E*)a.out + (long long)__builtin_amdgcn_readlane(tok, j0 + j) * a.c.ld_table + col, a.c.scale);
        }
        open = false;
#pragma unroll
        for (int k = 0; k < P::n; ++k) sum.v[k] = 0.f;
      }
    }
  }
  if (!(breaks >> (n - 1) & 1) && has) partial(open ? 0 : 1);
}

// ---- gradient: runs that cross blocks, at the block where they begin; the blocks behind it in four parts
template <typename E, bool WIDE>
__global__ __launch_bounds__(256) void embed_join_kernel(EmbedArgs a) {
  using P = Piece<E, WIDE>;
  __shared__ float part[4][64][P::n];
  __shared__ int found;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int pieces = (a.c.D + P::n - 1) / P::n, across = (pieces + 63) / 64;
  const int block = blockIdx.x / across, piece = (blockIdx.x - block * across) * 64 + lane;
  const int M = *a.total;
  const long long next = (long long)(block + 1) * EMBED_RUN;
  if (next >= M) return;
  const int first = block * EMBED_RUN, tok = a.token[next - 1];
  if (a.token[next] != tok) return;
  if (a.token[first] == tok && first > 0 && a.token[first - 1] == tok) return;
  // blocks behind this one that begin with the token
  const int blocks = (int)((M + EMBED_RUN - 1LL) / EMBED_RUN);
  int end = blocks;
  for (int b0 = block + 1; b0 < blocks; b0 += 256) {
    if (threadIdx.x == 0) found = blocks;
    __syncthreads();
    const int b = b0 + threadIdx.x;
    if (b < blocks && a.token[(long long)b * EMBED_RUN] != tok) atomicMin(&found, b);
    __syncthreads();
    end = found;
    __syncthreads();
    if (end < blocks) break;
  }
  const int n = end - (block + 1), per = (n + 3) / 4;
  const int from = block + 1 + wave * per, to = min(from + per, end);
  const int col = min(piece, pieces - 1) * P::n;
  float sum[P::n];
#pragma unroll
  for (int k = 0; k < P::n; ++k) sum[k] = wave == 0 ? a.part[(2LL * block + 1) * a.c.D + col + k] : 0.f;
  for (int b = from; b < to; ++b)
#pragma unroll
    for (int k = 0; k < P::n; ++k) sum[k] += a.part[2LL * b * a.c.D + col + k];
#pragma unroll
  for (int k = 0; k < P::n; ++k) part[wave][lane][k] = sum[k];
  __syncthreads();
  if (wave || piece >= pieces) return;
  P v;
#pragma unroll
  for (int k = 0; k < P::n; ++k)
    v.v[k] = (part[0][lane][k] + part[1][lane][k]) + (part[2][lane][k] + part[3][lane][k]);
  v.store((E*)a.out + (long long)tok * a.c.ld_table + col, a.c.scale);
}

// ---- launches
static bool wide_rows(const void* p, long long ld, int D, int size) {
  return (uintptr_t)p % 16 == 0 && ld * size % 16 == 0 && (long long)D * size % 16 == 0;
}
static size_t embed_piece(size_t n) { return (n + 255) / 256 * 256; }
size_t embed_workspace(const embed_cfg& c) {
  const size_t N = (size_t)c.N, blocks = (N + EMBED_RUN - 1) / EMBED_RUN;
  return 256 + 2 * embed_piece(4 * N) + 8 * blocks * c.D;
}
template <typename E, bool WIDE>
static hipError_t embed_lookup_start(const EmbedArgs& a, hipStream_t s) {
  const long long pieces = (a.c.D + Piece<E, WIDE>::n - 1) / Piece<E, WIDE>::n, n = (a.c.N * pieces + 255) / 256;
  if (!launchable(n, 256)) return TOO_LARGE;
  hipLaunchKernelGGL((embed_lookup_kernel<E, WIDE>), dim3((unsigned)n), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename E, bool WIDE>
static hipError_t embed_backward_start(const EmbedArgs& a, hipStream_t s) {
  const long long pieces = (a.c.D + Piece<E, WIDE>::n - 1) / Piece<E, WIDE>::n, across = (pieces + 63) / 64;
  const long long items = ((a.c.N + EMBED_RUN - 1LL) / EMBED_RUN) * across;
  if (!launchable(items, 256)) return TOO_LARGE;
  // ranges that leave a few hundred workgroups
  const int V = a.c.V;
  const dim3 t(PLAN_THREADS);
  if (V <= 256 * 128) hipLaunchKernelGGL((embed_plan_kernel<E, WIDE, 128>), dim3((V + 127) / 128), t, 0, s, a);
  else if (V <= 256 * 512) hipLaunchKernelGGL((embed_plan_kernel<E, WIDE, 512>), dim3((V + 511) / 512), t, 0, s, a);
  else hipLaunchKernelGGL((embed_plan_kernel<E, WIDE, 2048>), dim3((V + 2047) / 2048), t, 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((embed_sum_kernel<E, WIDE>), dim3((unsigned)((items + 3) / 4)), dim3(256), 0, s, a);
  if ((e = hipGetLastError()) != hipSuccess || a.c.N <= EMBED_RUN) return e;
  hipLaunchKernelGGL((embed_join_kernel<E, WIDE>), dim3((unsigned)items), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename E>
static hipError_t embed_start(const EmbedArgs& a, bool backward, hipStream_t s) {
  const bool wide = wide_rows(a.in, backward ? a.c.ld_out : a.c.ld_table, a.c.D, sizeof(E)) &&
                    wide_rows(a.out, backward ? a.c.ld_table : a.c.ld_out, a.c.D, sizeof(E));
  if (backward) return wide ? embed_backward_start<E, true>(a, s) : embed_backward_start<E, false>(a, s);
  return wide ? embed_lookup_start<E, true>(a, s) : embed_lookup_start<E, false>(a, s);
}
static hipError_t embed_typed(const EmbedArgs& a, bool backward, hipStream_t s) {
  if (a.c.dtype == MGRIT_F32) return embed_start<float>(a, backward, s);
  if (a.c.dtype == MGRIT_BF16) return embed_start<Bf16>(a, backward, s);
  return embed_start<F16>(a, backward, s);
}
hipError_t launch_embed_lookup(const EmbedArgs& a, hipStream_t s) { return embed_typed(a, false, s); }
hipError_t launch_embed_backward(EmbedArgs a, char* ws, hipStream_t s) {
  a.total = (int*)ws;
  a.place = (int*)(ws + 256);
  a.token = (int*)(ws + 256 + embed_piece(4 * (size_t)a.c.N));
  a.part = (float*)(ws + 256 + 2 * embed_piece(4 * (size_t)a.c.N));
  return embed_typed(a, true, s);
}

}  // namespace mg
