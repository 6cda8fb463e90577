// Embedding of tokens and the gradient of its table (include/mgrit_tokens.h).
//
// The gradient sorts: a workgroup owns a range of the vocabulary and looks through all tokens of the call twice.  The first
// time it counts those below its range, which is where its own will stand, and, per wave, those of each of its own tokens;
// the second time every wave puts the places of its part behind those of the waves before it.  (Of many tokens several
// workgroups of the range each place a part, having counted all.)  Places are therefore in order of token and place,
// whatever runs first.  Other workgroups of the launch, which waits for its loads most of the time, clear the table
// meanwhile. Then a wave adds up a block of 8 or 32 sorted places, however they fall into runs of one token; sums of runs
// that cross blocks meet in a third launch, at the block where the run begins.  A run of many blocks is the work of a
// workgroup there, 64 pieces of the width wide, so that a token that is most of all takes longer than many do: gradients of
// width 1024 in bf16, us, tokens spread / half of them one / all one, of 32768: 16384 33 / 41 / 49, 65536 71 / 102 / 147, 2^20
// 869 / 1729 / 2747; of 1000: 65536 52 / 93, 2^20 639 / 1619; of 2, one of them 80 %: 65536 123, 2^20 2282.
//
// 16384 tokens, most of them few, of 32768 x 1024 bf16: sort and clearing (64 MB) 14 us, sums (34 MB read) 12, join 6; lookup
// 67 MB in 10.8 us.  The sort takes 9.6 us of it, most of them waiting for tokens that all its workgroups look at.
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

// ---- gradient: places of the tokens of a range, in order; the table cleared
constexpr int PLAN_WAVES = 16, PLAN_THREADS = 64 * PLAN_WAVES;
// Tokens that a workgroup places at least, and ranges times parts at most: a part spares its workgroup the second look, but all
// parts count all tokens, which has to be at once.  Sort in us, one part / parts of 4096 / of 4096 with no more than 256
// workgroups, in ranges of 128: 16384 tokens of 1000 15.1 / 8.8 / 8.7, of 32768 15.0 / 20.2 / 14.9; 65536 of 1000 48.8 / 17.5 /
// 17.4, of 32768 45 / 141 / 45.4; 262144 of 1000 183 / 55 / 52, of 32768 158 / 494 / 158.
constexpr int PLAN_PART = 4096, PLAN_GROUPS = 256, PLAN_PARTS = 32;
// Rows CLEAR_ROWS group .. of the table, a wave a row.
constexpr int CLEAR_ROWS = 64;
template <typename E, bool WIDE>
__device__ inline void clear_rows(const EmbedArgs& a, int group) {
  using P = Piece<E, WIDE>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int pieces = (a.c.D + P::n - 1) / P::n;
  P zero;
#pragma unroll
  for (int k = 0; k < P::n; ++k) zero.v[k] = 0.f;
  for (int r = CLEAR_ROWS * group + wave; r < min(CLEAR_ROWS * (group + 1), a.c.V); r += PLAN_WAVES) {
    E* out = (E*)a.out + r * a.c.ld_table;
    for (int i = lane; i < pieces; i += 64) zero.store(out + (long long)i * P::n, 1.f);
  }
}
template <typename E, bool WIDE, int RANGE>
__global__ __launch_bounds__(PLAN_THREADS) void embed_plan_kernel(EmbedArgs a, int ranges, int parts) {
  if ((int)blockIdx.x >= ranges * parts) {
    clear_rows<E, WIDE>(a, (int)blockIdx.x - ranges * parts);
    return;
  }
  __shared__ int count[PLAN_WAVES][RANGE];
  __shared__ int other[2][RANGE];                    // tokens before and behind the workgroup's part
  __shared__ int part[PLAN_WAVES], below;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int range = blockIdx.x / parts, lo = range * RANGE, hi = min(lo + RANGE, a.c.V);
  for (int i = tid; i < PLAN_WAVES * RANGE; i += PLAN_THREADS) (&count[0][0])[i] = 0;
  for (int i = tid; i < 2 * RANGE; i += PLAN_THREADS) (&other[0][0])[i] = 0;
  if (tid == 0) below = 0;
  __syncthreads();
  const int N = a.c.N, per = (N + parts * PLAN_THREADS - 1) / (parts * PLAN_THREADS) * 64;      // places of a wave
  const auto place_of = [&](int i) { return (int)min((long long)N, (long long)i * per); };
  const int first = (blockIdx.x - range * parts) * PLAN_WAVES;
  const int begin = place_of(first + wave), end = place_of(first + wave + 1);
  // (eight tokens a lane at a time: what the loads wait for is most of the time)
  auto load = [&](int i0, int to, long long (&k)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) k[j] = i0 + 64 * j + lane < to ? a.tokens[i0 + 64 * j + lane] : -1;
  };
  int less = 0;
  auto look = [&](int from, int to, int step, int* counts) {
    for (int i0 = from; i0 < to; i0 += step) {
      long long k[8];
      load(i0, to, k);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        less += k[j] >= 0 && k[j] < lo;
        if (k[j] >= lo && k[j] < hi) atomicAdd(&counts[(int)k[j] - lo], 1);
      }
    }
  };
  look(begin, end, 512, count[wave]);
  const int before = place_of(first), behind = place_of(first + PLAN_WAVES);
  look(wave * 512, before, 512 * PLAN_WAVES, other[0]);
  look(behind + wave * 512, N, 512 * PLAN_WAVES, other[1]);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) less += __shfl_xor(less, o, 64);
  if (lane == 0) atomicAdd(&below, less);
  __syncthreads();
  // where each token's places start: behind those of the smaller ones; then where each wave's do
  constexpr int PER = (RANGE + PLAN_THREADS - 1) / PLAN_THREADS;
  int own[PER], sum = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int r = tid * PER + j;
    own[j] = 0;
    if (r < RANGE) {
      own[j] = other[0][r] + other[1][r];
      for (int w = 0; w < PLAN_WAVES; ++w) own[j] += count[w][r];
    }
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
    int pos = at + other[0][r];
    for (int w = 0; w < PLAN_WAVES; ++w) {
      const int n = count[w][r];
      count[w][r] = pos;
      pos += n;
    }
    at += own[j];
  }
  if (range == ranges - 1 && first == 0 && tid == PLAN_THREADS - 1) *a.total = at;
  __syncthreads();
  for (int i0 = begin; i0 < end; i0 += 512) {
    long long k[8];
    load(i0, end, k);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool mine = k[j] >= lo && k[j] < hi;
      const unsigned long long some = __ballot(mine);
      if (!some) continue;
      // the lanes with the same token, bit by bit
      const int r = mine ? (int)k[j] - lo : 0;
      unsigned who[2] = {(unsigned)some, (unsigned)(some >> 32)};
#pragma unroll
      for (int bit = 0; 1 << bit < RANGE; ++bit) {
        const unsigned long long set = __ballot(r >> bit & 1);
        const unsigned without = (r >> bit & 1) - 1;   // all bits where the lane's is 0
        who[0] &= (unsigned)set ^ without;
        who[1] &= (unsigned)(set >> 32) ^ without;
      }
      if (mine) {
        const int before = __builtin_amdgcn_mbcnt_hi(who[1], __builtin_amdgcn_mbcnt_lo(who[0], 0));
        const int pos = count[wave][r], to = pos + before;
        a.place[to] = i0 + 64 * j + lane;
        a.token[to] = (int)k[j];
        if (before == 0) count[wave][r] = pos + __popc(who[0]) + __popc(who[1]);
      }
      // (what one lane has written, all lanes of the wave read in the next round: LDS serves a wave in order, and nothing
      // has to wait for the places to be stored)
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
  }
}

// ---- gradient: sums of a block of RUN sorted places, in one wave per 64 pieces of the width, up to 16 rows under way (8 of 32:
// 12.6 us)
template <typename E, bool WIDE, int RUN>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs a) {
  using P = Piece<E, WIDE>;
  constexpr int AHEAD = RUN < 16 ? RUN : 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int pieces = (a.c.D + P::n - 1) / P::n, across = (pieces + 63) / 64;
  const long long item = (long long)blockIdx.x * 4 + wave;
  const int block = (int)(item / across), piece = (int)(item - (long long)block * across) * 64 + lane;
  const int M = *a.total;
  const int first = block * RUN;
  if (first >= M) return;
  const int n = min(RUN, M - first), col = min(piece, pieces - 1) * P::n;
  const bool has = piece < pieces;
  // a lane for each place: its token, and whether its run ends there
  const int i = first + min(lane, n - 1);
  const int tok = a.token[i], place = a.place[i];
  const bool ends = lane < n && (i + 1 >= M || a.token[i + 1] != tok);
  const unsigned long long breaks = __ballot(ends);
  const bool before = first > 0 && a.token[first - 1] == __builtin_amdgcn_readfirstlane(tok);
  // for the join: the token of a run that begins here and goes on
  const int tail = __builtin_amdgcn_readlane(tok, n - 1);
  const bool goes_on = !(breaks >> (n - 1) & 1);
  if (piece == 0)
    a.crosses[block] = goes_on && !(before && tail == __builtin_amdgcn_readfirstlane(tok)) ? tail : -1;
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
  if (goes_on && has) partial(open ? 0 : 1);
}

// ---- gradient: runs that cross blocks, at the block where they begin; the blocks behind it in four parts
constexpr int JOIN_WAVES = 4;
template <typename E, bool WIDE>
__global__ __launch_bounds__(64 * JOIN_WAVES) void embed_join_kernel(EmbedArgs a) {
  using P = Piece<E, WIDE>;
  __shared__ float part[JOIN_WAVES][64][P::n];
  __shared__ int found;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int pieces = (a.c.D + P::n - 1) / P::n, across = (pieces + 63) / 64;
  const int block = blockIdx.x / across, piece = (blockIdx.x - block * across) * 64 + lane;
  const int M = *a.total, run = a.run;
  const int tok = a.crosses[block];                  // (anything, where no place of the block is used)
  if ((block + 1LL) * run >= M || tok < 0) return;
  // blocks behind this one that begin with the token
  const int blocks = (int)((M + run - 1LL) / run);
  int end = blocks;
  for (int b0 = block + 1; b0 < blocks; b0 += 64 * JOIN_WAVES) {
    if (threadIdx.x == 0) found = blocks;
    __syncthreads();
    const int b = b0 + threadIdx.x;
    if (b < blocks && a.token[(long long)b * run] != tok) atomicMin(&found, b);
    __syncthreads();
    end = found;
    __syncthreads();
    if (end < blocks) break;
  }
  const int n = end - (block + 1), per = (n + JOIN_WAVES - 1) / JOIN_WAVES;
  const int from = block + 1 + wave * per, to = min(from + per, end);
  const int col = min(piece, pieces - 1) * P::n;
  float sum[P::n];
#pragma unroll
  for (int k = 0; k < P::n; ++k) sum[k] = wave == 0 ? a.part[(2LL * block + 1) * a.c.D + col + k] : 0.f;
#pragma unroll 8
  for (int b = from; b < to; ++b) {
    const float* p = a.part + 2LL * b * a.c.D + col;
#pragma unroll
    for (int k = 0; k < P::n; ++k) sum[k] += p[k];
  }
#pragma unroll
  for (int k = 0; k < P::n; ++k) part[wave][lane][k] = sum[k];
  __syncthreads();
  if (wave || piece >= pieces) return;
  P v;
#pragma unroll
  for (int k = 0; k < P::n; ++k) {
    v.v[k] = part[0][lane][k];
#pragma unroll
    for (int w = 1; w < JOIN_WAVES; ++w) v.v[k] += part[w][lane][k];
  }
  v.store((E*)a.out + (long long)tok * a.c.ld_table + col, a.c.scale);
}

// ---- launches
static bool wide_rows(const void* p, long long ld, int D, int size) {
  return (uintptr_t)p % 16 == 0 && ld * size % 16 == 0 && (long long)D * size % 16 == 0;
}
static size_t embed_piece(size_t n) { return (n + 255) / 256 * 256; }
// Sorted places that a wave adds up: few make the sums of few tokens short, but leave more to join.  Both directions, us,
// runs of 8 / 16 / 32: 1003 tokens of 32768 x 1024 bf16 24.1 / 25.4 / 26.8, of 50021 x 500 floats 26.9 / 27.8 / 29.0; 4096
// 28.7 / 29.5 / 30.9, 30.1 / 31.2 / 32.7; 16384 45.4 / 42.9 / 42.8, 47.2 / 46.1 / 46.3.
static int embed_run(int N) { return N <= 4096 ? 8 : 32; }
// The total, places, tokens, runs that cross blocks, sums.
size_t embed_workspace(const embed_cfg& c) {
  const size_t N = (size_t)c.N, blocks = (N + embed_run(c.N) - 1) / embed_run(c.N);
  return 256 + 2 * embed_piece(4 * N) + embed_piece(4 * blocks) + 8 * blocks * c.D;
}
template <typename E, bool WIDE>
static hipError_t embed_lookup_start(const EmbedArgs& a, hipStream_t s) {
  const long long pieces = (a.c.D + Piece<E, WIDE>::n - 1) / Piece<E, WIDE>::n, n = (a.c.N * pieces + 255) / 256;
  if (!launchable(n, 256)) return TOO_LARGE;
  hipLaunchKernelGGL((embed_lookup_kernel<E, WIDE>), dim3((unsigned)n), dim3(256), 0, s, a);
  return hipGetLastError();
}
// RANGE tokens of the vocabulary for a workgroup of the sort.
template <typename E, bool WIDE, int RANGE>
static hipError_t embed_backward_range(const EmbedArgs& a, hipStream_t s) {
  const long long pieces = (a.c.D + Piece<E, WIDE>::n - 1) / Piece<E, WIDE>::n, across = (pieces + 63) / 64;
  const long long items = ((a.c.N + a.run - 1LL) / a.run) * across;
  const int ranges = (a.c.V + RANGE - 1) / RANGE, clears = (a.c.V + CLEAR_ROWS - 1) / CLEAR_ROWS;
  const int parts = max(1, min(min((a.c.N + PLAN_PART - 1) / PLAN_PART, PLAN_GROUPS / ranges), PLAN_PARTS));
  if (!launchable(items, 64 * JOIN_WAVES)) return TOO_LARGE;
  hipLaunchKernelGGL((embed_plan_kernel<E, WIDE, RANGE>), dim3(ranges * parts + clears), dim3(PLAN_THREADS), 0, s, a, ranges,
                     parts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 groups((unsigned)((items + 3) / 4));
  if (a.run == 8) hipLaunchKernelGGL((embed_sum_kernel<E, WIDE, 8>), groups, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((embed_sum_kernel<E, WIDE, 32>), groups, dim3(256), 0, s, a);
  if ((e = hipGetLastError()) != hipSuccess || a.c.N <= a.run) return e;
  hipLaunchKernelGGL((embed_join_kernel<E, WIDE>), dim3((unsigned)items), dim3(64 * JOIN_WAVES), 0, s, a);
  return hipGetLastError();
}
template <typename E, bool WIDE>
static hipError_t embed_backward_start(const EmbedArgs& a, hipStream_t s) {
  // Small ranges leave more workgroups, large ones more parts of many tokens.  Sort in us for ranges of 128 / 512 / 2048:
  // 1000 tokens of 32768 8.0 / 8.1 / 10.2, of 131072 23.5 / 11.5 / 12.0; 16384 of 1000 8.7 / 9.3 / -, of 32768 14.9 / 9.6 / -,
  // of 10^6 206 / 80 / 72; 65536 of 8192 21.3 / 16.3 / 17.7, of 32768 45 / 23.5 / 20.4, of 131072 - / 51 / 29.5; 262144 of 1000
  // 52 / 53 / 59, of 8192 67 / 47 / 45, of 32768 158 / 72 / 51, of 131072 - / 180 / 79.
  if (a.c.N <= 8192 && a.c.V <= 256 * 128) return embed_backward_range<E, WIDE, 128>(a, s);
  if (a.c.V <= 16 * 512 || (a.c.N <= 32768 && a.c.V <= 256 * 512)) return embed_backward_range<E, WIDE, 512>(a, s);
  return embed_backward_range<E, WIDE, 2048>(a, s);
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
  a.run = embed_run(a.c.N);
  a.total = (int*)ws;
  ws += 256;
  a.place = (int*)ws;
  ws += embed_piece(4 * (size_t)a.c.N);
  a.token = (int*)ws;
  ws += embed_piece(4 * (size_t)a.c.N);
  a.crosses = (int*)ws;
  ws += embed_piece(4 * (((size_t)a.c.N + a.run - 1) / a.run));
  a.part = (float*)ws;
  return embed_typed(a, true, s);
}

}  // namespace mg
