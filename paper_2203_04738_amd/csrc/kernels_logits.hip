// Rows of logits (include/mgrit_ops.h): log probabilities with entropy and top alternatives, and the distillation
// loss with its gradient.
//
// A team of 1, 4 or 16 waves holds a row, or a segment of a long one, in registers as it was stored, 16 bytes per
// load: one pass over memory, and everything after it (maximum, sums, alternatives, gradient) reads registers.  Rows
// longer than a team holds are cut into segments whose statistics a second kernel joins.
//
// Alternatives.  A value's key is a whole number that rises with it; the largest key of a group of lanes is a lower
// bound of the k-th largest of all, if there are k groups with keys as large.  The K-th largest of the groups'
// largest keys (found bit by bit, by counting) leaves little more than K candidates of the whole row, which go to LDS
// with their indices and are ranked by counting how many beat each.  Keys with indices are all different, so the
// result does not depend on the order in which candidates arrive.  Where there are more candidates than LDS takes
// (rows of equal values), the alternatives are found one after the other, each the largest below the last.
#include <type_traits>

#include "elem.h"
#include "ops.h"

namespace mg {

typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

// Waves and 16-byte loads per thread of a team.
template <typename E, int NW>
struct TeamOf {
  static constexpr int per_load = 16 / (int)sizeof(E);       // elements
  static constexpr int loads = NW == 1 ? (sizeof(E) == 4 ? 4 : 2) : sizeof(E) == 4 ? 8 : 4;
  static constexpr int threads = NW * 64;
  static constexpr int block = NW == 1 ? 256 : threads;      // threads of a workgroup
  static constexpr int teams = block / threads;
  static constexpr int chunks = threads * loads;             // 16-byte pieces a team holds
  static constexpr int elems = chunks * per_load;
  static constexpr int cand = NW == 1 ? elems : 1024;        // candidates that fit LDS
};

__device__ inline unsigned key_of(float v) {                 // -0 as +0, NaN above all
  if (v != v) return 0xffffffffu;
  const unsigned b = __float_as_uint(v + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float value_of(unsigned key) {
  if (key == 0xffffffffu) return __uint_as_float(0x7fc00000u);
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
// Larger for lower indices; neither 0 nor all bits set.
__device__ inline u64 full_key(unsigned key, unsigned idx) { return (u64)key << 32 | (0x7fffffffu - idx); }
__device__ inline int64_t index_of(u64 f) { return (int64_t)(0x7fffffffu - (unsigned)f); }

// Sums and maxima over a wave, the same bits in every lane and run.
__device__ inline float wave_sum(float v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ inline float wave_max(float v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ inline u64 wave_max(u64 v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 w = __shfl_xor(v, o, 64);
    v = w > v ? w : v;
  }
  return v;
}

// The largest of three (of those that are not NaN), in one instruction: fmaxf would first make each of the stored
// values canonical.
__device__ inline float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

template <int NW>
__device__ inline void team_sync() {
  if constexpr (NW > 1) {
    __syncthreads();
  } else {                                                   // one wave: what its lanes left in LDS
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
  }
}

// The 16 bytes of a row from element i on, at a 16-byte boundary; what lies outside lo .. hi-1 is -inf.
template <typename E>
__device__ inline uintx4 load_piece(const E* row, int i, int lo, int hi) {
  constexpr int PER = 16 / (int)sizeof(E);
  if (i >= lo && i + PER <= hi) return *reinterpret_cast<const uintx4*>(row + i);
  E e[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) e[k] = elem_of<E>(-__builtin_inff());
  if (i < hi)
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (i + k >= lo && i + k < hi) e[k] = row[i + k];
  return __builtin_bit_cast(uintx4, e);
}
template <typename E>
__device__ inline float piece_at(const uintx4& raw, int k) {
  return word_elem<E>(raw[k / ELEMS_PER_WORD<E>], k % ELEMS_PER_WORD<E>);
}

// The elements lo .. hi-1 of a row that a thread of the team holds: load j holds the 16 bytes (j * threads + thread)
// of the segment, counted from the 16-byte boundary at or before the row's start.  What lies outside is -inf.
template <typename E, int NW>
struct Held {
  using T = TeamOf<E, NW>;
  uintx4 raw[T::loads];
  int first;                                                 // index of the thread's first element

  // base: the row; hi <= V
  __device__ inline void load(const E* row, int lo, int hi, int shift, int tid) {
    first = lo + tid * T::per_load - shift;
#pragma unroll
    for (int j = 0; j < T::loads; ++j) {
      raw[j] = load_piece(row, first + j * T::threads * T::per_load, lo, hi);
    }
  }
  __device__ inline int index(int j, int k) const { return first + j * T::threads * T::per_load + k; }
  __device__ inline float at(int j, int k) const {
    return piece_at<E>(raw[j], k);
  }
};

// Maximum (of what is not NaN), and with c = log2(e) / t: s = sum 2^(c (x - m)), u = sum of the same times
// c (x - m).  A row of nothing but -inf: m = -inf, s = 0.
struct Stats {
  float m, s, u;
};
__device__ inline float finite_max(float m) { return m == -__builtin_inff() ? 0.f : m; }

// How an exponent c (x - m) is computed for every x of a row: as one multiply-add fma(x, c, -r) with r = c m rounded,
// whose rounding d = c m - r is the same for the whole row, or, where d could pass 1/2 (|r| from 2^24 on: rows whose
// largest value is the type's lowest, for one), as it is written.
constexpr float ONE_FMA = 0x1p24f;
struct Exponent {
  float c, m, r;
  bool one;
  __device__ inline Exponent(float c_, float max) : c(c_), m(finite_max(max)), r(m * c_), one(fabsf(r) < ONE_FMA) {}
  // 2^-d, what a sum of 2^fma(x, c, -r) is to be multiplied by
  __device__ inline float scale() const { return one ? __builtin_amdgcn_exp2f(-rest()) : 1.f; }
  __device__ inline float rest() const { return one ? fmaf(m, c, -r) : 0.f; }
};
template <bool ONE>
__device__ inline float exponent(const Exponent& x, float v) {
  return ONE ? fmaf(v, x.c, -x.r) : (v - x.m) * x.c;
}

// (largest: of each of the thread's loads)
template <typename E, int NW, bool ENTROPY>
__device__ inline Stats team_stats(const Held<E, NW>& x, float c, int tid, float (*part)[2],
                                   float (&largest)[TeamOf<E, NW>::loads]) {
  using T = TeamOf<E, NW>;
  Stats st;
  float m = -__builtin_inff();
#pragma unroll
  for (int j = 0; j < T::loads; ++j) {
    largest[j] = -__builtin_inff();
#pragma unroll
    for (int k = 0; k < T::per_load; k += 2) largest[j] = max3(largest[j], x.at(j, k), x.at(j, k + 1));
    m = fmaxf(m, largest[j]);
  }
  m = wave_max(m);
  if constexpr (NW > 1) {
    if ((tid & 63) == 0) part[tid >> 6][0] = m;
    __syncthreads();
    m = part[tid & (NW - 1)][0];
#pragma unroll
    for (int o = 1; o < NW; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    __syncthreads();
  }
  const Exponent ex(c, m);
  float s = 0.f, u = 0.f;
  auto sum = [&](auto one) {
#pragma unroll
    for (int j = 0; j < T::loads; ++j)
#pragma unroll
      for (int k = 0; k < T::per_load; ++k) {
        const float z = exponent<decltype(one)::value>(ex, x.at(j, k));
        const float e = __builtin_amdgcn_exp2f(z);
        s += e;
        if (ENTROPY) u = fmaf(e, fmaxf(z, -1e30f), u);       // (0 times -inf is 0 here)
      }
  };
  if (ex.one) sum(std::true_type{});
  else sum(std::false_type{});
  s = wave_sum(s);
  if (ENTROPY) u = wave_sum(u);
  if constexpr (NW > 1) {
    if ((tid & 63) == 0) {
      part[tid >> 6][0] = s;
      part[tid >> 6][1] = u;
    }
    __syncthreads();
    s = part[tid & (NW - 1)][0];
    if (ENTROPY) u = part[tid & (NW - 1)][1];
#pragma unroll
    for (int o = 1; o < NW; o <<= 1) {
      s += __shfl_xor(s, o, 64);
      if (ENTROPY) u += __shfl_xor(u, o, 64);
    }
  }
  const float f = ex.scale();
  st.m = m;
  st.s = s * f;
  st.u = (u - ex.rest() * s) * f;
  return st;
}

// w (x - m), w >= 0: the difference of two floats may be beyond them where w times it is not.  What a mask leaves out
// (-inf) stays that, also where w m is beyond the floats.
__device__ inline float below(float x, float m, float w) {
  const float d = x - m;
  if (x == -__builtin_inff()) return x;
  return w < 1.f && fabsf(d) == __builtin_inff() ? x * w - m * w : d * w;
}
// log p of a logit, from the statistics of its row
__device__ inline float log_prob(float x, const Stats& r, float inv_t) {
  if (r.s == 0.f) return -__builtin_inff();
  return below(x, r.m, inv_t) - logf(r.s);
}
__device__ inline float entropy_of(const Stats& r) { return r.s == 0.f ? 0.f : logf(r.s) - r.u * LN2 / r.s; }

// K-th largest of the 64 * PER keys that the lanes of a wave hold (0: no key), or a little less: its top 16
// bits (all that a 16-bit type has).  0 if there are fewer than K.
template <int PER>
__device__ inline unsigned kth_key(const unsigned (&key)[PER], int K) {
  unsigned t = 0;
#pragma unroll 1
  for (int bit = 31; bit >= 16; --bit) {
    const unsigned u = t | (1u << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) n += __popcll(__ballot(key[i] >= u));
    if (n >= K) t = u;
  }
  return t;
}

template <int NW, int CAND>
struct TopShared {
  u64 cand[CAND];
  unsigned keys[NW > 1 ? 256 : 1];
  u64 best[NW > 1 ? 16 : 1];
  unsigned threshold;
  int n;
};

// The K largest of the entries lo .. hi-1 of a row, in falling order: put(rank, full key).  own: the thread's own
// largest value; ordinary: no NaN and no +inf; scan(bound, take): calls take(key, index) for the thread's values >=
// bound.  (What few rows need reads the row from the caches, in loops: it would cost the others registers.)
template <typename E, int NW, int CAND, typename SCAN, typename PUT>
__device__ inline void team_top(const E* row, int lo, int hi, int K, int tid, float own, bool ordinary,
                                TopShared<NW, CAND>& sh, SCAN scan, PUT put) {
  constexpr int THREADS = NW * 64;
  // (-inf, all that lies outside the row is, cannot be told from what is in it: no bound then)
  unsigned most = own > -__builtin_inff() ? key_of(own) : 0;
  if (tid == 0) sh.n = 0;
  unsigned threshold;
  if constexpr (NW == 1) {
    const unsigned one[1] = {most};
    threshold = kth_key<1>(one, K);
  } else {
    if constexpr (NW == 16) {                                // groups of four lanes
      most = max(most, (unsigned)__shfl_xor((int)most, 1, 64));
      most = max(most, (unsigned)__shfl_xor((int)most, 2, 64));
      if ((tid & 3) == 0) sh.keys[tid >> 2] = most;
    } else {
      sh.keys[tid] = most;
    }
    __syncthreads();
    if (tid < 64) {
      unsigned four[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) four[i] = sh.keys[tid + 64 * i];
      threshold = kth_key<4>(four, K);
      if (tid == 0) sh.threshold = threshold;
    }
    __syncthreads();
    threshold = sh.threshold;
  }
  team_sync<NW>();
  auto take = [&](unsigned key, int i) {
    const int at = atomicAdd(&sh.n, 1);
    if (at < CAND) sh.cand[at] = full_key(key, (unsigned)i);
  };
  if (ordinary && threshold != 0) {                          // values compare as their keys do
    scan(value_of(threshold), take);
  } else {                                                   // fewer than K groups above -inf: all that is
    for (int i = lo + tid; i < hi; i += THREADS) {
      const float v = elem_f32(row[i]);
      if (ordinary ? v > -__builtin_inff() : key_of(v) >= threshold) take(key_of(v), i);
    }
  }
  team_sync<NW>();
  const int n = sh.n;
  if (n <= CAND) {
    for (int i = tid; i < n; i += THREADS) {
      const u64 mine = sh.cand[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += sh.cand[j] > mine;
      if (rank < K) put(rank, mine);
    }
    if (n < K && tid < 64)                                   // -inf at the lowest indices
      for (int i0 = lo, rank = n; rank < K; i0 += 64) {
        const bool inf = i0 + tid < hi && elem_f32(row[i0 + tid]) == -__builtin_inff();
        const u64 mask = __ballot(inf);
        const int mine = rank + __popcll(mask & ((1ull << tid) - 1));
        if (inf && mine < K) put(mine, full_key(key_of(-__builtin_inff()), (unsigned)(i0 + tid)));
        rank += __popcll(mask);
      }
    return;
  }
  if constexpr (NW > 1) {
    u64 last = ~0ull;
    for (int r = 0; r < K; ++r) {
      u64 best = 0;
      for (int i = lo + tid; i < hi; i += THREADS) {
        const u64 f = full_key(key_of(elem_f32(row[i])), (unsigned)i);
        if (f < last && f > best) best = f;
      }
      best = wave_max(best);
      if ((tid & 63) == 0) sh.best[tid >> 6] = best;
      __syncthreads();
      best = sh.best[tid & (NW - 1)];
#pragma unroll
      for (int o = 1; o < NW; o <<= 1) {
        const u64 w = __shfl_xor(best, o, 64);
        best = w > best ? w : best;
      }
      if (tid == 0) put(r, best);
      last = best;
      __syncthreads();
    }
  }
}
// The same of what a team holds; largest: that of each of the thread's loads.
template <typename E, int NW, typename PUT>
__device__ inline void held_top(const Held<E, NW>& x, const E* row, int lo, int hi, int K, int tid,
                                const float (&largest)[TeamOf<E, NW>::loads], bool ordinary,
                                TopShared<NW, TeamOf<E, NW>::cand>& sh, PUT put) {
  using T = TeamOf<E, NW>;
  float own = largest[0];
#pragma unroll
  for (int j = 1; j < T::loads; ++j) own = fmaxf(own, largest[j]);
  team_top<E, NW>(row, lo, hi, K, tid, own, ordinary, sh, [&](float bound, auto take) {
#pragma unroll
    for (int j = 0; j < T::loads; ++j) {
      if (!(largest[j] >= bound)) continue;
#pragma unroll
      for (int k = 0; k < T::per_load; ++k) {
        const float v = x.at(j, k);
        if (v >= bound) take(key_of(v), x.index(j, k));
      }
    }
  }, put);
}

// How the rows of a call are cut.
struct RowShape {
  int segs;                  // segments per row
  int seg;                   // 16-byte pieces of a segment
};
// Elements between the 16-byte boundary at or before p and p.
template <typename E>
__device__ inline int row_shift(const E* p) {
  return (int)((uintptr_t)p / sizeof(E) % (16 / sizeof(E)));
}

// Statistics and alternatives of a row's segment, in the workspace.
struct SegOut {
  float *m, *s, *u;          // [N][segs]
  u64* top;                  // [N][segs][K]
};
static SegOut seg_out(char* ws, long long N, int segs) {
  const long long n = N * segs;
  return {(float*)ws, (float*)ws + n, (float*)ws + 2 * n, (u64*)(ws + (3 * n * 4 + 15) / 16 * 16)};
}

struct RowArgs {
  const void* logits;
  const int64_t* tokens;
  float *logp, *entropy, *top_logp;
  int64_t* top_ids;
  int N, V, K;
  long long ld;
  float inv_t;
  RowShape shape;
  SegOut out;                // segs > 1
};

// What token_logprobs writes for a row once its statistics are known (the thread that calls it writes).
template <typename E>
__device__ inline void put_token(const RowArgs& a, long long row, const E* x, const Stats& st) {
  if (a.entropy) a.entropy[row] = entropy_of(st);
  if (a.tokens) {
    const long long t = a.tokens[row];
    float v = 0.f;
    if (t >= a.V) v = __uint_as_float(0x7fc00000u);
    else if (t >= 0) v = log_prob(elem_f32(x[t]), st, a.inv_t);
    a.logp[row] = v;
  }
}

// A team per row or segment.  What bounds few rows is latency: 8 rows of 32768 bf16, K = 20: 8.8 us for load, two
// sums, the search of the bound and the ranking; 100 rows of 51 floats: 6.1 us.
template <typename E, int NW, bool SEGS>
__global__ __launch_bounds__((TeamOf<E, NW>::block), NW == 16 ? 8 : 4) void logprobs_kernel(RowArgs a) {
  using T = TeamOf<E, NW>;
  __shared__ float part[NW == 1 ? 1 : NW][2];
  __shared__ TopShared<NW, T::cand> top[T::teams];
  const int team = NW == 1 ? threadIdx.x >> 6 : 0, tid = NW == 1 ? threadIdx.x & 63 : threadIdx.x;
  const long long item = (long long)blockIdx.x * T::teams + team;
  const long long row = SEGS ? item / a.shape.segs : item;
  const int seg = SEGS ? (int)(item - row * a.shape.segs) : 0;
  if (row >= a.N) return;                                    // (teams of one wave: whole waves)
  const E* x = (const E*)a.logits + row * a.ld;
  const int shift = row_shift(x);
  const int begin = seg * a.shape.seg * T::per_load - shift;
  const int lo = max(begin, 0);
  const int hi = SEGS ? (int)min((long long)a.V, begin + (long long)a.shape.seg * T::per_load) : a.V;
  Held<E, NW> held;
  held.load(x, lo, hi, lo - begin, tid);
  const float c = a.inv_t * LOG2E;
  float largest[T::loads];
  const Stats st = team_stats<E, NW, true>(held, c, tid, part, largest);
  const bool ordinary = st.s == st.s;                        // (no NaN, no +inf)
  if constexpr (SEGS) {
    if (tid == 0) {
      a.out.m[item] = st.m;
      a.out.s[item] = st.s;
      a.out.u[item] = st.u;
    }
    if (a.K > 0) {
      u64* out = a.out.top + item * a.K;
      for (int i = tid; i < a.K; i += T::threads)
        if (i >= hi - lo) out[i] = 0;                        // (a last segment of fewer than K entries)
      held_top<E, NW>(held, x, lo, hi, min(a.K, hi - lo), tid, largest, ordinary, top[team],
                     [&](int r, u64 f) { out[r] = f; });
    }
  } else {
    if (tid == 0) put_token(a, row, x, st);
    if (a.K > 0)
      held_top<E, NW>(held, x, lo, hi, a.K, tid, largest, ordinary, top[team], [&](int r, u64 f) {
        a.top_logp[row * a.K + r] = log_prob(value_of((unsigned)(f >> 32)), st, a.inv_t);
        a.top_ids[row * a.K + r] = index_of(f);
      });
  }
}

// Many long rows.  What bounds them is arithmetic: an exponential and four operations on every value, and what each
// wave does besides, so a thread goes through 128 values in a stream of pieces, four loaded ahead, and keeps of each
// piece its largest value alone; the few pieces that hold an alternative are read again.  The exponents are taken
// against a reference r of the thread's own, the largest of the first pieces, 2^(c x - r): it moves (and the sums
// with it) where a later piece is 2^32 times as large; threads and waves are brought to one reference at the end.
// 2048 x 131072 bf16, K = 8: 537 MB in 114 us traced (4.7 TB/s; calls behind each other 106 us with the join); held
// by teams of 4 waves, 32 values a thread, 182 us.
template <typename E>
struct StreamOf {
  static constexpr int per = 16 / (int)sizeof(E), batches = sizeof(E) == 4 ? 8 : 4;
  static constexpr int chunks = batches * 4 * 256;           // 16-byte pieces of a workgroup: 2^15 values
};
template <typename E, bool SEGS>
__global__ __launch_bounds__(256) void logprobs_stream_kernel(RowArgs a) {
  using T = StreamOf<E>;
  constexpr float NONE = -__builtin_inff();
  __shared__ float part[4][4];
  __shared__ TopShared<4, 1024> top;
  const int tid = threadIdx.x;
  const long long item = blockIdx.x, row = SEGS ? item / a.shape.segs : item;
  const int seg = SEGS ? (int)(item - row * a.shape.segs) : 0;
  const E* x = (const E*)a.logits + row * a.ld;
  const int begin = (SEGS ? seg * a.shape.seg * T::per : 0) - row_shift(x);
  const int lo = max(begin, 0);
  const int hi = SEGS ? (int)min((long long)a.V, begin + (long long)a.shape.seg * T::per) : a.V;
  const int first = begin + tid * T::per;
  const float c = a.inv_t * LOG2E;
  float largest[T::batches][4], r = NONE, s = 0.f, u = 0.f, own = NONE;
  uintx4 ahead[4];
  auto load = [&](int b) {
#pragma unroll
    for (int q = 0; q < 4; ++q) ahead[q] = load_piece(x, first + (4 * b + q) * 256 * T::per, lo, hi);
  };
  load(0);
#pragma unroll
  for (int b = 0; b < T::batches; ++b) {
    uintx4 raw[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      raw[q] = ahead[q];
      largest[b][q] = NONE;
    }
    if (begin + b * 1024 * T::per >= hi) continue;           // (the same in all threads)
    if (b + 1 < T::batches) load(b + 1);
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int k = 0; k < T::per; k += 2)
        largest[b][q] = max3(largest[b][q], piece_at<E>(raw[q], k), piece_at<E>(raw[q], k + 1));
    const float m = fmaxf(fmaxf(largest[b][0], largest[b][1]), fmaxf(largest[b][2], largest[b][3]));
    own = fmaxf(own, m);
    const float to = m * c;
    if (to - r > 32.f && to > -ONE_FMA) {                    // (also from no reference to the first)
      if (r != NONE) {
        const float d = r - to, f = __builtin_amdgcn_exp2f(d);
        u = fmaf(d, s, u) * f;
        s *= f;
      }
      r = to;
    }
    const float ref = r == NONE ? 0.f : r;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int k = 0; k < T::per; ++k) {
        const float z = fmaf(piece_at<E>(raw[q], k), c, -ref), e = __builtin_amdgcn_exp2f(z);
        s += e;
        u = fmaf(e, fmaxf(z, -1e30f), u);                    // (0 times -inf is 0 here)
      }
  }
  // one reference R for all; m: the largest value
  float m = wave_max(own), R = wave_max(r);
  if ((tid & 63) == 0) {
    part[tid >> 6][0] = m;
    part[tid >> 6][1] = R;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    m = fmaxf(m, part[w][0]);
    R = fmaxf(R, part[w][1]);
  }
  if (r != NONE) {
    const float d = r - R, f = __builtin_amdgcn_exp2f(d);
    u = fmaf(d, s, u) * f;
    s *= f;
  }
  s = wave_sum(s);
  u = wave_sum(u);
  if ((tid & 63) == 0) {
    part[tid >> 6][2] = s;
    part[tid >> 6][3] = u;
  }
  __syncthreads();
  s = (part[0][2] + part[1][2]) + (part[2][2] + part[3][2]);
  u = (part[0][3] + part[1][3]) + (part[2][3] + part[3][3]);
  Stats st = {m, s, u};
  const float d = fmaf(m, c, -R);                            // from R to c m
  if (fabsf(m * c) < ONE_FMA) {
    const float f = __builtin_amdgcn_exp2f(-d);
    st.u = fmaf(-d, s, u) * f;
    st.s = s * f;
  } else if (m != NONE && m < __builtin_inff()) {
    // so large that c x - r is too coarse: against the value itself (from the caches)
    s = u = 0.f;
    for (int i = lo + tid; i < hi; i += 256) {
      const float z = (elem_f32(x[i]) - m) * c, e = __builtin_amdgcn_exp2f(z);
      s += e;
      u = fmaf(e, fmaxf(z, -1e30f), u);
    }
    s = wave_sum(s);
    u = wave_sum(u);
    __syncthreads();
    if ((tid & 63) == 0) {
      part[tid >> 6][2] = s;
      part[tid >> 6][3] = u;
    }
    __syncthreads();
    st.s = (part[0][2] + part[1][2]) + (part[2][2] + part[3][2]);
    st.u = (part[0][3] + part[1][3]) + (part[2][3] + part[3][3]);
  }
  const bool ordinary = st.s == st.s;                        // (no NaN, no +inf)
  auto scan = [&](float bound, auto take) {
#pragma unroll
    for (int b = 0; b < T::batches; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (!(largest[b][q] >= bound)) continue;
        const int i = first + (4 * b + q) * 256 * T::per;
        const uintx4 raw = load_piece(x, i, lo, hi);
#pragma unroll
        for (int k = 0; k < T::per; ++k) {
          const float v = piece_at<E>(raw, k);
          if (v >= bound) take(key_of(v), i + k);
        }
      }
  };
  if constexpr (SEGS) {
    if (tid == 0) {
      a.out.m[item] = st.m;
      a.out.s[item] = st.s;
      a.out.u[item] = st.u;
    }
    if (a.K > 0) {
      u64* out = a.out.top + item * a.K;
      for (int i = tid; i < a.K; i += 256)
        if (i >= hi - lo) out[i] = 0;
      team_top<E, 4>(x, lo, hi, min(a.K, hi - lo), tid, own, ordinary, top, scan,
                     [&](int rank, u64 f) { out[rank] = f; });
    }
  } else {
    if (tid == 0) put_token(a, row, x, st);
    if (a.K > 0)
      team_top<E, 4>(x, lo, hi, a.K, tid, own, ordinary, top, scan, [&](int rank, u64 f) {
        a.top_logp[row * a.K + rank] = log_prob(value_of((unsigned)(f >> 32)), st, a.inv_t);
        a.top_ids[row * a.K + rank] = index_of(f);
      });
  }
}

// Statistics of a row from those of its segments, by one wave; the same bits in every lane.
__device__ inline Stats join_stats(const SegOut& o, long long row, int segs, float c, int lane) {
  float m = -__builtin_inff(), s = 0.f, u = 0.f;
  for (int i = lane; i < segs; i += 64) m = fmaxf(m, o.m[row * segs + i]);
  m = wave_max(m);
  const float m0 = finite_max(m);
  for (int i = lane; i < segs; i += 64) {
    const float d = (finite_max(o.m[row * segs + i]) - m0) * c, si = o.s[row * segs + i];
    const float f = si == 0.f ? 0.f : __builtin_amdgcn_exp2f(d);
    s += f * si;
    if (f != 0.f) u += f * fmaf(si, d, o.u[row * segs + i]);   // (d can be -inf: a segment of the lowest value)
  }
  return {m, wave_sum(s), wave_sum(u)};
}

constexpr int JOIN_SEGS = 33;                                // of a row at most: 2^20 entries and a piece, 2^15 each
template <typename E>
__global__ __launch_bounds__(256) void logprobs_join_kernel(RowArgs a) {
  __shared__ u64 cand[JOIN_SEGS * LOGPROBS_MAX_K];
  __shared__ u64 least;
  __shared__ int n;
  const long long row = blockIdx.x;
  const E* x = (const E*)a.logits + row * a.ld;
  const int tid = threadIdx.x, segs = a.shape.segs;
  const Stats st = join_stats(a.out, row, segs, a.inv_t * LOG2E, tid & 63);
  if (tid == 0) put_token(a, row, x, st);
  if (a.K == 0) return;
  const u64* top = a.out.top + row * segs * a.K;
  // the largest of the segments' K-th keys: K entries are as large
  if (tid < 64) {
    u64 v = 0;
    for (int i = tid; i < segs; i += 64) v = max(v, top[(long long)i * a.K + a.K - 1]);
    v = wave_max(v);
    if (tid == 0) {
      least = v;
      n = 0;
    }
  }
  __syncthreads();
  const u64 bound = max(least, (u64)1);
  for (int i = tid; i < segs * a.K; i += 256) {
    const u64 f = top[i];
    if (f >= bound) cand[atomicAdd(&n, 1)] = f;
  }
  __syncthreads();
  const int count = n;
  for (int i = tid; i < count; i += 256) {
    const u64 mine = cand[i];
    int rank = 0;
    for (int j = 0; j < count; ++j) rank += cand[j] > mine;
    if (rank < a.K) {
      a.top_logp[row * a.K + rank] = log_prob(value_of((unsigned)(mine >> 32)), st, a.inv_t);
      a.top_ids[row * a.K + rank] = index_of(mine);
    }
  }
}

// ---- distillation
// The teacher's side of a row, in LDS.
struct Teacher {
  float q[DISTILL_MAX_K];                                    // weights (0: padding)
  float x[DISTILL_MAX_K];                                    // the student's logits there
  int id[DISTILL_MAX_K];                                     // -1: padding
  float total;                                               // of the weights: 1, 0 (no teacher), NaN (an id >= V)
  float qlogq;                                               // sum q log q
};
// By one wave; row: the student's logits.  Weights from (teacher - largest) / t, as `below` has it: a teacher's value
// over t may be beyond a float.
template <typename E>
__device__ inline void read_teacher(const int64_t* ids, const float* teacher, int K, int V, float inv_t,
                                    const E* row, int lane, Teacher& t) {
  constexpr int PER = DISTILL_MAX_K / 64;
  float z[PER];
  bool bad = false;
  float m = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int k = lane + 64 * i;
    z[i] = -__builtin_inff();
    if (k >= K) continue;
    const long long id = ids[k];
    const bool entry = id >= 0;
    if (entry) z[i] = teacher[k];
    bad |= entry && id >= V;
    t.id[k] = entry && id < V ? (int)id : -1;
    t.x[k] = entry && id < V ? elem_f32(row[id]) : 0.f;
    m = fmaxf(m, z[i]);
  }
  m = finite_max(wave_max(m));
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    z[i] = below(z[i], m, inv_t);
    s += __builtin_amdgcn_exp2f(z[i] * LOG2E);
  }
  s = wave_sum(s);
  const float log_s = logf(s);
  float ql = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int k = lane + 64 * i;
    if (k >= K) continue;
    const float q = s == 0.f ? 0.f : __builtin_amdgcn_exp2f(z[i] * LOG2E) / s;
    t.q[k] = q;
    if (q != 0.f) ql = fmaf(q, z[i] - log_s, ql);
  }
  ql = wave_sum(ql);
  const bool any_bad = __any(bad);
  if (lane == 0) {
    t.total = any_bad ? __uint_as_float(0x7fc00000u) : s == 0.f ? 0.f : 1.f;
    t.qlogq = ql;
  }
}
// Loss of a row, by one wave.
__device__ inline float teacher_loss(const Teacher& t, int K, float m, float s, float inv_t, int lane) {
  if (t.total == 0.f) return 0.f;
  float dot = 0.f;
  for (int k = lane; k < K; k += 64)
    if (t.q[k] != 0.f) dot += below(t.x[k], finite_max(m), t.q[k] * inv_t);
  dot = wave_sum(dot);
  if (s == 0.f) return __builtin_inff() * t.total;
  return (t.qlogq - dot + logf(s)) * t.total;
}
// Weight of entry k and of those before and behind it with the same id.
__device__ inline float same_ids(const Teacher& t, int K, int k) {
  float q = 0.f;
  const int id = t.id[k];
  for (int i = 0; i < K; ++i) q += t.id[i] == id ? t.q[i] : 0.f;
  return q;
}

struct DistillArgs {
  const void* logits;
  const int64_t* ids;
  const float *teacher, *weight;
  float *loss, *stats;
  const float* stats_in;
  void* dlogits;
  int N, V, K;
  long long ld, ld_grad;
  float inv_t;
  RowShape shape;
  SegOut out;
  bool past;                 // gradients past the caches
};

// w (p - q) of what a team holds of a row, stored; scale = w total / s, then the entries of the teacher.  A row of
// nothing but -inf (s = 0) has p = 0, but for an id that does not exist (total is NaN), which makes it NaN.
template <typename E, int NW>
__device__ inline void put_gradient(const DistillArgs& a, const Held<E, NW>& x, E* out, int lo, int hi, float m,
                                    float s, float w, const Teacher& t, int tid) {
  using T = TeamOf<E, NW>;
  const Exponent ex(a.inv_t * LOG2E, m);
  const float f = s == 0.f ? 0.f * t.total : w * t.total / s * ex.scale();
  const bool wide = ((uintptr_t)(out + x.first) & 15) == 0;
  auto store = [&](auto one) {
#pragma unroll
    for (int j = 0; j < T::loads; ++j) {
      const int i = x.index(j, 0);
      uintx4 r;
#pragma unroll
      for (int k = 0; k < T::per_load; k += ELEMS_PER_WORD<E>) {
        float g[2];
#pragma unroll
        for (int e = 0; e < ELEMS_PER_WORD<E>; ++e)
          g[e] = f * __builtin_amdgcn_exp2f(exponent<decltype(one)::value>(ex, x.at(j, k + e)));
        if constexpr (sizeof(E) == 4) r[k] = __float_as_uint(g[0]);
        else r[k / 2] = pack2<E>(g[0], g[1]);
      }
      if (wide && i >= lo && i + T::per_load <= hi) {
        store_as(reinterpret_cast<uintx4*>(out + i), r, a.past);
      } else {
        E e[T::per_load];
        __builtin_memcpy(e, &r, 16);
#pragma unroll
        for (int k = 0; k < T::per_load; ++k)
          if (i + k >= lo && i + k < hi) out[i + k] = e[k];
      }
    }
  };
  if (ex.one) store(std::true_type{});
  else store(std::false_type{});
  // the entries, over what was stored there before the barrier
  team_sync<NW>();
  for (int k = tid; k < a.K; k += T::threads) {
    const int id = t.id[k];
    if (id < lo || id >= hi) continue;
    const float p = f * __builtin_amdgcn_exp2f(ex.one ? exponent<true>(ex, t.x[k]) : exponent<false>(ex, t.x[k]));
    out[id] = elem_of<E>(p - w * t.total * same_ids(t, a.K, k));
  }
}
template <typename E>
__device__ inline void put_zeros(E* out, int lo, int hi, int tid, int threads) {
  for (int i = lo + tid; i < hi; i += threads) out[i] = elem_of<E>(0.f);
}

// A row in one team: loss, statistics and, where it is asked for, the gradient.  8192 x 32768 bf16, 64 teacher
// logits: 1.07 GB in 215 us where calls follow each other (5.0 TB/s, a copy's is 6.2), 256 us as traced.
template <typename E, int NW>
__global__ __launch_bounds__((TeamOf<E, NW>::block)) void distill_kernel(DistillArgs a) {
  using T = TeamOf<E, NW>;
  __shared__ float part[NW == 1 ? 1 : NW][2];
  __shared__ Teacher teachers[T::teams];
  const int team = NW == 1 ? threadIdx.x >> 6 : 0, tid = NW == 1 ? threadIdx.x & 63 : threadIdx.x;
  const long long row = (long long)blockIdx.x * T::teams + team;
  if (row >= a.N) return;
  Teacher& t = teachers[team];
  const E* x = (const E*)a.logits + row * a.ld;
  Held<E, NW> held;
  held.load(x, 0, a.V, row_shift(x), tid);
  if (tid < 64) read_teacher(a.ids + row * a.K, a.teacher + row * a.K, a.K, a.V, a.inv_t, x, tid, t);
  team_sync<NW>();
  float largest[T::loads];
  const Stats st = team_stats<E, NW, false>(held, a.inv_t * LOG2E, tid, part, largest);
  const bool none = t.total == 0.f;
  if (tid < 64) {
    const float loss = teacher_loss(t, a.K, st.m, st.s, a.inv_t, tid);
    if (tid == 0) {
      a.loss[row] = loss;
      if (a.stats) {
        a.stats[2 * row] = none ? 0.f : st.m;
        a.stats[2 * row + 1] = none ? 1.f : st.s;
      }
    }
  }
  if (!a.dlogits) return;
  E* out = (E*)a.dlogits + row * a.ld_grad;
  const float w = (a.weight ? a.weight[row] : 1.f) * a.inv_t;
  if (none || w == 0.f) put_zeros(out, 0, a.V, tid, T::threads);
  else put_gradient<E, NW>(a, held, out, 0, a.V, st.m, st.s, w, t, tid);
}

// Statistics of a segment of a long row: 1003 x 50021 floats, 201 MB in 30 us (from the last-level cache in part),
// the gradient below 402 MB in 69 us (the logits from that cache in part).
template <typename E>
__global__ __launch_bounds__(1024) void distill_segment_kernel(DistillArgs a) {
  using T = TeamOf<E, 16>;
  __shared__ float part[16][2];
  const long long row = blockIdx.x / (unsigned)a.shape.segs;
  const int seg = (int)(blockIdx.x - row * a.shape.segs);
  const E* x = (const E*)a.logits + row * a.ld;
  const int begin = seg * a.shape.seg * T::per_load - row_shift(x);
  const int lo = max(begin, 0), hi = (int)min((long long)a.V, begin + (long long)a.shape.seg * T::per_load);
  Held<E, 16> held;
  held.load(x, lo, hi, lo - begin, threadIdx.x);
  float largest[T::loads];
  const Stats st = team_stats<E, 16, false>(held, a.inv_t * LOG2E, threadIdx.x, part, largest);
  if (threadIdx.x == 0) {
    a.out.m[blockIdx.x] = st.m;
    a.out.s[blockIdx.x] = st.s;
    a.out.u[blockIdx.x] = 0.f;
  }
}
// Loss and statistics of a long row from those of its segments; one wave.
template <typename E>
__global__ __launch_bounds__(64) void distill_join_kernel(DistillArgs a) {
  __shared__ Teacher t;
  const long long row = blockIdx.x;
  const int lane = threadIdx.x;
  const E* x = (const E*)a.logits + row * a.ld;
  read_teacher(a.ids + row * a.K, a.teacher + row * a.K, a.K, a.V, a.inv_t, x, lane, t);
  __syncthreads();
  const Stats st = join_stats(a.out, row, a.shape.segs, a.inv_t * LOG2E, lane);
  const float loss = teacher_loss(t, a.K, st.m, st.s, a.inv_t, lane);
  if (lane == 0) {
    const bool none = t.total == 0.f;
    a.loss[row] = loss;
    a.stats[2 * row] = none ? 0.f : st.m;
    a.stats[2 * row + 1] = none ? 1.f : st.s;
  }
}

// Gradient of a row, or of a segment of one, from its statistics.
template <typename E, int NW>
__global__ __launch_bounds__((TeamOf<E, NW>::block)) void distill_grad_kernel(DistillArgs a) {
  using T = TeamOf<E, NW>;
  __shared__ Teacher teachers[T::teams];
  const int team = NW == 1 ? threadIdx.x >> 6 : 0, tid = NW == 1 ? threadIdx.x & 63 : threadIdx.x;
  const long long item = (long long)blockIdx.x * T::teams + team;
  const long long row = item / a.shape.segs;
  const int seg = (int)(item - row * a.shape.segs);
  if (row >= a.N) return;
  Teacher& t = teachers[team];
  const E* x = (const E*)a.logits + row * a.ld;
  const int begin = seg * a.shape.seg * T::per_load - row_shift(x);
  const int lo = max(begin, 0), hi = (int)min((long long)a.V, begin + (long long)a.shape.seg * T::per_load);
  Held<E, NW> held;
  held.load(x, lo, hi, lo - begin, tid);
  if (tid < 64) read_teacher(a.ids + row * a.K, a.teacher + row * a.K, a.K, a.V, a.inv_t, x, tid, t);
  team_sync<NW>();
  E* out = (E*)a.dlogits + row * a.ld_grad;
  const float w = (a.weight ? a.weight[row] : 1.f) * a.inv_t;
  if (t.total == 0.f || w == 0.f) put_zeros(out, lo, hi, tid, T::threads);
  else put_gradient<E, NW>(a, held, out, lo, hi, a.stats_in[2 * row], a.stats_in[2 * row + 1], w, t, tid);
}

// ---- launches
static int elem_size(int dtype) { return dtype == MGRIT_F32 ? 4 : 2; }
static bool rows_aligned(const void* p, long long ld, int size) {
  return (uintptr_t)p % 16 == 0 && ld * size % 16 == 0;
}
// Waves of the smallest team that holds a row (0: none does).  Rows that do not start on a 16-byte
// boundary take up to a load more.
static int team_waves(int V, int size, bool aligned) {
  const int need = V + (aligned ? 0 : 16 / size - 1);
  if (need <= (size == 4 ? TeamOf<float, 1>::elems : TeamOf<Bf16, 1>::elems)) return 1;
  if (need <= (size == 4 ? TeamOf<float, 4>::elems : TeamOf<Bf16, 4>::elems)) return 4;
  if (need <= (size == 4 ? TeamOf<float, 16>::elems : TeamOf<Bf16, 16>::elems)) return 16;
  return 0;
}
// Segments of a row, all as long, of at most 2^15 values: what a team of 16 waves holds or a workgroup streams.
static RowShape segments(int V, int size, bool aligned) {
  const int per = 16 / size, most = size == 4 ? TeamOf<float, 16>::chunks : TeamOf<Bf16, 16>::chunks;
  static_assert(TeamOf<float, 16>::chunks == StreamOf<float>::chunks &&
                    TeamOf<Bf16, 16>::chunks == StreamOf<Bf16>::chunks,
                "both forms take segments of the same length");
  const int pieces = (V + (aligned ? 0 : per - 1) + per - 1) / per;
  RowShape s;
  s.segs = (pieces + most - 1) / most;
  s.seg = (pieces + s.segs - 1) / s.segs;
  return s;
}
// Whether token_logprobs streams rows longer than four waves hold (a workgroup of four waves for each 2^15 values)
// instead of holding them in teams of 16 waves.  K = 20, streamed : held, us: 32768 bf16, 512 rows 15.2 : 12.4, 768
// rows 18.4 : 18.4, 2048 rows 33.9 : 39.8; 32768 floats, 512 rows 19.3 : 17.9, 2048 rows 48.2 : 50.4; 131072 bf16 (4
// segments a row), 64 rows 18.2 : 14.9, 192 rows 24.9 : 23.6, 256 rows 28.1 : 28.4.
constexpr long long STREAM_SEGMENTS = 768;
// Whether rows, or their segments, can be a team each in one launch.
static bool teams_launchable(const logits_cfg& c, int size, bool aligned) {
  const int waves = team_waves(c.V, size, aligned);
  if (waves == 1) return launchable(((long long)c.N + 3) / 4, 256);
  return launchable((long long)c.N * segments(c.V, size, aligned).segs, waves == 4 ? 256 : 1024);
}
size_t logits_workspace(const logits_cfg& c) {
  const int size = elem_size(c.dtype);
  // (what is aligned is known with the arrays only: the larger of the two)
  if (team_waves(c.V, size, false)) return 0;
  const long long n = (long long)c.N * segments(c.V, size, false).segs;
  return (size_t)((3 * n * 4 + 15) / 16 * 16 + 8 * n * (c.K > LOGPROBS_MAX_K ? 0 : c.K) + 8LL * c.N);
}

template <typename E>
static hipError_t logprobs_start(const LogitsArgs& a, hipStream_t s) {
  RowArgs r{};
  r.logits = a.logits;
  r.tokens = a.ids;
  r.logp = a.logp;
  r.entropy = a.entropy;
  r.top_logp = a.top_logp;
  r.top_ids = a.top_ids;
  r.N = a.c.N;
  r.V = a.c.V;
  r.K = a.c.K;
  r.ld = a.c.ld;
  r.inv_t = 1.0f / a.c.temperature;
  const bool aligned = rows_aligned(a.logits, a.c.ld, sizeof(E));
  r.shape = {1, 0};
  const unsigned N = (unsigned)a.c.N;
  const int waves = team_waves(a.c.V, sizeof(E), aligned);
  const RowShape cut = segments(a.c.V, sizeof(E), aligned);
  const bool stream = (long long)N * cut.segs >= STREAM_SEGMENTS;
  const dim3 grid(N * (unsigned)cut.segs);
  // (a row's segments, or four rows in one workgroup)
  const int threads = waves == 1 || waves == 4 || stream ? 256 : 1024;
  if (!launchable(waves == 1 ? ((long long)N + 3) / 4 : (long long)N * cut.segs, threads)) return TOO_LARGE;
  switch (waves) {
    case 1:
      hipLaunchKernelGGL((logprobs_kernel<E, 1, false>), dim3((N + 3) / 4), dim3(256), 0, s, r);
      break;
    case 4:
      hipLaunchKernelGGL((logprobs_kernel<E, 4, false>), dim3(N), dim3(256), 0, s, r);
      break;
    case 16:
      if (stream) hipLaunchKernelGGL((logprobs_stream_kernel<E, false>), dim3(N), dim3(256), 0, s, r);
      else hipLaunchKernelGGL((logprobs_kernel<E, 16, false>), dim3(N), dim3(1024), 0, s, r);
      break;
    default: {
      r.shape = cut;
      r.out = seg_out(a.workspace, a.c.N, cut.segs);
      if (stream) hipLaunchKernelGGL((logprobs_stream_kernel<E, true>), grid, dim3(256), 0, s, r);
      else hipLaunchKernelGGL((logprobs_kernel<E, 16, true>), grid, dim3(1024), 0, s, r);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL((logprobs_join_kernel<E>), dim3(N), dim3(256), 0, s, r);
    }
  }
  return hipGetLastError();
}
hipError_t launch_token_logprobs(const LogitsArgs& a, hipStream_t s) {
  if (a.c.dtype == MGRIT_F32) return logprobs_start<float>(a, s);
  if (a.c.dtype == MGRIT_BF16) return logprobs_start<Bf16>(a, s);
  return logprobs_start<F16>(a, s);
}

static DistillArgs distill_args(const LogitsArgs& a) {
  DistillArgs d{};
  d.logits = a.logits;
  d.ids = a.ids;
  d.teacher = a.teacher;
  d.weight = a.weight;
  d.loss = a.loss;
  d.stats = a.stats;
  d.stats_in = a.stats_in;
  d.dlogits = a.dlogits;
  d.N = a.c.N;
  d.V = a.c.V;
  d.K = a.c.K;
  d.ld = a.c.ld;
  d.ld_grad = a.c.ld_grad;
  d.inv_t = 1.0f / a.c.temperature;
  d.past = results_past_caches((double)elem_size(a.c.dtype) * a.c.N * a.c.V, 180e6);
  return d;
}
template <typename E>
static hipError_t grad_start(const LogitsArgs& a, const float* stats, hipStream_t s) {
  DistillArgs d = distill_args(a);
  d.stats_in = stats;
  const bool aligned = rows_aligned(a.logits, a.c.ld, sizeof(E));
  const unsigned N = (unsigned)a.c.N;
  if (!teams_launchable(a.c, sizeof(E), aligned)) return TOO_LARGE;
  // (the boundary of a row moves its segments: the whole row has to be within the last one)
  switch (team_waves(a.c.V, sizeof(E), aligned)) {
    case 1:
      d.shape = {1, TeamOf<E, 1>::chunks};
      hipLaunchKernelGGL((distill_grad_kernel<E, 1>), dim3((N + 3) / 4), dim3(256), 0, s, d);
      break;
    case 4:
      d.shape = {1, TeamOf<E, 4>::chunks};
      hipLaunchKernelGGL((distill_grad_kernel<E, 4>), dim3(N), dim3(256), 0, s, d);
      break;
    case 16:
      d.shape = {1, TeamOf<E, 16>::chunks};
      hipLaunchKernelGGL((distill_grad_kernel<E, 16>), dim3(N), dim3(1024), 0, s, d);
      break;
    default:
      d.shape = segments(a.c.V, sizeof(E), aligned);
      hipLaunchKernelGGL((distill_grad_kernel<E, 16>), dim3(N * (unsigned)d.shape.segs), dim3(1024), 0, s, d);
  }
  return hipGetLastError();
}
template <typename E>
static hipError_t distill_start(const LogitsArgs& a, hipStream_t s) {
  DistillArgs d = distill_args(a);
  const bool aligned = rows_aligned(a.logits, a.c.ld, sizeof(E));
  const unsigned N = (unsigned)a.c.N;
  if (!teams_launchable(a.c, sizeof(E), aligned)) return TOO_LARGE;
  switch (team_waves(a.c.V, sizeof(E), aligned)) {
    case 1:
      hipLaunchKernelGGL((distill_kernel<E, 1>), dim3((N + 3) / 4), dim3(256), 0, s, d);
      return hipGetLastError();
    case 4:
      hipLaunchKernelGGL((distill_kernel<E, 4>), dim3(N), dim3(256), 0, s, d);
      return hipGetLastError();
    case 16:
      hipLaunchKernelGGL((distill_kernel<E, 16>), dim3(N), dim3(1024), 0, s, d);
      return hipGetLastError();
  }
  d.shape = segments(a.c.V, sizeof(E), aligned);
  d.out = seg_out(a.workspace, a.c.N, d.shape.segs);
  if (!d.stats) d.stats = (float*)d.out.top;                 // (no alternatives here: the space behind)
  hipLaunchKernelGGL((distill_segment_kernel<E>), dim3(N * (unsigned)d.shape.segs), dim3(1024), 0, s, d);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((distill_join_kernel<E>), dim3(N), dim3(64), 0, s, d);
  e = hipGetLastError();
  if (e != hipSuccess || !a.dlogits) return e;
  return grad_start<E>(a, d.stats, s);
}
hipError_t launch_distill(const LogitsArgs& a, hipStream_t s) {
  if (a.c.dtype == MGRIT_F32) return distill_start<float>(a, s);
  if (a.c.dtype == MGRIT_BF16) return distill_start<Bf16>(a, s);
  return distill_start<F16>(a, s);
}
hipError_t launch_distill_grad(const LogitsArgs& a, hipStream_t s) {
  if (a.c.dtype == MGRIT_F32) return grad_start<float>(a, a.stats_in, s);
  if (a.c.dtype == MGRIT_BF16) return grad_start<Bf16>(a, a.stats_in, s);
  return grad_start<F16>(a, a.stats_in, s);
}

}  // namespace mg
