// Rows of logits (include/mgrit_ops.h): log probabilities with entropy and top alternatives, and the
// distillation loss with its gradient.
//
// A team of 1, 4 or 16 waves holds a row, or a segment of a long one, in registers as it was stored, 16 bytes
// per load: one pass over memory, and everything after it (maximum, sums, alternatives, gradient) reads
// registers.  Rows longer than a team holds are cut into segments whose statistics a second kernel joins.
//
// Alternatives.  A value's key is a whole number that rises with it; the largest key of a group of lanes is a lower bound
// of the k-th largest of all, if there are k groups with keys as large.  The K-th largest of the groups' largest
// keys (found bit by bit, by counting) leaves little more than K candidates of the whole row, which go to LDS with their indices and
// are ranked by counting how many beat each.  Keys with indices are all different, so the result does not
// depend on the order in which candidates arrive.  Where there are more candidates than LDS takes (rows of
// equal values), the alternatives are found one after the other, each the largest below the last.
#include <type_traits>

#include "elem.h"
#include "ops.h"

namespace mg {

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

// Waves and 16-byte loads per thread of a team.
template <typename E, int NW>
struct TeamOf {
  static constexpr int per_load = 16 / (int)sizeof(E);       // elements
  static constexpr int loads = NW == 1 ? (sizeof(E) == 4 ? 4 : 2) : (sizeof(E) == 4 ? 8 : 4);
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

// The elements lo .. hi-1 of a row that a thread of the team holds: load j holds the 16 bytes (j * threads + thread) of the
// segment, counted from the 16-byte boundary at or before the row's start.  What lies outside is -inf.
template <typename E, int NW>
struct Held {
  using T = TeamOf<E, NW>;
  uintx4 raw[T::loads];
  int first;                                                 // index of the thread's first element

  static __device__ inline E low() { return elem_of<E>(-__builtin_inff()); }
  // base: the row; hi <= V
  __device__ inline void load(const E* row, int lo, int hi, int shift, int tid) {
    first = lo + tid * T::per_load - shift;
#pragma unroll
    for (int j = 0; j < T::loads; ++j) {
      const int i = first + j * T::threads * T::per_load;
      if (i >= hi) {
        E e[T::per_load];
#pragma unroll
        for (int k = 0; k < T::per_load; ++k) e[k] = low();
        raw[j] = __builtin_bit_cast(uintx4, e);
      } else if (i >= lo && i + T::per_load <= hi) {
        raw[j] = *reinterpret_cast<const uintx4*>(row + i);
      } else {
        E e[T::per_load];
#pragma unroll
        for (int k = 0; k < T::per_load; ++k) {
          e[k] = low();
          if (i + k >= lo && i + k < hi) e[k] = row[i + k];
        }
        raw[j] = __builtin_bit_cast(uintx4, e);
      }
    }
  }
  __device__ inline int index(int j, int k) const { return first + j * T::threads * T::per_load + k; }
  __device__ inline float at(int j, int k) const {
    return word_elem<E>(raw[j][k / ELEMS_PER_WORD<E>], k % ELEMS_PER_WORD<E>);
  }
};

// Maximum (of what is not NaN), and with c = log2(e) / t: s = sum 2^(c (x - m)), u = sum of the same times
// c (x - m).  A row of nothing but -inf: m = -inf, s = 0.
struct Stats {
  float m, s, u;
};
__device__ inline float finite_max(float m) { return m == -__builtin_inff() ? 0.f : m; }

// How an exponent c (x - m) is computed for every x of a row: as one multiply-add fma(x, c, -r) with r = c m rounded,
// whose rounding d = c m - r is the same for the whole row, or, where r is not finite (rows whose largest
// value is the type's lowest), as it is written.
struct Exponent {
  float c, m, r;
  bool one;
  __device__ inline Exponent(float c_, float max) : c(c_), m(finite_max(max)), r(m * c_), one(fabsf(r) < __builtin_inff()) {}
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
    largest[j] = x.at(j, 0);
#pragma unroll
    for (int k = 1; k < T::per_load; ++k) largest[j] = fmaxf(largest[j], x.at(j, k));
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

// log p of a logit, from the statistics of its row
__device__ inline float log_prob(float x, const Stats& r, float inv_t) {
  if (r.s == 0.f) return -__builtin_inff();
  return (x - r.m) * inv_t - logf(r.s);
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

// The K largest of the entries lo .. hi-1 of a row that the team holds, in falling order: put(rank, full key).  largest:
// that of each of the thread's loads; ordinary: no NaN and no +inf.  (What few rows need reads the row from the caches, in loops:
// it would cost the others registers.)
template <typename E, int NW, typename PUT>
__device__ inline void team_top(const Held<E, NW>& x, const E* row, int lo, int hi, int K, int tid,
                                const float (&largest)[TeamOf<E, NW>::loads], bool ordinary, TopShared<NW, TeamOf<E, NW>::cand>& sh, PUT put) {
  using T = TeamOf<E, NW>;
  // (-inf, all that lies outside the row is, cannot be told from what is in it: no bound then)
  float own = largest[0];
#pragma unroll
  for (int j = 1; j < T::loads; ++j) own = fmaxf(own, largest[j]);
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
    if (at < T::cand) sh.cand[at] = full_key(key, (unsigned)i);
  };
  const bool bounded = ordinary && threshold != 0;
  if (bounded) {                                             // values compare as their keys do
    const float bound = value_of(threshold);
#pragma unroll
    for (int j = 0; j < T::loads; ++j) {
      if (!(largest[j] >= bound)) continue;
#pragma unroll
      for (int k = 0; k < T::per_load; ++k) {
        const float v = x.at(j, k);
        if (v >= bound) take(key_of(v), x.index(j, k));
      }
    }
  } else {                                                   // fewer than K groups above -inf: all that is
    for (int i = lo + tid; i < hi; i += T::threads) {
      const float v = elem_f32(row[i]);
      if (ordinary ? v > -__builtin_inff() : key_of(v) >= threshold) take(key_of(v), i);
    }
  }
  team_sync<NW>();
  const int n = sh.n;
  if (n <= T::cand) {
    for (int i = tid; i < n; i += T::threads) {
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
      for (int i = lo + tid; i < hi; i += T::threads) {
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
      team_top<E, NW>(held, x, lo, hi, min(a.K, hi - lo), tid, largest, ordinary, top[team],
                     [&](int r, u64 f) { out[r] = f; });
    }
  } else {
    if (tid == 0) put_token(a, row, x, st);
    if (a.K > 0)
      team_top<E, NW>(held, x, lo, hi, a.K, tid, largest, ordinary, top[team], [&](int r, u64 f) {
        a.top_logp[row * a.K + r] = log_prob(value_of((unsigned)(f >> 32)), st, a.inv_t);
        a.top_ids[row * a.K + r] = index_of(f);
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
    if (si != 0.f) u += f * fmaf(si, d, o.u[row * segs + i]);
  }
  return {m, wave_sum(s), wave_sum(u)};
}

constexpr int JOIN_SEGS = 33;                                // of a row at most: 2^20 entries and a piece, 2^15 each, or 2^18, 2^13 each
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
// By one wave; row: the student's logits.
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
    if (entry) z[i] = teacher[k] * inv_t;
    bad |= entry && id >= V;
    t.id[k] = entry && id < V ? (int)id : -1;
    t.x[k] = entry && id < V ? elem_f32(row[id]) : 0.f;
    m = fmaxf(m, z[i]);
  }
  m = wave_max(m);
  const float m0 = finite_max(m);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) s += __builtin_amdgcn_exp2f((z[i] - m0) * LOG2E);
  s = wave_sum(s);
  const float log_s = logf(s);
  float ql = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int k = lane + 64 * i;
    if (k >= K) continue;
    const float q = s == 0.f ? 0.f : __builtin_amdgcn_exp2f((z[i] - m0) * LOG2E) / s;
    t.q[k] = q;
    if (q != 0.f) ql = fmaf(q, z[i] - m0 - log_s, ql);
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
    if (t.q[k] != 0.f) dot = fmaf(t.q[k], (t.x[k] - finite_max(m)) * inv_t, dot);
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
};

// w (p - q) of what a team holds of a row, stored; scale = w total / s, then the entries of the teacher.
template <typename E, int NW>
__device__ inline void put_gradient(const DistillArgs& a, const Held<E, NW>& x, E* out, int lo, int hi, float m,
                                    float s, float w, const Teacher& t, int tid) {
  using T = TeamOf<E, NW>;
  const Exponent ex(a.inv_t * LOG2E, m);
  const float f = t.total == 0.f || s == 0.f ? 0.f * s : w * t.total / s * ex.scale();
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
        *reinterpret_cast<uintx4*>(out + i) = r;
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
  if (t.total == 0.f) return;
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

// A row in one team: loss, statistics and, where it is asked for, the gradient.
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

// Statistics of a segment of a long row.
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
constexpr int CUT_ROWS = 512;
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
// Segments of a row, all as long, for teams of `waves` (4 or 16) waves.
static RowShape segments(int V, int size, bool aligned, int waves = 16) {
  const int per = 16 / size;
  const int most = (size == 4 ? TeamOf<float, 16>::chunks : TeamOf<Bf16, 16>::chunks) / 16 * waves;
  const int pieces = (V + (aligned ? 0 : per - 1) + per - 1) / per;
  RowShape s;
  s.segs = (pieces + most - 1) / most;
  s.seg = (pieces + s.segs - 1) / s.segs;
  return s;
}
// Waves of the teams that token_logprobs cuts long rows up for (their segments are joined in a second launch), 0 where
// it leaves rows whole.
static int logprobs_cut(int N, int V, int size, bool aligned) {
  const int whole = team_waves(V, size, aligned);
  if (whole == 1 || whole == 4) return 0;
  if (whole == 16 && N < CUT_ROWS) return 0;
  return V <= (1 << 18) ? 4 : 16;
}
size_t logits_workspace(const logits_cfg& c) {
  const int size = elem_size(c.dtype);
  // (what is aligned is known with the arrays only: the larger of the two)
  long long segs = team_waves(c.V, size, false) ? 0 : segments(c.V, size, false).segs;
  const int cut = logprobs_cut(c.N, c.V, size, false);
  if (cut) segs = segments(c.V, size, false, cut).segs;
  if (!segs) return 0;
  const long long n = c.N * segs;
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
  const int cut = logprobs_cut(a.c.N, a.c.V, sizeof(E), aligned);
  if (cut) {
    r.shape = segments(a.c.V, sizeof(E), aligned, cut);
    r.out = seg_out(a.workspace, a.c.N, r.shape.segs);
    const dim3 grid(N * (unsigned)r.shape.segs);
    if (cut == 4) hipLaunchKernelGGL((logprobs_kernel<E, 4, true>), grid, dim3(256), 0, s, r);
    else hipLaunchKernelGGL((logprobs_kernel<E, 16, true>), grid, dim3(1024), 0, s, r);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((logprobs_join_kernel<E>), dim3(N), dim3(256), 0, s, r);
    return hipGetLastError();
  }
  switch (team_waves(a.c.V, sizeof(E), aligned)) {
    case 1:
      hipLaunchKernelGGL((logprobs_kernel<E, 1, false>), dim3((N + 3) / 4), dim3(256), 0, s, r);
      break;
    case 4:
      hipLaunchKernelGGL((logprobs_kernel<E, 4, false>), dim3(N), dim3(256), 0, s, r);
      break;
    default:
      hipLaunchKernelGGL((logprobs_kernel<E, 16, false>), dim3(N), dim3(1024), 0, s, r);
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
  return d;
}
template <typename E>
static hipError_t grad_start(const LogitsArgs& a, const float* stats, hipStream_t s) {
  DistillArgs d = distill_args(a);
  d.stats_in = stats;
  const bool aligned = rows_aligned(a.logits, a.c.ld, sizeof(E));
  const unsigned N = (unsigned)a.c.N;
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
