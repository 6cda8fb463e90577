// Two neighbouring channels of one step of a sequence, exponentials and sigmoids of any size.
#pragma once
#include "elem.h"
#include "ops.h"

namespace mg {

// Raw words of two neighbouring channels of one step.
template <typename E>
struct RawPair {
  unsigned w[sizeof(E) / 2];
  __device__ inline void anew() {
#pragma unroll
    for (unsigned& x : w) asm volatile("" : "+v"(x));
  }
  __device__ inline void set(float x) {
    const E e = elem_of<E>(x);
    if constexpr (sizeof(E) == 4) w[0] = w[1] = __float_as_uint(e);
    else w[0] = (unsigned)e.bits * 0x10001u;
  }
  __device__ inline float at(int i) const {
    if constexpr (sizeof(E) == 4) return __uint_as_float(w[i]);
    else return word_elem<E>(w[0], i);
  }
};
// Channels c and c + 1 of a step at p; ALIGNED: as one word, with c + 1 < H.  Otherwise `second` says whether
// there is a channel c + 1.
template <typename E, bool ALIGNED>
__device__ inline RawPair<E> load_pair(const E* p, bool second) {
  RawPair<E> r;
  if constexpr (ALIGNED) {
    if constexpr (sizeof(E) == 4) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      r.w[0] = v.x;
      r.w[1] = v.y;
    } else {
      r.w[0] = *reinterpret_cast<const unsigned*>(p);
    }
  } else {
    const E a = p[0], b = p[second ? 1 : 0];
    if constexpr (sizeof(E) == 4) {
      r.w[0] = __float_as_uint(a);
      r.w[1] = __float_as_uint(b);
    } else {
      r.w[0] = (unsigned)a.bits | ((unsigned)b.bits << 16);
    }
  }
  return r;
}
template <typename E, bool ALIGNED>
__device__ inline void store_pair(E* p, float a, float b, bool second, bool past = false) {
  if constexpr (ALIGNED) {
    typedef float Word __attribute__((ext_vector_type(2)));
    if constexpr (sizeof(E) == 4) {
      const Word w = {a, b};
      store_as(reinterpret_cast<Word*>(p), w, past);
    } else {
      store_as(reinterpret_cast<unsigned*>(p), pack2<E>(a, b), past);
    }
  } else {
    p[0] = elem_of<E>(a);
    if (second) p[1] = elem_of<E>(b);
  }
}

// Whether two channels of every step of the array are one aligned word.
template <typename E>
inline bool pairs(const glr_seq& q, int H) {
  return H % 2 == 0 && q.stride_t % 2 == 0 && q.stride_b % 2 == 0 && (uintptr_t)q.data % (2 * sizeof(E)) == 0;
}

// exp(x), x of any size: 2^p with p = x log2(e) as rounded, and e^r for what the rounding left, r = x - p ln 2 (at
// most 2^-17 where 2^p is a number other than 0 and infinity).  Without the second factor the result is off by 7 units of
// 2^-24 at x = -6, 16 at -20, 62 at -80.  Where 2^p is 0 or infinity, it is the result, and r may be anything: the product is
// NaN there or the result, and the maximum with 2^p / 2, which is below any other result, takes the number (of NaN alone, NaN).
__device__ inline float exp_of(float x) {
  const float p = LOG2E * x, e = __builtin_amdgcn_exp2f(p);
  return fmaxf(fmaf(e, fmaf(-p, LN2, x), e), 0.5f * e);
}
// s = sigmoid(z), n = sigmoid(-z).  (Of a NaN they are numbers: each use multiplies by z.)
struct Sigmoid {
  float s, n;
  __device__ inline explicit Sigmoid(float z) {
    const float x = __builtin_amdgcn_fmed3f(-z, -104.f, 88.f), p = x * LOG2E;
    float e = __builtin_amdgcn_exp2f(p);
    e = fmaf(e, fmaf(-p, LN2, x), e);
    s = __builtin_amdgcn_rcpf(1.0f + e);
    n = e * s;
  }
};
// z as a factor of sigmoid(z), which is not quite 0 below -88: the lowest value of a type times that would be far from 0.
__device__ inline float gate_factor(float z) { return z < -104.f ? -104.f : z; }
__device__ inline float silu(float z) { return gate_factor(z) * Sigmoid(z).s; }
}  // namespace mg
