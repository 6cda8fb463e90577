// Elements of the three storage types: conversions, raw words and pairs.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mg {

struct Bf16 {
  unsigned short bits;
};
struct F16 {
  unsigned short bits;
};

__device__ inline float elem_f32(float v) { return v; }
__device__ inline float elem_f32(Bf16 v) { return __uint_as_float((unsigned)v.bits << 16); }
__device__ inline float elem_f32(F16 v) { return (float)__builtin_bit_cast(_Float16, v.bits); }
template <typename E>
__device__ inline E elem_of(float v);
template <>
__device__ inline float elem_of<float>(float v) { return v; }
template <>
__device__ inline Bf16 elem_of<Bf16>(float v) {
  return {__builtin_bit_cast(unsigned short, (__bf16)v)};
}
template <>
__device__ inline F16 elem_of<F16>(float v) {
  return {__builtin_bit_cast(unsigned short, (_Float16)v)};
}

// Word i of a group of raw 32-bit words as its elements: one float, or two 16-bit values.
template <typename E>
constexpr int ELEMS_PER_WORD = 4 / (int)sizeof(E);
template <typename E>
__device__ inline float word_elem(unsigned w, int i);
template <>
__device__ inline float word_elem<float>(unsigned w, int) { return __uint_as_float(w); }
template <>
__device__ inline float word_elem<Bf16>(unsigned w, int i) {
  return __uint_as_float(i ? w & 0xffff0000u : w << 16);
}
template <>
__device__ inline float word_elem<F16>(unsigned w, int i) {
  return elem_f32(F16{(unsigned short)(i ? w >> 16 : w)});
}
// Two values rounded into a word of 16-bit elements (a in the low half).
template <typename E>
__device__ inline unsigned pack2(float a, float b) {
  return (unsigned)elem_of<E>(a).bits | ((unsigned)elem_of<E>(b).bits << 16);
}
template <>
__device__ inline unsigned pack2<Bf16>(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef float floatx2 __attribute__((ext_vector_type(2)));
  const floatx2 v = {a, b};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}

// Stores a value, past the caches or not.  (The empty statements keep the compiler from making one ordinary store of
// the two.)
template <typename V>
__device__ inline void store_as(V* p, const V& v, bool past) {
  if (past) {
    asm volatile("" ::: "memory");
    __builtin_nontemporal_store(v, p);
    asm volatile("" ::: "memory");
  } else {
    *p = v;
  }
}

}  // namespace mg
