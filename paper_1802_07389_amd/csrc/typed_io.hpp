// typed_io.hpp -- values of the types the training-step operators read and
// write.  Arithmetic is in fp32 (or 64 bits); a conversion to fewer bits rounds
// once, half to even.
#pragma once

#include "tlc_internal.h"

namespace tlc {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// v rounded to Out.  An fp16 result's product is kept apart from its
// conversion: the compiler joins the two into one mixed-precision multiply-add
// whose result is not rounded to fp32 in between, and bits would differ from
// the two steps that the header states.
template <class Out>
__device__ __forceinline__ Out round_to(float v) {
  if constexpr (sizeof(Out) == 2 && __is_same(Out, f16_t)) asm("" : "+v"(v));
  return (Out)v;
}

// V neighbouring values at any address of their type: gfx950 moves 16 bytes
// there with the same instruction as at aligned ones, so rows of odd length and
// views need no path of their own.
template <class T, int V>
struct PackOf {
  typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
template <class T>
struct PackOf<T, 1> {
  typedef T type;
};
template <class T, int V>
struct Pack {
  typename PackOf<T, V>::type v;
  __device__ __forceinline__ float get(int i) const {
    if constexpr (V == 1)
      return (float)v;
    else
      return (float)v[i];
  }
  __device__ __forceinline__ void set(int i, float f) {
    if constexpr (V == 1)
      v = round_to<T>(f);
    else
      v[i] = round_to<T>(f);
  }
};
template <class T, int V, bool kStream = false>
__device__ __forceinline__ Pack<T, V> load_pack(const T* p) {
  typedef typename PackOf<T, V>::type type;
  Pack<T, V> r;
  if constexpr (kStream)
    r.v = __builtin_nontemporal_load(reinterpret_cast<const type*>(p));
  else
    r.v = *reinterpret_cast<const type*>(p);
  return r;
}
template <class T, int V, bool kStream = false>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, V>& r) {
  typedef typename PackOf<T, V>::type type;
  if constexpr (kStream)
    __builtin_nontemporal_store(r.v, reinterpret_cast<type*>(p));
  else
    *reinterpret_cast<type*>(p) = r.v;
}

// n / d for n < 2^31 by one product: with s = ceil(log2 d) and mul =
// floor(2^(31+s) / d) + 1 the product exceeds the quotient's by less than
// n / 2^31 of a step.
struct Divider {
  uint32_t d, mul, shift;
};
inline Divider divider(uint32_t d) {
  uint32_t s = 0;
  while (((uint64_t)1 << s) < d) ++s;
  return Divider{d, (uint32_t)((((uint64_t)1 << (31 + s)) / d) + 1), 31 + s};
}
__device__ __forceinline__ uint32_t quotient(uint32_t n, Divider v) {
  return (uint32_t)(((uint64_t)n * v.mul) >> v.shift);
}

// Calls f with a value of the C++ type of a TLC_F32, TLC_BF16 or TLC_F16.
template <class F>
inline auto with_type(int type, F&& f) {
  if (type == TLC_BF16) return f(bf16_t());
  if (type == TLC_F16) return f(f16_t());
  return f(float());
}

inline size_t type_bytes(int type) { return type == TLC_F32 ? 4 : 2; }

}  // namespace tlc
