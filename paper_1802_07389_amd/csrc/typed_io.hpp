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

// Calls f with a value of the C++ type of a TLC_F32, TLC_BF16 or TLC_F16.
template <class F>
inline auto with_type(int type, F&& f) {
  if (type == TLC_BF16) return f(bf16_t());
  if (type == TLC_F16) return f(f16_t());
  return f(float());
}

inline size_t type_bytes(int type) { return type == TLC_F32 ? 4 : 2; }

}  // namespace tlc
