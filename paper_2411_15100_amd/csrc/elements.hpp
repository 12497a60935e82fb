// Element types of logits and hidden states on the device.
#pragma once
#include <hip/hip_runtime.h>

#include "logits.hpp"

namespace xgm {

typedef unsigned long long u64;

template <Elem E> struct Type;
template <> struct Type<Elem::kF32> { typedef uint32_t bits; };
template <> struct Type<Elem::kBF16> { typedef uint16_t bits; };
template <> struct Type<Elem::kF16> { typedef uint16_t bits; };

template <Elem E> __device__ __forceinline__ float widened(typename Type<E>::bits v) {
  if constexpr (E == Elem::kF32) return __uint_as_float(v);
  if constexpr (E == Elem::kBF16) return __uint_as_float((uint32_t)v << 16);
  if constexpr (E == Elem::kF16) return (float)__builtin_bit_cast(_Float16, v);
}
// rounded to nearest, ties to even; a NaN stays one
template <Elem E> __device__ __forceinline__ typename Type<E>::bits narrowed(float f) {
  if constexpr (E == Elem::kF32) return __float_as_uint(f);
  if constexpr (E == Elem::kBF16) return __builtin_bit_cast(uint16_t, (__bf16)f);
  if constexpr (E == Elem::kF16) return __builtin_bit_cast(uint16_t, (_Float16)f);
}
// The same from 64 bits: one rounding, not one to 32 bits and another to the type.  The first one matters only where it ends on a middle of two numbers of the
// type, and those end in a one and 15 zeros (bf16) or in 12 zeros (f16; more below its normal numbers): there the number goes back a step to the side on which y lies.
// (Left to the compiler, which mends every number: 16384 rows of 4096 columns, 8 bits to f16, 75 us and not 44; to bf16 51 and 44.)
template <Elem E> __device__ __forceinline__ typename Type<E>::bits narrowed(double y) {
  float f = (float)y;
  if constexpr (E != Elem::kF32) {
    const uint32_t u = __float_as_uint(f);
    const bool middle = E == Elem::kBF16 ? (u & 0xffffu) == 0x8000u : (u & 0xfffu) == 0 && f != 0.0f;  // (what 32 bits make 0 is 0)
    if (__builtin_expect(middle, 0)) {
      const double back = (double)f;
      if (back < y || back > y) f = __uint_as_float(u + (fabs(back) < fabs(y) ? 1u : ~0u));
    }
  }
  return narrowed<E>(f);
}

}  // namespace xgm
