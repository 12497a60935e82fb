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
// The same from 64 bits: one rounding, not one to 32 bits and another to the type.
template <Elem E> __device__ __forceinline__ typename Type<E>::bits narrowed(double y) {
  if constexpr (E == Elem::kF32) return __float_as_uint((float)y);
  if constexpr (E == Elem::kBF16) return __builtin_bit_cast(uint16_t, (__bf16)y);
  if constexpr (E == Elem::kF16) return __builtin_bit_cast(uint16_t, (_Float16)y);
}

}  // namespace xgm
