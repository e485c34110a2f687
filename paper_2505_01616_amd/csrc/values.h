// Values of a row, eight at a time and at any alignment, and the matrix cores'
// operands (act.hip, experts.hip).
#pragma once

#include <type_traits>

#include "ops.h"

namespace netsim_ops {
namespace {

using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using s16x4 = __attribute__((ext_vector_type(4))) short;
using s16x8 = __attribute__((ext_vector_type(8))) short;
using f32x16 = __attribute__((ext_vector_type(16))) float;
using lds_s16x4 = __attribute__((address_space(3))) s16x4;

// Eight values of a row, as words (values of 16 bits two by two).
template <class T>
struct Eight {
  static constexpr int WORDS = 2 * sizeof(T);
  uint32_t w[WORDS];
};
// Reads of 16 bytes at any alignment of the elements.
typedef uint32_t words_at_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t words_at_4 __attribute__((ext_vector_type(4), aligned(4)));
template <class T>
__device__ __forceinline__ Eight<T> load_eight(const T* p) {
  using Words = std::conditional_t<sizeof(T) == 2, words_at_2, words_at_4>;
  Eight<T> out;
#pragma unroll
  for (int i = 0; i < Eight<T>::WORDS; i += 4) {
    const Words v = reinterpret_cast<const Words*>(p)[i / 4];
#pragma unroll
    for (int j = 0; j < 4; ++j) out.w[i + j] = v[j];
  }
  return out;
}
// The same with zeros beyond `left` values.
template <class T>
__device__ __forceinline__ Eight<T> load_some(const T* p, int left) {
  if (left >= 8) return load_eight(p);
  Eight<T> out;
#pragma unroll
  for (int i = 0; i < Eight<T>::WORDS; ++i) out.w[i] = 0;
  constexpr int PER = 4 / sizeof(T);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < left) {
      if constexpr (PER == 1)
        out.w[i] = reinterpret_cast<const uint32_t*>(p)[i];
      else
        out.w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << (16 * (i & 1));
    }
  return out;
}
template <class T>
__device__ __forceinline__ float value_of(const Eight<T>& v, int i) {
  if constexpr (sizeof(T) == 4)
    return __uint_as_float(v.w[i]);
  else
    return (float)__builtin_bit_cast(T, (uint16_t)(v.w[i / 2] >> (16 * (i & 1))));
}

template <class T>
__device__ __forceinline__ void store_some(T* p, const float (&v)[8], int left) {
  if (left >= 8) {
    using Words = std::conditional_t<sizeof(T) == 2, words_at_2, words_at_4>;
#pragma unroll
    for (int i = 0; i < Eight<T>::WORDS; i += 4) {
      Words w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4)
          w[j] = __float_as_uint(v[i + j]);
        else
          w[j] = (uint32_t)__builtin_bit_cast(uint16_t, (T)v[2 * (i + j)]) |
                 (uint32_t)__builtin_bit_cast(uint16_t, (T)v[2 * (i + j) + 1]) << 16;
      }
      reinterpret_cast<Words*>(p)[i / 4] = w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) p[i] = (T)v[i];
  }
}

}  // namespace
}  // namespace netsim_ops
