// Rows of 16- and 32-bit numbers as float32, eight at a time (library private).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dwkv.h"

namespace dwkv {

typedef float float8_t __attribute__((ext_vector_type(8), aligned(16)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8), aligned(16)));
typedef __bf16 brain8_t __attribute__((ext_vector_type(8), aligned(16)));

template <int T> struct RowType;
template <> struct RowType<DWKV_F16> { using one = _Float16; using eight = half8_t; };
template <> struct RowType<DWKV_BF16> { using one = __bf16; using eight = brain8_t; };
template <> struct RowType<DWKV_F32> { using one = float; using eight = float8_t; };
template <int T> using row_t = typename RowType<T>::one;
template <int T> using row8_t = typename RowType<T>::eight;

// Eight numbers at a 16-byte aligned place.
template <int T>
__device__ __forceinline__ float8_t load8(const row_t<T>* p) {
  return __builtin_convertvector(*reinterpret_cast<const row8_t<T>*>(p), float8_t);
}
// Rounded to nearest even; PAST: past the caches.
template <int T, bool PAST>
__device__ __forceinline__ void store8(row_t<T>* p, float8_t x) {
  const row8_t<T> v = __builtin_convertvector(x, row8_t<T>);
  if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<row8_t<T>*>(p));
  else *reinterpret_cast<row8_t<T>*>(p) = v;
}

// The same at any place that the type's own alignment allows.
template <int T> struct AnyPlace;
template <> struct AnyPlace<DWKV_F16> { typedef _Float16 eight __attribute__((ext_vector_type(8), aligned(2))); };
template <> struct AnyPlace<DWKV_BF16> { typedef __bf16 eight __attribute__((ext_vector_type(8), aligned(2))); };
template <> struct AnyPlace<DWKV_F32> { typedef float eight __attribute__((ext_vector_type(8), aligned(4))); };
template <int T>
__device__ __forceinline__ float8_t load8_any(const row_t<T>* p) {
  return __builtin_convertvector(*reinterpret_cast<const typename AnyPlace<T>::eight*>(p), float8_t);
}
template <int T>
__device__ __forceinline__ void store8_any(row_t<T>* p, float8_t x) {
  *reinterpret_cast<typename AnyPlace<T>::eight*>(p) = __builtin_convertvector(x, typename AnyPlace<T>::eight);
}

}  // namespace dwkv
