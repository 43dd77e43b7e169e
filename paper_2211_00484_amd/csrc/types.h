// Element types of device arrays that may be fp32, bf16 or fp16, and wide accesses to them.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

namespace tbs {

struct bf16 {
  uint16_t bits;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16 x) { return __uint_as_float((uint32_t)x.bits << 16); }
__device__ __forceinline__ float to_float(_Float16 x) { return (float)x; }
// Rounded to nearest, ties to even, by the hardware's conversions (NaN stays NaN).
template <class T>
__device__ __forceinline__ T from_float(float x) {
  return (T)x;
}
template <>
__device__ __forceinline__ bf16 from_float<bf16>(float x) {
  return bf16{__builtin_bit_cast(uint16_t, (__bf16)x)};
}

template <class T, int N>
struct Vec {
  T v[N];
};
// N elements at p, which is aligned to its elements only (one wide access all the same).
template <class T, int N>
__device__ __forceinline__ Vec<T, N> load_vec(const T* p) {
  Vec<T, N> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return r;
}
template <class T, int N>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, N>& r) {
  __builtin_memcpy(p, &r, sizeof(r));
}

}  // namespace tbs
