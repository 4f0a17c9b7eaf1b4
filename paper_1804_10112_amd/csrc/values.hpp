// The value types of caches and logits: conversions to and from 32 bits, 16 bytes at a time.
#pragma once
#include "common.hpp"

namespace spt {

using f16 = _Float16;
using bf16 = __bf16;

#if defined(__HIPCC__)

template <class T>
__device__ __forceinline__ float to_float(T v) { return static_cast<float>(v); }
template <class T>
__device__ __forceinline__ T from_float(float v) { return static_cast<T>(v); }  // to the nearest, ties to even

template <class T>
struct Vec16 {  // 16 bytes of T
  static constexpr int n = 16 / sizeof(T);
  T v[n];
};

#endif

}  // namespace spt
