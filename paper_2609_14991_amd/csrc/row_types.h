// Element types of rows that come in fp32, bf16 or fp16 (FUSION_F32 and on), and
// access to them 16 bytes at a time.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace fusion {

struct Half { uint16_t b; };   // fp16
struct Brain { uint16_t b; };  // bf16
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(Brain x) { return __uint_as_float((uint32_t)x.b << 16); }
__device__ __forceinline__ float to_float(Half x) { return (float)__builtin_bit_cast(_Float16, x.b); }
__device__ __forceinline__ void from_float(float v, float &o) { o = v; }
__device__ __forceinline__ void from_float(float v, Brain &o) { o.b = __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ void from_float(float v, Half &o) { o.b = __builtin_bit_cast(uint16_t, (_Float16)v); }

// 16 bytes of a row, at its elements' alignment
template <class T>
struct Pack {
  static constexpr int n = 16 / sizeof(T);
  T v[n];
};

}  // namespace fusion
