// Shared by the training-step operators (include/gd_train.h): element types, 16-byte pieces, small numerics.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gd_internal.cuh"
#include "gd_train.h"

namespace gd {

template <int DT>
struct Elem;
template <>
struct Elem<GD_DTYPE_FP32> {
  using type = float;
  static __device__ __forceinline__ float get(float x) { return x; }
  static __device__ __forceinline__ float put(float x) { return x; }
};
template <>
struct Elem<GD_DTYPE_BF16> {
  using type = __nv_bfloat16;
  static __device__ __forceinline__ float get(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ __nv_bfloat16 put(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct Elem<GD_DTYPE_FP16> {
  using type = __half;
  static __device__ __forceinline__ float get(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half put(float x) { return __float2half_rn(x); }
};

// Two 16-bit elements of a 32-bit word, element 0 in the low half.
template <int DT>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if constexpr (DT == GD_DTYPE_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <int DT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (DT == GD_DTYPE_BF16) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
  }
  const __half2 p = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&p);
}

inline bool is_16bit(int dt) { return dt == GD_DTYPE_BF16 || dt == GD_DTYPE_FP16; }
inline bool is_dtype(int dt) { return dt == GD_DTYPE_FP32 || is_16bit(dt); }
inline size_t dtype_bytes(int dt) { return dt == GD_DTYPE_FP32 ? 4 : 2; }
inline bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

}  // namespace gd
