// Vectors of 16 bytes of fp32, bfloat16 or fp16 elements.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace qb {

template <class T>
__device__ __forceinline__ float to_float(T e) {
  if constexpr (std::is_same_v<T, float>) return e;
  else if constexpr (std::is_same_v<T, __half>) return __half2float(e);
  else return __bfloat162float(e);
}
template <class T>
__device__ __forceinline__ T from_float(float f) {
  if constexpr (std::is_same_v<T, float>) return f;
  else if constexpr (std::is_same_v<T, __half>) return __float2half_rn(f);
  else return __float2bfloat16_rn(f);
}

// 16 / sizeof(T) neighbouring elements.
template <class T>
struct Vec16 {
  static constexpr int N = 16 / sizeof(T);
  uint4 raw;
  // from p (16-byte aligned) where the row has elements left there, which are a multiple of N then; else zeros
  __device__ __forceinline__ void load(const T* p, int64_t left) { raw = left > 0 ? *reinterpret_cast<const uint4*>(p) : make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void store(T* p, int64_t left) const {
    if (left > 0) *reinterpret_cast<uint4*>(p) = raw;
  }
  __device__ __forceinline__ void get(float (&f)[N]) const {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (std::is_same_v<T, float>) {
        f[j] = __uint_as_float(w[j]);
      } else if constexpr (std::is_same_v<T, __half>) {
        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
        f[2 * j] = v.x;
        f[2 * j + 1] = v.y;
      } else {
        f[2 * j] = __uint_as_float(w[j] << 16);
        f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ void set(const float (&f)[N]) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (std::is_same_v<T, float>) {
        w[j] = __float_as_uint(f[j]);
      } else if constexpr (std::is_same_v<T, __half>) {
        const __half2 h = __floats2half2_rn(f[2 * j], f[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&h);
      } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
    raw = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

}  // namespace qb
