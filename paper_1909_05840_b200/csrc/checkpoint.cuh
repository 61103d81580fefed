// Activations saved in 8 bits: int8 codes with one fp32 scale per row and block of 64 columns.
#pragma once

#include "common.cuh"

namespace qb {

constexpr int kCheckpointBlock = QB_CHECKPOINT_BLOCK;
inline __host__ __device__ int64_t checkpoint_blocks(int64_t K) { return (K + kCheckpointBlock - 1) / kCheckpointBlock; }

// The scale of a block whose largest magnitude is `top` (NaN where the block has one), and its codes.
struct CheckpointScale {
  float scale, inv;
  __device__ __forceinline__ explicit CheckpointScale(float top) {
    if (!(top < INFINITY)) {  // a NaN or an infinity: the block restores as NaN
      scale = __int_as_float(0x7fffffff);
      inv = 0.0f;
    } else if (top < 7.8886091e-31f) {  // 2^-100: counts as zeros (127 / top would leave fp32's range a little below)
      scale = 1.0f;
      inv = 0.0f;
    } else {
      scale = top / 127.0f;
      inv = 127.0f / top;
    }
  }
  // x * inv rounded to nearest even, by an addition that leaves nothing behind the point: its low byte is the code
  static constexpr float kShift = 12582912.0f;  // 1.5 * 2^23
  __device__ __forceinline__ float shifted(float x) const { return __fmaf_rn(x, inv, kShift); }
  __device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) const {
    const uint32_t lo = __byte_perm(__float_as_uint(shifted(a)), __float_as_uint(shifted(b)), 0x0040);
    const uint32_t hi = __byte_perm(__float_as_uint(shifted(c)), __float_as_uint(shifted(d)), 0x0040);
    return __byte_perm(lo, hi, 0x5410);
  }
};

// Byte `i` of a word of codes as a number.
__device__ __forceinline__ float code_value(uint32_t w, int i) { return (float)(int)(int8_t)(w >> (8 * i)); }

}  // namespace qb
