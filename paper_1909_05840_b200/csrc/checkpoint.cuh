// Activations saved in 8 bits: int8 codes with one fp32 scale per row and block of 64 columns.
#pragma once

#include "common.cuh"
#include "ptx_float.cuh"

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

// Byte `i` of a word of codes as a number: with its sign turned it is the low byte of 2^23 + 128 + code, which costs a permutation and an
// addition (a conversion of a whole number to fp32 takes the pipe of the exponentials).
__device__ __forceinline__ uint32_t turned_codes(uint32_t w) { return w ^ 0x80808080u; }
__device__ __forceinline__ float shifted_code(uint32_t turned, int i) { return __uint_as_float(__byte_perm(turned, 0x4B000000u, 0x7440 | i)); }
constexpr float kCodeShift = 8388736.0f;
// The values of four codes.
__device__ __forceinline__ void code_values(uint32_t word, float scale, float* p) {
  const uint32_t w = turned_codes(word);
  const uint64_t shift = ptx::pack_f32x2(-kCodeShift, -kCodeShift), s = ptx::pack_f32x2(scale, scale);
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const float2 f = ptx::unpack_f32x2(ptx::mul_f32x2(ptx::add_f32x2(ptx::pack_f32x2(shifted_code(w, i), shifted_code(w, i + 1)), shift), s));
    p[i] = f.x;
    p[i + 1] = f.y;
  }
}

}  // namespace qb
