// Activations saved in 8 bits: int8 codes with one fp32 scale per row and block of 64 columns.
#pragma once

#include "common.cuh"
#include "ptx_float.cuh"

namespace qb {

constexpr int kCheckpointBlock = QB_CHECKPOINT_BLOCK;
inline __host__ __device__ int64_t checkpoint_blocks(int64_t K) { return (K + kCheckpointBlock - 1) / kCheckpointBlock; }

__device__ __forceinline__ float checkpoint_scale(float top) {
  if (!(top < INFINITY)) return __int_as_float(0x7fffffff);  // a NaN or an infinity: the block restores as NaN
  if (top < 7.8886091e-31f) return 1.0f;                     // below 2^-100 it counts as zeros
  return fminf(top / 127.0f, __int_as_float(0x7c010203));    // 127 times the largest scale is still finite
}
// The codes of such a block, from quotients of 32 bits: step is 128 / top and scale 127 / top within 2^-22 of themselves (both 0 where every code is 0).
struct CheckpointCodes {
  float step, scale, top;
  __device__ __forceinline__ explicit CheckpointCodes(float top) : top(top) {
    // of top * 2^-6, so that the reciprocal of the largest numbers is not a subnormal one
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(top * 0.015625f));
    r = top >= 7.8886091e-31f && top < INFINITY ? r : 0.0f;
    step = r * 2.0f;
    scale = r * 1.984375f;
  }
  // Two quotients rounded to nearest even, by an addition that leaves nothing behind the point: a code is the low byte.
  static constexpr float kShift = 12582912.0f;  // 1.5 * 2^23
  __device__ __forceinline__ uint64_t shifted(uint64_t x) const { return ptx::fma_f32x2(x, ptx::pack_f32x2(scale, scale), ptx::pack_f32x2(kShift, kShift)); }
  // The same for x and top of at most 11 bits (16-bit types): 127 x is exact, so that one correction of the quotient by what it leaves of
  // 127 x gives the exact one, rounded once.  A quotient of such numbers that is not on the border of two codes is more than 2^-20 of
  // itself from it: the code is that of the exact quotient.
  __device__ __forceinline__ uint64_t exact16(uint64_t x) const {
    const uint64_t p = ptx::mul_f32x2(x, ptx::pack_f32x2(scale, scale));
    const float minus = top * -0.0078125f;  // all of it over 128: 127 x may be too large for fp32
    const uint64_t left = ptx::fma_f32x2(p, ptx::pack_f32x2(minus, minus), ptx::mul_f32x2(x, ptx::pack_f32x2(0.9921875f, 0.9921875f)));
    return ptx::add_f32x2(ptx::fma_f32x2(left, ptx::pack_f32x2(step, step), p), ptx::pack_f32x2(kShift, kShift));
  }
  static __device__ __forceinline__ uint32_t bytes4(uint64_t lo, uint64_t hi) {
    const float2 a = ptx::unpack_f32x2(lo), b = ptx::unpack_f32x2(hi);
    const uint32_t l = __byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040), h = __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040);
    return __byte_perm(l, h, 0x5410);
  }
  __device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) const {
    return bytes4(shifted(ptx::pack_f32x2(a, b)), shifted(ptx::pack_f32x2(c, d)));
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
