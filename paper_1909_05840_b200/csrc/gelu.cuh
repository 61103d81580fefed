// GELU x * Phi(x) (Phi the distribution function of the normal distribution) and its derivative, two values at a time.
//
// With u = |x| and e = exp(-x^2 / 2), Phi(-u) = e * R(u), where R (the Mills ratio over sqrt(2 pi)) falls smoothly from 1/2; and so
//     gelu(x) = max(x, 0) - u * e * R(u),        gelu'(x) = [x >= 0] + sign(x) * e * (u / sqrt(2 pi) - R(u)).
// R is a polynomial of degree 11 in u, fitted here to the function on 0 <= u <= 5.75 for the least largest of
// max(u, 1) * e * |error| / 1.5e-7 and |error / R| / 2^-12: one exponential and no division per value.  Beyond 5.75 u counts as 5.75 there
// (gelu is then below 5e-8 or within that of x).  Against 64 bits: gelu is off by at most 4e-7 and 2^-23 of its value where x > 0, for x
// < 0 by 2^-10 of its value or 4e-7, whichever is less (down to -5.75); gelu' by at most 4e-7.  Infinities and NaN come out as the limits.
#pragma once

#include "ptx_float.cuh"

namespace qb {

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

struct GeluTerms {
  uint64_t u, e;  // min(|x|, 5.75), exp(-x^2 / 2)
};
__device__ __forceinline__ GeluTerms gelu_terms(float a, float b) {
  GeluTerms t;
  t.u = ptx::pack_f32x2(fminf(fabsf(a), 5.75f), fminf(fabsf(b), 5.75f));
  const uint64_t x = ptx::pack_f32x2(a, b);
  const float half_log2e = -0.72134752f;
  const float2 p = ptx::unpack_f32x2(ptx::mul_f32x2(ptx::mul_f32x2(x, x), ptx::pack_f32x2(half_log2e, half_log2e)));
  t.e = ptx::pack_f32x2(exp2_approx(p.x), exp2_approx(p.y));
  return t;
}
// c0 + c1 u + (R's terms from the second degree on, with their signs turned)
__device__ __forceinline__ uint64_t gelu_poly(uint64_t u, float c0, float c1) {
  constexpr float c[10] = {-0.24984169006347656f, 0.13220742344856262f,    -0.06054938957095146f,  0.023666609078645706f,  -0.0075540607795119286f,
                           0.0018558446317911148f, -0.0003288344305474311f, 3.888118953909725e-05f, -2.715689788601594e-06f, 8.416543550993083e-08f};
  uint64_t p = ptx::pack_f32x2(c[9], c[9]);
#pragma unroll
  for (int i = 8; i >= 0; --i) p = ptx::fma_f32x2(p, u, ptx::pack_f32x2(c[i], c[i]));
  p = ptx::fma_f32x2(p, u, ptx::pack_f32x2(c1, c1));
  return ptx::fma_f32x2(p, u, ptx::pack_f32x2(c0, c0));
}
// gelu of both values
__device__ __forceinline__ float2 gelu2(float a, float b) {
  const GeluTerms t = gelu_terms(a, b);
  const uint64_t r = gelu_poly(t.u, -0.4999998211860657f, 0.3989296555519104f);  // -R
  return ptx::unpack_f32x2(ptx::fma_f32x2(ptx::mul_f32x2(t.u, t.e), r, ptx::pack_f32x2(fmaxf(a, 0.0f), fmaxf(b, 0.0f))));
}
// gelu' of both values
__device__ __forceinline__ float2 gelu_slope2(float a, float b) {
  const GeluTerms t = gelu_terms(a, b);
  const float2 s = ptx::unpack_f32x2(ptx::mul_f32x2(t.e, gelu_poly(t.u, -0.4999998211860657f, 0.3989296555519104f + 0.39894228f)));  // e (u / sqrt(2 pi) - R)
  return make_float2(a < 0.0f ? -s.x : 1.0f + s.x, b < 0.0f ? -s.y : 1.0f + s.y);
}

}  // namespace qb
