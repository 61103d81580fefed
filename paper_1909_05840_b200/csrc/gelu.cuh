// GELU x * Phi(x) (Phi the distribution function of the normal distribution) and its derivative, two values at a time.
//
// With u = |x| and e = exp(-x^2 / 2), Phi(-u) = e * R(u), where R (the Mills ratio over sqrt(2 pi)) falls smoothly from 1/2; and so
//     gelu(x) = max(x, 0) - u * e * R(u),        gelu'(x) = [x >= 0] + sign(x) * e * (u / sqrt(2 pi) - R(u)).
// R is a polynomial of degree 11 in u, fitted here to the function on 0 <= u <= 5.75 for the least largest of
// max(u, 1) * e * |error| / 1.5e-7 and |error / R| / 2^-12: one exponential and no division per value.  Beyond 5.75 u counts as 5.75 there
// (gelu is then below 5e-8 or within that of x).  Against 64 bits: gelu is off by at most 4e-7 and 2^-23 of its value where x > 0, for x
// < 0 by 2^-10 of its value or 4e-7, whichever is less (down to -5.75); gelu' by at most 4e-7
// (measured: 3.1e-7, 6.5e-4 of the value, 3.0e-7).  Infinities and NaN come out as the limits.
#pragma once

#include "ptx_float.cuh"

namespace qb {

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The terms of P pairs at a time, step by step for all of them: a pair's chain is some thirty dependent instructions, and one or two warps
// of a scheduler do not hide it.
template <int P>
struct GeluTerms {
  uint64_t u[P], e[P];  // min(|x|, 5.75), exp(-x^2 / 2)
  __device__ __forceinline__ explicit GeluTerms(const float* x) {
    const float half_log2e = -0.72134752f;
    const uint64_t scale = ptx::pack_f32x2(half_log2e, half_log2e);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const uint64_t v = ptx::pack_f32x2(x[2 * i], x[2 * i + 1]);
      e[i] = ptx::mul_f32x2(ptx::mul_f32x2(v, v), scale);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const float2 f = ptx::unpack_f32x2(e[i]);
      e[i] = ptx::pack_f32x2(exp2_approx(f.x), exp2_approx(f.y));
    }
#pragma unroll
    for (int i = 0; i < P; ++i) u[i] = ptx::pack_f32x2(fminf(fabsf(x[2 * i]), 5.75f), fminf(fabsf(x[2 * i + 1]), 5.75f));
  }
  // c0 + c1 u + (R's terms from the second degree on, with their signs turned)
  __device__ __forceinline__ void poly(float c0, float c1, uint64_t (&p)[P]) const {
    constexpr float c[10] = {-0.24984169006347656f, 0.13220742344856262f,    -0.06054938957095146f,  0.023666609078645706f,  -0.0075540607795119286f,
                             0.0018558446317911148f, -0.0003288344305474311f, 3.888118953909725e-05f, -2.715689788601594e-06f, 8.416543550993083e-08f};
#pragma unroll
    for (int i = 0; i < P; ++i) p[i] = ptx::fma_f32x2(u[i], ptx::pack_f32x2(c[9], c[9]), ptx::pack_f32x2(c[8], c[8]));
#pragma unroll
    for (int k = 7; k >= -2; --k) {
      const float f = k >= 0 ? c[k >= 0 ? k : 0] : (k == -1 ? c1 : c0);
#pragma unroll
      for (int i = 0; i < P; ++i) p[i] = ptx::fma_f32x2(p[i], u[i], ptx::pack_f32x2(f, f));
    }
  }
};
// gelu of 2 P values, in place
template <int P>
__device__ __forceinline__ void gelu_many(float* x) {
  const GeluTerms<P> t(x);
  uint64_t r[P];
  t.poly(-0.4999998211860657f, 0.3989296555519104f, r);  // -R
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const float2 f = ptx::unpack_f32x2(ptx::fma_f32x2(ptx::mul_f32x2(t.u[i], t.e[i]), r[i], ptx::pack_f32x2(fmaxf(x[2 * i], 0.0f), fmaxf(x[2 * i + 1], 0.0f))));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
// gelu' of 2 P values times g, in place of g: [x >= 0] + sign(x) s as 1/2 + sign(x) (1/2 + s)
template <int P>
__device__ __forceinline__ void times_gelu_slope(const float* x, float* g) {
  const GeluTerms<P> t(x);
  uint64_t r[P];
  t.poly(-0.4999998211860657f, 0.3989296555519104f + 0.39894228f, r);  // u / sqrt(2 pi) - R
  const uint64_t half = ptx::pack_f32x2(0.5f, 0.5f);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const float2 s = ptx::unpack_f32x2(ptx::fma_f32x2(t.e[i], r[i], half));
    const uint64_t slope = ptx::add_f32x2(ptx::pack_f32x2(copysignf(s.x, x[2 * i]), copysignf(s.y, x[2 * i + 1])), half);
    const float2 f = ptx::unpack_f32x2(ptx::mul_f32x2(slope, ptx::pack_f32x2(g[2 * i], g[2 * i + 1])));
    g[2 * i] = f.x;
    g[2 * i + 1] = f.y;
  }
}

}  // namespace qb
