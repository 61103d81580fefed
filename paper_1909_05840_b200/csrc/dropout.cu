// qb_dropout: y = (keep ? x / (1 - p) : 0) + residual, the mask made anew from a counter wherever it is needed.
//
// Word i % 4 of Philox4x32 with seven rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// SC 2011; seven is the least number of rounds that passes their whole battery of tests), counter
// (i / 4, offset + call) and key = seed, decides element i: it is kept when the word is at least p * 2^32.  The mask depends
// on the index alone, so that the backward pass is the same call on the gradient and nothing is stored.
//
// Bound by memory: one read (two with a residual) and one write.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "common.cuh"

namespace qb {

struct DropArgs {
  const uint64_t* rng;  // dev [2]: seed, offset
  uint64_t call;
  uint32_t threshold;  // keep when word >= threshold
  float scale;         // 1 / (1 - p)
};

__device__ __forceinline__ uint4 philox4x32_7(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

template <class T>
__device__ __forceinline__ float to_float(T v) {
  if constexpr (std::is_same_v<T, float>) return v;
  else if constexpr (std::is_same_v<T, __half>) return __half2float(v);
  else return __bfloat162float(v);
}
template <class T>
__device__ __forceinline__ T from_float(float v) {
  if constexpr (std::is_same_v<T, float>) return v;
  else if constexpr (std::is_same_v<T, __half>) return __float2half_rn(v);
  else return __float2bfloat16_rn(v);
}

// One vector of V elements at 16 bytes (VECTOR) or one element after the other.
template <class T, int V, bool VECTOR>
struct Vec {
  union {
    uint4 raw;
    T e[V];
  };
  __device__ __forceinline__ Vec() {}
  __device__ __forceinline__ void load(const T* p, int64_t left) {
    if constexpr (VECTOR) {
      if (left >= V) {
        raw = *reinterpret_cast<const uint4*>(p);
        return;
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j < left) e[j] = p[j];
  }
  __device__ __forceinline__ void store(T* p, int64_t left) const {
    if constexpr (VECTOR) {
      if (left >= V) {
        *reinterpret_cast<uint4*>(p) = raw;
        return;
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j < left) p[j] = e[j];
  }
};

constexpr int kDropThreads = 256;
constexpr int kDropUnroll = 4;  // vectors of 16 bytes that a thread has in flight

// A block takes kDropThreads * kDropUnroll vectors and ends.  DROP: p > 0 (with p = 0 nothing is drawn).  RES: a residual is
// added.
template <class T, bool VECTOR, bool DROP, bool RES>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const T* x, const T* residual, T* y, int64_t n, DropArgs a) {
  constexpr int V = 16 / sizeof(T), U = kDropUnroll;
  pdl_begin();
  const int64_t base = ((int64_t)blockIdx.x * (kDropThreads * U) + threadIdx.x) * V;
  Vec<T, V, VECTOR> v[U], r[RES ? U : 1];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t at = base + (int64_t)u * (kDropThreads * V);
    if (at < n) {
      v[u].load(x + at, n - at);
      if constexpr (RES) r[u].load(residual + at, n - at);
    }
  }
  uint32_t k0 = 0, k1 = 0, c2 = 0, c3 = 0;
  if constexpr (DROP) {
    const uint64_t seed = a.rng[0], sub = a.rng[1] + a.call;
    k0 = (uint32_t)seed;
    k1 = (uint32_t)(seed >> 32);
    c2 = (uint32_t)sub;
    c3 = (uint32_t)(sub >> 32);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t at = base + (int64_t)u * (kDropThreads * V);
    if (at >= n) return;
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
      uint32_t w[4] = {0, 0, 0, 0};
      if constexpr (DROP) {
        const uint64_t c = (uint64_t)at / 4 + q;
        const uint4 d = philox4x32_7((uint32_t)c, (uint32_t)(c >> 32), c2, c3, k0, k1);
        w[0] = d.x;
        w[1] = d.y;
        w[2] = d.z;
        w[3] = d.w;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float f = to_float(v[u].e[4 * q + j]);
        // a select, not a product with 0: what is dropped may be infinite or NaN
        if constexpr (DROP) f = w[j] >= a.threshold ? __fmul_rn(f, a.scale) : 0.0f;
        if constexpr (RES) f = __fadd_rn(f, to_float(r[u].e[4 * q + j]));
        v[u].e[4 * q + j] = from_float<T>(f);
      }
    }
    v[u].store(y + at, n - at);
  }
}

template <class T>
static qb_status launch_dropout(const void* x, const void* residual, void* y, int64_t n, bool vector, bool drop, const DropArgs& a,
                                cudaStream_t stream) {
  auto kernel = vector ? (drop ? (residual ? dropout_kernel<T, true, true, true> : dropout_kernel<T, true, true, false>)
                               : (residual ? dropout_kernel<T, true, false, true> : dropout_kernel<T, true, false, false>))
                       : (drop ? (residual ? dropout_kernel<T, false, true, true> : dropout_kernel<T, false, true, false>)
                               : (residual ? dropout_kernel<T, false, false, true> : dropout_kernel<T, false, false, false>));
  constexpr int64_t per_block = (int64_t)kDropThreads * kDropUnroll * (16 / sizeof(T));
  const unsigned grid = (unsigned)((n + per_block - 1) / per_block);  // n <= 2^40: at most 2^28 blocks
  QB_CUDA_TRY(launch_kernel(kernel, grid, kDropThreads, 0, stream, 1, false, static_cast<const T*>(x), static_cast<const T*>(residual),
                            static_cast<T*>(y), n, a));
  return QB_OK;
}

}  // namespace qb

extern "C" qb_status qb_dropout(const void* x, int type, int64_t n, double p, const uint64_t* rng, uint64_t call,
                                const void* residual, void* y, void* cuda_stream) {
  if (!x || !y || !rng || n <= 0 || n > QB_MAX_ELEMENTS || !(p >= 0.0 && p < 1.0) || type < QB_F32 || type > QB_F16) {
    qb::set_last_error("qb_dropout: invalid argument (n=%lld p=%g type=%d)", (long long)n, p, type);
    return QB_ERR_INVALID;
  }
  const uintptr_t all = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y) | reinterpret_cast<uintptr_t>(residual);
  if (all % (type == QB_F32 ? 4 : 2) != 0 || reinterpret_cast<uintptr_t>(rng) % 8 != 0) {
    qb::set_last_error("qb_dropout: x, residual and y must be aligned to their elements, rng to 8 bytes");
    return QB_ERR_ALIGN;
  }
  qb_status st = qb::require_sm100(nullptr);
  if (st != QB_OK) return st;
  qb::DropArgs a;
  a.rng = rng;
  a.call = call;
  a.threshold = (uint32_t)std::min(std::rint(p * 4294967296.0), 4294967295.0);
  a.scale = (float)(1.0 / (1.0 - p));
  const bool vector = all % 16 == 0;  // else the elements one by one: same values
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  switch (type) {
    case QB_F32: return qb::launch_dropout<float>(x, residual, y, n, vector, a.threshold != 0, a, stream);
    case QB_BF16: return qb::launch_dropout<__nv_bfloat16>(x, residual, y, n, vector, a.threshold != 0, a, stream);
    default: return qb::launch_dropout<__half>(x, residual, y, n, vector, a.threshold != 0, a, stream);
  }
}
