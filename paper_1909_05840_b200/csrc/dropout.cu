// qb_dropout: y = (keep ? x / (1 - p) : 0) + residual, the mask made anew from a counter wherever it is needed.
//
// Word i % 4 of Philox4x32 with seven rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// SC 2011; seven is the least number of rounds that passes their whole battery of tests), counter
// (i / 4, offset + call) and key = seed, decides element i: it is kept when the word is at least p * 2^32.  The mask depends
// on the index alone, so that the backward pass is the same call on the gradient and nothing is stored.
//
// Bound by memory: one read (two with a residual) and one write; at 16 bits without a residual by the generator's instructions
// (17 per element; ALU and multiplier pipes 60 % busy, DRAM at 4.4 TB/s, warps waiting for the pipes).  24,576 x 4,096: fp32 117 us
// (6.9 TB/s), fp16 77 us (5.2 TB/s), fp16 with a residual 87 us (7.0 TB/s).  Two vectors of 16 bytes a thread and eight blocks an SM:
// with one vector fp16 took 88 us, with four 79 and, with a residual, 95 to 149.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "common.cuh"

namespace qb {

struct DropArgs {
  const uint64_t* rng;  // dev [2]: seed, offset
  uint64_t call;
  uint32_t last;       // the largest word that drops: round(p * 2^32) - 1 (round(p * 2^32) may be 2^32, and nothing is kept)
  float scale;         // 1 / (1 - p)
};

// Seven rounds for counters that differ in their low word alone: what the other words and the keys give in the first rounds is
// formed once per thread (25 instead of 28 products and xors per four elements, and no key arithmetic).
struct Philox7 {
  uint32_t x1, y2, z2, w3, k0[5], k1[4];
  __device__ __forceinline__ void start(uint64_t seed, uint64_t sub, uint32_t c1) {
    uint32_t a = (uint32_t)seed, b = (uint32_t)(seed >> 32);
    const uint64_t p1 = (uint64_t)(uint32_t)sub * 0xCD9E8D57u;  // round 1: the third word
    x1 = (uint32_t)(sub >> 32) ^ b;
    const uint64_t p2 = (uint64_t)((uint32_t)(p1 >> 32) ^ c1 ^ a) * 0xD2511F53u;  // round 2: what the first word has become
    a += 0x9E3779B9u;
    b += 0xBB67AE85u;
    y2 = (uint32_t)p1 ^ a;
    z2 = (uint32_t)(p2 >> 32) ^ b;
    a += 0x9E3779B9u;
    b += 0xBB67AE85u;
    w3 = (uint32_t)p2 ^ b;
#pragma unroll
    for (int r = 0; r < 5; ++r) {
      k0[r] = a;
      if (r > 0) k1[r - 1] = b;
      a += 0x9E3779B9u;
      b += 0xBB67AE85u;
    }
  }
  __device__ __forceinline__ uint4 words(uint32_t c0) const {
    const uint64_t a1 = (uint64_t)c0 * 0xD2511F53u;
    const uint64_t b2 = (uint64_t)((uint32_t)(a1 >> 32) ^ x1) * 0xCD9E8D57u;
    uint32_t w0 = (uint32_t)(b2 >> 32) ^ y2, w1 = (uint32_t)b2, w2 = (uint32_t)a1 ^ z2, w3_;
    {
      const uint64_t a = (uint64_t)w0 * 0xD2511F53u, b = (uint64_t)w2 * 0xCD9E8D57u;
      w0 = (uint32_t)(b >> 32) ^ w1 ^ k0[0];
      w1 = (uint32_t)b;
      w2 = (uint32_t)(a >> 32) ^ w3;
      w3_ = (uint32_t)a;
    }
#pragma unroll
    for (int r = 1; r < 5; ++r) {
      const uint64_t a = (uint64_t)w0 * 0xD2511F53u, b = (uint64_t)w2 * 0xCD9E8D57u;
      w0 = (uint32_t)(b >> 32) ^ w1 ^ k0[r];
      w1 = (uint32_t)b;
      w2 = (uint32_t)(a >> 32) ^ w3_ ^ k1[r - 1];
      w3_ = (uint32_t)a;
    }
    return make_uint4(w0, w1, w2, w3_);
  }
};

// Two neighbouring elements at a time: one conversion instruction rounds and packs both.
template <class T>
__device__ __forceinline__ float2 pair_to_float(const T* e) {
  if constexpr (std::is_same_v<T, float>) return make_float2(e[0], e[1]);
  else if constexpr (std::is_same_v<T, __half>) return __half22float2(__halves2half2(e[0], e[1]));
  else return __bfloat1622float2(__halves2bfloat162(e[0], e[1]));
}
template <class T>
__device__ __forceinline__ void pair_from_float(T* e, float2 f) {
  if constexpr (std::is_same_v<T, float>) {
    e[0] = f.x;
    e[1] = f.y;
  } else if constexpr (std::is_same_v<T, __half>) {
    const __half2 h = __floats2half2_rn(f.x, f.y);
    e[0] = __low2half(h);
    e[1] = __high2half(h);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    e[0] = __low2bfloat16(h);
    e[1] = __high2bfloat16(h);
  }
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
constexpr int kDropUnroll = 2;  // vectors of 16 bytes that a thread has in flight

// A block takes kDropThreads * kDropUnroll vectors and ends.  DROP: p > 0 (with p = 0 nothing is drawn).  RES: a residual is
// added.
template <class T, bool VECTOR, bool DROP, bool RES>
__global__ void __launch_bounds__(kDropThreads, 8) dropout_kernel(const T* x, const T* residual, T* y, int64_t n, DropArgs a) {
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
  // a block's counters have one high word: its share of them is a power of two, and aligned to it
  constexpr int kCounters = kDropThreads * U * V / 4;
  static_assert((kCounters & (kCounters - 1)) == 0, "counters of a block");
  Philox7 philox;
  if constexpr (DROP) philox.start(a.rng[0], a.rng[1] + a.call, (uint32_t)((uint64_t)blockIdx.x * kCounters >> 32));
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t at = base + (int64_t)u * (kDropThreads * V);
    if (at >= n) return;
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
      uint32_t w[4] = {0, 0, 0, 0};
      if constexpr (DROP) {
        const uint4 d = philox.words((uint32_t)(at / 4) + q);
        w[0] = d.x;
        w[1] = d.y;
        w[2] = d.z;
        w[3] = d.w;
      }
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        float2 f = pair_to_float(&v[u].e[4 * q + j]);
        // a select, not a product with 0: what is dropped may be infinite or NaN
        if constexpr (DROP) {
          f.x = w[j] > a.last ? __fmul_rn(f.x, a.scale) : 0.0f;
          f.y = w[j + 1] > a.last ? __fmul_rn(f.y, a.scale) : 0.0f;
        }
        if constexpr (RES) {
          const float2 g = pair_to_float(&r[u].e[4 * q + j]);
          f.x = __fadd_rn(f.x, g.x);
          f.y = __fadd_rn(f.y, g.y);
        }
        pair_from_float(&v[u].e[4 * q + j], f);
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
  const unsigned grid = (unsigned)((n + per_block - 1) / per_block);  // n <= 2^40: at most 2^29 blocks
  QB_CUDA_TRY(launch_kernel<kMostL1>(kernel, grid, kDropThreads, 0, stream, 1, false, static_cast<const T*>(x), static_cast<const T*>(residual),
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
  const double threshold = std::rint(p * 4294967296.0);  // 0: nothing is dropped
  a.last = (uint32_t)std::max(threshold - 1.0, 0.0);
  a.scale = (float)(1.0 / (1.0 - p));
  const bool vector = all % 16 == 0;  // else the elements one by one: same values
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  switch (type) {
    case QB_F32: return qb::launch_dropout<float>(x, residual, y, n, vector, threshold > 0.0, a, stream);
    case QB_BF16: return qb::launch_dropout<__nv_bfloat16>(x, residual, y, n, vector, threshold > 0.0, a, stream);
    default: return qb::launch_dropout<__half>(x, residual, y, n, vector, threshold > 0.0, a, stream);
  }
}
