// qb_checkpoint, qb_restore, qb_gelu_backward: activations saved in 8 bits with a scale per row and block of 64 columns, and their use.
//
// A block's 64 values lie in 8 (16-bit types) or 16 (fp32) neighbouring lanes, 16 bytes each, which agree on the largest magnitude by
// shuffles; codes are rounded in 32 bits, and again in 64 where the quotient lies next to the border of two of them.
// Bound by memory: one read and one write of each tensor.
#include "checkpoint.cuh"
#include "common.cuh"
#include "gelu.cuh"
#include "vec16.cuh"

#include <algorithm>

namespace qb {

constexpr int kCheckpointThreads = 256;
constexpr int kCheckpointUnroll = 4;  // vectors that a thread has in flight

// Where vector `v` of a matrix of `blocks` blocks a row lies.  FLAT: rows are whole blocks, so that vectors follow one another.
template <int N, bool FLAT>
struct CheckpointAt {
  int64_t element, block, left;  // left: elements of the row from here on
  __device__ __forceinline__ CheckpointAt(int64_t v, int64_t K, int64_t blocks) {
    constexpr int kPer = kCheckpointBlock / N;
    block = v / kPer;
    if constexpr (FLAT) {
      element = v * N;
      left = N;
    } else {
      const int64_t row = (block | blocks) >> 32 ? block / blocks : (int64_t)((uint32_t)block / (uint32_t)blocks), col = (block - row * blocks) * kCheckpointBlock + (v % kPer) * N;
      element = row * K + col;
      left = K - col;
    }
  }
};

// The codes of N values as bytes.
template <int N>
__device__ __forceinline__ void store_codes(int8_t* p, const uint32_t (&w)[N / 4], int64_t left, bool vector) {
  if (vector) {
    if (left > 0) {
      if constexpr (N == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
      else *reinterpret_cast<uint32_t*>(p) = w[0];
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < left) p[j] = (int8_t)(w[j >> 2] >> (8 * (j & 3)));
  }
}
template <int N>
__device__ __forceinline__ void load_codes(const int8_t* p, uint32_t (&w)[N / 4], int64_t left, bool vector) {
#pragma unroll
  for (int j = 0; j < N / 4; ++j) w[j] = 0;
  if (vector) {
    if (left > 0) {
      if constexpr (N == 8) {
        const uint2 q = *reinterpret_cast<const uint2*>(p);
        w[0] = q.x;
        w[1] = q.y;
      } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < left) w[j >> 2] |= (uint32_t)(uint8_t)p[j] << (8 * (j & 3));
  }
}

// Codes whose 32-bit quotient may lie on the wrong side of a border, from the quotient in 64 bits (its error is far below the least
// distance of a quotient of two 24-bit numbers from a border that it does not lie on).
template <int N>
__device__ __noinline__ void exact_codes(const float (&f)[N], float top, uint32_t (&w)[N / 4]) {
#pragma unroll
  for (int j = 0; j < N / 4; ++j) w[j] = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) w[j >> 2] |= (uint32_t)(uint8_t)(int8_t)__double2int_rn((double)f[j] * 127.0 / (double)top) << (8 * (j & 3));
}

template <class T, bool FLAT, bool VECTOR>
__global__ void __launch_bounds__(kCheckpointThreads) checkpoint_kernel(const T* x, int8_t* codes, float* scales, int64_t vectors, int64_t K, int64_t blocks) {
  constexpr int N = Vec16<T>::N, kPer = kCheckpointBlock / N, U = kCheckpointUnroll;
  pdl_begin();
  const int64_t base = (int64_t)blockIdx.x * (kCheckpointThreads * U) + threadIdx.x;
  Vec16<T> v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = base + u * kCheckpointThreads;
    if (i < vectors) {
      const CheckpointAt<N, FLAT> at(i, K, blocks);
      v[u].template load<VECTOR>(x + at.element, at.left);
    } else {
      v[u].raw = make_uint4(0u, 0u, 0u, 0u);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float f[N];
    v[u].get(f);
    float top = 0.0f;
#pragma unroll
    for (int j = 0; j < N; j += 2) top = max3_nan(top, fabsf(f[j]), fabsf(f[j + 1]));
#pragma unroll
    for (int d = 1; d < kPer; d *= 2) top = max3_nan(top, __shfl_xor_sync(0xffffffffu, top, d), 0.0f);
    const int64_t i = base + u * kCheckpointThreads;
    if (i < vectors) {
      const CheckpointAt<N, FLAT> at(i, K, blocks);
      const CheckpointScale cs(top);
      float far = 0.0f;  // the largest distance of a quotient from its code
#pragma unroll
      for (int j = 0; j < N; ++j) far = fmaxf(far, fabsf(__fmaf_rn(f[j], cs.inv, CheckpointScale::kShift - cs.shifted(f[j]))));
      uint32_t w[N / 4];
#pragma unroll
      for (int j = 0; j < N / 4; ++j) w[j] = cs.codes4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]);
      // x * inv is off by 127 * 2^-24 at most
      if (far > 0.5f - 1.0e-5f) exact_codes(f, top, w);
      store_codes<N>(codes + at.element, w, at.left, VECTOR);
      if (i % kPer == 0) scales[at.block] = cs.scale;
    }
  }
}

// What is formed from the saved value p: itself, gelu(p), grad_y * gelu'(p).
enum ActivationUse { kValue = 0, kActivation = 1, kSlopeOf = 2 };

// CODES: p from codes and scales, else from `pre`.
template <class T, int USE, bool CODES, bool FLAT, bool VECTOR>
__global__ void __launch_bounds__(kCheckpointThreads) activation_kernel(const T* grad_y, const T* pre, const int8_t* codes, const float* scales, T* y, int64_t vectors,
                                                                        int64_t K, int64_t blocks) {
  constexpr int N = Vec16<T>::N, U = kCheckpointUnroll;
  pdl_begin();
  const int64_t base = (int64_t)blockIdx.x * (kCheckpointThreads * U) + threadIdx.x;
  Vec16<T> g[USE == kSlopeOf ? U : 1], v[CODES ? 1 : U];
  uint32_t w[CODES ? U : 1][N / 4];
  float scale[CODES ? U : 1];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = base + u * kCheckpointThreads;
    if (i < vectors) {
      const CheckpointAt<N, FLAT> at(i, K, blocks);
      if constexpr (USE == kSlopeOf) g[u].template load<VECTOR>(grad_y + at.element, at.left);
      if constexpr (CODES) {
        load_codes<N>(codes + at.element, w[u], at.left, VECTOR);
        scale[u] = scales[at.block];
      } else {
        v[u].template load<VECTOR>(pre + at.element, at.left);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = base + u * kCheckpointThreads;
    if (i >= vectors) return;
    float p[N], d[N];
    if constexpr (CODES) {
#pragma unroll
      for (int j = 0; j < N / 4; ++j) code_values(w[u][j], scale[u], p + 4 * j);
    } else {
      v[u].get(p);
    }
    if constexpr (USE == kActivation) gelu_many<N / 2>(p);
    if constexpr (USE == kSlopeOf) {
      g[u].get(d);
      times_gelu_slope<N / 2>(p, d);
    }
    const CheckpointAt<N, FLAT> at(i, K, blocks);
    Vec16<T> out;
    out.set(USE == kSlopeOf ? d : p);
    out.template store<VECTOR>(y + at.element, at.left);
  }
}

template <class T>
struct CheckpointShape {
  int64_t vectors, blocks;
  unsigned grid;
  bool flat, vector;
  CheckpointShape(int64_t M, int64_t K, bool aligned) {
    constexpr int N = Vec16<T>::N;
    blocks = checkpoint_blocks(K);
    vectors = M * blocks * (kCheckpointBlock / N);
    constexpr int64_t per = (int64_t)kCheckpointThreads * kCheckpointUnroll;
    grid = (unsigned)((vectors + per - 1) / per);
    vector = aligned && K % N == 0;
    flat = vector && K % kCheckpointBlock == 0;
  }
};

template <class T>
static qb_status launch_checkpoint(const void* x, int64_t M, int64_t K, int8_t* codes, float* scales, cudaStream_t stream) {
  const CheckpointShape<T> s(M, K, aligned16(x));
  auto kernel = s.flat ? checkpoint_kernel<T, true, true> : (s.vector ? checkpoint_kernel<T, false, true> : checkpoint_kernel<T, false, false>);
  QB_CUDA_TRY(launch_kernel<kMostL1>(kernel, s.grid, kCheckpointThreads, 0, stream, 1, false, static_cast<const T*>(x), codes, scales, s.vectors, K, s.blocks));
  return QB_OK;
}
template <class T, int USE, bool CODES>
static qb_status launch_activation(const void* grad_y, const void* pre, const int8_t* codes, const float* scales, int64_t M, int64_t K, void* y, cudaStream_t stream) {
  const CheckpointShape<T> s(M, K, aligned16(grad_y) && aligned16(pre) && aligned16(y));
  auto kernel = s.flat ? activation_kernel<T, USE, CODES, true, true>
                       : (s.vector ? activation_kernel<T, USE, CODES, false, true> : activation_kernel<T, USE, CODES, false, false>);
  QB_CUDA_TRY(launch_kernel<kMostL1>(kernel, s.grid, kCheckpointThreads, 0, stream, 1, false, static_cast<const T*>(grad_y), static_cast<const T*>(pre), codes, scales,
                                     static_cast<T*>(y), s.vectors, K, s.blocks));
  return QB_OK;
}

static bool impossible_checkpoint(int64_t M, int64_t K) {
  return M <= 0 || K <= 0 || K > QB_MAX_ELEMENTS || checkpoint_blocks(K) > QB_MAX_ELEMENTS / kCheckpointBlock / M;
}
static qb_status check_checkpoint(const char* what, bool pointers, int type, int64_t M, int64_t K) {
  if (pointers && type >= QB_F32 && type <= QB_F16 && !impossible_checkpoint(M, K)) return QB_OK;
  set_last_error("%s: invalid argument (M=%lld K=%lld type=%d)", what, (long long)M, (long long)K, type);
  return QB_ERR_INVALID;
}
static bool to_elements(const void* p, int type) { return reinterpret_cast<uintptr_t>(p) % (type == QB_F32 ? 4 : 2) == 0; }

}  // namespace qb

extern "C" qb_status qb_checkpoint(const void* x, int type, int64_t M, int64_t K, int8_t* codes, float* scales, void* cuda_stream) {
  using namespace qb;
  qb_status st = check_checkpoint("qb_checkpoint", x && codes && scales, type, M, K);
  if (st != QB_OK) return st;
  if (!to_elements(x, type) || !aligned16(codes) || !to_elements(scales, QB_F32)) {
    set_last_error("qb_checkpoint: x and scales must be aligned to their elements, codes to 16 bytes");
    return QB_ERR_ALIGN;
  }
  if ((st = require_sm100(nullptr)) != QB_OK) return st;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  switch (type) {
    case QB_F32: return launch_checkpoint<float>(x, M, K, codes, scales, stream);
    case QB_BF16: return launch_checkpoint<__nv_bfloat16>(x, M, K, codes, scales, stream);
    default: return launch_checkpoint<__half>(x, M, K, codes, scales, stream);
  }
}

extern "C" qb_status qb_restore(const int8_t* codes, const float* scales, int64_t M, int64_t K, int activation, int type, void* y, void* cuda_stream) {
  using namespace qb;
  qb_status st = check_checkpoint("qb_restore", codes && scales && y && activation >= QB_IDENTITY && activation <= QB_GELU, type, M, K);
  if (st != QB_OK) return st;
  if (!aligned16(codes) || !to_elements(scales, QB_F32) || !to_elements(y, type)) {
    set_last_error("qb_restore: codes must be 16-byte aligned, scales and y aligned to their elements");
    return QB_ERR_ALIGN;
  }
  if ((st = require_sm100(nullptr)) != QB_OK) return st;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  const auto run = [&](auto zero) {
    using T = decltype(zero);
    return activation == QB_GELU ? launch_activation<T, kActivation, true>(nullptr, nullptr, codes, scales, M, K, y, stream)
                                 : launch_activation<T, kValue, true>(nullptr, nullptr, codes, scales, M, K, y, stream);
  };
  switch (type) {
    case QB_F32: return run(float());
    case QB_BF16: return run(__nv_bfloat16());
    default: return run(__half());
  }
}

extern "C" qb_status qb_gelu_backward(const void* grad_y, int type, const void* pre, const int8_t* pre_codes, const float* pre_scales, int64_t M, int64_t K,
                                      void* grad_x, void* cuda_stream) {
  using namespace qb;
  const bool one = pre ? !pre_codes && !pre_scales : pre_codes && pre_scales;
  qb_status st = check_checkpoint("qb_gelu_backward", grad_y && grad_x && one, type, M, K);
  if (st != QB_OK) return st;
  if (!to_elements(grad_y, type) || !to_elements(grad_x, type) || !to_elements(pre, type) || !aligned16(pre_codes) || !to_elements(pre_scales, QB_F32)) {
    set_last_error("qb_gelu_backward: codes must be 16-byte aligned, the others aligned to their elements");
    return QB_ERR_ALIGN;
  }
  if ((st = require_sm100(nullptr)) != QB_OK) return st;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  const auto run = [&](auto zero) {
    using T = decltype(zero);
    return pre ? launch_activation<T, kSlopeOf, false>(grad_y, pre, nullptr, nullptr, M, K, grad_x, stream)
               : launch_activation<T, kSlopeOf, true>(grad_y, nullptr, pre_codes, pre_scales, M, K, grad_x, stream);
  };
  switch (type) {
    case QB_F32: return run(float());
    case QB_BF16: return run(__nv_bfloat16());
    default: return run(__half());
  }
}
