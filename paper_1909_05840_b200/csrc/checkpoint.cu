// qb_checkpoint, qb_restore, qb_gelu_backward: activations saved in 8 bits with a scale per row and block of 64 columns, and their use.
//
// A block's 64 values lie in 8 (16-bit types) or 16 (fp32) neighbouring lanes, 16 bytes each, which agree on the largest magnitude by
// shuffles.  The quotients are exact for 16-bit types; in fp32 they are formed again in 64 bits where they lie next to the border of two codes.
// Bound by memory: one read and one write of each tensor.  24,576 x 4,096: saved from bfloat16 50 us (6.1 TB/s), from fp32 78 (6.6),
// restored to bfloat16 48 (6.4), GELU formed anew 74 (4.1: two thirds of the issue slots, a block's loads and
// arithmetic one after the other), GELU's gradient from codes 80 (6.4).  Codes rounded again in 64 bits
// wherever a 32-bit quotient lies near a border took 127 us in bfloat16: exact halves of the block's maximum are common there, and one
// correction of the quotient decides them.  Rows that are not made of vectors: 5,003 x 1,023 bfloat16 saved in 15.6 us.
#include "checkpoint.cuh"
#include "common.cuh"
#include "gelu.cuh"
#include "vec16.cuh"

#include <algorithm>

namespace qb {

constexpr int kCheckpointThreads = 256;
constexpr int kCheckpointUnroll = 4;  // vectors that a thread has in flight

// Turns of the kernel that saves, two vectors each.
template <class T>
constexpr int kCheckpointTurns = sizeof(T) == 4 ? 4 : 2;

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

// The codes of N values as bytes, where the row has them (left > 0).
template <int N>
__device__ __forceinline__ void store_codes(int8_t* p, const uint32_t (&w)[N / 4], int64_t left) {
  if (left <= 0) return;
  if constexpr (N == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint32_t*>(p) = w[0];
}
template <int N>
__device__ __forceinline__ void load_codes(const int8_t* p, uint32_t (&w)[N / 4], int64_t left) {
#pragma unroll
  for (int j = 0; j < N / 4; ++j) w[j] = 0;
  if (left <= 0) return;
  if constexpr (N == 8) {
    const uint2 q = *reinterpret_cast<const uint2*>(p);
    w[0] = q.x;
    w[1] = q.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// A code whose 32-bit quotient may lie on the wrong side of a border, from the quotient in 64 bits (its error is far below the least
// distance of a quotient of two 24-bit numbers from a border that it does not lie on).
__device__ __forceinline__ int8_t exact_code(float x, float top) { return (int8_t)__double2int_rn((double)x * 127.0 / (double)top); }
constexpr float kNearBorder = 0.5f - 4.0e-5f;  // x * scale is off by 127 * 2^-22 at most

// A thread takes two neighbouring vectors of a block, U times.
template <class T, bool FLAT>
__global__ void __launch_bounds__(kCheckpointThreads) checkpoint_kernel(const T* x, int8_t* codes, float* scales, int64_t vectors, int64_t K, int64_t blocks) {
  constexpr int N = Vec16<T>::N, kPer = kCheckpointBlock / N / 2, U = kCheckpointTurns<T>;
  pdl_begin();
  const int64_t base = ((int64_t)blockIdx.x * (kCheckpointThreads * U) + threadIdx.x) * 2;
  Vec16<T> v[U][2];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = base + u * (2 * kCheckpointThreads);
    if (i < vectors) {
      const CheckpointAt<N, FLAT> at(i, K, blocks);
      v[u][0].load(x + at.element, at.left);
      v[u][1].load(x + at.element + N, at.left - (FLAT ? 0 : N));
    } else {
      v[u][0].raw = v[u][1].raw = make_uint4(0u, 0u, 0u, 0u);
    }
  }
  float top[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    top[u] = 0.0f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float f[N];
      v[u][h].get(f);
#pragma unroll
      for (int j = 0; j < N; j += 2) top[u] = max3_nan(top[u], fabsf(f[j]), fabsf(f[j + 1]));
    }
  }
#pragma unroll
  for (int d = 1; d < kPer; d *= 2) {
#pragma unroll
    for (int u = 0; u < U; ++u) top[u] = max3_nan(top[u], __shfl_xor_sync(0xffffffffu, top[u], d), 0.0f);
  }
  // one division a thread: lane u of a block's writes the scale of its block of turn u
  static_assert(U <= kPer, "lanes of a block");
  const int lane = threadIdx.x % kPer;
  float scale = top[0];
#pragma unroll
  for (int u = 1; u < U; ++u) scale = lane == u ? top[u] : scale;
  scale = checkpoint_scale(scale);
  if (lane < U) {
    const int64_t i = base - 2 * lane + (int64_t)lane * (2 * kCheckpointThreads);
    if (i < vectors) scales[CheckpointAt<N, FLAT>(i, K, blocks).block] = scale;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = base + u * (2 * kCheckpointThreads);
    if (i >= vectors) return;
    const CheckpointAt<N, FLAT> at(i, K, blocks);
    const CheckpointCodes cs(top[u]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float f[N];
      v[u][h].get(f);
      bool exact = false;
      uint64_t q[N / 2];
      uint32_t w[N / 4];
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int j = 0; j < N / 2; ++j) q[j] = cs.exact16(ptx::pack_f32x2(f[2 * j], f[2 * j + 1]));
      } else {
        float far = 0.0f;  // the largest distance of a quotient from its code
        const uint64_t minus_shift = ptx::pack_f32x2(-CheckpointCodes::kShift, -CheckpointCodes::kShift), minus_scale = ptx::pack_f32x2(-cs.scale, -cs.scale);
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
          const uint64_t x2 = ptx::pack_f32x2(f[2 * j], f[2 * j + 1]);
          q[j] = cs.shifted(x2);
          const float2 d = ptx::unpack_f32x2(ptx::fma_f32x2(x2, minus_scale, ptx::add_f32x2(q[j], minus_shift)));
          far = fmaxf(far, fmaxf(fabsf(d.x), fabsf(d.y)));
        }
        exact = far > kNearBorder;
      }
#pragma unroll
      for (int j = 0; j < N / 4; ++j) w[j] = CheckpointCodes::bytes4(q[2 * j], q[2 * j + 1]);
      const int64_t left = FLAT ? N : at.left - h * N;
      store_codes<N>(codes + at.element + h * N, w, left);
      if (sizeof(T) == 4 && exact && left > 0) {  // rare: x is read again rather than kept
#pragma unroll 1
        for (int j = 0; j < N; ++j) codes[at.element + h * N + j] = exact_code(to_float(x[at.element + h * N + j]), top[u]);
      }
    }
  }
}

// What is formed from the saved value p: itself, gelu(p), grad_y * gelu'(p).
enum ActivationUse { kValue = 0, kActivation = 1, kSlopeOf = 2 };

// CODES: p from codes and scales, else from `pre`.
template <class T, int USE, bool CODES, bool FLAT>
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
      if constexpr (USE == kSlopeOf) g[u].load(grad_y + at.element, at.left);
      if constexpr (CODES) {
        load_codes<N>(codes + at.element, w[u], at.left);
        scale[u] = scales[at.block];
      } else {
        v[u].load(pre + at.element, at.left);
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
    out.store(y + at.element, at.left);
  }
}

// Rows of any length and alignment: a warp a block of 64, two values a lane, U blocks at a time.
constexpr int kAnyBlocks = 4;
struct AnyBlock {
  int64_t block, element, col;
  __device__ __forceinline__ AnyBlock(int64_t b, int64_t K, int64_t blocks) : block(b) {
    const int64_t row = (b | blocks) >> 32 ? b / blocks : (int64_t)((uint32_t)b / (uint32_t)blocks);
    col = (b - row * blocks) * kCheckpointBlock;
    element = row * K + col;
  }
  __device__ __forceinline__ int cols(int64_t K) const { return (int)min((int64_t)kCheckpointBlock, K - col); }
  __device__ __forceinline__ void next(int64_t K) {
    ++block;
    element += cols(K);
    col += kCheckpointBlock;
    if (col >= K) col = 0;
  }
};
template <class T>
__global__ void __launch_bounds__(kCheckpointThreads) checkpoint_any_kernel(const T* x, int8_t* codes, float* scales, int64_t count, int64_t K, int64_t blocks) {
  constexpr int U = kAnyBlocks;
  pdl_begin();
  const int lane = threadIdx.x & 31;
  const int64_t first = ((int64_t)blockIdx.x * (kCheckpointThreads / 32) + (threadIdx.x >> 5)) * U;
  const AnyBlock begin(first, K, blocks);
  AnyBlock at = begin;
  float f[U][2];
#pragma unroll
  for (int u = 0; u < U; ++u, at.next(K)) {
    f[u][0] = f[u][1] = 0.0f;
    if (first + u < count) {
      if (lane < at.cols(K)) f[u][0] = to_float(x[at.element + lane]);
      if (lane + 32 < at.cols(K)) f[u][1] = to_float(x[at.element + lane + 32]);
    }
  }
  float top[U];
#pragma unroll
  for (int u = 0; u < U; ++u) top[u] = max3_nan(fabsf(f[u][0]), fabsf(f[u][1]), 0.0f);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
#pragma unroll
    for (int u = 0; u < U; ++u) top[u] = max3_nan(top[u], __shfl_xor_sync(0xffffffffu, top[u], d), 0.0f);
  }
  at = begin;
#pragma unroll
  for (int u = 0; u < U; ++u, at.next(K)) {
    if (first + u >= count) return;
    const CheckpointCodes cs(top[u]);
    const uint64_t x2 = ptx::pack_f32x2(f[u][0], f[u][1]);
    float2 q;
    if constexpr (sizeof(T) == 2) {
      q = ptx::unpack_f32x2(cs.exact16(x2));
    } else {
      q = ptx::unpack_f32x2(cs.shifted(x2));
      const float d0 = __fmaf_rn(f[u][0], -cs.scale, q.x - CheckpointCodes::kShift), d1 = __fmaf_rn(f[u][1], -cs.scale, q.y - CheckpointCodes::kShift);
      if (fmaxf(fabsf(d0), fabsf(d1)) > kNearBorder) {
        q.x = __int_as_float(exact_code(f[u][0], top[u]));
        q.y = __int_as_float(exact_code(f[u][1], top[u]));
      }
    }
    if (lane < at.cols(K)) codes[at.element + lane] = (int8_t)__float_as_uint(q.x);
    if (lane + 32 < at.cols(K)) codes[at.element + lane + 32] = (int8_t)__float_as_uint(q.y);
    if (lane == 0) scales[at.block] = checkpoint_scale(top[u]);
  }
}
template <class T, int USE, bool CODES>
__global__ void __launch_bounds__(kCheckpointThreads) activation_any_kernel(const T* grad_y, const T* pre, const int8_t* codes, const float* scales, T* y, int64_t count,
                                                                            int64_t K, int64_t blocks) {
  constexpr int U = kAnyBlocks;
  pdl_begin();
  const int lane = threadIdx.x & 31;
  const int64_t first = ((int64_t)blockIdx.x * (kCheckpointThreads / 32) + (threadIdx.x >> 5)) * U;
  const AnyBlock begin(first, K, blocks);
  AnyBlock at = begin;
  float p[2 * U], g[2 * U];
#pragma unroll
  for (int u = 0; u < U; ++u, at.next(K)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      p[2 * u + h] = g[2 * u + h] = 0.0f;
      if (first + u < count) {
        const int c = lane + 32 * h;
        if (c < at.cols(K)) {
          if constexpr (CODES) p[2 * u + h] = (float)codes[at.element + c] * scales[at.block];
          else p[2 * u + h] = to_float(pre[at.element + c]);
          if constexpr (USE == kSlopeOf) g[2 * u + h] = to_float(grad_y[at.element + c]);
        }
      }
    }
  }
  if constexpr (USE == kActivation) gelu_many<U>(p);
  if constexpr (USE == kSlopeOf) times_gelu_slope<U>(p, g);
  at = begin;
#pragma unroll
  for (int u = 0; u < U; ++u, at.next(K)) {
    if (first + u >= count) return;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (lane + 32 * h < at.cols(K)) y[at.element + lane + 32 * h] = from_float<T>(USE == kSlopeOf ? g[2 * u + h] : p[2 * u + h]);
  }
}

// Vectors, blocks of a row, and whether rows are made of whole vectors and of whole blocks.
template <class T>
struct CheckpointShape {
  int64_t count, vectors, blocks;
  bool flat, vector;
  CheckpointShape(int64_t M, int64_t K, bool aligned) {
    constexpr int N = Vec16<T>::N;
    blocks = checkpoint_blocks(K);
    count = M * blocks;
    vectors = count * (kCheckpointBlock / N);
    vector = aligned && K % N == 0;
    flat = vector && K % kCheckpointBlock == 0;
  }
  // blocks of threads whose threads take `turns` vectors each (no vectors: whose warps take kAnyBlocks blocks)
  unsigned grid(int turns) const {
    const int64_t per = vector ? (int64_t)kCheckpointThreads * turns : kCheckpointThreads / 32 * kAnyBlocks, all = vector ? vectors : count;
    return (unsigned)((all + per - 1) / per);
  }
};

template <class T>
static qb_status launch_checkpoint(const void* x_data, int64_t M, int64_t K, int8_t* codes, float* scales, cudaStream_t stream) {
  const T* const x = static_cast<const T*>(x_data);
  const CheckpointShape<T> s(M, K, aligned16(x));
  const unsigned grid = s.grid(2 * kCheckpointTurns<T>);
  if (s.vector)
    QB_CUDA_TRY(launch_kernel<kMostL1>(s.flat ? checkpoint_kernel<T, true> : checkpoint_kernel<T, false>, grid, kCheckpointThreads, 0, stream, 1, false, x, codes, scales,
                                       s.vectors, K, s.blocks));
  else
    QB_CUDA_TRY(launch_kernel<kMostL1>(checkpoint_any_kernel<T>, grid, kCheckpointThreads, 0, stream, 1, false, x, codes, scales, s.count, K, s.blocks));
  return QB_OK;
}
template <class T, int USE, bool CODES>
static qb_status launch_activation(const void* grad_y, const void* pre, const int8_t* codes, const float* scales, int64_t M, int64_t K, void* y, cudaStream_t stream) {
  const CheckpointShape<T> s(M, K, aligned16(grad_y) && aligned16(pre) && aligned16(y));
  const unsigned grid = s.grid(kCheckpointUnroll);
  const T *const g = static_cast<const T*>(grad_y), *const p = static_cast<const T*>(pre);
  if (s.vector)
    QB_CUDA_TRY(launch_kernel<kMostL1>(s.flat ? activation_kernel<T, USE, CODES, true> : activation_kernel<T, USE, CODES, false>, grid, kCheckpointThreads, 0, stream, 1,
                                       false, g, p, codes, scales, static_cast<T*>(y), s.vectors, K, s.blocks));
  else
    QB_CUDA_TRY(launch_kernel<kMostL1>(activation_any_kernel<T, USE, CODES>, grid, kCheckpointThreads, 0, stream, 1, false, g, p, codes, scales, static_cast<T*>(y), s.count,
                                       K, s.blocks));
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
static bool to_elements(const void* p, int type) { return aligned_to(p, type == QB_F32 ? 4 : 2); }

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
