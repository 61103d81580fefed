// qb_layer_norm, qb_layer_norm_backward.
//
// A row of up to 1,024 elements is held by one warp, 32 elements a lane; up to 8,192 by two, four or eight warps, which join their sums
// through shared memory; beyond, a block goes over it as often as it needs it (the second time from L2).  Each element is read once into
// registers, so that the variance is a sum of squared differences from the mean that is known by then (and of what rounding the mean left).
// Backward: a block keeps the sums of grad_y * xhat and grad_y over its rows in registers, a pair a column, and leaves them in the
// workspace at its end; a second kernel sums the blocks', always in the same order.
// Bound by memory: one read and one write of the tensor forward, two reads and one write backward.  24,576 x 1,024: bfloat16 forward 19.9 us
// (5.1 TB/s), backward 30.5 (4.9), fp32 34.7 (5.8) and 53 (5.7); 5,003 x 1,024 bfloat16 6.9 and 13.1; 32 x 768 2.4 and 4.3.  About 4 us
// of a backward pass are its start, its blocks' sums and the second kernel.  Rows on their way in shared memory cost no registers (forward 0.9 us
// more with the next row in registers, 8 with one row a warp and a block that ends).  Tried and not kept, backward, 24,576 x 1,024 bfloat16: two warps a row with
// sixteen elements a lane 45 us, two blocks per SM with gamma in shared memory 41, two rows a warp at a time 31.  Forward, where rows are not made of
// vectors, 8 to 92 bytes a thread are spilled (weights: two blocks per SM leave 128 registers).
#include "common.cuh"
#include "ptx_float.cuh"
#include "vec16.cuh"

#include <algorithm>
#include <atomic>

namespace qb {

constexpr int kNormThreads = 256;
constexpr int kNormElements = 32;  // of a row that a lane holds
constexpr int kNormMostHeld = 8 * 32 * kNormElements;

// Where a lane's elements lie: vector i begins at column (i * lanes of the row + lane in the row) * V.
template <class T, int WPR, bool VECTOR>
struct NormRow {
  // 16-bit and fp32 vectors of 16 bytes; rows that are not made of them: an element a lane
  static constexpr int V = VECTOR ? Vec16<T>::N : 1;
  static constexpr int kVectors = kNormElements / V;
  static constexpr int kStride = WPR * 32 * V;
  static constexpr int kRegs = VECTOR ? kVectors * 4 : kVectors;
  uint32_t raw[kRegs];
  __device__ __forceinline__ void load(const T* row, int first, int D) {
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
      const int c = first + i * kStride;
      if constexpr (VECTOR) {
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        if (c < D) w = *reinterpret_cast<const uint4*>(row + c);
        raw[4 * i] = w.x;
        raw[4 * i + 1] = w.y;
        raw[4 * i + 2] = w.z;
        raw[4 * i + 3] = w.w;
      } else {
        raw[i] = 0u;
        if (c < D) {
          if constexpr (sizeof(T) == 4) raw[i] = *reinterpret_cast<const uint32_t*>(row + c);
          else raw[i] = *reinterpret_cast<const uint16_t*>(row + c);
        }
      }
    }
  }
  __device__ __forceinline__ void get(int i, float* f) const {
    if constexpr (VECTOR) {
      Vec16<T> v;
      v.raw = make_uint4(raw[4 * i], raw[4 * i + 1], raw[4 * i + 2], raw[4 * i + 3]);
      float e[V];
      v.get(e);
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = e[j];
    } else if constexpr (sizeof(T) == 4) {
      f[0] = __uint_as_float(raw[i]);
    } else {
      const uint16_t h = (uint16_t)raw[i];
      f[0] = to_float(*reinterpret_cast<const T*>(&h));
    }
  }
  static __device__ __forceinline__ void put(T* row, int c, const float (&f)[V]) {
    if constexpr (VECTOR) {
      Vec16<T> v;
      v.set(f);
      *reinterpret_cast<uint4*>(row + c) = v.raw;
    } else {
      row[c] = from_float<T>(f[0]);
    }
  }
};
// Rows on their way: a ring of stages in shared memory, filled by copies of 16 bytes that need no registers.  A thread copies and reads its
// own bytes alone, so that nobody waits for anybody.  TENSORS rows a stage.
template <class T, int WPR, int TENSORS>
struct NormRing {
  using Row = NormRow<T, WPR, true>;
  static constexpr int kStageBytes = TENSORS * Row::kVectors * 16 * kNormThreads;
  // forward: two blocks per SM
  static constexpr int kStages = TENSORS == 1 ? 98304 / kStageBytes : 196608 / kStageBytes;
  // behind the rows, backward: mean and rstd, a copy of each for every lane (loads that are waited for within a row's turn cost 24,576 x
  // 1,024 bfloat16 10 us of 40)
  static constexpr int kStatsBytes = TENSORS == 1 ? 0 : kStages * kNormThreads * 8;
  static constexpr int kBytes = kStages * kStageBytes + kStatsBytes;
  static_assert(kStages >= 3, "stages");
  uint32_t mine;
  __device__ __forceinline__ explicit NormRing(const void* smem) : mine(ptx::smem_u32(smem) + threadIdx.x * 16) {}
  __device__ __forceinline__ uint32_t at(int stage, int tensor, int i) const {
    return mine + (uint32_t)((stage * TENSORS + tensor) * Row::kVectors + i) * (16 * kNormThreads);
  }
  __device__ __forceinline__ void fetch(int stage, int tensor, const T* row, int first, int end) const {
#pragma unroll
    for (int i = 0; i < Row::kVectors; ++i) {
      const int c = first + i * Row::kStride;
      if (c < end) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at(stage, tensor, i)), "l"(row + c) : "memory");
    }
  }
  __device__ __forceinline__ uint32_t stats_at(int stage) const { return mine + kStages * kStageBytes - threadIdx.x * 8 + stage * (kNormThreads * 8); }
  __device__ __forceinline__ void fetch_stats(int stage, const float* mean, const float* rstd) const {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(stats_at(stage)), "l"(mean) : "memory");
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(stats_at(stage) + 4), "l"(rstd) : "memory");
  }
  __device__ __forceinline__ void read_stats(int stage, float& mean, float& rstd) const {
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(mean), "=f"(rstd) : "r"(stats_at(stage)) : "memory");
  }
  static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  static __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory"); }
  static __device__ __forceinline__ void wait_all() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }
  // (vectors behind the row's end were not copied, and are zeros)
  __device__ __forceinline__ void read(int stage, int tensor, Row& r, int first, int end) const {
#pragma unroll
    for (int i = 0; i < Row::kVectors; ++i) {
      uint32_t* const w = r.raw + 4 * i;
      w[0] = w[1] = w[2] = w[3] = 0u;
      if (first + i * Row::kStride < end)
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at(stage, tensor, i)) : "memory");
    }
  }
};

// V weights from column c on (fp32, 16-byte aligned where V is above 1 and VECTOR), or `instead` of them.
template <int V>
__device__ __forceinline__ void norm_weights(const float* w, int c, float instead, bool vector, float* f) {
#pragma unroll
  for (int j = 0; j < V; ++j) f[j] = instead;
  if (!w) return;
  if (V >= 4 && vector) {
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
      const float4 q = *reinterpret_cast<const float4*>(w + c + 4 * j);
      f[4 * j] = q.x;
      f[4 * j + 1] = q.y;
      f[4 * j + 2] = q.z;
      f[4 * j + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = w[c + j];
  }
}

// Arithmetic on one value, or on two at a time where a lane's values come in pairs.
template <int V>
struct NormMath {
  static constexpr int W = V > 1 ? 2 : 1;
  typedef std::conditional_t<V == 1, float, uint64_t> F;
  static __device__ __forceinline__ F all(float a) {
    if constexpr (V == 1) return a;
    else return ptx::pack_f32x2(a, a);
  }
  static __device__ __forceinline__ F from(const float* p) {
    if constexpr (V == 1) return p[0];
    else return ptx::pack_f32x2(p[0], p[1]);
  }
  static __device__ __forceinline__ void to(float* p, F a) {
    if constexpr (V == 1) {
      p[0] = a;
    } else {
      const float2 f = ptx::unpack_f32x2(a);
      p[0] = f.x;
      p[1] = f.y;
    }
  }
  static __device__ __forceinline__ F add(F a, F b) {
    if constexpr (V == 1) return a + b;
    else return ptx::add_f32x2(a, b);
  }
  static __device__ __forceinline__ F mul(F a, F b) {
    if constexpr (V == 1) return a * b;
    else return ptx::mul_f32x2(a, b);
  }
  static __device__ __forceinline__ F fma(F a, F b, F c) {
    if constexpr (V == 1) return __fmaf_rn(a, b, c);
    else return ptx::fma_f32x2(a, b, c);
  }
  static __device__ __forceinline__ float sum(F a) {
    if constexpr (V == 1) {
      return a;
    } else {
      const float2 f = ptx::unpack_f32x2(a);
      return f.x + f.y;
    }
  }
};

template <class A>
__device__ __forceinline__ A warp_sum(A s) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  return s;
}
// The sum over the WPR warps of a row.  `slots`: of this call alone until every warp of the block has met the next one's barrier.
template <int WPR, class A>
__device__ __forceinline__ A row_sum(A s, A* slots, int warp, int lane) {
  s = warp_sum(s);
  if constexpr (WPR > 1) {
    if (lane == 0) slots[warp] = s;
    __syncthreads();
    s = 0;
    const int first = warp / WPR * WPR;
#pragma unroll
    for (int i = 0; i < WPR; ++i) s += slots[first + i];
  }
  return s;
}

struct NormArgs {
  const float *gamma, *beta;
  float* mean;
  float* rstd;
  int64_t M;
  int32_t D;
  float eps, inv_d;
  double inv64;
  int32_t vector_weights;
};

// A row's mean: an fp32 number next to it, and what that leaves, `delta`.  Rows whose mean is far above their deviations need both (with a
// mean one unit of its last place off, a constant row gives rstd times that unit), and a sum that is good for them: 16-bit values of one
// binade have 11 bits, so that 8,192 of them add up in fp32 without rounding; of fp32 values a lane sums the differences from its first
// one, and the lanes' sums are added in 64 bits; longer rows are summed as differences, twice.  24,576 x 1,024: bfloat16 19.9 us (19.1
// with the mean alone), fp32 34.7 (34.0); all sums as differences, twice: 20.9 and 34.7; fp32 element by element in 64 bits: 34.7, 32 x 768 2.75 instead of 2.6.
struct NormMean {
  float mean, delta;
  __device__ __forceinline__ NormMean(float mean, float delta) : mean(mean), delta(delta) {}
  __device__ __forceinline__ NormMean(float sum, int D, float inv_d, double) {
    mean = sum * inv_d;
    mean = fmaf(fmaf(-mean, (float)D, sum), inv_d, mean);
    delta = fmaf(-mean, (float)D, sum) * inv_d;
  }
  __device__ __forceinline__ NormMean(double sum, int D, float inv_d, double inv64) {
    mean = (float)(sum * inv64);
    delta = (float)fma(-(double)mean, (double)D, sum) * inv_d;
  }
  // 1 / sqrt(variance + eps) from the sum of (x - mean)^2
  __device__ __forceinline__ float rstd(float sum2, float inv_d, float eps) const {
    const float var = fmaf(-delta, delta, sum2 * inv_d);
    return 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);  // (a NaN stays one)
  }
};

// A block goes over its share of the rows with the weights in registers and the next rows on their way.
template <class T, int WPR, bool VECTOR>
__global__ void __launch_bounds__(kNormThreads, 2) layer_norm_kernel(const T* x, T* y, const NormArgs a) {
  using Row = NormRow<T, WPR, VECTOR>;
  constexpr int V = Row::V;
  typedef NormMath<V> Math;
  typedef typename Math::F F;
  constexpr int W = Math::W;
  typedef std::conditional_t<sizeof(T) == 4, double, float> Sum;
  __shared__ Sum slots[2][8];
  __shared__ float slots2[2][8];
  pdl_begin();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = a.D;
  const int first = ((warp % WPR) * 32 + lane) * V;
  const int64_t step = (int64_t)gridDim.x * (8 / WPR);
  int64_t m = (int64_t)blockIdx.x * (8 / WPR) + warp / WPR;
  using Ring = NormRing<T, WPR, 1>;
  extern __shared__ __align__(16) float room[];
  const Ring ring(room);
  const auto fetch = [&](int stage, int64_t row) {
    if (row < a.M) ring.fetch(stage, 0, x + row * D, first, D);
    Ring::commit();
  };
  if constexpr (VECTOR) {
#pragma unroll
    for (int k = 0; k < Ring::kStages - 1; ++k) fetch(k, m + k * step);
  }
  int stage = 0;
  float gamma[kNormElements], beta[kNormElements];
#pragma unroll
  for (int i = 0; i < Row::kVectors; ++i) {
    const int c = first + i * Row::kStride;
    if (c < D) {
      norm_weights<V>(a.gamma, c, 1.0f, a.vector_weights, gamma + i * V);
      norm_weights<V>(a.beta, c, 0.0f, a.vector_weights, beta + i * V);
    }
  }
  float n = 0.0f;  // how many of a row's elements are the lane's
#pragma unroll
  for (int i = 0; i < Row::kVectors; ++i) n += first + i * Row::kStride < D ? (float)V : 0.0f;
  int turn = 0;
  for (int64_t m0 = (int64_t)blockIdx.x * (8 / WPR); m0 < a.M; m0 += step, m += step, turn ^= 1) {
    const int end = m < a.M ? D : 0;
    Row r;
    if constexpr (VECTOR) {
      Ring::wait();
      ring.read(stage, 0, r, first, end);
      fetch(stage == 0 ? Ring::kStages - 1 : stage - 1, m + (Ring::kStages - 1) * step);  // where the row before was
      if (++stage == Ring::kStages) stage = 0;
    } else {
      r.load(x + (end ? m : 0) * D, first, end);
    }
    F s = Math::all(0.0f);
    Sum sum;
    if constexpr (sizeof(T) == 4) {  // the lane's elements: n times the first one, and the differences from it
      float one[V];
      r.get(0, one);
      const F minus_one = Math::all(-one[0]);
#pragma unroll
      for (int i = 0; i < Row::kVectors; ++i) {
        if (first + i * Row::kStride < end) {
          float f[V];
          r.get(i, f);
#pragma unroll
          for (int j = 0; j < V; j += W) s = Math::add(s, Math::add(Math::from(f + j), minus_one));
        }
      }
      sum = fma((double)n, (double)one[0], (double)Math::sum(s));
    } else {
#pragma unroll
      for (int i = 0; i < Row::kVectors; ++i) {
        float f[V];
        r.get(i, f);
#pragma unroll
        for (int j = 0; j < V; j += W) s = Math::add(s, Math::from(f + j));
      }
      sum = Math::sum(s);
    }
    const NormMean st(row_sum<WPR>(sum, slots[turn], warp, lane), D, a.inv_d, a.inv64);
    const F minus_mean = Math::all(-st.mean);
    s = Math::all(0.0f);
#pragma unroll
    for (int i = 0; i < Row::kVectors; ++i) {
      if (first + i * Row::kStride < end) {
        float f[V];
        r.get(i, f);
#pragma unroll
        for (int j = 0; j < V; j += W) {
          const F d = Math::add(Math::from(f + j), minus_mean);
          s = Math::fma(d, d, s);
        }
      }
    }
    const float rstd = st.rstd(row_sum<WPR>(Math::sum(s), slots2[turn], warp, lane), a.inv_d, a.eps);
    const F all_rstd = Math::all(rstd), minus_delta = Math::all(-st.delta * rstd);
#pragma unroll
    for (int i = 0; i < Row::kVectors; ++i) {
      const int c = first + i * Row::kStride;
      if (c < end) {
        float f[V];
        r.get(i, f);
#pragma unroll
        for (int j = 0; j < V; j += W)
          Math::to(f + j, Math::fma(Math::fma(Math::add(Math::from(f + j), minus_mean), all_rstd, minus_delta), Math::from(gamma + i * V + j), Math::from(beta + i * V + j)));
        Row::put(y + m * D, c, f);
      }
    }
    if (a.mean && end && warp % WPR == 0 && lane == 0) {
      a.mean[m] = st.mean;
      a.rstd[m] = rstd;
    }
  }
}

__device__ __forceinline__ float block_sum(float s, float* slots) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  s = warp_sum(s);
  __syncthreads();
  if (lane == 0) slots[warp] = s;
  __syncthreads();
  s = slots[0];
#pragma unroll
  for (int i = 1; i < kNormThreads / 32; ++i) s += slots[i];
  return s;
}

// Rows that registers do not hold: a block a row.
template <class T>
__global__ void __launch_bounds__(kNormThreads) layer_norm_long_kernel(const T* x, T* y, const NormArgs a) {
  __shared__ float slots[8];
  pdl_begin();
  const int D = a.D;
  for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
    const T* const row = x + m * D;
    const float shift = to_float(row[0]);
    float s = 0.0f, s2 = 0.0f;
    for (int c = threadIdx.x; c < D; c += kNormThreads) s += to_float(row[c]) - shift;
    const float mean = fmaf(block_sum(s, slots), a.inv_d, shift);
    s = 0.0f;
    for (int c = threadIdx.x; c < D; c += kNormThreads) {
      const float d = to_float(row[c]) - mean;
      s += d;
      s2 = __fmaf_rn(d, d, s2);
    }
    const NormMean st(mean, block_sum(s, slots) * a.inv_d);
    const float rstd = st.rstd(block_sum(s2, slots), a.inv_d, a.eps), minus_delta = -st.delta * rstd;
    for (int c = threadIdx.x; c < D; c += kNormThreads)  // (y may be x: each element is read and written by one thread)
      y[m * D + c] = from_float<T>(__fmaf_rn(__fmaf_rn(to_float(row[c]) - mean, rstd, minus_delta), a.gamma ? a.gamma[c] : 1.0f, a.beta ? a.beta[c] : 0.0f));
    if (a.mean && threadIdx.x == 0) {
      a.mean[m] = mean + st.delta;
      a.rstd[m] = rstd;
    }
  }
}

struct NormBackArgs {
  const float *gamma, *mean, *rstd;
  float* parts;  // [blocks][2][D]
  int64_t M;
  int32_t D;
  float inv_d;
  int32_t vector_weights;
};

// As the forward kernel.  A lane's sums of its columns lie in the parts in the order of registers and lanes (norm_column).
template <class T, int WPR, bool VECTOR>
__global__ void __launch_bounds__(kNormThreads, 1) layer_norm_backward_kernel(const T* grad_y, const T* x, T* grad_x, const NormBackArgs a) {
  using Row = NormRow<T, WPR, VECTOR>;
  constexpr int V = Row::V, kRows = 8 / WPR, kLanes = WPR * 32;
  typedef NormMath<V> Math;
  typedef typename Math::F F;
  constexpr int W = Math::W;
  extern __shared__ __align__(16) float room[];
  float* const columns = room;  // [rows of the block][2][registers][lanes of a row], behind the last row
  __shared__ float slots[2][2][8];
  pdl_begin();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = a.D;
  const int first = ((warp % WPR) * 32 + lane) * V;
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t m = (int64_t)blockIdx.x * kRows + warp / WPR;
  using Ring = NormRing<T, WPR, 2>;
  const Ring ring(room);
  const auto fetch = [&](int stage, int64_t row) {
    if (row < a.M) {
      ring.fetch(stage, 0, grad_y + row * D, first, D);
      ring.fetch(stage, 1, x + row * D, first, D);
      ring.fetch_stats(stage, a.mean + row, a.rstd + row);
    }
    Ring::commit();
  };
  if constexpr (VECTOR) {
#pragma unroll
    for (int k = 0; k < Ring::kStages - 1; ++k) fetch(k, m + k * step);
  }
  int stage = 0;
  float gamma[kNormElements];
#pragma unroll
  for (int i = 0; i < Row::kVectors; ++i)
    if (first + i * Row::kStride < D) norm_weights<V>(a.gamma, first + i * Row::kStride, 1.0f, a.vector_weights, gamma + i * V);
  float sum_gx[kNormElements] = {}, sum_g[kNormElements] = {};
  int turn = 0;
  for (int64_t m0 = (int64_t)blockIdx.x * kRows; m0 < a.M; m0 += step, m += step, turn ^= 1) {
    const int end = m < a.M ? D : 0;
    Row gy, xr;
    float mean = 0.0f, rstd = 0.0f;
    if constexpr (VECTOR) {
      Ring::wait();
      ring.read(stage, 0, gy, first, end);
      ring.read(stage, 1, xr, first, end);
      if (end) ring.read_stats(stage, mean, rstd);
      fetch(stage == 0 ? Ring::kStages - 1 : stage - 1, m + (Ring::kStages - 1) * step);  // where the row before was
      if (++stage == Ring::kStages) stage = 0;
    } else {
      gy.load(grad_y + (end ? m : 0) * D, first, end);
      xr.load(x + (end ? m : 0) * D, first, end);
      mean = a.mean[end ? m : 0];
      rstd = a.rstd[end ? m : 0];
    }
    const F minus_mean = Math::all(-mean), all_rstd = Math::all(rstd);
    F s2 = Math::all(0.0f), sx2 = Math::all(0.0f);
#pragma unroll
    for (int i = 0; i < Row::kVectors; ++i) {
      if (first + i * Row::kStride < end) {
        float g[V], f[V];
        gy.get(i, g);
        xr.get(i, f);
#pragma unroll
        for (int j = 0; j < V; j += W) {
          const int k = i * V + j;
          const F gj = Math::from(g + j), xhat = Math::mul(Math::add(Math::from(f + j), minus_mean), all_rstd), gw = Math::mul(gj, Math::from(gamma + k));
          Math::to(sum_gx + k, Math::fma(gj, xhat, Math::from(sum_gx + k)));
          Math::to(sum_g + k, Math::add(gj, Math::from(sum_g + k)));
          s2 = Math::add(s2, gw);
          sx2 = Math::fma(gw, xhat, sx2);
        }
      }
    }
    float s = Math::sum(s2), sx = Math::sum(sx2);
    s = warp_sum(s);
    sx = warp_sum(sx);
    if constexpr (WPR > 1) {
      if (lane == 0) {
        slots[turn][0][warp] = s;
        slots[turn][1][warp] = sx;
      }
      __syncthreads();
      s = sx = 0.0f;
      const int begin = warp / WPR * WPR;
#pragma unroll
      for (int i = 0; i < WPR; ++i) {
        s += slots[turn][0][begin + i];
        sx += slots[turn][1][begin + i];
      }
    }
    const F minus_s = Math::all(-s * a.inv_d), minus_sx = Math::all(-sx * a.inv_d);
#pragma unroll
    for (int i = 0; i < Row::kVectors; ++i) {
      const int c = first + i * Row::kStride;
      if (c < end) {
        float g[V], f[V];
        gy.get(i, g);
        xr.get(i, f);
#pragma unroll
        for (int j = 0; j < V; j += W) {
          const F xhat = Math::mul(Math::add(Math::from(f + j), minus_mean), all_rstd);
          const F inner = Math::fma(Math::from(g + j), Math::from(gamma + i * V + j), minus_s);
          Math::to(f + j, Math::mul(all_rstd, Math::fma(xhat, minus_sx, inner)));
        }
        Row::put(grad_x + m * D, c, f);
      }
    }
  }
  if (!a.parts) return;
  if constexpr (VECTOR && kRows > 1) {  // the sums take the ring's place
    Ring::wait_all();
    __syncthreads();
  }
  // the block's sums: its rows' warps in their order
  float* const part = a.parts + (int64_t)blockIdx.x * (2 * kNormElements * kLanes);
  const int at = (warp % WPR) * 32 + lane;
#pragma unroll
  for (int i = 0; i < kNormElements; ++i) {
    if (kRows > 1) {
      columns[((warp / WPR * 2) * kNormElements + i) * kLanes + at] = sum_gx[i];
      columns[((warp / WPR * 2 + 1) * kNormElements + i) * kLanes + at] = sum_g[i];
    } else {
      part[i * kLanes + at] = sum_gx[i];
      part[(kNormElements + i) * kLanes + at] = sum_g[i];
    }
  }
  if constexpr (kRows > 1) {
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * kNormElements * kLanes; i += kNormThreads) {
      float s = columns[i];
#pragma unroll
      for (int r = 1; r < kRows; ++r) s += columns[r * (2 * kNormElements * kLanes) + i];
      part[i] = s;
    }
  }
}
// The column of register i of lane `at` of a row (`lanes` of them), vectors of V.
__device__ __forceinline__ int norm_column(int i, int at, int lanes, int V) { return (i / V * lanes + at) * V + i % V; }

template <class T>
__global__ void __launch_bounds__(kNormThreads) layer_norm_long_backward_kernel(const T* grad_y, const T* x, T* grad_x, const NormBackArgs a) {
  __shared__ float slots[8];
  pdl_begin();
  const int D = a.D;
  float* const part = a.parts ? a.parts + (int64_t)blockIdx.x * 2 * D : nullptr;
  bool begun = false;
  for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
    const float mean = a.mean[m], rstd = a.rstd[m];
    float s = 0.0f, sx = 0.0f;
    for (int c = threadIdx.x; c < D; c += kNormThreads) {
      const float g = to_float(grad_y[m * D + c]), xhat = (to_float(x[m * D + c]) - mean) * rstd, gw = g * (a.gamma ? a.gamma[c] : 1.0f);
      s += gw;
      sx = __fmaf_rn(gw, xhat, sx);
      if (part) {  // each column by one thread
        part[c] = begun ? __fmaf_rn(g, xhat, part[c]) : g * xhat;
        part[D + c] = begun ? part[D + c] + g : g;
      }
    }
    begun = true;
    s = block_sum(s, slots) * a.inv_d;
    sx = block_sum(sx, slots) * a.inv_d;
    for (int c = threadIdx.x; c < D; c += kNormThreads) {
      const float g = to_float(grad_y[m * D + c]), xhat = (to_float(x[m * D + c]) - mean) * rstd;
      grad_x[m * D + c] = from_float<T>(rstd * (__fmaf_rn(g, a.gamma ? a.gamma[c] : 1.0f, -s) - xhat * sx));
    }
  }
}

// Sums over the blocks: 32 sums a block, 32 groups of blocks side by side (few loads one after the other: the launch is as long as these
// take), joined in their order.  `lanes`: of a row, in whose order the sums lie (half of them gamma's), or 0: in the columns' order.
constexpr int kNormJoinGroups = 32;
__global__ void __launch_bounds__(32 * kNormJoinGroups) layer_norm_join_kernel(const float* parts, int blocks, int32_t sums, int32_t lanes, int32_t V, int32_t D,
                                                                               float* grad_gamma, float* grad_beta) {
  __shared__ float joined[kNormJoinGroups][32];
  pdl_begin();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int k = (int)blockIdx.x * 32 + lane, run = (blocks + kNormJoinGroups - 1) / kNormJoinGroups, last = min((warp + 1) * run, blocks);
  float s = 0.0f;
  if (k < sums) {
#pragma unroll 8
    for (int b = warp * run; b < last; ++b) s += parts[(int64_t)b * sums + k];
  }
  joined[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && k < sums) {
#pragma unroll
    for (int w = 1; w < kNormJoinGroups; ++w) s += joined[w][lane];
    const int at = k < sums / 2 ? k : k - sums / 2;
    const int c = lanes ? norm_column(at / lanes, at % lanes, lanes, V) : at;
    float* const to = k < sums / 2 ? grad_gamma : grad_beta;
    if (to && c < D) to[c] = s;
  }
}

constexpr size_t kNormPartsOff = 1024;
static int norm_warps(int64_t D) { return D <= 1024 ? 1 : (D <= 2048 ? 2 : (D <= 4096 ? 4 : 8)); }
// Sums that a block of the backward pass leaves: two for each register of the row's lanes, or for each column.
static int64_t norm_sums(int64_t D) { return D > kNormMostHeld ? 2 * D : 2 * kNormElements * 32 * norm_warps(D); }

// Lets a kernel have `bytes` of dynamic shared memory (once per device).
template <auto KERNEL>
static qb_status norm_room(size_t bytes) {
  static std::atomic<bool> set[64] = {};
  int dev = 0;
  QB_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64 || !set[dev].load(std::memory_order_acquire)) {
    QB_CUDA_TRY(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    if (dev >= 0 && dev < 64) set[dev].store(true, std::memory_order_release);
  }
  return QB_OK;
}

template <class T, int WPR, bool VECTOR>
static qb_status launch_norm_form(const T* x, T* y, const NormArgs& a, int sms, cudaStream_t stream) {
  constexpr size_t smem = VECTOR ? NormRing<T, WPR, 1>::kBytes : 0;
  constexpr int kRows = 8 / WPR;
  qb_status st = norm_room<layer_norm_kernel<T, WPR, VECTOR>>(smem);
  if (st != QB_OK) return st;
  QB_CUDA_TRY(launch_kernel(layer_norm_kernel<T, WPR, VECTOR>, (unsigned)std::min<int64_t>((a.M + kRows - 1) / kRows, (int64_t)sms * 2), kNormThreads, smem, stream,
                            1, false, x, y, a));
  return QB_OK;
}
template <class T>
static qb_status launch_norm(const void* x_data, void* y_data, const NormArgs& a, int sms, cudaStream_t stream) {
  const T* const x = static_cast<const T*>(x_data);
  T* const y = static_cast<T*>(y_data);
  if (a.D > kNormMostHeld) {
    QB_CUDA_TRY(launch_kernel(layer_norm_long_kernel<T>, (unsigned)std::min<int64_t>(a.M, (int64_t)sms * 8), kNormThreads, 0, stream, 1, false, x, y, a));
    return QB_OK;
  }
  const bool vector = a.D % Vec16<T>::N == 0 && aligned16(x) && aligned16(y);
  switch (norm_warps(a.D)) {
    case 1: return vector ? launch_norm_form<T, 1, true>(x, y, a, sms, stream) : launch_norm_form<T, 1, false>(x, y, a, sms, stream);
    case 2: return vector ? launch_norm_form<T, 2, true>(x, y, a, sms, stream) : launch_norm_form<T, 2, false>(x, y, a, sms, stream);
    case 4: return vector ? launch_norm_form<T, 4, true>(x, y, a, sms, stream) : launch_norm_form<T, 4, false>(x, y, a, sms, stream);
    default: return vector ? launch_norm_form<T, 8, true>(x, y, a, sms, stream) : launch_norm_form<T, 8, false>(x, y, a, sms, stream);
  }
}

template <class T, int WPR, bool VECTOR>
static qb_status launch_norm_backward_form(const T* grad_y, const T* x, T* grad_x, const NormBackArgs& a, int blocks, cudaStream_t stream) {
  constexpr size_t sums = WPR < 8 ? (size_t)2 * kNormElements * 32 * 8 * 4 : 0;
  constexpr size_t smem = VECTOR ? std::max(sums, (size_t)NormRing<T, WPR, 2>::kBytes) : sums;
  qb_status st = norm_room<layer_norm_backward_kernel<T, WPR, VECTOR>>(smem);
  if (st != QB_OK) return st;
  QB_CUDA_TRY(launch_kernel(layer_norm_backward_kernel<T, WPR, VECTOR>, (unsigned)blocks, kNormThreads, smem, stream, 1, false, grad_y, x, grad_x, a));
  return QB_OK;
}
// V: receives the vector length, which the order of the sums goes by.
template <class T>
static qb_status launch_norm_backward(const void* grad_y, const void* x_data, void* grad_x, const NormBackArgs& a, int blocks, int* V, cudaStream_t stream) {
  const T *const gy = static_cast<const T*>(grad_y), *const x = static_cast<const T*>(x_data);
  T* const gx = static_cast<T*>(grad_x);
  if (a.D > kNormMostHeld) {
    QB_CUDA_TRY(launch_kernel(layer_norm_long_backward_kernel<T>, (unsigned)blocks, kNormThreads, 0, stream, 1, false, gy, x, gx, a));
    return QB_OK;
  }
  const bool vector = a.D % Vec16<T>::N == 0 && aligned16(x) && aligned16(gy) && aligned16(gx);
  *V = vector ? Vec16<T>::N : 1;
  switch (norm_warps(a.D)) {
    case 1: return vector ? launch_norm_backward_form<T, 1, true>(gy, x, gx, a, blocks, stream) : launch_norm_backward_form<T, 1, false>(gy, x, gx, a, blocks, stream);
    case 2: return vector ? launch_norm_backward_form<T, 2, true>(gy, x, gx, a, blocks, stream) : launch_norm_backward_form<T, 2, false>(gy, x, gx, a, blocks, stream);
    case 4: return vector ? launch_norm_backward_form<T, 4, true>(gy, x, gx, a, blocks, stream) : launch_norm_backward_form<T, 4, false>(gy, x, gx, a, blocks, stream);
    default: return vector ? launch_norm_backward_form<T, 8, true>(gy, x, gx, a, blocks, stream) : launch_norm_backward_form<T, 8, false>(gy, x, gx, a, blocks, stream);
  }
}

static qb_status check_norm(const char* what, bool pointers, int type, int64_t M, int64_t D) {
  if (pointers && type >= QB_F32 && type <= QB_F16 && M > 0 && M <= QB_MAX_MN && D > 0 && D <= QB_MAX_K) return QB_OK;
  set_last_error("%s: invalid argument (M=%lld D=%lld type=%d)", what, (long long)M, (long long)D, type);
  return QB_ERR_INVALID;
}

}  // namespace qb

extern "C" size_t qb_layer_norm_workspace_bytes(int64_t M, int64_t D) {
  if (M <= 0 || M > QB_MAX_MN || D <= 0 || D > QB_MAX_K) return 0;
  return qb::kNormPartsOff + (size_t)std::min<int64_t>(M, 2 * qb::kRingMaxCtas) * (size_t)qb::norm_sums(D) * 4;
}

extern "C" qb_status qb_layer_norm(const void* x, int type, const float* gamma, const float* beta, double eps, int64_t M, int64_t D, void* y, float* mean, float* rstd,
                                   void* cuda_stream) {
  using namespace qb;
  qb_status st = check_norm("qb_layer_norm", x && y && (mean != nullptr) == (rstd != nullptr) && eps >= 0.0 && eps < 3.0e38, type, M, D);
  if (st != QB_OK) return st;
  const size_t e = type == QB_F32 ? 4 : 2;
  if (!aligned_to(x, e) || !aligned_to(y, e) || !aligned_to(gamma, 4) || !aligned_to(beta, 4) || !aligned_to(mean, 4) || !aligned_to(rstd, 4)) {
    set_last_error("qb_layer_norm: every array must be aligned to its elements");
    return QB_ERR_ALIGN;
  }
  int sms = 0;
  if ((st = require_sm100(&sms)) != QB_OK) return st;
  const NormArgs a = {gamma, beta, mean, rstd, M, (int32_t)D, (float)eps, (float)(1.0 / (double)D), 1.0 / (double)D, aligned16(gamma) && aligned16(beta)};
  switch (type) {
    case QB_F32: return launch_norm<float>(x, y, a, sms, (cudaStream_t)cuda_stream);
    case QB_BF16: return launch_norm<__nv_bfloat16>(x, y, a, sms, (cudaStream_t)cuda_stream);
    default: return launch_norm<__half>(x, y, a, sms, (cudaStream_t)cuda_stream);
  }
}

extern "C" qb_status qb_layer_norm_backward(const void* grad_y, const void* x, int type, const float* gamma, const float* mean, const float* rstd, int64_t M, int64_t D,
                                            void* grad_x, float* grad_gamma, float* grad_beta, void* ws, size_t ws_bytes, void* cuda_stream) {
  using namespace qb;
  qb_status st = check_norm("qb_layer_norm_backward", grad_y && x && mean && rstd && grad_x, type, M, D);
  if (st != QB_OK) return st;
  const size_t e = type == QB_F32 ? 4 : 2;
  if (!aligned_to(grad_y, e) || !aligned_to(x, e) || !aligned_to(grad_x, e) || !aligned_to(gamma, 4) || !aligned_to(mean, 4) || !aligned_to(rstd, 4) || !aligned_to(grad_gamma, 4) ||
      !aligned_to(grad_beta, 4)) {
    set_last_error("qb_layer_norm_backward: every array must be aligned to its elements");
    return QB_ERR_ALIGN;
  }
  const bool sums = grad_gamma || grad_beta;
  if (sums && (!ws || !aligned16(ws) || ws_bytes < qb_layer_norm_workspace_bytes(M, D))) {
    set_last_error("qb_layer_norm_backward: workspace null, not 16-byte aligned or too small");
    return QB_ERR_WORKSPACE;
  }
  int sms = 0;
  if ((st = require_sm100(&sms)) != QB_OK) return st;
  sms = std::min(sms, kRingMaxCtas);
  const int warps = norm_warps(D), rows = D > kNormMostHeld ? 1 : 8 / warps;
  const int blocks = (int)std::min<int64_t>((M + rows - 1) / rows, sms);  // what is resident
  float* const parts = sums ? reinterpret_cast<float*>(static_cast<char*>(ws) + kNormPartsOff) : nullptr;
  const NormBackArgs a = {gamma, mean, rstd, parts, M, (int32_t)D, (float)(1.0 / (double)D), aligned16(gamma)};
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  int V = 1;
  switch (type) {
    case QB_F32: st = launch_norm_backward<float>(grad_y, x, grad_x, a, blocks, &V, stream); break;
    case QB_BF16: st = launch_norm_backward<__nv_bfloat16>(grad_y, x, grad_x, a, blocks, &V, stream); break;
    default: st = launch_norm_backward<__half>(grad_y, x, grad_x, a, blocks, &V, stream);
  }
  if (st != QB_OK || !sums) return st;
  const int32_t count = (int32_t)norm_sums(D);
  QB_CUDA_TRY(launch_kernel(layer_norm_join_kernel, (unsigned)((count + 31) / 32), 32 * kNormJoinGroups, 0, stream, 1, false, parts, blocks, count,
                            D > kNormMostHeld ? 0 : 32 * warps, V, (int32_t)D, grad_gamma, grad_beta));
  return QB_OK;
}
