// qb_quantize_fp8 and qb_quantize_fp8_weights: 8-bit floating point codes with one power-of-two scale per block of 128.
//
// Per block: e is the least integer with max|x| * 2^-e <= the format's largest value (448 = 1.75 * 2^8 for e4m3,
// 57344 = 1.75 * 2^15 for e5m2), code = rn(x * 2^-e).  The scaling is exact, so a value is rounded once; nothing saturates.
// The scale is kept as the byte e + 127, which is the form in which the tensor cores take it (qb_gemm_fp8).
//
// max|x| is taken on the bit patterns (as unsigned integers they order like the magnitudes, infinities and NaN above every
// finite value), so that one integer reduction gives the maximum and says whether the block is finite.
//
// Bound by memory: x is read once; 1 byte per value and form is written, plus 1/128 for the scales.  24,576 x 4,096 bfloat16: rows 46 us
// (6.6 TB/s, the copy bandwidth; float16 46), both forms at once 68 us (5.9 TB/s; fp32 95 us, 6.4 TB/s; float16 74), weights with both
// forms 64 us.  The column sums come on top with a launch of their own: 9 us there, 4 at 6,144 x 4,096 (bfloat16 19.6 without), 1.5 at
// 613 x 768 (4.4).  Rows that are not aligned to four values: 24,576 x 4,095 bfloat16 rows 68 us, both forms 101.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "common.cuh"
#include "fp8.cuh"

namespace qb {

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// The byte e + 127 for a block whose largest magnitude has these bits (of fp32).  With max = 1.m * 2^E: e = E - 8 (e5m2: E - 15), one
// more where 1.m > 1.75.  Where the result is below 2^-127 (max|x| < 2^-119) it is held there.  0 and what is not finite: 1.
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits) {
  if (bits == 0u || bits >= 0x7F800000u) return 127u;
  const int e = (int)(bits >> 23) - (FMT == QB_E4M3 ? 8 : 15) + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(e, 0);
}

// Four codes, the first in the low byte.  cvt would turn infinities into the largest finite value.
template <int FMT>
__device__ __forceinline__ uint32_t codes_of(float x, float y, float z, float w) {
  uint16_t lo, hi;
  if constexpr (FMT == QB_E4M3) {
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(y), "f"(x));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(w), "f"(z));
  } else {
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(y), "f"(x));
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(w), "f"(z));
  }
  return (uint32_t)lo | ((uint32_t)hi << 16);
}
__device__ __forceinline__ float finite_or_nan(float f) {
  return (__float_as_uint(f) & 0x7FFFFFFFu) >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : f;
}

// Four consecutive values of a row as they lie in memory.  The loads of a thread are all issued before the first value is
// touched: a conversion beside its load would wait for it, one load after the other.
//
// Magnitudes stay packed (two 16-bit patterns are compared by one instruction): `Mag` is what the columns keep, `key` orders the
// largest of the four (the largest key of a warp, then `bits`, gives the magnitude as fp32 bits).  `Inv` is 2^-e as the scaling
// takes it: fp32, or bfloat16 twice, whose products with bfloat16 values are exact (what falls below its least
// normal number is far below the formats' and becomes 0 either way).
template <class T>
struct Quad {
  static constexpr bool kWide = sizeof(T) == 4;
  static constexpr bool kBf16 = std::is_same_v<T, __nv_bfloat16>;
  typedef typename std::conditional<kWide, uint4, uint2>::type Raw;
  typedef typename std::conditional<kWide, uint4, uint2>::type Mag;
  typedef typename std::conditional<kBf16, uint32_t, float>::type Inv;
  Raw raw;
  __device__ __forceinline__ void clear() { raw = {}; }
  __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const Raw*>(p); }
  // the first `left` of four values of any alignment
  __device__ __forceinline__ void load_each(const T* p, int left) {
    uint32_t e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      e[i] = 0u;
      if (i < left) {
        if constexpr (kWide) e[i] = reinterpret_cast<const uint32_t*>(p)[i];
        else e[i] = reinterpret_cast<const uint16_t*>(p)[i];
      }
    }
    if constexpr (kWide) raw = make_uint4(e[0], e[1], e[2], e[3]);
    else raw = make_uint2(e[0] | e[1] << 16, e[2] | e[3] << 16);
  }
  // Rows of any alignment are read by the aligned quads that have something of them: the four values that start `shift` (1 to 3) values
  // into this quad end in `next`.
  static __device__ __forceinline__ uint32_t part(uint32_t lo, uint32_t hi, int shift) { return shift & 1 ? __funnelshift_r(lo, hi, 16) : lo; }
  __device__ __forceinline__ void shift(const Quad& next, int shift) {
    if (shift == 0) return;
    if constexpr (kWide) {
      const Raw a = raw, b = next.raw;
      if (shift == 1) raw = make_uint4(a.y, a.z, a.w, b.x);
      else if (shift == 2) raw = make_uint4(a.z, a.w, b.x, b.y);
      else raw = make_uint4(a.w, b.x, b.y, b.z);
    } else {
      const uint32_t w0 = shift < 2 ? raw.x : raw.y, w1 = shift < 2 ? raw.y : next.raw.x, w2 = shift < 2 ? next.raw.x : next.raw.y;
      raw = make_uint2(part(w0, w1, shift), part(w1, w2, shift));
    }
  }
  // the quad of the lane that follows; lane 31 gets lane 0's `wrap`
  static __device__ __forceinline__ Quad of_next_lane(const Quad& q, const Quad& wrap, int lane) {
    Quad r;
    const int from = (lane + 1) & 31;
    r.raw.x = __shfl_sync(0xffffffffu, lane == 0 ? wrap.raw.x : q.raw.x, from);
    r.raw.y = __shfl_sync(0xffffffffu, lane == 0 ? wrap.raw.y : q.raw.y, from);
    if constexpr (kWide) {
      r.raw.z = __shfl_sync(0xffffffffu, lane == 0 ? wrap.raw.z : q.raw.z, from);
      r.raw.w = __shfl_sync(0xffffffffu, lane == 0 ? wrap.raw.w : q.raw.w, from);
    }
    return r;
  }
  // nothing behind the first `left` values
  __device__ __forceinline__ void keep(int left) {
    if (left >= 4) return;
    if constexpr (kWide) {
      raw = make_uint4(left > 0 ? raw.x : 0u, left > 1 ? raw.y : 0u, left > 2 ? raw.z : 0u, 0u);
    } else {
      raw = make_uint2(left > 1 ? raw.x : (left > 0 ? raw.x & 0xFFFFu : 0u), left > 2 ? raw.y & 0xFFFFu : 0u);
    }
  }
  __device__ __forceinline__ Mag magnitudes() const {
    if constexpr (kWide) return make_uint4(raw.x & 0x7FFFFFFFu, raw.y & 0x7FFFFFFFu, raw.z & 0x7FFFFFFFu, raw.w & 0x7FFFFFFFu);
    else return make_uint2(raw.x & 0x7FFF7FFFu, raw.y & 0x7FFF7FFFu);
  }
  static __device__ __forceinline__ Mag larger(Mag a, Mag b) {
    if constexpr (kWide) return make_uint4(max(a.x, b.x), max(a.y, b.y), max(a.z, b.z), max(a.w, b.w));
    else return make_uint2(max_u16x2(a.x, b.x), max_u16x2(a.y, b.y));
  }
  static __device__ __forceinline__ uint32_t key(Mag m) {
    if constexpr (kWide) {
      return max(max(m.x, m.y), max(m.z, m.w));
    } else {
      const uint32_t r = max_u16x2(m.x, m.y);
      return max(r, r << 16);  // the larger half on top decides
    }
  }
  // fp32 bits of a magnitude that is a key, or the upper half of a word
  static __device__ __forceinline__ uint32_t bits(uint32_t k) {
    if constexpr (kWide) return k;
    else if constexpr (kBf16) return k & 0xFFFF0000u;
    else return __float_as_uint(__half2float(__ushort_as_half((unsigned short)(k >> 16))));
  }
  static __device__ __forceinline__ uint32_t column_bits(Mag m, int j) {
    if constexpr (kWide) {
      return j == 0 ? m.x : (j == 1 ? m.y : (j == 2 ? m.z : m.w));
    } else {
      const uint32_t w = j < 2 ? m.x : m.y;
      return bits(j & 1 ? w : w << 16);
    }
  }
  static __device__ __forceinline__ Inv inverse(uint32_t byte) {
    if constexpr (kBf16) return (254u - byte) * 0x00800080u;
    else return __uint_as_float((254u - byte) << 23);
  }
  // the inverses of columns 2 i and 2 i + 1, and of a whole row, as `codes` takes them
  struct Pair {
    Inv a, b;
  };
  static __device__ __forceinline__ Pair columns(uint32_t byte0, uint32_t byte1) {
    if constexpr (kBf16) {
      const uint32_t both = (254u - byte0) << 7 | (254u - byte1) << 23;
      return {both, both};
    } else {
      return {inverse(byte0), inverse(byte1)};
    }
  }
  __device__ __forceinline__ float4 values() const {
    if constexpr (kWide) {
      return make_float4(__uint_as_float(raw.x), __uint_as_float(raw.y), __uint_as_float(raw.z), __uint_as_float(raw.w));
    } else if constexpr (kBf16) {
      return make_float4(__uint_as_float(raw.x << 16), __uint_as_float(raw.x & 0xFFFF0000u), __uint_as_float(raw.y << 16),
                         __uint_as_float(raw.y & 0xFFFF0000u));
    } else {
      const __half* const e = reinterpret_cast<const __half*>(&raw);
      return make_float4(__half2float(e[0]), __half2float(e[1]), __half2float(e[2]), __half2float(e[3]));
    }
  }
  // `lo` for the first two, `hi` for the last two values.  FINITE: the block has no NaN or infinity.
  template <int FMT, bool FINITE>
  __device__ __forceinline__ uint32_t codes(Pair lo, Pair hi) const {
    if constexpr (kBf16) {
      if constexpr (FINITE) {
        Quad q;
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(q.raw.x) : "r"(raw.x), "r"(lo.a));
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(q.raw.y) : "r"(raw.y), "r"(hi.a));
        const float4 f = q.values();
        return codes_of<FMT>(f.x, f.y, f.z, f.w);
      }
      const auto wide = [](uint32_t pair, bool upper) { return __uint_as_float(upper ? pair & 0xFFFF0000u : pair << 16); };
      const float4 f = values();
      return codes_of<FMT>(finite_or_nan(f.x) * wide(lo.a, false), finite_or_nan(f.y) * wide(lo.a, true), finite_or_nan(f.z) * wide(hi.a, false),
                           finite_or_nan(f.w) * wide(hi.a, true));
    } else {
      float4 f = values();
      if constexpr (!FINITE) f = make_float4(finite_or_nan(f.x), finite_or_nan(f.y), finite_or_nan(f.z), finite_or_nan(f.w));
      return codes_of<FMT>(__fmul_rn(f.x, lo.a), __fmul_rn(f.y, lo.b), __fmul_rn(f.z, hi.a), __fmul_rn(f.w, hi.b));
    }
  }
};

constexpr size_t kSumsOff = 1024;  // of the tiles' column sums in the workspace

struct Fp8Args {
  int64_t M, K;      // x [M][K]
  int64_t Kp, Mp;    // rounded up to 128
  uint8_t* q;        // [M][Kp]
  uint8_t* scale;    // of q
  uint8_t* qt;       // [K][Mp] or NULL
  uint8_t* scale_t;
  float* sums;       // [Mp / 128][K]: the sums of the tiles' columns, or NULL
  void* ws;
  int vector;        // every row starts aligned to four values
};

// Rows only: a warp takes two segments of 512 columns of a row (of neighbouring rows at a row's end); lane l holds values
// 4 l .. 4 l + 3 of each of the eight blocks, so that loads and stores are whole lines and a block's maximum is one warp
// reduction.  Lane j finishes block j (its scale, the byte), and the factors come back by shuffle.
constexpr int kRowThreads = 256;
template <class T, int FMT>
__global__ void __launch_bounds__(kRowThreads) fp8_rows_kernel(const T* x, Fp8Args a) {
  const int lane = threadIdx.x & 31;
  const uint32_t kq = (uint32_t)fp8_scale_words(a.Kp), items = (uint32_t)a.M * kq;  // at most 2^30
  const uint32_t it = 2 * (blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5));
  pdl_begin();
  if (it >= items) return;
  uint32_t row[2], q[2];
  row[0] = it / kq;
  q[0] = it - row[0] * kq;
  const bool wrap = q[0] + 1 == kq;
  row[1] = row[0] + (wrap ? 1 : 0);
  q[1] = wrap ? 0 : q[0] + 1;
  const int K = (int)a.K;
  Quad<T> v[8];
  if (a.vector) {  // every row begins with a quad, and K is a multiple of four: what is left of a row is too
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int c0 = (int)q[s] * 512 + lane * 4;
      const T* const p = x + (int64_t)row[s] * a.K + c0;
      const int left = (s == 0 || it + 1 < items) ? K - c0 : 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[4 * s + j].clear();
        if (left > j * 128) v[4 * s + j].load(p + j * 128);
      }
    }
  } else {
    Quad<T> behind[2];  // lane 0: the quad behind the segment
    int off[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int64_t base = (int64_t)row[s] * a.K + (int)q[s] * 512;
      const T* const p = x + base;
      off[s] = (int)(reinterpret_cast<uintptr_t>(p) / sizeof(T)) & 3;
      const int left = (s == 0 || it + 1 < items) ? K - (int)q[s] * 512 : 0;  // of the segment and what follows
      behind[s].clear();
      if (fp8_at_edge(base, base, left, 512, a.M * a.K)) {  // the first and the last segment of x
        off[s] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * s + j].load_each(p + j * 128 + lane * 4, left - j * 128 - lane * 4);
        continue;
      }
      // a quad is read where it has something of the row
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = fp8_quad_at(j, lane, off[s]);
        v[4 * s + j].clear();
        if (at < left && left > 0) v[4 * s + j].load(p + at);
      }
      if (lane == 0 && fp8_needs_behind(512, off[s], left)) behind[s].load(p + 512 - off[s]);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int left = (s == 0 || it + 1 < items) ? K - (int)q[s] * 512 - lane * 4 : 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const Quad<T> next = Quad<T>::of_next_lane(v[4 * s + j], j < 3 ? v[4 * s + (j + 1) % 4] : behind[s], lane);
        v[4 * s + j].shift(next, off[s]);
        v[4 * s + j].keep(left - j * 128);
      }
    }
  }
  uint32_t mine = 0;  // lane j: the largest key of block j
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t top = __reduce_max_sync(0xffffffffu, Quad<T>::key(v[j].magnitudes()));
    if (lane == j) mine = top;
  }
  const uint32_t top = Quad<T>::bits(mine), byte = scale_byte<FMT>(top);
  const bool finite = __all_sync(0xffffffffu, top < 0x7F800000u);
  if (lane < 8) {
    const uint32_t s = lane >> 2, block = 4 * (s ? q[1] : q[0]) + (lane & 3);
    if (it + s < items) a.scale[fp8_scale_offset(s ? row[1] : row[0], block, kq)] = (uint8_t)byte;
    if (top >= 0x7F800000u) report_status(a.ws, QB_ERR_NONFINITE);
  }
  const typename Quad<T>::Inv inv = Quad<T>::inverse(byte);
  const auto write = [&](auto all_finite) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (s == 1 && it + 1 >= items) break;
      const int c0 = (int)q[s] * 512 + lane * 4;
      uint8_t* const out = a.q + (int64_t)row[s] * a.Kp + c0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const typename Quad<T>::Inv i = __shfl_sync(0xffffffffu, inv, 4 * s + j);
        const uint32_t code = v[4 * s + j].template codes<FMT, decltype(all_finite)::value>({i, i}, {i, i});
        if (c0 + j * 128 < (int)a.Kp) *reinterpret_cast<uint32_t*>(out + j * 128) = code;
      }
    }
  };
  if (finite) write(std::true_type());
  else write(std::false_type());
}

// A tile of 128 x 128 values per block, held in registers (warp w: rows 16 w .. 16 w + 15, lane l: columns 4 l .. 4 l + 3).
// SQUARE: one scale for the tile (weights), else one per row for the codes and one per column for the transposed codes.
// The transposed codes cross shared memory, where a thread's 16 rows of a column are one 16-byte store, and leave as whole
// lines.
// BLOCKS per SM: what a block waits for is hidden by the others.
template <class T, int FMT, bool SQUARE, int BLOCKS>
__global__ void __launch_bounds__(256, BLOCKS) fp8_tile_kernel(const T* x, Fp8Args a) {
  typedef typename Quad<T>::Mag Mag;
  typedef typename Quad<T>::Pair Pair;
  __shared__ Mag tops[8][32];
  __shared__ uint32_t squares[8];
  __shared__ float4 sums[SQUARE ? 1 : 8][32];
  __shared__ uint4 turned[128 * 8];  // [column][8 pieces of 16 rows], piece p of column c at p ^ (c / 4 % 8)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t k_tiles = (uint32_t)(a.Kp / 128), mt = blockIdx.x / k_tiles, kt = blockIdx.x - mt * k_tiles;
  const int m0 = (int)mt * 128 + warp * 16, k0 = (int)kt * 128 + lane * 4;
  const int rows = (int)a.M - m0, left = (int)a.K - k0;  // rows of this warp's 16 and columns of this lane's four that exist
  pdl_begin();
  Quad<T> v[16];
  const T* const p = x + (int64_t)m0 * a.K + k0;
  if (a.vector && rows >= 16 && (int)kt * 128 + 128 <= (int)a.K) {  // all there, every row begins with a quad
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i].load(p + i * a.K);
  } else {
    // as in the rows form
    const T* const first = x + (int64_t)m0 * a.K + (int64_t)kt * 128;
    const int wide = (int)a.K - (int)kt * 128;  // columns of the tile and behind it
    if (fp8_at_edge(first - x, first - x + (min(rows, 16) - 1) * a.K, wide, 128, a.M * a.K)) {  // x's first and last rows
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        v[i].load_each(p + i * a.K, i < rows ? left : 0);
        asm volatile("" ::: "memory");  // a row at a time: 64 loads in flight would not leave room in 64 registers
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const T* const r = first + i * a.K;
        const int at = fp8_quad_at(0, lane, (int)(reinterpret_cast<uintptr_t>(r) / sizeof(T)) & 3);
        v[i].clear();
        if (i < rows && at < wide) v[i].load(r + at);
      }
      // the quads behind the tile's columns: lane i has row i's
      Quad<T> behind;
      behind.clear();
      if (lane < 16 && lane < rows) {
        const T* const r = first + lane * a.K;
        const int off = (int)(reinterpret_cast<uintptr_t>(r) / sizeof(T)) & 3;
        if (fp8_needs_behind(128, off, wide)) behind.load(r + 128 - off);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int off = (int)(reinterpret_cast<uintptr_t>(first + i * a.K) / sizeof(T)) & 3;
        Quad<T> wrap;
        wrap.raw.x = __shfl_sync(0xffffffffu, behind.raw.x, i);
        wrap.raw.y = __shfl_sync(0xffffffffu, behind.raw.y, i);
        if constexpr (sizeof(T) == 4) {
          wrap.raw.z = __shfl_sync(0xffffffffu, behind.raw.z, i);
          wrap.raw.w = __shfl_sync(0xffffffffu, behind.raw.w, i);
        }
        v[i].shift(Quad<T>::of_next_lane(v[i], wrap, lane), off);
        v[i].keep(i < rows ? left : 0);
      }
    }
  }
  Mag col = v[0].magnitudes();
  uint32_t row_key = 0;  // lane i: of row i
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const Mag m = v[i].magnitudes();
    if (i > 0) col = Quad<T>::larger(col, m);
    if constexpr (!SQUARE) {
      const uint32_t top = __reduce_max_sync(0xffffffffu, Quad<T>::key(m));
      if (lane == i) row_key = top;
    }
  }
  if constexpr (SQUARE) {
    const uint32_t mine = __reduce_max_sync(0xffffffffu, Quad<T>::key(col));
    if (lane == 0) squares[warp] = mine;
  } else {
    if (a.qt) tops[warp][lane] = col;
    if (a.sums) {
      float4 t = v[0].values();
#pragma unroll
      for (int i = 1; i < 16; ++i) {
        const float4 f = v[i].values();
        t.x += f.x;
        t.y += f.y;
        t.z += f.z;
        t.w += f.w;
      }
      sums[warp][lane] = t;
    }
  }
  __syncthreads();
  if constexpr (!SQUARE) {
    if (a.sums && warp == 0) {
      float4 t = sums[0][lane];
#pragma unroll
      for (int w = 1; w < 8; ++w) {
        const float4 f = sums[w][lane];
        t.x += f.x;
        t.y += f.y;
        t.z += f.z;
        t.w += f.w;
      }
      const float part[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < left) a.sums[(int64_t)mt * a.K + k0 + j] = part[j];
    }
  }
  if constexpr (SQUARE) {
#pragma unroll
    for (int w = 0; w < 8; ++w) row_key = max(row_key, squares[w]);
  }
  const uint32_t row_top = Quad<T>::bits(row_key), row_byte = scale_byte<FMT>(row_top);
  if (lane < 16 && lane < rows) {
    a.scale[fp8_scale_offset(m0 + lane, kt, fp8_scale_words(a.Kp))] = (uint8_t)row_byte;
    if (row_top >= 0x7F800000u) report_status(a.ws, QB_ERR_NONFINITE);
  }
  const bool rows_finite = __all_sync(0xffffffffu, row_top < 0x7F800000u);
  const typename Quad<T>::Inv row_inv = Quad<T>::inverse(row_byte);
  uint8_t* const out = a.q + (int64_t)m0 * a.Kp + k0;
  uint32_t code[16];
  const auto write = [&](auto all_finite) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const typename Quad<T>::Inv inv = SQUARE ? row_inv : __shfl_sync(0xffffffffu, row_inv, i);
      code[i] = v[i].template codes<FMT, decltype(all_finite)::value>(Pair{inv, inv}, Pair{inv, inv});
      if (i < rows) *reinterpret_cast<uint32_t*>(out + i * a.Kp) = code[i];
    }
  };
  if (rows_finite) write(std::true_type());
  else write(std::false_type());
  if (!a.qt) return;
  if constexpr (!SQUARE) {  // the columns' own scales
#pragma unroll
    for (int w = 0; w < 8; ++w) col = Quad<T>::larger(col, tops[w][lane]);
    uint32_t byte[4];
    bool finite = true;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t top = Quad<T>::column_bits(col, j);
      byte[j] = scale_byte<FMT>(top);
      finite = finite && top < 0x7F800000u;
      if (warp == 0 && j < left) a.scale_t[fp8_scale_offset(k0 + j, mt, fp8_scale_words(a.Mp))] = (uint8_t)byte[j];
    }
    const Pair lo = Quad<T>::columns(byte[0], byte[1]), hi = Quad<T>::columns(byte[2], byte[3]);
    if (__all_sync(0xffffffffu, finite)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) code[i] = v[i].template codes<FMT, true>(lo, hi);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) code[i] = v[i].template codes<FMT, false>(lo, hi);
    }
  } else if (warp == 0) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) a.scale_t[fp8_scale_offset(k0 + j, mt, fp8_scale_words(a.Mp))] = (uint8_t)row_byte;
  }
  // 16 rows x 4 columns of codes, column by column
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t sel = (uint32_t)(j | ((j + 4) << 4));
      const uint32_t lo = __byte_perm(code[4 * i], code[4 * i + 1], sel), hi = __byte_perm(code[4 * i + 2], code[4 * i + 3], sel);
      w[i] = __byte_perm(lo, hi, 0x5410);
    }
    turned[(lane * 4 + j) * 8 + (warp ^ (lane & 7))] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = i * 256 + threadIdx.x, c = at >> 3, piece = at & 7;
    if ((int)kt * 128 + c < a.K)
      *reinterpret_cast<uint4*>(a.qt + ((int64_t)kt * 128 + c) * a.Mp + (int64_t)mt * 128 + piece * 16) = turned[c * 8 + (piece ^ ((c >> 2) & 7))];
  }
}

// out[k] = the tiles' sums of column k: every warp of a block adds up every eighth tile, then the warps are joined in order.
__global__ void __launch_bounds__(256) fp8_sums_kernel(const float* parts, int tiles, int K, float* out) {
  __shared__ float joined[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = blockIdx.x * 32 + lane;
  pdl_begin();
  float t = 0.0f;
  if (k < K) {
#pragma unroll 8
    for (int i = warp; i < tiles; i += 8) t += parts[(int64_t)i * K + k];
  }
  joined[warp][lane] = t;
  __syncthreads();
  if (warp != 0 || k >= K) return;
#pragma unroll
  for (int w = 1; w < 8; ++w) t += joined[w][lane];
  out[k] = t;
}

template <class T, int FMT>
static qb_status launch_fp8(const T* x, const Fp8Args& a, bool square, int sms, cudaStream_t stream) {
  if (!square && !a.qt) {
    const int64_t items = a.M * fp8_scale_words(a.Kp), blocks = (items + kRowThreads / 16 - 1) / (kRowThreads / 16);
    QB_CUDA_TRY(launch_kernel<kMostL1>(fp8_rows_kernel<T, FMT>, (unsigned)blocks, kRowThreads, 0, stream, 1, false, x, a));
    return QB_OK;
  }
  const int64_t tiles = (a.Mp / 128) * (a.Kp / 128);
  // 16 bits: three blocks per SM where they take all tiles at once, else four (bfloat16, rows and columns, 18,944 x 384: 6.3 us, with
  // four 7.5; 24,576 x 4,096: 73.3 and 68.2; weights 4.9 and 5.6, 64.5 and 63.6).  fp16's rows and columns do not fit 64 registers.
  constexpr bool kWide = sizeof(T) == 4;
  constexpr int kFew = kWide ? 2 : 3, kMany = kWide ? 2 : 4, kManyBoth = std::is_same_v<T, __nv_bfloat16> ? 4 : kFew;
  const bool many = tiles > (int64_t)kFew * sms;
  auto kernel = square ? (many ? fp8_tile_kernel<T, FMT, true, kMany> : fp8_tile_kernel<T, FMT, true, kFew>)
                       : (many ? fp8_tile_kernel<T, FMT, false, kManyBoth> : fp8_tile_kernel<T, FMT, false, kFew>);
  QB_CUDA_TRY(launch_kernel(kernel, (unsigned)tiles, 256, 0, stream, 1, false, x, a));
  return QB_OK;
}
template <class T>
static qb_status launch_fp8_format(const void* x, int format, const Fp8Args& a, bool square, int sms, cudaStream_t stream) {
  return format == QB_E4M3 ? launch_fp8<T, QB_E4M3>(static_cast<const T*>(x), a, square, sms, stream)
                           : launch_fp8<T, QB_E5M2>(static_cast<const T*>(x), a, square, sms, stream);
}

static qb_status quantize_fp8_entry(const char* who, const void* x, int type, int64_t M, int64_t K, int format, uint8_t* q, uint8_t* scale,
                                    uint8_t* qt, uint8_t* scale_t, float* sums, void* ws, size_t ws_bytes, void* cuda_stream, bool square) {
  if (!x || !q || !scale || (qt == nullptr) != (scale_t == nullptr) || (sums && !qt) || M <= 0 || K <= 0 || M > QB_MAX_MN || K > QB_MAX_MN ||
      type < QB_F32 || type > QB_F16 || format < QB_E4M3 || format > QB_E5M2) {
    set_last_error("%s: invalid argument (M=%lld K=%lld type=%d format=%d)", who, (long long)M, (long long)K, type, format);
    return QB_ERR_INVALID;
  }
  const int64_t Kp = (K + 127) / 128 * 128, Mp = (M + 127) / 128 * 128;
  if ((Mp / 128) * (Kp / 128) > (int64_t)1 << 30 || M * fp8_scale_words(Kp) > (int64_t)1 << 30) {
    set_last_error("%s: more than 2^30 blocks of 128 x 128 or segments of 512 (M=%lld K=%lld)", who, (long long)M, (long long)K);
    return QB_ERR_INVALID;
  }
  const size_t size = type == QB_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(x) % size != 0 || !aligned16(q) || !aligned16(scale) || !aligned16(qt) || !aligned16(scale_t) ||
      reinterpret_cast<uintptr_t>(sums) % 4 != 0) {
    set_last_error("%s: x and the sums must be aligned to their elements, codes and scales to 16 bytes", who);
    return QB_ERR_ALIGN;
  }
  const size_t need = sums ? qb_fp8_sums_workspace_bytes(M, K) : kWsMinBytes;
  if (!ws || ws_bytes < need || reinterpret_cast<uintptr_t>(ws) % 4 != 0) {
    set_last_error("%s: workspace null, not aligned or smaller than %zu bytes", who, need);
    return QB_ERR_WORKSPACE;
  }
  int sms = 0;
  qb_status st = require_sm100(&sms);
  if (st != QB_OK) return st;
  Fp8Args a;
  a.M = M;
  a.K = K;
  a.Kp = Kp;
  a.Mp = Mp;
  a.q = q;
  a.scale = scale;
  a.qt = qt;
  a.scale_t = scale_t;
  a.sums = sums ? reinterpret_cast<float*>(static_cast<char*>(ws) + kSumsOff) : nullptr;
  a.ws = ws;
  a.vector = reinterpret_cast<uintptr_t>(x) % (4 * size) == 0 && K % 4 == 0;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  switch (type) {
    case QB_F32: st = launch_fp8_format<float>(x, format, a, square, sms, stream); break;
    case QB_BF16: st = launch_fp8_format<__nv_bfloat16>(x, format, a, square, sms, stream); break;
    default: st = launch_fp8_format<__half>(x, format, a, square, sms, stream);
  }
  if (st != QB_OK || !sums) return st;
  QB_CUDA_TRY(launch_kernel(fp8_sums_kernel, (unsigned)((K + 31) / 32), 256, 0, stream, 1, false, a.sums, (int)(Mp / 128), (int)K, sums));
  return QB_OK;
}

}  // namespace qb

extern "C" size_t qb_fp8_scale_bytes(int64_t rows, int64_t K) {
  if (rows <= 0 || K <= 0 || rows > QB_MAX_MN || K > QB_MAX_MN) return 0;
  return (size_t)((rows + 127) / 128 * qb::fp8_scale_words((K + 127) / 128 * 128) * 512);
}

extern "C" size_t qb_fp8_sums_workspace_bytes(int64_t M, int64_t K) {
  if (M <= 0 || K <= 0 || M > QB_MAX_MN || K > QB_MAX_MN) return 0;
  return (size_t)(qb::kSumsOff + (M + 127) / 128 * K * 4);
}

extern "C" qb_status qb_quantize_fp8(const void* x, int type, int64_t M, int64_t K, int format, uint8_t* xq, uint8_t* x_scale,
                                     uint8_t* xqt, uint8_t* xt_scale, float* col_sums, void* ws, size_t ws_bytes, void* cuda_stream) {
  return qb::quantize_fp8_entry("qb_quantize_fp8", x, type, M, K, format, xq, x_scale, xqt, xt_scale, col_sums, ws, ws_bytes, cuda_stream, false);
}

extern "C" qb_status qb_quantize_fp8_weights(const void* w, int type, int64_t N, int64_t K, int format, uint8_t* wq, uint8_t* w_scale,
                                             uint8_t* wqt, uint8_t* wt_scale, void* ws, size_t ws_bytes, void* cuda_stream) {
  return qb::quantize_fp8_entry("qb_quantize_fp8_weights", w, type, N, K, format, wq, w_scale, wqt, wt_scale, nullptr, ws, ws_bytes, cuda_stream, true);
}
