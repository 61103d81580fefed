// qb_quantize_fp8 and qb_quantize_fp8_weights: 8-bit floating point codes with one power-of-two scale per block of 128.
//
// Per block: e is the least integer with max|x| * 2^-e <= the format's largest value (448 = 1.75 * 2^8 for e4m3,
// 57344 = 1.75 * 2^15 for e5m2), code = rn(x * 2^-e).  The scaling is exact, so a value is rounded once; nothing saturates.
// The scale is kept as the byte e + 127, which is the form in which the tensor cores take it (qb_gemm_fp8).
//
// max|x| is taken on the bit patterns (as unsigned integers they order like the magnitudes, infinities and NaN above every
// finite value), so that one integer reduction gives the maximum and says whether the block is finite.
//
// Bound by memory: x is read once; 1 byte per value and form is written, plus 1/128 for the scales.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "common.cuh"
#include "fp8.cuh"

namespace qb {

template <class T>
__device__ __forceinline__ float widen(T v) {
  if constexpr (std::is_same_v<T, float>) return v;
  else if constexpr (std::is_same_v<T, __half>) return __half2float(v);
  else return __bfloat162float(v);
}

// Four consecutive values of a row as they lie in memory.  The loads of a thread are all issued before the first value is
// widened: a conversion beside its load would wait for it, one load after the other.
template <class T>
struct Quad {
  typename std::conditional<sizeof(T) == 4, float4, uint2>::type raw;
  __device__ __forceinline__ void clear() { raw = {}; }
  __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const decltype(raw)*>(p); }
  // the first `left` of them, one by one: rows that are not aligned to four values, and a row's end
  __device__ __forceinline__ void load_some(const T* p, int64_t left) {
    clear();
    T* const e = reinterpret_cast<T*>(&raw);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) e[j] = p[j];
  }
  __device__ __forceinline__ float4 values() const {
    if constexpr (sizeof(T) == 4) {
      return raw;
    } else {
      const T* const e = reinterpret_cast<const T*>(&raw);
      return make_float4(widen(e[0]), widen(e[1]), widen(e[2]), widen(e[3]));
    }
  }
};

__device__ __forceinline__ uint32_t magnitude(float f) { return __float_as_uint(f) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t magnitude4(float4 v) {
  return max(max(magnitude(v.x), magnitude(v.y)), max(magnitude(v.z), magnitude(v.w)));
}

// The byte e + 127 for a block whose largest magnitude has these bits.  With max = 1.m * 2^E: e = E - 8 (e5m2: E - 15), one more
// where 1.m > 1.75.  Where the result is below 2^-127 (max|x| < 2^-119) it is held there.  0 and what is not finite: 1.
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits) {
  if (bits == 0u || bits >= 0x7F800000u) return 127u;
  const int e = (int)(bits >> 23) - (FMT == QB_E4M3 ? 8 : 15) + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(e, 0);
}
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Four codes, the first in the low byte.  cvt would turn infinities into the largest finite value: they become NaN here.
template <int FMT>
__device__ __forceinline__ uint32_t codes4(float4 v, float4 inv, bool finite) {
  if (!finite) {
    const float nan = __uint_as_float(0x7FC00000u);
    if (magnitude(v.x) >= 0x7F800000u) v.x = nan;
    if (magnitude(v.y) >= 0x7F800000u) v.y = nan;
    if (magnitude(v.z) >= 0x7F800000u) v.z = nan;
    if (magnitude(v.w) >= 0x7F800000u) v.w = nan;
  }
  v.x = __fmul_rn(v.x, inv.x);
  v.y = __fmul_rn(v.y, inv.y);
  v.z = __fmul_rn(v.z, inv.z);
  v.w = __fmul_rn(v.w, inv.w);
  uint16_t lo, hi;
  if constexpr (FMT == QB_E4M3) {
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(v.y), "f"(v.x));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(v.w), "f"(v.z));
  } else {
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(v.y), "f"(v.x));
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(v.w), "f"(v.z));
  }
  return (uint32_t)lo | ((uint32_t)hi << 16);
}
template <int FMT>
__device__ __forceinline__ uint32_t codes4(float4 v, float inv, bool finite) {
  return codes4<FMT>(v, make_float4(inv, inv, inv, inv), finite);
}

struct Fp8Args {
  int64_t M, K;      // x [M][K]
  int64_t Kp, Mp;    // rounded up to 128
  uint8_t* q;        // [M][Kp]
  uint8_t* scale;    // of q
  uint8_t* qt;       // [K][Mp] or NULL
  uint8_t* scale_t;
  void* ws;
  int vector;        // every row starts aligned to four values
};

// Rows only: a warp takes a segment of 512 columns of a row; lane l holds values 4 l .. 4 l + 3 of each of its four blocks, so
// that loads and stores are whole lines and a block's maximum is one warp reduction.
constexpr int kRowThreads = 256;
template <class T, int FMT>
__global__ void __launch_bounds__(kRowThreads) fp8_rows_kernel(const T* x, Fp8Args a) {
  const int lane = threadIdx.x & 31;
  const uint32_t kq = (uint32_t)fp8_scale_words(a.Kp), items = (uint32_t)a.M * kq;  // M <= 2^24, kq <= 2^7
  const uint32_t it = blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  pdl_begin();
  if (it >= items) return;
  const uint32_t row = it / kq, q = it - row * kq;
  const int c0 = (int)q * 512 + lane * 4, left = (int)a.K - c0;
  const T* const p = x + (int64_t)row * a.K + c0;
  Quad<T> v[4];
  if (a.vector) {  // K is a multiple of four: what is left of a row is too
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j].clear();
      if (left > j * 128) v[j].load(p + j * 128);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j].load_some(p + j * 128, left - j * 128);
  }
  uint8_t* const out = a.q + (int64_t)row * a.Kp + c0;
  uint32_t word = 0;
  bool finite = true;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float4 f = v[j].values();
    const uint32_t top = __reduce_max_sync(0xffffffffu, magnitude4(f));
    const uint32_t byte = scale_byte<FMT>(top);
    word |= byte << (8 * j);
    finite = finite && top < 0x7F800000u;
    const uint32_t code = codes4<FMT>(f, inverse_scale(byte), top < 0x7F800000u);
    if (c0 + j * 128 < (int)a.Kp) *reinterpret_cast<uint32_t*>(out + j * 128) = code;
  }
  if (lane == 0) {
    *reinterpret_cast<uint32_t*>(a.scale + fp8_scale_offset(row, 4 * q, kq)) = word;
    if (!finite) report_status(a.ws, QB_ERR_NONFINITE);
  }
}

// A tile of 128 x 128 values per block, held in registers (warp w: rows 16 w .. 16 w + 15, lane l: columns 4 l .. 4 l + 3).
// SQUARE: one scale for the tile (weights), else one per row for the codes and one per column for the transposed codes.
// The transposed codes cross shared memory, where a thread's 16 rows of a column are one 16-byte store, and leave as whole
// lines.
template <class T, int FMT, bool SQUARE>
__global__ void __launch_bounds__(256, 2) fp8_tile_kernel(const T* x, Fp8Args a) {
  __shared__ uint32_t tops[8][128];
  __shared__ uint4 turned[128 * 8];  // [column][8 pieces of 16 rows], piece p of column c at p ^ (c / 4 % 8)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t k_tiles = (uint32_t)(a.Kp / 128), mt = blockIdx.x / k_tiles, kt = blockIdx.x - mt * k_tiles;
  const int m0 = (int)mt * 128 + warp * 16, k0 = (int)kt * 128 + lane * 4;
  const int rows = (int)a.M - m0, left = (int)a.K - k0;  // rows of this warp's 16 and columns of this lane's four that exist
  pdl_begin();
  Quad<T> v[16];
  const T* const p = x + (int64_t)m0 * a.K + k0;
  if (a.vector) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      v[i].clear();
      if (i < rows && left > 0) v[i].load(p + i * a.K);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i].load_some(p + i * a.K, i < rows ? left : 0);
  }
  uint32_t col[4] = {0, 0, 0, 0};
  uint32_t row_top = 0;  // lane i: of row i
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float4 f = v[i].values();
    const uint32_t m[4] = {magnitude(f.x), magnitude(f.y), magnitude(f.z), magnitude(f.w)};
#pragma unroll
    for (int j = 0; j < 4; ++j) col[j] = max(col[j], m[j]);
    if constexpr (!SQUARE) {
      const uint32_t top = __reduce_max_sync(0xffffffffu, max(max(m[0], m[1]), max(m[2], m[3])));
      if (lane == i) row_top = top;
    }
  }
  if constexpr (SQUARE) {
    const uint32_t mine = __reduce_max_sync(0xffffffffu, max(max(col[0], col[1]), max(col[2], col[3])));
    if (lane == 0) tops[warp][0] = mine;
  } else {
    if (a.qt) *reinterpret_cast<uint4*>(&tops[warp][lane * 4]) = make_uint4(col[0], col[1], col[2], col[3]);
  }
  __syncthreads();
  if constexpr (SQUARE) {
#pragma unroll
    for (int w = 0; w < 8; ++w) row_top = max(row_top, tops[w][0]);
  }
  const uint32_t row_byte = scale_byte<FMT>(row_top);
  if (lane < 16 && lane < rows) {
    a.scale[fp8_scale_offset(m0 + lane, kt, fp8_scale_words(a.Kp))] = (uint8_t)row_byte;
    if (row_top >= 0x7F800000u) report_status(a.ws, QB_ERR_NONFINITE);
  }
  const bool rows_finite = __all_sync(0xffffffffu, row_top < 0x7F800000u);
  const float row_inv = inverse_scale(row_byte);
  uint8_t* const out = a.q + (int64_t)m0 * a.Kp + k0;
  uint32_t code[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float inv = SQUARE ? row_inv : __shfl_sync(0xffffffffu, row_inv, i);
    code[i] = codes4<FMT>(v[i].values(), inv, rows_finite);
    if (i < rows) *reinterpret_cast<uint32_t*>(out + i * a.Kp) = code[i];
  }
  if (!a.qt) return;
  if constexpr (!SQUARE) {  // the columns' own scales
    uint32_t top[4] = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const uint4 t = *reinterpret_cast<const uint4*>(&tops[w][lane * 4]);
      top[0] = max(top[0], t.x);
      top[1] = max(top[1], t.y);
      top[2] = max(top[2], t.z);
      top[3] = max(top[3], t.w);
    }
    float inv[4];
    bool finite = true;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t byte = scale_byte<FMT>(top[j]);
      inv[j] = inverse_scale(byte);
      finite = finite && top[j] < 0x7F800000u;
      if (warp == 0 && j < left) a.scale_t[fp8_scale_offset(k0 + j, mt, fp8_scale_words(a.Mp))] = (uint8_t)byte;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) code[i] = codes4<FMT>(v[i].values(), make_float4(inv[0], inv[1], inv[2], inv[3]), finite);
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

template <class T, int FMT>
static qb_status launch_fp8(const T* x, const Fp8Args& a, bool square, cudaStream_t stream) {
  if (!square && !a.qt) {
    const int64_t items = a.M * fp8_scale_words(a.Kp), blocks = (items + kRowThreads / 32 - 1) / (kRowThreads / 32);
    QB_CUDA_TRY(launch_kernel(fp8_rows_kernel<T, FMT>, (unsigned)blocks, kRowThreads, 0, stream, 1, false, x, a));
    return QB_OK;
  }
  auto kernel = square ? fp8_tile_kernel<T, FMT, true> : fp8_tile_kernel<T, FMT, false>;
  QB_CUDA_TRY(launch_kernel(kernel, (unsigned)((a.Mp / 128) * (a.Kp / 128)), 256, 0, stream, 1, false, x, a));
  return QB_OK;
}
template <class T>
static qb_status launch_fp8_format(const void* x, int format, const Fp8Args& a, bool square, cudaStream_t stream) {
  return format == QB_E4M3 ? launch_fp8<T, QB_E4M3>(static_cast<const T*>(x), a, square, stream)
                           : launch_fp8<T, QB_E5M2>(static_cast<const T*>(x), a, square, stream);
}

static qb_status quantize_fp8_entry(const char* who, const void* x, int type, int64_t M, int64_t K, int format, uint8_t* q, uint8_t* scale,
                                    uint8_t* qt, uint8_t* scale_t, void* ws, size_t ws_bytes, void* cuda_stream, bool square) {
  if (!x || !q || !scale || (qt == nullptr) != (scale_t == nullptr) || M <= 0 || K <= 0 || M > QB_MAX_MN ||
      K > (qt ? QB_MAX_MN : QB_MAX_K) || type < QB_F32 || type > QB_F16 || format < QB_E4M3 || format > QB_E5M2) {
    set_last_error("%s: invalid argument (M=%lld K=%lld type=%d format=%d)", who, (long long)M, (long long)K, type, format);
    return QB_ERR_INVALID;
  }
  const int64_t Kp = (K + 127) / 128 * 128, Mp = (M + 127) / 128 * 128;
  if ((Mp / 128) * (Kp / 128) > (int64_t)1 << 30) {
    set_last_error("%s: more than 2^30 blocks of 128 x 128 (M=%lld K=%lld)", who, (long long)M, (long long)K);
    return QB_ERR_INVALID;
  }
  const size_t size = type == QB_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(x) % size != 0 || !aligned16(q) || !aligned16(scale) || !aligned16(qt) || !aligned16(scale_t)) {
    set_last_error("%s: x must be aligned to its elements, codes and scales to 16 bytes", who);
    return QB_ERR_ALIGN;
  }
  if (!ws || ws_bytes < kWsMinBytes) {
    set_last_error("%s: workspace null or too small", who);
    return QB_ERR_WORKSPACE;
  }
  qb_status st = require_sm100(nullptr);
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
  a.ws = ws;
  a.vector = reinterpret_cast<uintptr_t>(x) % (4 * size) == 0 && K % 4 == 0;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  switch (type) {
    case QB_F32: return launch_fp8_format<float>(x, format, a, square, stream);
    case QB_BF16: return launch_fp8_format<__nv_bfloat16>(x, format, a, square, stream);
    default: return launch_fp8_format<__half>(x, format, a, square, stream);
  }
}

}  // namespace qb

extern "C" size_t qb_fp8_scale_bytes(int64_t rows, int64_t K) {
  if (rows <= 0 || K <= 0 || rows > QB_MAX_MN || K > QB_MAX_MN) return 0;
  return (size_t)((rows + 127) / 128 * qb::fp8_scale_words((K + 127) / 128 * 128) * 512);
}

extern "C" qb_status qb_quantize_fp8(const void* x, int type, int64_t M, int64_t K, int format, uint8_t* xq, uint8_t* x_scale,
                                     uint8_t* xqt, uint8_t* xt_scale, void* ws, size_t ws_bytes, void* cuda_stream) {
  return qb::quantize_fp8_entry("qb_quantize_fp8", x, type, M, K, format, xq, x_scale, xqt, xt_scale, ws, ws_bytes, cuda_stream, false);
}

extern "C" qb_status qb_quantize_fp8_weights(const void* w, int type, int64_t N, int64_t K, int format, uint8_t* wq, uint8_t* w_scale,
                                             uint8_t* wqt, uint8_t* wt_scale, void* ws, size_t ws_bytes, void* cuda_stream) {
  return qb::quantize_fp8_entry("qb_quantize_fp8_weights", w, type, N, K, format, wq, w_scale, wqt, wt_scale, ws, ws_bytes, cuda_stream, true);
}
