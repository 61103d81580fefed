// qb_linear, qb_linear_grad_x, qb_linear_grad_w: the three products of a linear in 16-bit floating point,
//     y = act(x w^T + bias) + residual,     grad_x = (grad_y w) * gelu'(p) + residual,     grad_w = grad_y^T x,
// with everything behind the product done on its way out of tensor memory.
//
// One product kernel for all of them, out[m][n] = sum_k A(m, k) B(n, k): persistent CTAs (tcgen05 kind::f16, fp32 accumulators), K blocks
// of 64, two blocks a stage.  An operand lies in shared memory as its tensor has it: contraction along its rows (K-major: x and w of
// the forward pass, grad_y of grad_x) or down its columns (MN-major: w of grad_x, both operands of grad_w), so that nothing is
// transposed in memory.  20 warps:
//   warp 0        TMA producer (one lane)
//   warp 1        issues tcgen05.mma, owns the tensor memory (one lane)
//   warps 2..3    idle (one thread leaves the call's mark: begin_under)
//   warps 4..19   epilogue, four per TMEM lane quarter: tcgen05.ld -> bias, GELU or its slope, residual -> shared memory -> TMA store
// A tile is 128 rows of A per CTA x BT rows of B; TMEM lane = row, column = column of the output.  Large products run as CTA pairs
// (cta_group::2, 256 x 256 or 256 x 128).  No load is multicast.  Two accumulators, so that a tile's epilogue overlaps the products of the
// next.  Every wait is bounded: on expiry the CTA records QB_ERR_TIMEOUT and leaves through the normal exit path.
//
// Bound by the tensor cores' operands (after a pause, in us): 24,576 x 4,096, K = 1,024 140 (1,470 TFLOP/s; a library's product 149), 24,576 x
// 1,024, K = 4,096 140 (141), grad_w 24,576 x 4,096 x 1,024 in fp32 143 (138).  A pair's K block is 64 KB for 512 cycles of products; shared memory is
// written and read at 64 bytes a clock each, its whole bandwidth, and the tensor pipe is busy for 75 %.  What the epilogue adds shows where K is
// 1,024 or less: GELU 150, a residual 157 (200 MB more through L2, where the operands come from too), GELU with the
// pre-activation saved in 8 bits 170 or in 16 bits 171, the gradient through GELU 166 (13 of an element's instructions are GELU's slope).  Small products by
// their chain: 32 x 768 x 768 4.7 us, of which 0.9 until the kernel before has ended, 0.9 until the first operands are there, 1.6 for six
// stages, 0.8 from the accumulator to memory.
// Sixteen epilogue warps on 32 columns each (eight on 64 columns took as long, with GELU for eight values at a time instead of
// two 10 to 50 us less at 24,576 x 4,096 x 1,024).  Tried and not kept: fp32 sums added up in memory by TMA (10 us more, and longer runs), the columns'
// sums of grad_bias by the epilogue out of shared memory (14 to 59 us more).  Twenty warps leave 96 registers a thread: tiles of 256 x 256 with fp32 outputs
// spill 64 bytes, the 16-bit forms 12 at most.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>

#include "checkpoint.cuh"
#include "common.cuh"
#include "gelu.cuh"
#include "mbar_wait.cuh"
#include "ptx_float.cuh"
#include "tensormap.cuh"

namespace qb {

// How an operand lies and is loaded, two K blocks of 64 at a time: K-major (rows x 2 groups of 64 columns) or MN-major (128 rows along
// K x groups of 64 columns); one box of three dimensions, or, where rows are no multiple of 128 bytes, a box per group.
enum LinearForm { kRows = 0, kRows2 = 1, kCols = 2, kCols2 = 3 };
// The output: of the operands' type, fp32, or of their type from several runs over K.
enum LinearOut { kOut16 = 0, kOut32 = 1, kOut16Runs = 2 };
// What the epilogue does with the product besides bias, residual and what is saved.
enum LinearMode { kPlain = 0, kGelu = 1, kSlope = 2 };

struct LinearParams {
  CUtensorMap tma, tmb;  // operands
  CUtensorMap tmb_half;  // pairs: B for a tile of half the width
  CUtensorMap tmy;       // out (or the splits' parts, one after the other) in boxes of 32 rows x 64 bytes
  const float* bias;     // or NULL
  const void* side;      // residual, or 16-bit pre-activation (kSlope), [M][N] of out's type; or NULL
  const int8_t* codes;   // kSlope: the pre-activation in 8 bits, or NULL
  const float* scales;
  void* out;
  void* pre;             // receives the pre-activation in 16 bits, or NULL
  int8_t* pre_codes;     // receives it in 8 bits, or NULL
  float* pre_scales;
  void* ws;
  int32_t M, N;
  int32_t a_form, b_form;
  int32_t n_tiles, tiles;
  uint32_t n_tiles_inv, split_tiles_inv;  // quick_inverse
  int32_t whole;         // tiles below this are BT wide; pairs: the others are halves, two after the other
  int32_t split_tiles;   // tiles of one split of K (split s writes rows s * M .. of out, fp32)
  int32_t split_blocks;  // K blocks of 64 per split, even where there are several
  int32_t k_blocks;      // of all splits
  int32_t run_blocks;    // K blocks that one accumulator sums; even where there are several such runs, which registers add up
  int32_t tma_store;     // 1: rows of out are 16-byte aligned
  int32_t vector;        // 1: rows of side and of pre are 16-byte aligned, 2: 32-byte aligned
  int32_t vector_codes;  // the same of the codes'
  uint32_t idesc;
  uint32_t mark;         // even where a kernel of this call will run under this one: left in the workspace (begin_under)
};

constexpr int kLinEpilogueWarps = 16;
constexpr int kLinFirstEpilogueWarp = 4;
constexpr int kLinThreads = 32 * (kLinFirstEpilogueWarp + kLinEpilogueWarps);

template <int BT, int CG>
struct LinCfg {
  static constexpr int kABytes = 2 * 128 * 128;          // 128 rows, two K blocks of 128 bytes
  static constexpr int kBBytes = 2 * (BT / CG) * 128;
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kStages = BT / CG == 64 ? 4 : 3;
  static constexpr int kOutBytes = kLinEpilogueWarps * 2048;
  static constexpr int kBarBytes = 256;
  static constexpr int kBiasBytes = kLinEpilogueWarps * 32 * 4;
  static constexpr int kSmemBytes = kStages * kStageBytes + kOutBytes + kBarBytes + kBiasBytes;
  static constexpr int kTmemCols = 2 * BT;
  static_assert(kSmemBytes <= 232448, "shared memory");
};

// Shared-memory descriptor of an operand with 128-byte swizzle.  K-major: 1024 bytes between groups of eight rows.  MN-major: 64
// consecutive elements of M or N are a row of 128 bytes, the next 64 are 16384 bytes on (leading offset), the next eight of K 1024
// bytes (stride offset).  Version 1 (bits 46-47), SWIZZLE_128B (61-63 = 2).
__device__ __forceinline__ uint64_t lin_desc(uint32_t smem_addr, bool mn) {
  return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | (uint64_t)(mn ? 16384 >> 4 : 1) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}
// Instruction descriptor for kind::f16 without N >> 3 (bits 17-22): D fp32 (bits 4-5 = 1), A and B of one type (7-9, 10-12: fp16 0,
// bfloat16 1), MN-major A and B (15, 16), M >> 4 (24-28).
static uint32_t lin_idesc(bool half_type, bool a_mn, bool b_mn, int mma_m) {
  const uint32_t t = half_type ? 0u : 1u;
  return (1u << 4) | (t << 7) | (t << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(mma_m >> 4) << 24);
}

// t / d for 0 <= t < 2^31 and d > 0 by a product with quick_inverse(d) = 2^32 / d rounded down (for 1: 2^32 - 1): short of the quotient by one
// at most (t / 2^32 and a unit of the last place).
static uint32_t quick_inverse(uint32_t d) { return d == 1 ? 0xFFFFFFFFu : (uint32_t)(((uint64_t)1 << 32) / d); }
__device__ __forceinline__ int quick_divide(int t, int d, uint32_t inverse) {
  const int q = (int)__umulhi((uint32_t)t, inverse);
  return q + (t - q * d >= d ? 1 : 0);
}

// Where tile t lies: first row and column, columns, split and its range of K blocks.
template <int BT, int CG>
struct LinTile {
  int m0, n0, width, split, k0, k1;
  __device__ __forceinline__ LinTile(const LinearParams& gp, int t) {
    split = quick_divide(t, gp.split_tiles, gp.split_tiles_inv);
    t -= split * gp.split_tiles;
    k0 = split * gp.split_blocks;
    k1 = min(k0 + gp.split_blocks, gp.k_blocks);
    width = BT;
    int half = 0;
    if (CG == 2 && t >= gp.whole) {
      half = (t - gp.whole) & 1;
      t = gp.whole + ((t - gp.whole) >> 1);
      width = BT / 2;
    }
    m0 = quick_divide(t, gp.n_tiles, gp.n_tiles_inv);
    n0 = (t - m0 * gp.n_tiles) * BT + half * (BT / 2);
    m0 *= 128 * CG;
  }
};

// Two 16-bit values of a word, and back.
__device__ __forceinline__ float2 unpack16(uint32_t w, bool half_type) {
  if (half_type) return __half22float2(*reinterpret_cast<const __half2*>(&w));
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ uint32_t pack16(float lo, float hi, bool half_type) {
  if (half_type) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// A warp's staging buffer: 32 rows of 64 bytes, 16-byte pieces swizzled as TMA does it (64-byte swizzle), so that the lanes meet
// different banks with a row a lane.
__device__ __forceinline__ uint4* staged(uint8_t* buf, int row, int piece) {
  return reinterpret_cast<uint4*>(buf + row * 64 + ((piece ^ ((row >> 1) & 3)) << 4));
}

// Two values added to z[0] and z[1].
__device__ __forceinline__ void add2(float* z, float a, float b) {
  const float2 f = ptx::unpack_f32x2(ptx::add_f32x2(ptx::pack_f32x2(z[0], z[1]), ptx::pack_f32x2(a, b)));
  z[0] = f.x;
  z[1] = f.y;
}

// Eight columns of an accumulator added to z.
__device__ __forceinline__ void add_accumulator(uint32_t taddr, float* z) {
  uint32_t w[8];
  ptx::tmem_ld_32x32b_x8(taddr, w);
  ptx::tmem_ld_wait();
  ptx::tmem_ld_regs_ready(w);
#pragma unroll
  for (int c = 0; c < 8; c += 2) add2(z + c, __uint_as_float(w[c]), __uint_as_float(w[c + 1]));
}

// 32 bytes of a row, `wide`: whole sectors, where 16 bytes a lane would touch each of them twice; else 16 and, if `second`, the other 16.
__device__ __forceinline__ void load_row(const void* p, bool wide, bool second, uint4& a, uint4& b) {
  if (wide) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w)
                 : "l"(p));
  } else {
    a = *static_cast<const uint4*>(p);
    if (second) b = static_cast<const uint4*>(p)[1];
  }
}
__device__ __forceinline__ void store32(void* p, const uint4& a, const uint4& b) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z),
               "r"(b.w)
               : "memory");
}

// `rows` rows of `cols` 16-bit values from the staging buffer to rows of any alignment, `pitch` elements apart: two rows at a time, the
// lanes on consecutive words of them.
__device__ __forceinline__ void send_rows16(const uint8_t* buf, uint16_t* to, int64_t pitch, int rows, int cols, int lane) {
  const int first_odd = (int)(reinterpret_cast<uintptr_t>(to) >> 1) & 1, step = (int)(pitch & 1);
  const auto word = [&](int r, int col) {  // columns col and col + 1 of a row, col even
    return *reinterpret_cast<const uint32_t*>(buf + r * 64 + (((col >> 3) ^ ((r >> 1) & 3)) << 4) + (col & 6) * 2);
  };
  for (int r = lane >> 4; r < rows; r += 2) {
    // columns odd and odd + 1, odd + 2 and odd + 3 .. are the words of the row
    const int odd = first_odd ^ (step & r), c = 2 * (lane & 15) + odd;
    uint32_t w = word(r, 2 * (lane & 15));
    if (odd) w = __byte_perm(w, word(r, min(2 * (lane & 15) + 2, 30)), 0x5432);
    if (c + 1 < cols) *reinterpret_cast<uint32_t*>(to + r * pitch + c) = w;
  }
  if (lane < rows) {  // the single columns at the ends, of all rows at once
    const int odd = first_odd ^ (step & lane);
    uint16_t* const at = to + lane * pitch;
    if (odd) at[0] = (uint16_t)word(lane, 0);
    if ((cols - odd) & 1) at[cols - 1] = (uint16_t)(word(lane, (cols - 1) & ~1) >> ((cols - 1) & 1) * 16);
  }
}

// A chunk is 64 bytes of out: 16 or 32 columns.  HALF: the 16-bit tensors are fp16, else bfloat16.
template <int BT, int CG, int OUT, int MODE, bool HALF>
__global__ void __launch_bounds__(kLinThreads, 1) linear_kernel(const __grid_constant__ LinearParams gp) {
  using Cfg = LinCfg<BT, CG>;
  constexpr bool OUT32 = OUT == kOut32;
  constexpr int kStages = Cfg::kStages;
  const uint32_t rank = CG == 2 ? ptx::cluster_ctarank() : 0u;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t smem_base = ptx::smem_u32(smem);
  uint8_t* const out_ptr = smem + kStages * Cfg::kStageBytes;  // 1024-byte aligned
  uint8_t* const bar_ptr = out_ptr + Cfg::kOutBytes;
  const uint32_t bar_base = ptx::smem_u32(bar_ptr);
  auto full = [&](int s) { return bar_base + 8u * s; };
  auto empty = [&](int s) { return bar_base + 8u * (kStages + s); };
  auto acc_full = [&](int a) { return bar_base + 8u * (2 * kStages + a); };
  auto acc_empty = [&](int a) { return bar_base + 8u * (2 * kStages + 2 + a); };
  const uint32_t drain_bar = bar_base + 8u * (2 * kStages + 4);
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bar_ptr + 8 * (2 * kStages + 5));
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if ((smem_base & 1023u) != 0u) {  // never expected; the swizzle needs it
    pdl_begin();
    if (threadIdx.x == 0) report_status(gp.ws, QB_ERR_CUDA, (int)smem_base);
    return;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      ptx::mbar_init(full(s), 1);
      ptx::mbar_init(empty(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(acc_full(a), 1);
      ptx::mbar_init(acc_empty(a), kLinEpilogueWarps * CG);
    }
    ptx::mbar_init(drain_bar, 1);
    *abort_flag = 0;
    ptx::fence_mbar_init();
  }
  if (threadIdx.x == 32 * kLinFirstEpilogueWarp) {  // (the maps are arguments: nothing that a kernel before this one writes)
    ptx::prefetch_tensormap(&gp.tma);
    ptx::prefetch_tensormap(&gp.tmb);
    ptx::prefetch_tensormap(&gp.tmy);
  }
  if (warp == 1) {
    ptx::tmem_alloc_cg<CG>(ptx::smem_u32(tmem_slot), Cfg::kTmemCols);
    ptx::tmem_relinquish_cg<CG>();
  }
  ptx::tcgen05_fence_before_sync();
  __syncthreads();
  if constexpr (CG == 2) ptx::cluster_sync_all();
  ptx::tcgen05_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  pdl_begin();
  // the barriers that the issuer waits on live in the group's first CTA
  auto lead = [&](uint32_t bar) { return CG == 2 ? ptx::map_to_cta(bar, 0) : bar; };

  const int groups = (int)gridDim.x / CG, group = (int)blockIdx.x / CG;
  bool timed_out = false;
  int where = 0;

  if (warp == 0) {
    // ---------------- TMA producer ------------------------------------------------------------------
    if (ptx::elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      for (int t = group; t < gp.tiles && !timed_out; t += groups) {
        const LinTile<BT, CG> tile(gp, t);
        const bool half = CG == 2 && tile.width < BT;
        const int a_mn = tile.m0 + (int)rank * 128, b_rows = tile.width / CG, b_mn = tile.n0 + (int)rank * b_rows;
        const CUtensorMap* const tmb = half ? &gp.tmb_half : &gp.tmb;
        const uint32_t bytes = CG * (Cfg::kABytes + (half ? Cfg::kBBytes / 2 : Cfg::kBBytes));
        for (int kb = tile.k0; kb < tile.k1; kb += 2) {
          if (!wait_barrier_relaxed(empty(stage), phase ^ 1u, abort_flag)) {
            timed_out = true;
            where = (0 << 16) | stage;
            break;
          }
          const uint32_t a_smem = smem_base + stage * Cfg::kStageBytes, b_smem = a_smem + Cfg::kABytes;
          if (rank == 0) ptx::mbar_arrive_expect_tx(full(stage), bytes);
          auto load2 = [&](uint32_t dst, const CUtensorMap* tm, int x, int y) {
            if constexpr (CG == 2) ptx::tma_load_2d_pair(dst, tm, lead(full(stage)), x, y);
            else ptx::tma_load_2d(dst, tm, full(stage), x, y);
          };
          auto load3 = [&](uint32_t dst, const CUtensorMap* tm, int y, int z) {
            if constexpr (CG == 2) ptx::tma_load_3d_pair(dst, tm, lead(full(stage)), 0, y, z);
            else ptx::tma_load_3d(dst, tm, full(stage), 0, y, z);
          };
          auto load = [&](uint32_t dst, const CUtensorMap* tm, int form, int mn, int rows) {
            if (form == kRows) {
              load3(dst, tm, mn, kb);
            } else if (form == kCols) {
              load3(dst, tm, kb * 64, mn / 64);
            } else if (form == kRows2) {
              load2(dst, tm, kb * 64, mn);
              load2(dst + rows * 128, tm, kb * 64 + 64, mn);
            } else {
              load2(dst, tm, mn, kb * 64);
              if (rows > 64) load2(dst + 16384, tm, mn + 64, kb * 64);
            }
          };
          load(a_smem, &gp.tma, gp.a_form, a_mn, 128);
          load(b_smem, tmb, gp.b_form, b_mn, b_rows);
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      if (timed_out) {  // let copies in flight land before the CTA's shared memory is released
        const long long t0 = clock64();
        while (clock64() - t0 < 400000ll) {
        }
      }
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer (of a pair: in its first CTA only) ----------------------------------
    if (rank == 0 && ptx::elect_one()) {
      const bool a_mn = gp.a_form >= kCols, b_mn = gp.b_form >= kCols;
      const uint64_t a_desc0 = lin_desc(smem_base, a_mn), b_desc0 = lin_desc(smem_base + Cfg::kABytes, b_mn);
      // 16 elements of K per instruction: 32 bytes of a row, or 16 rows of 128 bytes
      const uint32_t a_step = a_mn ? 2048 >> 4 : 32 >> 4, b_step = b_mn ? 2048 >> 4 : 32 >> 4;
      int stage = 0, it = 0;
      uint32_t phase = 0;
      int t = group, run = 0;
      while (t < gp.tiles && !timed_out) {
        const int a = it & 1;
        const uint32_t d = tmem_base + (uint32_t)(a * BT);
        const LinTile<BT, CG> tile(gp, t);
        const int first = tile.k0 + run, last = min(first + gp.run_blocks, tile.k1);
        const uint32_t idesc = gp.idesc | ((uint32_t)(tile.width >> 3) << 17);
        const uint32_t a_next = a_mn ? 8192 >> 4 : 16384 >> 4, b_next = b_mn ? 8192 >> 4 : (uint32_t)(tile.width / CG * 128) >> 4;  // second K block
        if (!wait_barrier(acc_empty(a), ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_flag)) {
          timed_out = true;
          where = (1 << 16) | 0x100 | a;
          break;
        }
        for (int kb = first; kb < last; kb += 2) {
          if (!wait_barrier(full(stage), phase, abort_flag)) {
            timed_out = true;
            where = (1 << 16) | stage;
            break;
          }
          ptx::tcgen05_fence_after_sync();
          const uint64_t a_desc = a_desc0 + (uint64_t)(stage * (Cfg::kStageBytes >> 4));
          const uint64_t b_desc = b_desc0 + (uint64_t)(stage * (Cfg::kStageBytes >> 4));
#pragma unroll
          for (int j = 0; j < 4; ++j)
            ptx::mma_f16_ss_cg<CG>(d, a_desc + (uint64_t)(a_step * j), b_desc + (uint64_t)(b_step * j), idesc, kb != first || j != 0 ? 1u : 0u);
          if (kb + 1 < last) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              ptx::mma_f16_ss_cg<CG>(d, a_desc + (uint64_t)(a_next + a_step * j), b_desc + (uint64_t)(b_next + b_step * j), idesc, 1u);
          }
          ptx::mma_commit_cg<CG>(empty(stage));
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
        if (!timed_out) ptx::mma_commit_cg<CG>(acc_full(a));
        ++it;
        run += gp.run_blocks;
        if (last == tile.k1) {
          t += groups;
          run = 0;
        }
      }
      if (timed_out) {  // wait (bounded) for what was issued before tensor memory is freed
        ptx::mma_commit_cg<CG>(drain_bar);
        const long long t0 = clock64();
        while (!ptx::mbar_try_wait(drain_bar, 0) && clock64() - t0 < 400000000ll) {
        }
      }
    }
  } else if (warp >= kLinFirstEpilogueWarp) {
    // ---------------- epilogue ----------------------------------------------------------------------
    constexpr int kCols = OUT32 ? 16 : 32;  // columns of a chunk
    constexpr int kESize = OUT32 ? 4 : 2;
    const int ew = warp - kLinFirstEpilogueWarp, quarter = warp & 3, part = ew >> 2;
    float* const bias_at = reinterpret_cast<float*>(bar_ptr + Cfg::kBarBytes) + ew * 32;  // of the warp's chunk
    constexpr bool half_type = HALF;
    uint8_t* const buf = out_ptr + ew * 2048;
    const uint32_t lanes = tmem_base + ((uint32_t)(quarter * 32) << 16);
    auto arrive = [&](uint32_t bar) {  // this warp has read all it needs from the accumulator
      ptx::tcgen05_fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        if (CG == 2 && rank != 0) ptx::mbar_arrive_remote(lead(bar));
        else ptx::mbar_arrive(bar);
      }
    };
    int it = 0;
    for (int t = group; t < gp.tiles; t += groups) {
      const LinTile<BT, CG> tile(gp, t);
      const float* const bias = gp.bias;
      const void* const side = gp.side;
      int m0 = tile.m0 + (int)rank * 128 + quarter * 32, n0 = tile.n0;
      int chunks = m0 < gp.M ? max(0, min(tile.width / kCols, (gp.N - n0 + kCols - 1) / kCols)) : 0;
      asm volatile("" : "+r"(m0), "+r"(n0), "+r"(chunks));  // formed before the wait, not behind it
      // The warp's chunks, one a turn: every fourth one, or, where pairs of them are the blocks of codes, every fourth pair.
      const bool paired = !OUT32 && MODE != kSlope && gp.pre_codes != nullptr;
      const auto chunk = [&](int turn) { return paired ? 2 * part + (turn & 1) + 8 * (turn >> 1) : part + 4 * turn; };
      // Their biases, a column a lane: of two turns each (fp32 out: of four).  Every warp waits and goes on by itself: with the tile's
      // biases shared behind a barrier of all of them, they did the same things at the same time and waited for one another.
      float biases[2] = {0.0f, 0.0f};
      if (MODE != kSlope && bias) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int c = OUT32 ? chunk(2 * h + (lane >> 4)) * 16 + (lane & 15) : chunk(h) * 32 + lane;
          if (n0 + c < gp.N && c < tile.width) biases[h] = bias[n0 + c];
        }
      }
      const int rows = min(32, gp.M - m0);
      const bool mine = lane < rows;
      // The chunk's part of the tensor beside the product (residual, pre-activation, codes of it): the lane's row, fetched while the
      // products run.
      // (Rows that are 16-byte aligned only: by vectors for a slope, where there are registers for both kinds, else by way of the buffer.)
      constexpr int kLeast = MODE == kSlope ? 1 : 2;
      uint4 s[4];
      auto fetch = [&](int c0) {
        const int64_t corner = (int64_t)(m0 + lane) * gp.N + n0 + c0;
        if (MODE == kSlope && gp.codes) {
          if (!gp.vector_codes) return;
          s[0] = s[1] = make_uint4(0u, 0u, 0u, 0u);
          if (mine && n0 + c0 < gp.N) load_row(gp.codes + corner, gp.vector_codes > 1, n0 + c0 + 16 < gp.N, s[0], s[1]);
        } else if (side && gp.vector >= kLeast) {
          const uint8_t* const from = static_cast<const uint8_t*>(side) + corner * kESize;
#pragma unroll
          for (int k = 0; k < 4; k += 2) {
            s[k] = s[k + 1] = make_uint4(0u, 0u, 0u, 0u);
            const int c = n0 + c0 + k * (16 / kESize);
            if (mine && c < gp.N) load_row(from + 16 * k, MODE != kSlope || gp.vector > 1, c + 16 / kESize < gp.N, s[k], s[k + 1]);
          }
        }
      };
      // Waits for the accumulator of run `it`.
      auto wait_run = [&]() {
        if (!wait_barrier_warp(acc_full(it & 1), (uint32_t)(it >> 1) & 1u, abort_flag)) {
          timed_out = true;
          where = (3 << 16) | (it & 1);
          return false;
        }
        ptx::tcgen05_fence_after_sync();
        return true;
      };
      auto read = [&](int column, float* z) {
        uint32_t w[kCols];
        const uint32_t from = lanes + (uint32_t)((it & 1) * BT + column);
        if constexpr (OUT32) ptx::tmem_ld_32x32b_x16(from, w);
        else ptx::tmem_ld_32x32b_x32(from, w);
        ptx::tmem_ld_wait();
        ptx::tmem_ld_regs_ready(w);
#pragma unroll
        for (int j = 0; j < kCols; ++j) z[j] = __uint_as_float(w[j]);
      };
      auto add_bias = [&](int turn, float* z) {
        if (MODE == kSlope || !bias) return;
        __syncwarp();
        if constexpr (OUT32) {
          if ((lane >> 4) == (turn & 1)) bias_at[lane & 15] = biases[turn >> 1];
        } else {
          bias_at[lane] = turn == 0 ? biases[0] : biases[1];
        }
        __syncwarp();
        const float4* const b4 = reinterpret_cast<const float4*>(bias_at);
#pragma unroll
        for (int j = 0; j < kCols / 4; ++j) {
          const float4 q = b4[j];
          add2(z + 4 * j, q.x, q.y);
          add2(z + 4 * j + 2, q.z, q.w);
        }
      };
      // What becomes of the chunk's z (the product and the bias), from there to memory.  top: the largest magnitude of its block.
      auto emit = [&](int i, int next, float* v, float top) {
        const int c0 = i * kCols, cols = min(kCols, gp.N - n0 - c0);
        const int64_t corner = (int64_t)m0 * gp.N + n0 + c0;  // of the chunk, in elements
        const int64_t block = (int64_t)(m0 + lane) * checkpoint_blocks(gp.N) + (n0 + c0) / kCheckpointBlock;  // the row's, in scales
        float scale = 1.0f;
        if (MODE == kSlope && gp.codes && mine) scale = gp.scales[block];
        if constexpr (OUT32) fetch(c0);
        bool waited = false;  // for the chunk before to have left the buffer
        auto buffer_free = [&]() {
          if (waited) return;
          waited = true;
          if (lane == 0) ptx::tma_store_wait_read0();
          __syncwarp();
        };
        // rows of any alignment come by way of the buffer
        if (MODE == kSlope && gp.codes && !gp.vector_codes) {
          buffer_free();
          for (int r0 = 0; r0 < rows; r0 += 8) {  // eight rows on their way at a time
            int8_t e[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) e[r] = lane < cols && r0 + r < rows ? gp.codes[corner + (int64_t)(r0 + r) * gp.N + lane] : (int8_t)0;
#pragma unroll
            for (int r = 0; r < 8; ++r) reinterpret_cast<int8_t*>(staged(buf, r0 + r, lane >> 4))[lane & 15] = e[r];
          }
          __syncwarp();
#pragma unroll
          for (int k = 0; k < 2; ++k) s[k] = *staged(buf, lane, k);
          __syncwarp();
        } else if (side && gp.vector < kLeast) {
          buffer_free();
          if constexpr (OUT32) {
            for (int r = lane >> 4; r < rows; r += 2) {
              const int c = lane & 15;
              reinterpret_cast<float*>(staged(buf, r, c >> 2))[c & 3] = c < cols ? static_cast<const float*>(side)[corner + (int64_t)r * gp.N + c] : 0.0f;
            }
          } else {
            for (int r0 = 0; r0 < rows; r0 += 8) {
              uint16_t e[8];
#pragma unroll
              for (int r = 0; r < 8; ++r) e[r] = lane < cols && r0 + r < rows ? static_cast<const uint16_t*>(side)[corner + (int64_t)(r0 + r) * gp.N + lane] : (uint16_t)0;
#pragma unroll
              for (int r = 0; r < 8; ++r) reinterpret_cast<uint16_t*>(staged(buf, r0 + r, lane >> 3))[lane & 7] = e[r];
            }
          }
          __syncwarp();
#pragma unroll
          for (int k = 0; k < 4; ++k) s[k] = *staged(buf, lane, k);
          __syncwarp();
        }
        if constexpr (!OUT32 && MODE != kSlope) {
          if (gp.pre_codes) {  // z in 8 bits
            const CheckpointCodes cs(top);
            if (mine && (c0 & 32) == 0) gp.pre_scales[block] = checkpoint_scale(top);
            uint4 c[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              c[k].x = cs.codes4(v[16 * k], v[16 * k + 1], v[16 * k + 2], v[16 * k + 3]);
              c[k].y = cs.codes4(v[16 * k + 4], v[16 * k + 5], v[16 * k + 6], v[16 * k + 7]);
              c[k].z = cs.codes4(v[16 * k + 8], v[16 * k + 9], v[16 * k + 10], v[16 * k + 11]);
              c[k].w = cs.codes4(v[16 * k + 12], v[16 * k + 13], v[16 * k + 14], v[16 * k + 15]);
            }
            int8_t* const to = gp.pre_codes + corner;
            if (gp.vector_codes >= kLeast) {
              if (mine) store32(to + (int64_t)lane * gp.N, c[0], c[1]);
            } else {
              buffer_free();
#pragma unroll
              for (int k = 0; k < 2; ++k) *staged(buf, lane, k) = c[k];
              __syncwarp();
              if (lane < cols)
                for (int r = 0; r < rows; ++r) to[(int64_t)r * gp.N + lane] = reinterpret_cast<const int8_t*>(staged(buf, r, lane >> 4))[lane & 15];
              __syncwarp();
            }
          } else if (gp.pre) {  // z in 16 bits
            uint16_t* const to = static_cast<uint16_t*>(gp.pre) + corner;
            uint4 c[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
              c[k] = make_uint4(pack16(v[8 * k], v[8 * k + 1], half_type), pack16(v[8 * k + 2], v[8 * k + 3], half_type), pack16(v[8 * k + 4], v[8 * k + 5], half_type),
                                pack16(v[8 * k + 6], v[8 * k + 7], half_type));
            if (gp.vector >= kLeast) {
#pragma unroll
              for (int k = 0; k < 4; k += 2)
                if (mine && 8 * k < cols) store32(to + (int64_t)lane * gp.N + 8 * k, c[k], c[k + 1]);
            } else {
              buffer_free();
#pragma unroll
              for (int k = 0; k < 4; ++k) *staged(buf, lane, k) = c[k];
              __syncwarp();
              send_rows16(buf, to, gp.N, rows, cols, lane);
              __syncwarp();
            }
          }
        }
        if constexpr (MODE == kGelu) {
#pragma unroll
          for (int j = 0; j < kCols; j += 8) gelu_many<4>(v + j);
        }
        if constexpr (MODE == kSlope) {
#pragma unroll
          for (int j = 0; j < kCols; j += 8) {
            float p[8];
            if (gp.codes) {
              const uint4& q = s[j >> 4];
              code_values((j & 8) ? q.z : q.x, scale, p);
              code_values((j & 8) ? q.w : q.y, scale, p + 4);
            } else {
              const uint4& q = s[j >> 3];
              const uint32_t in[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
              for (int h = 0; h < 4; ++h) {
                const float2 f = unpack16(in[h], half_type);
                p[2 * h] = f.x;
                p[2 * h + 1] = f.y;
              }
            }
            times_gelu_slope<4>(p, v + j);
          }
        } else if (side) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t in[4] = {s[k].x, s[k].y, s[k].z, s[k].w};
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              if constexpr (OUT32) {
                v[4 * k + h] += __uint_as_float(in[h]);
              } else {
                const float2 r = unpack16(in[h], half_type);
                add2(v + 8 * k + 2 * h, r.x, r.y);
              }
            }
          }
        }
        if (!OUT32 && next < chunks) fetch(next * kCols);
        buffer_free();
#pragma unroll
        for (int k = 0; k < 4; ++k) {  // 16 bytes of the row at a time
          if constexpr (OUT32)
            *staged(buf, lane, k) = make_uint4(__float_as_uint(v[4 * k]), __float_as_uint(v[4 * k + 1]), __float_as_uint(v[4 * k + 2]), __float_as_uint(v[4 * k + 3]));
          else
            *staged(buf, lane, k) = make_uint4(pack16(v[8 * k], v[8 * k + 1], half_type), pack16(v[8 * k + 2], v[8 * k + 3], half_type),
                                               pack16(v[8 * k + 4], v[8 * k + 5], half_type), pack16(v[8 * k + 6], v[8 * k + 7], half_type));
        }
        const int64_t first_row = (int64_t)tile.split * gp.M;
        if (gp.tma_store) {
          ptx::fence_proxy_async_smem();  // every lane: its own stores
          __syncwarp();
          if (lane == 0) {
            ptx::tma_store_3d(&gp.tmy, ptx::smem_u32(buf), n0 + c0, m0, tile.split);
            ptx::tma_store_commit();
          }
        } else if constexpr (OUT32) {  // two rows at a time, the lanes on consecutive values of them
          __syncwarp();
          const int c = lane & 15;
          if (c < cols) {
            float* const to = static_cast<float*>(gp.out) + first_row * gp.N + corner + c;
            for (int r = lane >> 4; r < rows; r += 2) to[(int64_t)r * gp.N] = reinterpret_cast<const float*>(staged(buf, r, c >> 2))[c & 3];
          }
          __syncwarp();
        } else {
          __syncwarp();
          send_rows16(buf, static_cast<uint16_t*>(gp.out) + first_row * gp.N + corner, gp.N, rows, cols, lane);
          __syncwarp();
        }
      };
      const bool beside = !OUT32 && chunk(0) < chunks;
      if (OUT != kOut16Runs && beside) fetch(chunk(0) * kCols);
      bool ok;
      if constexpr (OUT != kOut16) {  // the runs before the last are added up in registers, and to the last one where it lies
        constexpr int kChunks = OUT32 ? BT / kCols / 4 : 2;  // of a warp
        float sums[kChunks][kCols] = {};
        int run = tile.k0;
        while (true) {
          ok = wait_run();
          if (!ok || run + gp.run_blocks >= tile.k1) break;
#pragma unroll
          for (int j = 0; j < kChunks; ++j) {
            if (chunk(j) < chunks) {
#pragma unroll
              for (int h = 0; h < kCols; h += 8) {
                add_accumulator(lanes + (uint32_t)((it & 1) * BT + chunk(j) * kCols + h), sums[j] + h);
              }
            }
          }
          arrive(acc_empty(it & 1));
          ++it;
          run += gp.run_blocks;
        }
        if (ok && run > tile.k0) {
#pragma unroll
          for (int j = 0; j < kChunks; ++j) {
            if (chunk(j) < chunks) {
#pragma unroll
              for (int h = 0; h < kCols; h += 8) {
                const uint32_t at = lanes + (uint32_t)((it & 1) * BT + chunk(j) * kCols + h);
                add_accumulator(at, sums[j] + h);
                ptx::tmem_st_32x32b_x8(at, sums[j] + h);
              }
            }
          }
          ptx::tmem_st_wait();
        }
      } else {
        ok = wait_run();
      }
      if (OUT == kOut16Runs && beside) fetch(chunk(0) * kCols);  // (behind the sums, which take the registers)
      if (!ok) break;
      if (chunk(0) >= chunks) arrive(acc_empty(it & 1));
      float top = 0.0f;
#pragma unroll 1
      for (int turn = 0; chunk(turn) < chunks; ++turn) {
        const int i = chunk(turn), next = chunk(turn + 1);
        float v[kCols];
        const auto highest = [&]() {
#pragma unroll
          for (int j = 0; j < kCols; j += 2) top = max3_nan(top, fabsf(v[j]), fabsf(v[j + 1]));
        };
        if (paired && (turn & 1) == 0) {  // the block's second chunk is read ahead, for its largest magnitude
          top = 0.0f;
          if (next < chunks) {
            read(next * kCols, v);
            add_bias(turn + 1, v);
            highest();
          }
        }
        read(i * kCols, v);
        if (next >= chunks) arrive(acc_empty(it & 1));
        add_bias(turn, v);
        if (paired && (turn & 1) == 0) highest();
        emit(i, next, v, top);
      }
      ++it;
    }
    if (lane == 0) ptx::tma_store_wait_read0();  // the buffers are in use until then
  } else if (gp.mark != 0 && blockIdx.x == 0 && threadIdx.x == 64) {  // (by an idle warp)
    st_release(&static_cast<WsHeader*>(gp.ws)->begun, gp.mark);
  }
  if (timed_out) {
    *abort_flag = 1;
    report_status(gp.ws, QB_ERR_TIMEOUT, where);
  }
  ptx::tcgen05_fence_before_sync();
  __syncthreads();
  if constexpr (CG == 2) ptx::cluster_sync_all();  // the other CTA's MMAs and arrivals reach into this CTA
  if (warp == 1) {
    __syncwarp();
    ptx::tcgen05_fence_after_sync();
    ptx::tmem_dealloc_cg<CG>(tmem_base, Cfg::kTmemCols);
  }
}

template <int BT, int CG, int OUT, int MODE, bool HALF>
static qb_status launch_linear_form(const LinearParams& gp, int sms, cudaStream_t stream) {
  using Cfg = LinCfg<BT, CG>;
  auto kernel = linear_kernel<BT, CG, OUT, MODE, HALF>;
  static std::atomic<bool> attr_set[64] = {};
  int dev = 0;
  QB_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
    QB_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmemBytes));
    if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
  }
  const int grid = std::min(gp.tiles, sms / CG) * CG;
  QB_CUDA_TRY(launch_kernel(kernel, (unsigned)grid, kLinThreads, Cfg::kSmemBytes, stream, CG, false, gp));
  return QB_OK;
}
template <int BT, int CG, int OUT, bool HALF>
static qb_status launch_linear_mode(const LinearParams& gp, int mode, int sms, cudaStream_t stream) {
  if constexpr (OUT != kOut32) {
    if (mode == kSlope) return launch_linear_form<BT, CG, OUT, kSlope, HALF>(gp, sms, stream);
  }
  return mode == kGelu ? launch_linear_form<BT, CG, OUT, kGelu, HALF>(gp, sms, stream) : launch_linear_form<BT, CG, OUT, kPlain, HALF>(gp, sms, stream);
}
template <int BT, int CG>
static qb_status launch_linear(const LinearParams& gp, int out, int mode, bool half_type, int sms, cudaStream_t stream) {
  // (with fp32 out the type of the 16-bit tensors is in the instruction descriptor alone)
  if (out == kOut32) return launch_linear_mode<BT, CG, kOut32, false>(gp, mode, sms, stream);
  if (out == kOut16Runs) return half_type ? launch_linear_mode<BT, CG, kOut16Runs, true>(gp, mode, sms, stream) : launch_linear_mode<BT, CG, kOut16Runs, false>(gp, mode, sms, stream);
  return half_type ? launch_linear_mode<BT, CG, kOut16, true>(gp, mode, sms, stream) : launch_linear_mode<BT, CG, kOut16, false>(gp, mode, sms, stream);
}

// What stands behind a product, as the join of a split one needs it.
struct LinearTail {
  const float* bias;
  const void* side;
  const int8_t* codes;
  const float* scales;
  void* out;
  void* pre;
  int32_t mode, out_type, type;
  bool vector;  // out is 16-byte aligned
};
__device__ __forceinline__ float load_value(const void* p, int64_t i, int type) {
  if (type == QB_F32) return static_cast<const float*>(p)[i];
  if (type == QB_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  return __half2float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_value(void* p, int64_t i, int type, float v) {
  if (type == QB_F32) static_cast<float*>(p)[i] = v;
  else if (type == QB_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else static_cast<__half*>(p)[i] = __float2half_rn(v);
}
__device__ __forceinline__ float gelu_one(float z) {
  float f[2] = {z, z};
  gelu_many<1>(f);
  return f[0];
}
// out = what stands behind the splits' sum, taken in their order.  Four parts at a time are on their way.
template <int V>
__global__ void __launch_bounds__(256) linear_join_kernel(const float* parts, int splits, int64_t MN, int N, const LinearTail tail) {
  constexpr int kAtOnce = 4;
  pdl_begin();
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V; i < MN; i += (int64_t)gridDim.x * 256 * V) {
    float v[V] = {};
    for (int s = 0; s < splits; s += kAtOnce) {
      float w[kAtOnce][V];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        if (s + k < splits) {
          if constexpr (V == 4) *reinterpret_cast<float4*>(w[k]) = *reinterpret_cast<const float4*>(parts + (s + k) * MN + i);
          else w[k][0] = parts[(s + k) * MN + i];
        }
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        if (s + k < splits) {
#pragma unroll
          for (int j = 0; j < V; ++j) v[j] = s + k == 0 ? w[k][j] : v[j] + w[k][j];
        }
      }
    }
    if (V == 4 && !tail.bias && !tail.side && !tail.codes && !tail.pre && tail.mode == kPlain && tail.vector) {  // a weight's gradient
      if (tail.out_type == QB_F32)
        *reinterpret_cast<float4*>(static_cast<float*>(tail.out) + i) = make_float4(v[0], v[V > 1], v[V > 2 ? 2 : 0], v[V > 3 ? 3 : 0]);
      else
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(tail.out) + i) =
            make_uint2(pack16(v[0], v[V > 1], tail.out_type == QB_F16), pack16(v[V > 2 ? 2 : 0], v[V > 3 ? 3 : 0], tail.out_type == QB_F16));
      continue;
    }
    const int64_t m = i / N;
    const int n = (int)(i - m * N);
#pragma unroll
    for (int j = 0; j < V; ++j) {  // (vectors: N is a multiple of 4)
      float z = v[j];
      if (tail.bias) z += tail.bias[n + j];
      if (tail.pre) store_value(tail.pre, i + j, tail.type, z);
      if (tail.mode == kGelu) z = gelu_one(z);
      if (tail.mode == kSlope) {
        const float p = tail.codes ? (float)tail.codes[i + j] * tail.scales[m * checkpoint_blocks(N) + (n + j) / kCheckpointBlock]
                                   : load_value(tail.side, i + j, tail.type);
        const float x[2] = {p, p};
        float g[2] = {z, z};
        times_gelu_slope<1>(x, g);
        z = g[0];
      } else if (tail.side) {
        z += load_value(tail.side, i + j, tail.out_type);
      }
      store_value(tail.out, i + j, tail.out_type, z);
    }
  }
}

// Rows of any length as rows of a multiple of 16 bytes, zeros behind them (what a TMA load needs).  Eight elements a thread, read as the
// words that hold them and shifted where they begin inside one; none that the tensor does not have is read.
__global__ void __launch_bounds__(256) pad_rows_kernel(const uint16_t* from, uint16_t* to, int64_t rows, int32_t cols, int32_t pitch) {
  pdl_begin();
  const int per_row = pitch / 8;
  const int64_t n = rows * per_row, all = rows * cols;
#pragma unroll 2
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = n >> 32 ? i / per_row : (int64_t)((uint32_t)i / (uint32_t)per_row);
    const int c = (int)(i - r * per_row) * 8, left = cols - c;
    const int64_t first = r * cols + c;
    uint32_t w[5];
    if (first + 10 <= all) {
      const uint32_t* const words = reinterpret_cast<const uint32_t*>(from) + (first >> 1);  // (`from` is 16-byte aligned)
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = words[j];
      w[4] = 0u;
      if (first & 1) {
        w[4] = words[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __funnelshift_r(w[j], w[j + 1], 16);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = first + 2 * j < all ? from[first + 2 * j] : 0, hi = first + 2 * j + 1 < all ? from[first + 2 * j + 1] : 0;
        w[j] = lo | hi << 16;
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {  // what the next row begins with is not this row's
      if (2 * j >= left) w[j] = 0u;
      else if (2 * j + 1 >= left) w[j] &= 0xffffu;
    }
    *reinterpret_cast<uint4*>(to + i * 8) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// Sums of the columns of g [M][N] over its rows, first over runs of rows into parts [runs][N], then over the runs, in their order.
// UNDER: the kernel before this one on the stream is of this call, the product or the join of its parts, which neither writes what is read
// here nor touches the parts, so that this kernel does not wait for its end, and runs on SMs that it leaves (24,576 x 4,096, K = 1,024: grad_w
// 143 us, with grad_bias 151, one after the other 181).  One block waits at its end, so that the kernels that follow find both done.
//
// What the kernels before the product wrote is visible to the product, which has waited for it (pdl_begin), but not thereby to a grid that has
// not waited itself.  So the product leaves a mark of its call behind its wait, by a release; who acquires it has behind him all that the
// product had.  A block that does not find it within some microseconds waits for the product's end instead.  The last kernel of the
// call takes the mark away, and every call has one of its own, so that none is mistaken for that of an earlier replay or of a call
// whose later launches failed.
__device__ __forceinline__ void begin_under(const void* ws, uint32_t mark) {
  const int seen = threadIdx.x == 0 && poll_word(&static_cast<const WsHeader*>(ws)->begun, mark, 20000);
  if (!__syncthreads_or(seen)) pdl_begin();
}
static uint32_t next_mark() {
  static std::atomic<uint32_t> last{0};
  uint32_t mark;
  while ((mark = last.fetch_add(1, std::memory_order_relaxed) + 1) == 0) {
  }
  return mark;
}
template <bool VECTOR, bool UNDER>
__global__ void __launch_bounds__(256) column_parts_kernel(const uint16_t* g, int64_t M, int32_t N, int64_t run, int col_blocks, int half_type, float* parts,
                                                          const void* ws, uint32_t mark) {
  __shared__ float sums[8][256];
  if constexpr (UNDER) begin_under(ws, mark);
  else pdl_begin();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t which = blockIdx.x / col_blocks, first = which * run, last = min(first + run, M);
  const int n0 = ((int)blockIdx.x - (int)which * col_blocks) * 256;
  float s[8] = {};
  if constexpr (VECTOR) {
    const int c = n0 + lane * 8;
    if (c < N) {
#pragma unroll 4
      for (int64_t m = first + warp; m < last; m += 8) {
        const uint4 w = *reinterpret_cast<const uint4*>(g + m * N + c);
        const uint32_t in[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = unpack16(in[j], half_type != 0);
          s[2 * j] += f.x;
          s[2 * j + 1] += f.y;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[warp][lane * 8 + j] = s[j];
  } else {
    for (int64_t m = first + warp; m < last; m += 8)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = n0 + lane + 32 * j;
        if (c < N) s[j] += unpack16(g[m * N + c], half_type != 0).x;
      }
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[warp][lane + 32 * j] = s[j];
  }
  __syncthreads();
  const int c = n0 + (int)threadIdx.x;
  if (c < N) {
    float t = sums[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < 8; ++w) t += sums[w][threadIdx.x];
    parts[which * N + c] = t;
  }
  if (UNDER && blockIdx.x == 0) pdl_begin();  // (a block that waits keeps its place from those that have not begun)
}
// 32 columns a block, 32 groups of runs side by side, joined in their order.  ws: where the mark of begin_under is, or NULL.
constexpr int kColumnGroups = 32;
__global__ void __launch_bounds__(32 * kColumnGroups) column_join_kernel(const float* parts, int runs, int32_t N, float* sums, void* ws) {
  __shared__ float joined[kColumnGroups][32];
  pdl_begin();
  if (ws && blockIdx.x == 0 && threadIdx.x == 0) static_cast<WsHeader*>(ws)->begun = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = (int)blockIdx.x * 32 + lane;
  const int group = (runs + kColumnGroups - 1) / kColumnGroups, last = min((warp + 1) * group, runs);
  float t = 0.0f;
  if (c < N) {
#pragma unroll 8
    for (int r = warp * group; r < last; ++r) t += parts[(int64_t)r * N + c];
  }
  joined[warp][lane] = t;
  __syncthreads();
  if (warp == 0 && c < N) {
#pragma unroll
    for (int w = 1; w < kColumnGroups; ++w) t += joined[w][lane];
    sums[c] = t;
  }
}

// The same for a few columns and rows (kFewColumns, kFewValues), by one block in one launch: 2^k threads a column, joined as a tree.
constexpr int kFewColumns = 256;
constexpr int64_t kFewValues = 65536;
template <bool UNDER>
__global__ void __launch_bounds__(1024) column_few_kernel(const uint16_t* g, int64_t M, int32_t N, int half_type, float* sums, void* ws, uint32_t mark) {
  __shared__ float joined[1024];
  if constexpr (UNDER) begin_under(ws, mark);
  else pdl_begin();
  int lanes = 1;
  while (2 * lanes * N <= 1024) lanes *= 2;
  const int c = (int)threadIdx.x % N, lane = (int)threadIdx.x / N;
  float t = 0.0f;
  if (lane < lanes) {
#pragma unroll 8
    for (int64_t r = lane; r < M; r += lanes) t += unpack16(g[r * N + c], half_type != 0).x;
  }
  for (int step = lanes / 2; step > 0; step /= 2) {
    joined[threadIdx.x] = t;
    __syncthreads();
    if (lane < step) t += joined[threadIdx.x + step * N];
    __syncthreads();
  }
  if (lane == 0) sums[c] = t;
  if constexpr (UNDER) {
    pdl_begin();
    if (threadIdx.x == 0) static_cast<WsHeader*>(ws)->begun = 0;
  }
}

static int64_t lin_up(int64_t n, int64_t m) { return (n + m - 1) / m; }

// The tensor cores cut an accumulator off at its last place at each addition of 16 products, always towards zero: the error grows
// with their number (24,576 products of random signs: 2.8e-5 of the result's norm).  fp32 outputs are summed in runs of this many K blocks,
// which the epilogue's registers add up, rounded to nearest: the error is then that of fp32 products.
constexpr int kLinRunBlocks = 8;
// 16-bit outputs are summed in one run as long as that costs less than a tenth of their own rounding (2.1e-4 of the norm in fp16, 1.7e-3 in
// bfloat16), else in runs of 8,192 products (1e-5).  The sums of runs take registers that a single run's epilogue has for itself: a kernel that can do both took
// 156 us instead of 150 at 24,576 x 4,096 x 1,024 with GELU, with the pre-activation saved in codes 188 instead of 173 (80 to 150 bytes a thread
// are spilled).
constexpr int kLinRunBlocks16 = 128;
static int64_t single_run_blocks(bool half_type) { return half_type ? 256 : 1024; }
constexpr size_t kLinScratchOff = 1024;  // of what calls keep in the workspace besides its header

// The form of a product: CTAs per tile, columns, for pairs how many tiles are whole, and splits of K.
struct LinearChoice {
  int cg, bt;
  int32_t tiles, whole, splits, split_blocks;
};
// The cheapest by what a launch and each of its rounds of tiles take, in hundredths of a microsecond: a tile a part per K block of 64 and
// a fixed part, the launch the time until the first tile and of the last epilogue.  Fitted to M from 32 to 5,003, N and K from 768 to
// 4,096: 5,003 x 768 x 768 9.4 us by tiles of 256 x 256, 8.8 by 256 x 128, 9.8 by 128 x 128, 11.6 by 128 x 64; 5,003 x 2,304 x 768 15.7,
// 17.0, 19.6, 24.9; 613 x 768 x 768 6.3, 6.3, 6.0, 5.2.  A last round that fills at most half of the pairs is cut into tiles of half the
// width (5,003 x 1,024 x 4,096 42.9 -> 34.8 us).  Where a long K meets few tiles, K is split into runs whose sums a second kernel joins: that
// costs its launch and the traffic of the parts.
static LinearChoice choose_linear(int64_t M, int64_t N, int64_t K, int sms, size_t scratch) {
  static constexpr struct {
    int cg, bt, block, fixed, launch;
  } kForms[] = {{2, 256, 29, 40, 560}, {2, 128, 16, 70, 370}, {1, 128, 20, 80, 300}, {1, 64, 16, 20, 290}};
  const int64_t blocks = lin_up(K, 64);
  LinearChoice best = {};
  int64_t best_cost = 0;
  for (const auto& f : kForms) {
    if (f.cg == 2 && sms < 2) continue;
    const int64_t groups = sms / f.cg, tiles = lin_up(M, 128 * f.cg) * lin_up(N, f.bt);
    for (int64_t splits = 1; splits == 1 || (4 * splits <= blocks && tiles * (splits - 1) < groups && splits * M * N * 4 <= (int64_t)scratch); ++splits) {
      const int64_t run = splits == 1 ? blocks : lin_up(lin_up(blocks, splits), 2) * 2;
      if (lin_up(blocks, run) != splits) continue;
      const int64_t tile = f.block * run + f.fixed, all = tiles * splits, last = all % groups;
      const bool halves = f.bt == 256 && splits == 1 && last > 0 && 2 * last <= groups;
      const int64_t cost = f.launch + (all / groups) * tile + (halves ? tile * 6 / 10 : (last > 0 ? tile : 0)) + (splits > 1 ? 200 + splits * M * N / 15000 : 0);
      if (best.cg == 0 || cost < best_cost) {
        best_cost = cost;
        best = {f.cg, f.bt, (int32_t)(halves ? all + last : all), (int32_t)(halves ? all - last : all), (int32_t)splits, (int32_t)run};
      }
    }
  }
  return best;
}
static bool impossible_linear(int64_t M, int64_t N, int64_t K) {
  if (M <= 0 || N <= 0 || K <= 0 || M > QB_MAX_MN || N > QB_MAX_MN || K > QB_MAX_MN) return true;
  const int64_t most = (int64_t)1 << 30;  // tiles of each of the three products
  return lin_up(M, 128) * lin_up(N, 64) > most || lin_up(M, 128) * lin_up(K, 64) > most || lin_up(N, 128) * lin_up(K, 64) > most;
}

// A call's part of the workspace behind its header, handed out piece by piece.
struct LinearScratch {
  char* at;
  size_t left;
  LinearScratch(void* ws, size_t bytes) : at(static_cast<char*>(ws) + kLinScratchOff), left(bytes > kLinScratchOff ? bytes - kLinScratchOff : 0) {}
  void* take(size_t bytes) {
    bytes = (bytes + 255) / 256 * 256;
    if (bytes > left) return nullptr;
    void* const p = at;
    at += bytes;
    left -= bytes;
    return p;
  }
};
static size_t pad_bytes(int64_t rows, int64_t cols) { return cols % 8 == 0 ? 0 : ((size_t)rows * (size_t)lin_up(cols, 8) * 16 + 255) / 256 * 256; }

// An operand: a tensor [rows][cols] whose rows (K-major) or columns (MN-major) the product contracts.
struct LinearOperand {
  const void* data;
  int64_t rows, cols;
  bool mn;  // contraction along the rows of the tensor
};
// The operand as TMA can read it: itself, or a copy with longer rows.
static qb_status padded(LinearOperand* o, int64_t* pitch, LinearScratch* scratch, int sms, const char* what, cudaStream_t stream) {
  *pitch = lin_up(o->cols, 8) * 8;
  if (*pitch == o->cols) return QB_OK;
  uint16_t* const copy = static_cast<uint16_t*>(scratch->take(pad_bytes(o->rows, o->cols)));
  if (!copy) {
    set_last_error("%s: the workspace is too small for rows that are no multiple of 8 elements (qb_linear_workspace_bytes)", what);
    return QB_ERR_WORKSPACE;
  }
  const unsigned grid = (unsigned)std::min<int64_t>(lin_up(o->rows * *pitch, 2048), (int64_t)sms * 16);
  QB_CUDA_TRY(launch_kernel(pad_rows_kernel, grid, 256, 0, stream, 1, false, static_cast<const uint16_t*>(o->data), copy, o->rows, (int32_t)o->cols, (int32_t)*pitch));
  o->data = copy;
  return QB_OK;
}
// Map and form of an operand for boxes of `extent` rows or columns of the output.
static qb_status operand_map(CUtensorMap* tm, int32_t* form, const LinearOperand& o, int64_t pitch, int extent, bool half_type) {
  const CUtensorMapDataType t = half_type ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  const bool whole = o.cols % 64 == 0;
  *form = o.mn ? (whole ? kCols : kCols2) : (whole ? kRows : kRows2);
  if (whole) return make_group_map(tm, t, 2, o.data, o.rows, pitch * 2, o.mn ? 128 : extent, o.mn ? extent / 64 : 2);
  return make_matrix_map(tm, t, o.data, o.rows, o.cols, pitch * 2, o.mn ? 128 : extent, 64, CU_TENSOR_MAP_SWIZZLE_128B);
}

// out [M][N] = A B^T over K, and what `tail` says.  `pre_codes`: saved in 8 bits by the epilogue (then K is not split).  `mark`: of the call, for a
// kernel that runs under this one, or 0.
static qb_status run_linear(const char* what, LinearOperand a, LinearOperand b, int64_t M, int64_t N, int64_t K, const LinearTail& tail, int8_t* pre_codes,
                            float* pre_scales, void* ws, LinearScratch scratch, uint32_t mark, int sms, cudaStream_t stream) {
  const bool half_type = tail.type == QB_F16;
  int64_t a_pitch, b_pitch;
  qb_status st;
  if ((st = padded(&a, &a_pitch, &scratch, sms, what, stream)) != QB_OK) return st;
  if ((st = padded(&b, &b_pitch, &scratch, sms, what, stream)) != QB_OK) return st;
  const int64_t blocks = lin_up(K, 64);
  const LinearChoice choice = choose_linear(M, N, K, sms, pre_codes ? 0 : scratch.left);
  const int cg = choice.cg, bt = choice.bt;
  const bool split = choice.splits > 1;
  const bool out32 = split || tail.out_type == QB_F32;
  const int out = out32 ? kOut32 : (blocks > single_run_blocks(half_type) ? kOut16Runs : kOut16);
  float* const parts = reinterpret_cast<float*>(scratch.at);
  LinearParams gp;
  if ((st = operand_map(&gp.tma, &gp.a_form, a, a_pitch, 128, half_type)) != QB_OK) return st;
  if ((st = operand_map(&gp.tmb, &gp.b_form, b, b_pitch, bt / cg, half_type)) != QB_OK) return st;
  gp.tmb_half = gp.tmb;
  if (choice.whole < choice.tiles && (st = operand_map(&gp.tmb_half, &gp.b_form, b, b_pitch, bt / 4, half_type)) != QB_OK) return st;
  const int64_t row_bytes = N * (out32 ? 4 : 2);
  gp.tma_store = row_bytes % 16 == 0 && (split || aligned16(tail.out));
  gp.tmy = gp.tma;
  if (gp.tma_store && (st = make_parts_map(&gp.tmy, out32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : (half_type ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16),
                                           split ? parts : tail.out, choice.splits, M, N, row_bytes, 32, out32 ? 16 : 32, CU_TENSOR_MAP_SWIZZLE_64B)) != QB_OK)
    return st;
  gp.bias = split ? nullptr : tail.bias;
  gp.side = split || tail.codes ? nullptr : tail.side;
  gp.codes = split ? nullptr : tail.codes;
  gp.scales = tail.scales;
  gp.out = split ? parts : tail.out;
  gp.pre = split ? nullptr : tail.pre;
  gp.pre_codes = pre_codes;
  gp.pre_scales = pre_scales;
  const auto vectors = [](int64_t pitch, const void* p, const void* q) {
    return pitch % 32 == 0 && aligned_to(p, 32) && aligned_to(q, 32) ? 2 : (pitch % 16 == 0 && aligned16(p) && aligned16(q) ? 1 : 0);
  };
  gp.vector = vectors(row_bytes, tail.side, tail.pre);
  gp.vector_codes = vectors(N, tail.codes, pre_codes);
  gp.ws = ws;
  gp.M = (int32_t)M;
  gp.N = (int32_t)N;
  gp.n_tiles = (int32_t)lin_up(N, bt);
  gp.tiles = choice.tiles;
  gp.whole = choice.whole;
  gp.split_tiles = choice.tiles / choice.splits;
  gp.n_tiles_inv = quick_inverse((uint32_t)gp.n_tiles);
  gp.split_tiles_inv = quick_inverse((uint32_t)gp.split_tiles);
  gp.split_blocks = choice.split_blocks;
  gp.k_blocks = (int32_t)blocks;
  gp.run_blocks = out == kOut32 ? kLinRunBlocks : (out == kOut16Runs ? kLinRunBlocks16 : (int32_t)blocks);
  gp.idesc = lin_idesc(half_type, a.mn, b.mn, 128 * cg);
  gp.mark = mark;
  const int mode = split ? kPlain : tail.mode;
  if (cg == 2 && bt == 128) st = launch_linear<128, 2>(gp, out, mode, half_type, sms, stream);
  else if (cg == 2) st = launch_linear<256, 2>(gp, out, mode, half_type, sms, stream);
  else if (bt == 128) st = launch_linear<128, 1>(gp, out, mode, half_type, sms, stream);
  else st = launch_linear<64, 1>(gp, out, mode, half_type, sms, stream);
  if (st != QB_OK) return st;
  if (!split) return QB_OK;
  const bool vector = N % 4 == 0;
  QB_CUDA_TRY(launch_kernel(vector ? linear_join_kernel<4> : linear_join_kernel<1>, (unsigned)std::min<int64_t>(lin_up(M * N, vector ? 1024 : 256), (int64_t)sms * 8), 256, 0,
                            stream, 1, false, parts, choice.splits, M * N, (int)N, tail));
  return QB_OK;
}

// Runs of rows for the column sums: about eight blocks per SM, no run shorter than 32 rows.
static int64_t column_runs(int64_t M, int64_t N, int sms) {
  return std::max<int64_t>(1, std::min<int64_t>(lin_up(M, 32), std::max<int64_t>(1, (int64_t)sms * 8 / lin_up(N, 256))));
}

static qb_status check_linear(const char* what, const void* const (&needed)[4], int type, int out_type, int64_t M, int64_t N, int64_t K) {
  bool ok = (type == QB_BF16 || type == QB_F16) && (out_type == type || out_type == QB_F32) && !impossible_linear(M, N, K);
  for (const void* p : needed) ok = ok && p;
  if (ok) return QB_OK;
  set_last_error("%s: invalid argument (M=%lld N=%lld K=%lld type %d, output type %d)", what, (long long)M, (long long)N, (long long)K, type, out_type);
  return QB_ERR_INVALID;
}
static qb_status no_room_for_bias() {
  set_last_error("qb_linear_grad_w: the workspace is too small for the bias's gradient (qb_linear_workspace_bytes)");
  return QB_ERR_WORKSPACE;
}
static qb_status check_linear_ws(const char* what, const void* ws, size_t ws_bytes) {
  if (ws && aligned16(ws) && ws_bytes >= kWsMinBytes) return QB_OK;
  set_last_error("%s: workspace null, not 16-byte aligned or too small", what);
  return QB_ERR_WORKSPACE;
}

}  // namespace qb

extern "C" size_t qb_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  using namespace qb;
  if (impossible_linear(M, N, K)) return 0;
  const size_t pads = pad_bytes(M, K) + pad_bytes(N, K) + pad_bytes(M, N);
  const size_t sums = ((size_t)column_runs(M, N, kRingMaxCtas) * (size_t)N * 4 + 255) / 256 * 256;
  // parts of a split product: where its output is small against the device
  const int64_t outs[3] = {M * N, M * K, N * K};
  size_t parts = 0;
  for (int64_t n : outs) parts = std::max(parts, (size_t)std::min<int64_t>(n * 16, (int64_t)16 << 20) * 4);
  return kLinScratchOff + pads + sums + parts;
}

extern "C" int32_t qb_linear_tile_columns(int64_t M, int64_t N, int64_t K, size_t ws_bytes, int32_t* rows, int32_t* half_tiles, int32_t* splits) {
  using namespace qb;
  if (impossible_linear(M, N, K)) return 0;
  int sms = 148;
  require_sm100(&sms);  // without a device: for a 148-SM part
  const LinearChoice c = choose_linear(M, N, K, sms, ws_bytes > kLinScratchOff ? ws_bytes - kLinScratchOff : 0);
  if (rows) *rows = 128 * c.cg;
  if (half_tiles) *half_tiles = c.tiles - c.whole;
  if (splits) *splits = c.splits;
  return c.bt;
}

extern "C" qb_status qb_linear(const void* x, const void* w, int type, const float* bias, int activation, const void* residual, int64_t M, int64_t N, int64_t K,
                               int out_type, void* y, void* pre, int8_t* pre_codes, float* pre_scales, void* ws, size_t ws_bytes, void* cuda_stream) {
  using namespace qb;
  const char* const what = "qb_linear";
  qb_status st = check_linear(what, {x, w, y, y}, type, out_type, M, N, K);
  if (st != QB_OK) return st;
  if (activation < QB_IDENTITY || activation > QB_GELU || (pre_codes != nullptr) != (pre_scales != nullptr) || (pre && pre_codes) ||
      ((pre || pre_codes) && out_type != type)) {
    set_last_error("qb_linear: invalid activation (%d), or a pre-activation saved in both forms, without its scales or beside an fp32 output", activation);
    return QB_ERR_INVALID;
  }
  const size_t e = out_type == QB_F32 ? 4 : 2;
  if (!aligned16(x) || !aligned16(w) || !aligned_to(bias, 4) || !aligned_to(residual, e) || !aligned_to(y, e) || !aligned_to(pre, 2) || !aligned_to(pre_scales, 4)) {
    set_last_error("qb_linear: x and w must be 16-byte aligned, the others aligned to their elements");
    return QB_ERR_ALIGN;
  }
  if ((st = check_linear_ws(what, ws, ws_bytes)) != QB_OK) return st;
  int sms = 0;
  if ((st = require_sm100(&sms)) != QB_OK) return st;
  const LinearTail tail = {bias, residual, nullptr, nullptr, y, pre, activation == QB_GELU ? kGelu : kPlain, out_type, type, aligned16(y)};
  return run_linear(what, {x, M, K, false}, {w, N, K, false}, M, N, K, tail, pre_codes, pre_scales, ws, LinearScratch(ws, ws_bytes), 0, sms, (cudaStream_t)cuda_stream);
}

extern "C" qb_status qb_linear_grad_x(const void* grad_y, const void* w, int type, const void* pre, const int8_t* pre_codes, const float* pre_scales,
                                      const void* residual, int64_t M, int64_t N, int64_t K, void* grad_x, void* ws, size_t ws_bytes, void* cuda_stream) {
  using namespace qb;
  const char* const what = "qb_linear_grad_x";
  qb_status st = check_linear(what, {grad_y, w, grad_x, grad_x}, type, type, M, N, K);
  if (st != QB_OK) return st;
  if ((pre_codes != nullptr) != (pre_scales != nullptr) || (pre && pre_codes) || (residual && (pre || pre_codes))) {
    set_last_error("qb_linear_grad_x: a pre-activation in both forms, codes without scales, or a residual beside a pre-activation");
    return QB_ERR_INVALID;
  }
  if (!aligned16(grad_y) || !aligned16(w) || !aligned_to(residual, 2) || !aligned_to(grad_x, 2) || !aligned_to(pre, 2) || !aligned_to(pre_scales, 4)) {
    set_last_error("qb_linear_grad_x: grad_y and w must be 16-byte aligned, the others aligned to their elements");
    return QB_ERR_ALIGN;
  }
  if ((st = check_linear_ws(what, ws, ws_bytes)) != QB_OK) return st;
  int sms = 0;
  if ((st = require_sm100(&sms)) != QB_OK) return st;
  const LinearTail tail = {nullptr, pre ? pre : residual, pre_codes, pre_scales, grad_x, nullptr, pre || pre_codes ? kSlope : kPlain, type, type, aligned16(grad_x)};
  return run_linear(what, {grad_y, M, N, false}, {w, N, K, true}, M, K, N, tail, nullptr, nullptr, ws, LinearScratch(ws, ws_bytes), 0, sms, (cudaStream_t)cuda_stream);
}

extern "C" qb_status qb_linear_grad_w(const void* grad_y, const void* x, int type, int64_t M, int64_t N, int64_t K, int out_type, void* grad_w, float* grad_bias,
                                      void* ws, size_t ws_bytes, void* cuda_stream) {
  using namespace qb;
  const char* const what = "qb_linear_grad_w";
  const void* const either = grad_w ? grad_w : grad_bias;
  qb_status st = check_linear(what, {grad_y, grad_w ? x : grad_y, either, either}, type, out_type, M, N, K);
  if (st != QB_OK) return st;
  if (!aligned16(grad_y) || !aligned16(x) || !aligned_to(grad_w, out_type == QB_F32 ? 4 : 2) || !aligned_to(grad_bias, 4)) {
    set_last_error("qb_linear_grad_w: grad_y and x must be 16-byte aligned, the others aligned to their elements");
    return QB_ERR_ALIGN;
  }
  if ((st = check_linear_ws(what, ws, ws_bytes)) != QB_OK) return st;
  int sms = 0;
  if ((st = require_sm100(&sms)) != QB_OK) return st;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  LinearScratch scratch(ws, ws_bytes);
  const bool few = N <= kFewColumns && M * N <= kFewValues;
  const int64_t run = lin_up(M, column_runs(M, N, sms)), runs = lin_up(M, run);
  float* const parts = grad_bias && !few ? static_cast<float*>(scratch.take((size_t)runs * (size_t)N * 4)) : nullptr;
  if (grad_bias && !few && !parts) return no_room_for_bias();
  const uint32_t mark = grad_w && grad_bias ? next_mark() : 0;
  if (grad_w) {
    const LinearTail tail = {nullptr, nullptr, nullptr, nullptr, grad_w, nullptr, kPlain, out_type, type, aligned16(grad_w)};
    if ((st = run_linear(what, {grad_y, M, N, true}, {x, M, K, true}, N, K, M, tail, nullptr, nullptr, ws, scratch, mark, sms, stream)) != QB_OK) return st;
  }
  // behind the product, under which it runs where that leaves SMs
  if (grad_bias && few) {
    QB_CUDA_TRY(launch_kernel(grad_w ? column_few_kernel<true> : column_few_kernel<false>, 1, 1024, 0, stream, 1, false, static_cast<const uint16_t*>(grad_y), M, (int32_t)N,
                              (int)(type == QB_F16), grad_bias, ws, mark));
  } else if (grad_bias) {
    const int col_blocks = (int)lin_up(N, 256);
    auto sum = N % 8 == 0 ? (grad_w ? column_parts_kernel<true, true> : column_parts_kernel<true, false>)
                          : (grad_w ? column_parts_kernel<false, true> : column_parts_kernel<false, false>);
    QB_CUDA_TRY(launch_kernel(sum, (unsigned)(col_blocks * runs), 256, 0, stream, 1, false, static_cast<const uint16_t*>(grad_y), M, (int32_t)N, run, col_blocks,
                              (int)(type == QB_F16), parts, static_cast<const void*>(ws), mark));
    QB_CUDA_TRY(launch_kernel(column_join_kernel, (unsigned)lin_up(N, 32), 32 * kColumnGroups, 0, stream, 1, false, parts, (int)runs, (int32_t)N, grad_bias,
                              grad_w ? ws : nullptr));
  }
  return QB_OK;
}
