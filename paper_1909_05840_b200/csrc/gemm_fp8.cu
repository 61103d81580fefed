// qb_gemm_fp8: y[m][n] = sum over K of a[m][k] * b[n][k] + bias[n] on 8-bit floating point codes with one power-of-two scale per
// row and block of 128 along K (qb_quantize_fp8, qb_quantize_fp8_weights).
//
// The scales enter inside the tensor cores: tcgen05.mma kind::mxf8f6f4 multiplies each row's 32 products of an instruction
// by 2^(ea - 127) * 2^(eb - 127), the bytes taken from tensor memory, and accumulates in fp32, so that a tile is summed over all of
// K in tensor memory at the full 8-bit rate and leaves it once (scales applied outside would cost an accumulator read per
// block of 128).  A word holds the bytes of four blocks; the instruction descriptor names the byte, so that the scales are copied
// to tensor memory once per 512 elements of K.
//
// One persistent CTA per SM, 12 warps:
//   warp 0        TMA producer (one lane): codes of A and B (128-byte swizzle, K block of 128), every fourth block the scales
//   warp 1        issues tcgen05.cp (scales) and tcgen05.mma, owns the tensor memory (one lane)
//   warps 2..3    idle
//   warps 4..11   epilogue, two per TMEM lane quarter: tcgen05.ld -> bias -> round -> shared memory -> TMA store
// A tile is 128 rows of A per CTA x BT rows of B; TMEM lane = row of A, column = row of B.  Large products run as CTA pairs
// (cta_group::2, 256 x 256): each CTA stages its own 128 rows of A and half of B's rows.  No load is multicast.
// Two accumulators, so that the epilogue of a tile overlaps the products of the next.  At BT = 256 they and the scales
// do not fit the 512 columns side by side: the accumulators overlap by 32 columns, which the epilogue reads first.
// Every wait is bounded: on expiry the CTA records QB_ERR_TIMEOUT and leaves through the normal exit path.
//
// Bound by loads for long K (24,576 x 1,024 x 4,096: bfloat16 out 75 us, 2,750 TFLOP/s, of which the MMAs alone take 62 us, fp32 out
// 81: a K block of a pair is 64 KB, and comes at 50 to 60 bytes per clock and SM), by the epilogue up to K = 768 (5,003 x 2,304 x
// 768: 11.4 us) and by writing y (24,576 x 4,096 x 1,024: 88 us, 74 without the stores).  y leaves by TMA: staging and store pipes are
// what the epilogue waits for (18,944 x 4,096, K = 128 46.4 us with stores by the warps, 40.4 by TMA; 384 51.0 and 43.8; 768 59.2 and
// 58.0; 1,024 69.1 and 71.1; 2,048 120.1 and 119.7).  Rows that are not 16-byte aligned are stored by words (6,235 x 3,501 x 753: 40
// us, with 3,504 columns 22).
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>

#include "common.cuh"
#include "fp8.cuh"
#include "mbar_wait.cuh"
#include "ptx_float.cuh"
#include "tensormap.cuh"

namespace qb {

struct Fp8Params {
  CUtensorMap tma, tmb;    // codes, box 128 bytes of K x the CTA's rows
  CUtensorMap tmb_half;    // pairs: B's rows for a tile of half the width
  CUtensorMap tmsa, tmsb;  // scales as rows of 512 bytes
  CUtensorMap tmy;         // y (or the splits' parts, one after the other) in boxes of 32 rows x 128 bytes
  const float* bias;
  void* y;
  void* ws;
  int32_t M, N, K;
  int32_t n_tiles, tiles;
  int32_t whole;        // tiles below this are BT wide; pairs: the others are halves, two after the other
  int32_t split_tiles;  // tiles of one split of K (split s writes rows s * M .. of y, fp32)
  int32_t split_blocks; // blocks of 128 of K per split, a multiple of 4 where there are several
  int32_t words;        // rows of 512 bytes of scales per 128 rows of codes
  int32_t a_last, b_last;  // last block of 128 rows of A's and of B's scales
  int32_t tma_store;    // 1: rows of y are 16-byte aligned
  uint32_t idesc;       // fp8_idesc
};

constexpr int kFp8EpilogueWarps = 8;
constexpr int kFp8FirstEpilogueWarp = 4;
constexpr int kFp8Threads = 32 * (kFp8FirstEpilogueWarp + kFp8EpilogueWarps);

template <int BT, int CG>
struct Fp8Cfg {
  static constexpr int kABytes = 128 * 128;
  static constexpr int kBBytes = BT / CG * 128;
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kScaleBlocksB = (BT + 127) / 128;  // blocks of 128 rows of B's scales that a tile needs
  static constexpr int kScaleBytes = 512 * (1 + kScaleBlocksB);
  static constexpr int kStages = BT == 64 ? 6 : 5;
  static constexpr int kOutBytes = kFp8EpilogueWarps * 32 * 128;
  static constexpr int kBarBytes = 256;
  static constexpr int kBiasBytes = 2 * 256 * 4;
  static constexpr int kSmemBytes = kStages * (kStageBytes + kScaleBytes) + kOutBytes + kBarBytes + kBiasBytes;
  static constexpr int kScaleCols = 4 * (1 + kScaleBlocksB);
  static constexpr int kTmemCols = BT == 64 ? 256 : 512;
  // the second accumulator's first column: behind the first where scales fit too, else 32 columns back
  static constexpr int kAcc1 = 2 * BT + kScaleCols <= kTmemCols ? BT : BT - 32;
  static constexpr bool kOverlap = kAcc1 < BT;
  static constexpr int kScaleCol = kAcc1 + BT;
  static_assert(kScaleCol + kScaleCols <= kTmemCols, "tensor memory");
  static_assert(kSmemBytes <= 232448, "shared memory");
};

// Shared-memory matrix descriptor of a K-major operand with 128-byte swizzle: start address >> 4 (bits 0-13), leading offset
// (16-29, unused here), 1024 bytes between groups of eight rows (32-45), version 1 (46-47), SWIZZLE_128B (61-63 = 2).
__device__ __forceinline__ uint64_t fp8_operand_desc(uint32_t smem_addr) {
  return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// The same for 32 rows of 16 bytes without swizzle (scales): 128 bytes between groups of eight rows.
__device__ __forceinline__ uint64_t fp8_scale_desc(uint32_t smem_addr) {
  return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}
// Instruction descriptor for kind::mxf8f6f4 without N >> 3 (bits 17-22) and the byte numbers of the scales (A's in bits 29-30, B's
// in 4-5): formats in bits 7-9 and 10-12 (e4m3 0, e5m2 1), both operands K-major, scales UE8M0 (23), M >> 4 in 24-28.
static uint32_t fp8_idesc(int a_format, int b_format, int mma_m) {
  return ((uint32_t)a_format << 7) | ((uint32_t)b_format << 10) | (1u << 23) | ((uint32_t)(mma_m >> 4) << 24);
}

// Where tile t lies: first row and column, columns, split and its range of K blocks.
template <int BT, int CG>
struct Fp8Tile {
  int m0, n0, width, split, k0, k1;
  __device__ __forceinline__ Fp8Tile(const Fp8Params& gp, int t) {
    split = t / gp.split_tiles;
    t -= split * gp.split_tiles;
    k0 = split * gp.split_blocks;
    k1 = min(k0 + gp.split_blocks, gp.K / 128);
    width = BT;
    int half = 0;
    if (CG == 2 && t >= gp.whole) {
      half = (t - gp.whole) & 1;
      t = gp.whole + ((t - gp.whole) >> 1);
      width = BT / 2;
    }
    m0 = t / gp.n_tiles;
    n0 = (t - m0 * gp.n_tiles) * BT + half * (BT / 2);
    m0 *= 128 * CG;
  }
};

// Barrier over the epilogue warps (named barrier 1) that also ORs a predicate over them.
__device__ __forceinline__ bool fp8_epilogue_sync_or(bool pred) {
  uint32_t res;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbar.red.or.pred p, 1, %2, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(res)
      : "r"((uint32_t)pred), "n"(32 * kFp8EpilogueWarps)
      : "memory");
  return res != 0;
}

template <int BT, int CG, bool BF16>
__global__ void __launch_bounds__(kFp8Threads, 1) gemm_fp8_kernel(const __grid_constant__ Fp8Params gp) {
  using Cfg = Fp8Cfg<BT, CG>;
  constexpr int kStages = Cfg::kStages;
  const uint32_t rank = CG == 2 ? ptx::cluster_ctarank() : 0u;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t smem_base = ptx::smem_u32(smem);
  uint8_t* const out_ptr = smem + kStages * Cfg::kStageBytes;  // 1024-byte aligned
  const uint32_t scale_base = smem_base + kStages * Cfg::kStageBytes + Cfg::kOutBytes;
  uint8_t* const bar_ptr = smem + kStages * (Cfg::kStageBytes + Cfg::kScaleBytes) + Cfg::kOutBytes;
  const uint32_t bar_base = ptx::smem_u32(bar_ptr);
  auto full = [&](int s) { return bar_base + 8u * s; };
  auto empty = [&](int s) { return bar_base + 8u * (kStages + s); };
  auto acc_full = [&](int a) { return bar_base + 8u * (2 * kStages + a); };
  auto acc_empty = [&](int a) { return bar_base + 8u * (2 * kStages + 2 + a); };
  const uint32_t overlap_read = bar_base + 8u * (2 * kStages + 4);  // the columns that both accumulators have were read
  const uint32_t drain_bar = bar_base + 8u * (2 * kStages + 5);
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bar_ptr + 8 * (2 * kStages + 6));
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* const bias_tile = reinterpret_cast<float*>(bar_ptr + Cfg::kBarBytes);  // [2][256]
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
      ptx::mbar_init(acc_empty(a), kFp8EpilogueWarps * CG);
    }
    ptx::mbar_init(overlap_read, 4 * CG);
    ptx::mbar_init(drain_bar, 1);
    *abort_flag = 0;
    ptx::fence_mbar_init();
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
        const Fp8Tile<BT, CG> tile(gp, t);
        const bool half = CG == 2 && tile.width < BT;
        const int m0 = tile.m0 + (int)rank * 128, n0 = tile.n0;
        const int sa = min(m0 / 128, gp.a_last) * gp.words;
        const int b_row = n0 + (int)rank * (tile.width / CG);
        const CUtensorMap* const tmb = half ? &gp.tmb_half : &gp.tmb;
        const uint32_t bytes = CG * (Cfg::kABytes + (half ? Cfg::kBBytes / 2 : Cfg::kBBytes));
        for (int kb = tile.k0; kb < tile.k1; ++kb) {
          if (!wait_barrier_relaxed(empty(stage), phase ^ 1u, abort_flag)) {
            timed_out = true;
            where = (0 << 16) | stage;
            break;
          }
          const bool scales = (kb & 3) == 0;
          const uint32_t a_smem = smem_base + stage * Cfg::kStageBytes, b_smem = a_smem + Cfg::kABytes;
          const uint32_t s_smem = scale_base + stage * Cfg::kScaleBytes;
          if (rank == 0) ptx::mbar_arrive_expect_tx(full(stage), bytes + (scales ? CG * Cfg::kScaleBytes : 0));
          auto load = [&](uint32_t dst, const CUtensorMap* tm, int x, int y) {
            if constexpr (CG == 2) ptx::tma_load_2d_pair(dst, tm, lead(full(stage)), x, y);
            else ptx::tma_load_2d(dst, tm, full(stage), x, y);
          };
          if (scales) {
            load(s_smem, &gp.tmsa, 0, sa + kb / 4);
#pragma unroll
            for (int j = 0; j < Cfg::kScaleBlocksB; ++j)
              load(s_smem + 512 * (1 + j), &gp.tmsb, 0, min(n0 / 128 + j, gp.b_last) * gp.words + kb / 4);
          }
          load(a_smem, &gp.tma, kb * 128, m0);
          load(b_smem, tmb, kb * 128, b_row);
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
      const uint64_t a_desc0 = fp8_operand_desc(smem_base), b_desc0 = fp8_operand_desc(smem_base + Cfg::kABytes);
      const uint64_t s_desc0 = fp8_scale_desc(scale_base);
      const uint32_t sfa = tmem_base + Cfg::kScaleCol, sfb0 = sfa + 4;
      int stage = 0, it = 0;
      uint32_t phase = 0;
      for (int t = group; t < gp.tiles && !timed_out; t += groups, ++it) {
        const int a = it & 1;
        const uint32_t d = tmem_base + (a ? Cfg::kAcc1 : 0);
        const Fp8Tile<BT, CG> tile(gp, t);
        const uint32_t sfb = sfb0 + (uint32_t)(tile.n0 % 128 / 32);  // where the tile begins in its block of 128 scales
        const uint32_t idesc0 = gp.idesc | ((uint32_t)(tile.width >> 3) << 17);
        bool ok = wait_barrier(acc_empty(a), ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_flag);
        if (Cfg::kOverlap && ok && it > 0) ok = wait_barrier(overlap_read, (uint32_t)(it - 1) & 1u, abort_flag);
        if (!ok) {
          timed_out = true;
          where = (1 << 16) | 0x100 | a;
          break;
        }
        for (int kb = tile.k0; kb < tile.k1; ++kb) {
          if (!wait_barrier(full(stage), phase, abort_flag)) {
            timed_out = true;
            where = (1 << 16) | stage;
            break;
          }
          ptx::tcgen05_fence_after_sync();
          const uint32_t id = (uint32_t)kb & 3u;
          if (id == 0) {
            const uint64_t s_desc = s_desc0 + (uint64_t)(stage * (Cfg::kScaleBytes >> 4));
#pragma unroll
            for (int j = 0; j <= Cfg::kScaleBlocksB; ++j) ptx::tmem_copy_scales_cg<CG>(sfa + 4 * j, s_desc + (uint64_t)(j * (512 >> 4)));
          }
          const uint32_t idesc = idesc0 | (id << 29) | (id << 4);
          const uint64_t a_desc = a_desc0 + (uint64_t)(stage * (Cfg::kStageBytes >> 4));
          const uint64_t b_desc = b_desc0 + (uint64_t)(stage * (Cfg::kStageBytes >> 4));
#pragma unroll
          for (int j = 0; j < 4; ++j)  // 32 elements of K per instruction: 32 bytes
            ptx::mma_mxf8_ss_cg<CG>(d, a_desc + 2u * j, b_desc + 2u * j, idesc, sfa, sfb, kb != tile.k0 || j != 0 ? 1u : 0u);
          ptx::mma_commit_cg<CG>(empty(stage));
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
        if (!timed_out) ptx::mma_commit_cg<CG>(acc_full(a));
      }
      if (timed_out) {  // wait (bounded) for what was issued before tensor memory is freed
        ptx::mma_commit_cg<CG>(drain_bar);
        const long long t0 = clock64();
        while (!ptx::mbar_try_wait(drain_bar, 0) && clock64() - t0 < 400000000ll) {
        }
      }
    }
  } else if (warp >= kFp8FirstEpilogueWarp) {
    // ---------------- epilogue ----------------------------------------------------------------------
    constexpr int kCols = BF16 ? 64 : 32;  // columns of a chunk: 128 bytes of y
    const int ew = warp - kFp8FirstEpilogueWarp, quarter = warp & 3, half = ew >> 2;
    const int e = threadIdx.x - 32 * kFp8FirstEpilogueWarp;
    uint8_t* const buf = out_ptr + ew * (32 * 128);
    const uint32_t lanes = tmem_base + ((uint32_t)(quarter * 32) << 16);
    auto arrive = [&](uint32_t bar) {  // this warp has read from tensor memory what it announces
      ptx::tcgen05_fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        if (CG == 2 && rank != 0) ptx::mbar_arrive_remote(lead(bar));
        else ptx::mbar_arrive(bar);
      }
    };
    int it = 0;
    for (int t = group; t < gp.tiles; t += groups, ++it) {
      const int a = it & 1;
      const Fp8Tile<BT, CG> tile(gp, t);
      int m0 = tile.m0 + (int)rank * 128 + quarter * 32, n0 = tile.n0;
      int chunks = m0 < gp.M ? max(0, min(tile.width / kCols, (gp.N - n0 + kCols - 1) / kCols)) : 0;
      // formed before the wait: the compiler would do the divisions behind it, where the next tile's products wait for this
      // tile's first columns (18,944 x 4,096 x 1,024: 68.7 us, so 68.2)
      asm volatile("" : "+r"(m0), "+r"(n0), "+r"(chunks));
      bias_tile[a * 256 + e] = gp.bias && e < BT && n0 + e < gp.N ? gp.bias[n0 + e] : 0.0f;
      const bool ok = ew != 0 || wait_barrier_warp(acc_full(a), (uint32_t)(it >> 1) & 1u, abort_flag);
      if (fp8_epilogue_sync_or(!ok)) {  // publishes the bias, and all eight warps give up together
        timed_out = true;
        where = (3 << 16) | a;
        break;
      }
      ptx::tcgen05_fence_after_sync();
      const uint32_t acc = lanes + (a ? Cfg::kAcc1 : 0);
      // accumulator 0 shares its last 32 columns, accumulator 1 its first: they are read first, by the quarter's first warp
      const bool down = Cfg::kOverlap && a == 0;
      if (Cfg::kOverlap && half == 0 && (down ? chunks < BT / kCols : chunks == 0)) arrive(overlap_read);
      if (half >= chunks) arrive(acc_empty(a));
#pragma unroll 1
      for (int i = half; i < chunks; i += 2) {
        const int c0 = (down ? chunks - 1 - i : i) * kCols;
        uint32_t v[kCols / 32][32];
#pragma unroll
        for (int p = 0; p < kCols / 32; ++p) ptx::tmem_ld_32x32b_x32(acc + (uint32_t)(c0 + 32 * p), v[p]);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int p = 0; p < kCols / 32; ++p) ptx::tmem_ld_regs_ready(v[p]);
        if (Cfg::kOverlap && i == 0 && (!down || chunks == BT / kCols)) arrive(overlap_read);
        if (i + 2 >= chunks) arrive(acc_empty(a));
        const float4* const b4 = reinterpret_cast<const float4*>(bias_tile + a * 256 + c0);
        if (lane == 0) ptx::tma_store_wait_read0();  // the chunk before has left the buffer
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j) {  // 16 bytes of the row at a time; the swizzle keeps the lanes on different banks
          uint4 w;
          if constexpr (BF16) {
            const float4 b0 = b4[2 * j], b1 = b4[2 * j + 1];
            const uint32_t* const s = &v[j >> 2][(j & 3) * 8];
            const __nv_bfloat162 p0 = __floats2bfloat162_rn(__uint_as_float(s[0]) + b0.x, __uint_as_float(s[1]) + b0.y);
            const __nv_bfloat162 p1 = __floats2bfloat162_rn(__uint_as_float(s[2]) + b0.z, __uint_as_float(s[3]) + b0.w);
            const __nv_bfloat162 p2 = __floats2bfloat162_rn(__uint_as_float(s[4]) + b1.x, __uint_as_float(s[5]) + b1.y);
            const __nv_bfloat162 p3 = __floats2bfloat162_rn(__uint_as_float(s[6]) + b1.z, __uint_as_float(s[7]) + b1.w);
            w.x = *reinterpret_cast<const uint32_t*>(&p0);
            w.y = *reinterpret_cast<const uint32_t*>(&p1);
            w.z = *reinterpret_cast<const uint32_t*>(&p2);
            w.w = *reinterpret_cast<const uint32_t*>(&p3);
          } else {
            const float4 b0 = b4[j];
            const uint32_t* const s = &v[0][j * 4];
            w.x = __float_as_uint(__uint_as_float(s[0]) + b0.x);
            w.y = __float_as_uint(__uint_as_float(s[1]) + b0.y);
            w.z = __float_as_uint(__uint_as_float(s[2]) + b0.z);
            w.w = __float_as_uint(__uint_as_float(s[3]) + b0.w);
          }
          *reinterpret_cast<uint4*>(buf + lane * 128 + ((j ^ (lane & 7)) << 4)) = w;
        }
        __syncwarp();
        const int rows = min(32, gp.M - m0);
        const size_t first_row = (size_t)tile.split * gp.M;
        if (gp.tma_store) {
          ptx::fence_proxy_async_smem();  // every lane: its own stores
          __syncwarp();
          if (lane == 0) {
            ptx::tma_store_3d(&gp.tmy, ptx::smem_u32(buf), n0 + c0, m0, tile.split);
            ptx::tma_store_commit();
          }
        } else if constexpr (BF16) {  // rows of y of any alignment: a row at a time, the lanes on consecutive words of it
          const int cols = min(kCols, gp.N - n0 - c0);
          uint16_t* const to = static_cast<uint16_t*>(gp.y) + (first_row + m0) * gp.N + n0 + c0;
          const int first_odd = (int)(reinterpret_cast<uintptr_t>(to) >> 1) & 1, step = gp.N & 1;
          const auto word = [&](int r, int col) {  // columns col and col + 1 of a row, col even
            return *reinterpret_cast<const uint32_t*>(buf + r * 128 + (((col >> 3) ^ (r & 7)) << 4) + (col & 6) * 2);
          };
          for (int r = 0; r < rows; ++r) {
            // columns odd and odd + 1, odd + 2 and odd + 3 .. are the words of y
            const int odd = first_odd ^ (step & r), c = 2 * lane + odd;
            uint32_t w = word(r, 2 * lane);
            if (odd) w = __byte_perm(w, word(r, min(2 * lane + 2, kCols - 2)), 0x5432);
            if (c + 1 < cols) *reinterpret_cast<uint32_t*>(to + (size_t)r * gp.N + c) = w;
          }
          if (lane < rows) {  // the single columns at the ends, of all rows at once
            const int odd = first_odd ^ (step & lane);
            uint16_t* const at = to + (size_t)lane * gp.N;
            if (odd) at[0] = (uint16_t)word(lane, 0);
            if ((cols - odd) & 1) at[cols - 1] = (uint16_t)(word(lane, (cols - 1) & ~1) >> ((cols - 1) & 1) * 16);
          }
        } else {  // the lanes on consecutive values of a row
          const int col = n0 + c0 + lane;
          if (col < gp.N) {
            float* const to = static_cast<float*>(gp.y) + (first_row + m0) * gp.N + col;
            for (int r = 0; r < rows; ++r)
              to[(size_t)r * gp.N] = *reinterpret_cast<const float*>(buf + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4);
          }
        }
      }
    }
    if (lane == 0) ptx::tma_store_wait_read0();  // the buffers are in use until then
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

template <int BT, int CG, bool BF16>
static qb_status launch_gemm_fp8(const Fp8Params& gp, int sms, cudaStream_t stream) {
  using Cfg = Fp8Cfg<BT, CG>;
  auto kernel = gemm_fp8_kernel<BT, CG, BF16>;
  static std::atomic<bool> attr_set[64] = {};
  int dev = 0;
  QB_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
    QB_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmemBytes));
    if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
  }
  const int grid = std::min(gp.tiles, sms / CG) * CG;
  QB_CUDA_TRY(launch_kernel(kernel, (unsigned)grid, kFp8Threads, Cfg::kSmemBytes, stream, CG, false, gp));
  return QB_OK;
}

// y = the splits' sum, in their order, + bias.
template <bool BF16, bool VECTOR>
__global__ void __launch_bounds__(256) fp8_join_kernel(const float* parts, int splits, int64_t MN, int N, const float* bias, void* y) {
  constexpr int V = VECTOR ? 4 : 1;
  pdl_begin();
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V; i < MN; i += (int64_t)gridDim.x * 256 * V) {
    float v[V];
    if constexpr (VECTOR) *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(parts + i);
    else v[0] = parts[i];
    for (int s = 1; s < splits; ++s) {
      float w[V];
      if constexpr (VECTOR) *reinterpret_cast<float4*>(w) = *reinterpret_cast<const float4*>(parts + s * MN + i);
      else w[0] = parts[s * MN + i];
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] += w[j];
    }
    const int n = (int)(i % N);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (bias) v[j] += bias[n + j];  // (vectors: N is a multiple of 4)
      if constexpr (BF16) static_cast<__nv_bfloat16*>(y)[i + j] = __float2bfloat16_rn(v[j]);
      else static_cast<float*>(y)[i + j] = v[j];
    }
  }
}

constexpr size_t kPartsOff = 1024;  // of a split product's parts in the workspace
static int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m; }
static bool impossible_product(int64_t M, int64_t N, int64_t K) {
  if (M <= 0 || N <= 0 || K <= 0 || M > QB_MAX_MN || N > QB_MAX_MN || K > QB_MAX_MN) return true;
  return up(M, 128) * up(N, 64) > (int64_t)1 << 30 || std::max(up(M, 128), up(N, 128)) * fp8_scale_words(K) > (int64_t)1 << 30;
}

// The form of a product: CTAs per tile, columns, for pairs how many tiles are whole, and splits of K.
struct Fp8Choice {
  int cg, bt;
  int32_t tiles, whole, splits, split_blocks;
};
// The cheapest by what a launch and each of its rounds of tiles take, in hundredths of a microsecond: a tile a part per block of 128
// of K and a fixed part, but no less than its epilogue, the launch the time until the first tile and of the last epilogue.  Fitted
// to M = 18,944, 1 to 16 rounds, bfloat16 out (K = 128, 768, 4,096; four rounds of pairs 12.1, 16.2 and 58.0 us, eight of 128 columns
// 11.9, 18.9 and 74.8, 16 of 64 columns 18.3, 27.1 and 107).  With few rounds of short tiles the smaller ones are ahead: 2,048 x 2,304 x
// 768 6.5 us in two rounds of 128 columns, 7.6 in one of pairs; 5,003 x 2,304 x 768 12.0 by pairs, 12.9 by 128 columns.  A last round
// that fills at most half of the pairs is cut into tiles of half the width, which take about 0.7 of the time (6,144 x 1,024 x 4,096, 96
// tiles: 25.4 -> 22.1 us).  Where a long K meets few tiles, K is split into runs that are a multiple of 512 (a word of
// scales), whose sums a second kernel joins: that costs its launch and the traffic of the parts.
static Fp8Choice choose_fp8(int64_t M, int64_t N, int64_t K, int sms, size_t scratch) {
  static constexpr struct {
    int cg, bt, block, fixed, least, launch;
  } kForms[] = {{2, 256, 41, 20, 220, 480}, {1, 128, 27, 37, 120, 310}, {1, 64, 20, 25, 100, 300}};
  const int64_t blocks = K / 128;
  Fp8Choice best = {};
  int64_t best_cost = 0;
  for (const auto& f : kForms) {
    if (f.cg == 2 && sms < 2) continue;
    const int64_t groups = sms / f.cg, tiles = up(M, 128 * f.cg) * up(N, f.bt);
    for (int64_t splits = 1; splits == 1 || (4 * splits <= blocks && tiles * (splits - 1) < groups && splits * M * N * 4 <= (int64_t)scratch); ++splits) {
      const int64_t run = splits == 1 ? blocks : up(up(blocks, splits), 4) * 4;
      if (up(blocks, run) != splits) continue;
      const int64_t tile = std::max<int64_t>(f.block * run + f.fixed, f.least), all = tiles * splits, last = all % groups;
      const bool halves = f.cg == 2 && splits == 1 && last > 0 && 2 * last <= groups;
      const int64_t cost = f.launch + (all / groups) * tile + (halves ? tile * 7 / 10 : (last > 0 ? tile : 0)) + (splits > 1 ? 250 + splits * M * N / 7500 : 0);
      if (best.cg == 0 || cost < best_cost) {
        best_cost = cost;
        best = {f.cg, f.bt, (int32_t)(halves ? all + last : all), (int32_t)(halves ? all - last : all), (int32_t)splits, (int32_t)run};
      }
    }
  }
  return best;
}

}  // namespace qb

extern "C" int32_t qb_gemm_fp8_tile_columns(int64_t M, int64_t N, int64_t K, size_t ws_bytes, int32_t* half_tiles, int32_t* splits) {
  if (qb::impossible_product(M, N, K) || K % 128 != 0) return 0;
  int sms = 148;
  qb::require_sm100(&sms);  // without a device: for a 148-SM part
  const qb::Fp8Choice c = qb::choose_fp8(M, N, K, sms, ws_bytes > qb::kPartsOff ? ws_bytes - qb::kPartsOff : 0);
  if (half_tiles) *half_tiles = c.tiles - c.whole;
  if (splits) *splits = c.splits;
  return c.bt;
}

extern "C" qb_status qb_gemm_fp8(const uint8_t* a, const uint8_t* a_scale, int a_format, const uint8_t* b, const uint8_t* b_scale,
                                 int b_format, const float* bias, int64_t M, int64_t N, int64_t K, int out_type, void* y, void* ws,
                                 size_t ws_bytes, void* cuda_stream) {
  using namespace qb;
  if (!a || !a_scale || !b || !b_scale || !y || M <= 0 || N <= 0 || K <= 0 || M > QB_MAX_MN || N > QB_MAX_MN || K > QB_MAX_MN ||
      a_format < QB_E4M3 || a_format > QB_E5M2 || b_format < QB_E4M3 || b_format > QB_E5M2 || out_type < QB_F32 || out_type > QB_BF16) {
    set_last_error("qb_gemm_fp8: invalid argument (M=%lld N=%lld K=%lld formats %d, %d, output type %d)", (long long)M, (long long)N,
                   (long long)K, a_format, b_format, out_type);
    return QB_ERR_INVALID;
  }
  if (K % 128 != 0 || !aligned16(a) || !aligned16(b) || !aligned16(a_scale) || !aligned16(b_scale) ||
      reinterpret_cast<uintptr_t>(bias) % 4 != 0 || reinterpret_cast<uintptr_t>(y) % (out_type == QB_F32 ? 4 : 2) != 0) {
    set_last_error("qb_gemm_fp8: K must be a multiple of 128, codes and scales 16-byte aligned, bias and y aligned to their elements");
    return QB_ERR_ALIGN;
  }
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 4 != 0 || ws_bytes < kWsMinBytes) {
    set_last_error("qb_gemm_fp8: workspace null, not aligned or too small");
    return QB_ERR_WORKSPACE;
  }
  if (impossible_product(M, N, K)) {
    set_last_error("qb_gemm_fp8: more than 2^30 tiles, or pieces of scales (M=%lld N=%lld K=%lld)", (long long)M, (long long)N, (long long)K);
    return QB_ERR_INVALID;
  }
  int sms = 0;
  qb_status st = require_sm100(&sms);
  if (st != QB_OK) return st;
  const bool roomy = ws_bytes > kPartsOff && reinterpret_cast<uintptr_t>(ws) % 16 == 0;
  const Fp8Choice choice = choose_fp8(M, N, K, sms, roomy ? ws_bytes - kPartsOff : 0);
  const int cg = choice.cg, bt = choice.bt;
  Fp8Params gp;
  const CUtensorMapDataType u8 = CU_TENSOR_MAP_DATA_TYPE_UINT8, u32 = CU_TENSOR_MAP_DATA_TYPE_UINT32;
  gp.words = (int32_t)fp8_scale_words(K);
  if ((st = make_matrix_map(&gp.tma, u8, a, M, K, K, 128, 128, CU_TENSOR_MAP_SWIZZLE_128B)) != QB_OK) return st;
  if ((st = make_matrix_map(&gp.tmb, u8, b, N, K, K, bt / cg, 128, CU_TENSOR_MAP_SWIZZLE_128B)) != QB_OK) return st;
  gp.tmb_half = gp.tmb;
  if (choice.whole < choice.tiles && (st = make_matrix_map(&gp.tmb_half, u8, b, N, K, K, bt / 4, 128, CU_TENSOR_MAP_SWIZZLE_128B)) != QB_OK) return st;
  if ((st = make_matrix_map(&gp.tmsa, u32, a_scale, up(M, 128) * gp.words, 128, 512, 1, 128, CU_TENSOR_MAP_SWIZZLE_NONE)) != QB_OK) return st;
  if ((st = make_matrix_map(&gp.tmsb, u32, b_scale, up(N, 128) * gp.words, 128, 512, 1, 128, CU_TENSOR_MAP_SWIZZLE_NONE)) != QB_OK) return st;
  const bool split = choice.splits > 1;
  float* const parts = reinterpret_cast<float*>(static_cast<char*>(ws) + kPartsOff);
  const bool bf16 = out_type == QB_BF16 && !split;
  gp.tma_store = N * (bf16 ? 2 : 4) % 16 == 0 && (split || aligned16(y));
  gp.tmy = gp.tma;
  if (gp.tma_store && (st = make_parts_map(&gp.tmy, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, split ? parts : y,
                                           choice.splits, M, N, N * (bf16 ? 2 : 4), 32, bf16 ? 64 : 32)) != QB_OK)
    return st;
  gp.bias = split ? nullptr : bias;
  gp.y = split ? parts : y;
  gp.split_blocks = choice.split_blocks;
  gp.split_tiles = choice.tiles / choice.splits;
  gp.ws = ws;
  gp.M = (int32_t)M;
  gp.N = (int32_t)N;
  gp.K = (int32_t)K;
  gp.n_tiles = (int32_t)up(N, bt);
  gp.tiles = choice.tiles;
  gp.whole = choice.whole;
  gp.a_last = (int32_t)up(M, 128) - 1;
  gp.b_last = (int32_t)up(N, 128) - 1;
  gp.idesc = fp8_idesc(a_format, b_format, 128 * cg);
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (cg == 2) st = bf16 ? launch_gemm_fp8<256, 2, true>(gp, sms, stream) : launch_gemm_fp8<256, 2, false>(gp, sms, stream);
  else if (bt == 128) st = bf16 ? launch_gemm_fp8<128, 1, true>(gp, sms, stream) : launch_gemm_fp8<128, 1, false>(gp, sms, stream);
  else st = bf16 ? launch_gemm_fp8<64, 1, true>(gp, sms, stream) : launch_gemm_fp8<64, 1, false>(gp, sms, stream);
  if (st != QB_OK || !split) return st;
  const bool vector = N % 4 == 0;
  auto join = out_type == QB_BF16 ? (vector ? fp8_join_kernel<true, true> : fp8_join_kernel<true, false>)
                                  : (vector ? fp8_join_kernel<false, true> : fp8_join_kernel<false, false>);
  QB_CUDA_TRY(launch_kernel(join, (unsigned)std::min<int64_t>(up(M * N, vector ? 1024 : 256), (int64_t)sms * 8), 256, 0, stream, 1, false, parts,
                            choice.splits, M * N, (int)N, bias, y));
  return QB_OK;
}
