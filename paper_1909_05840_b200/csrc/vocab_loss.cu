// qb_vocab_loss, qb_vocab_loss_backward: softmax cross entropy of hidden states h [T][D] over a vocabulary w [V][D], logits
// z = h w^T + bias, without keeping the logits.
//
// Forward: tiles of 256 tokens x 256 words (up to 128 tokens: of 256 words x the tokens) are multiplied on the tensor cores and reduced
// to a maximum and a sum of exponentials per token on their way out of tensor memory; a second kernel joins the tiles of a token.
// Backward: with the forward pass's lse, g[v][t] = grad_loss[t] * (exp(z[t][v] - lse[t]) - [v = target[t]]) needs no reduction.
// The vocabulary is taken in pieces: for one piece g is formed (the logits again) and rounded to bfloat16 into the workspace,
// transposed, while the two products of the piece before it (bfloat16 because the tensor cores take both operands in one type, h's and w's:
// more bits would be a second bfloat16 term, two instructions for one in both products and twice g's bytes; the gradients
// come out 0.0021 to 0.0026 of their norm off, where rounding the exact ones to bfloat16 gives 0.0017),
//     grad_w [piece][D] = g h      and      grad_h [T][D] += g^T w,
// run in the same launch: the three kinds of tile are dealt over the SMs so that all end together.  grad_h is summed over the
// pieces in fp32 in the workspace (each element by one addition per launch, or into a slab of its own: the order is always the
// same); a last kernel rounds it and sums the bias's gradient, whose terms never were bfloat16.
//
// One product kernel for all of it: CTA pairs (tcgen05 cta_group::2, kind::f16, bfloat16 operands, fp32 accumulators), tiles of
// 256 x 256, K blocks of 64, a ring of three stages of two blocks (64 KB per CTA), two accumulators in tensor memory.  An operand lies in
// shared memory as the tensor has it: contraction along its rows (K-major) or down its columns (MN-major), so that nothing is
// transposed in memory.  12 warps: 0 loads (TMA), 1 issues MMAs, 4..11 epilogue, two per TMEM lane quarter.  Every wait is
// bounded, as in qb_gemm.
//
// Bound by the tensor cores (replayed from a graph after a pause; many passes in a row run under the power cap, a fifth slower):
// 4,096 x 30,522 x 768 forward 119 us (1,613 TFLOP/s, the tensor pipe busy for 84 %; the MMAs alone 109), backward 446; 3,686 x
// 30,522 x 1,024 forward 149, backward 510 us (1,355 TFLOP/s over the three products, 70 % busy; the MMAs alone 381, loads alone 284).  With
// few tokens by reading w: 77 tokens x 30,522 x 768 forward 13.7 us (w alone 7.3).
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "common.cuh"
#include "mbar_wait.cuh"
#include "ptx_float.cuh"
#include "tensormap.cuh"

namespace qb {

constexpr int kVocabTile = 256;
constexpr int kVocabEpilogueWarps = 8;
constexpr int kVocabThreads = 32 * (4 + kVocabEpilogueWarps);
constexpr int kVocabStages = 3;
constexpr int kVocabStageBytes = 65536;  // 128 rows of A and 128 of B, two K blocks of 64 each
constexpr int kVocabOutBytes = kVocabEpilogueWarps * 2048;
constexpr int kVocabBarBytes = 256;
// Backward: per accumulator three values of each of the tile's columns.  Forward with few tokens: a maximum and a sum per lane
// quarter and token.
constexpr int kVocabColBytes = 2 * 3 * 256 * 4;
constexpr int kFewTokens = 128;
static_assert(4 * kFewTokens * 8 <= kVocabColBytes, "columns' values");
constexpr int kVocabSmemBytes = kVocabStages * kVocabStageBytes + kVocabOutBytes + kVocabBarBytes + kVocabColBytes;
constexpr int kMaxPairs = 80;
constexpr float kLog2e = 1.4426950408889634f;

// How an operand lies and is loaded, two K blocks of 64 at a time: K-major (128 rows x 2 groups of 64 columns) or MN-major (128 rows x
// 2 groups of 64 columns, the rows along K); one box of three dimensions, or, where rows are no multiple of 128 bytes, two boxes
// of one group.  A box costs the TMA unit about 100 ns whatever it holds: with boxes of 8 KB 4,096 x 30,522 x 768 forward took 165 us, of
// 16 KB 129, of 32 KB 119.
enum VocabForm { kRows = 0, kRows2 = 1, kCols = 2, kCols2 = 3 };
enum VocabKind { kLogits = 0, kGradZ = 1, kGradW = 2, kGradH = 3 };
// FEW: up to kFewTokens tokens.  They are then the columns of the tiles of logits in the forward pass too, and the tiles are as wide
// as the tokens (rounded up to 32): a pair loads 256 words and those tokens, not 256 rows of mostly nothing (77 tokens, 30,522
// x 768: forward 21.8 -> 17.1 us, backward 69 -> 61).  With more tokens narrower tiles do not pay: loads bound the K blocks, so
// that 613 tokens as 3 x 224 columns took as long as 3 x 256, and the logits are reduced with a token per lane, which needs no
// exchange between lanes.

// One kind of tile of a launch.
struct VocabProblem {
  int32_t kind;
  int32_t map_a, map_b;    // tensor maps of the operands
  int32_t a_form, b_form;
  int32_t n_tiles;         // tile t of a split: row tile t / n_tiles, column tile t % n_tiles
  int32_t width;           // columns of a tile (FEW, logits; else 256)
  int32_t m_tiles;         // not 0: column tile t / m_tiles, row tile t % m_tiles
  int32_t split_tiles;     // tiles per split of the contraction
  int32_t k_blocks;        // of one split
  int32_t k_end;           // of all splits
  int32_t a_row0, b_row0;  // where the operands' rows begin in their tensors (rows of the tile, or of K where MN-major)
  int32_t start[kMaxPairs + 1];  // pair g has tiles start[g] .. start[g + 1] - 1
};

enum { kMapH = 0, kMapHTile, kMapW, kMapG, kMaps };

struct VocabParams {
  CUtensorMap map[kMaps];  // h, h with boxes of a narrower column tile's rows, w, g of the piece before
  VocabProblem prob[3];
  int32_t count;
  int32_t T, V, D;
  int32_t v0;           // first word of the piece whose logits are formed
  int32_t out_v0;       // first word of the piece that grad_w gets
  int32_t add;          // grad_h is added to what the slabs hold
  int32_t g_pitch;      // tokens rounded up to 64
  uint16_t* g_new;      // [words of a piece][g_pitch]
  uint16_t* grad_w;     // [V][D]
  float* slabs;         // [splits][T][D]
  const float* bias;
  const int32_t* targets;
  const float* lse;
  const float* grad_loss;
  float2* part;         // forward: [2 * word tile + half][T], maximum and sum of exponentials
  float* z_target;      // forward: [T]
  float* part_bias;     // backward: [2 * token tile + half][V], or NULL
  void* ws;
};

// Operand of 128 rows (or columns) x 128 elements of K, 128-byte swizzle.  K-major: 1024 bytes between groups of eight rows.
// MN-major: 64 consecutive elements of M or N are a row of 128 bytes, the next 64 are 16384 bytes on (leading offset), the next
// eight of K 1024 bytes (stride offset).  Version 1, SWIZZLE_128B as in qb_gemm.
__device__ __forceinline__ uint64_t vocab_desc(uint32_t smem_addr, int mn) {
  return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | (uint64_t)(mn ? 16384 >> 4 : 1) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}
// Instruction descriptor for kind::f16: D fp32 (bits 4-5 = 1), A and B bfloat16 (7-9, 10-12 = 1), MN-major A and B (15, 16),
// N >> 3 (17-22), M >> 4 (24-28).
__device__ __forceinline__ uint32_t vocab_idesc(int a_mn, int b_mn, int width) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(width >> 3) << 17) |
         ((uint32_t)(kVocabTile >> 4) << 24);
}

__device__ __forceinline__ bool vocab_epilogue_sync_or(bool pred) {
  uint32_t res;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbar.red.or.pred p, 1, %2, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(res)
      : "r"((uint32_t)pred), "n"(32 * kVocabEpilogueWarps)
      : "memory");
  return res != 0;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// e^d for a difference of logits.  The difference comes first and is scaled then: logits that are scaled before they are subtracted
// are rounded at their own size (at -5e9, a finite mask, by hundreds, so that e^0 became infinite or 0), and those below -2.4e38
// have no scaled value.
__device__ __forceinline__ float exp_fast(float d) { return exp2_fast(d * kLog2e); }
// What is subtracted for a maximum of `most`: itself, or, where that is infinite, the finite value next to it (no difference of
// infinities: -infinity alone sums to 0, a +infinity makes the sum infinite).  A NaN among the logits reaches the sum by its own term.
__device__ __forceinline__ float exp_base(float most) { return fminf(fmaxf(most, -FLT_MAX), FLT_MAX); }
// sum of e^(z - base), two values an instruction
__device__ __forceinline__ float exp_sum(const float (&z)[32], float base) {
  const uint64_t base2 = ptx::pack_f32x2(-base, -base), log2e2 = ptx::pack_f32x2(kLog2e, kLog2e);
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < 32; j += 2) {
    const float2 d = ptx::unpack_f32x2(ptx::mul_f32x2(ptx::add_f32x2(ptx::pack_f32x2(z[j], z[j + 1]), base2), log2e2));
    s[j & 3] += exp2_fast(d.x);
    s[(j & 3) + 1] += exp2_fast(d.y);
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// A pair's walk over its tiles, all kinds one after the other.
struct VocabCursor {
  int i, t, end;
  __device__ __forceinline__ bool first(const VocabParams& gp, int g) {
    i = -1;
    t = end = 0;
    return next(gp, g);
  }
  __device__ __forceinline__ bool next(const VocabParams& gp, int g) {
    if (i >= 0) ++t;
    while (t >= end) {
      if (++i >= gp.count) return false;
      t = gp.prob[i].start[g];
      end = gp.prob[i].start[g + 1];
    }
    return true;
  }
};
struct VocabTileAt {
  int m, n, split, k0, k1;  // row and column tile, split, range of K blocks
  __device__ __forceinline__ VocabTileAt(const VocabProblem& p, int t) {
    split = t / p.split_tiles;
    t -= split * p.split_tiles;
    if (p.m_tiles) {
      n = t / p.m_tiles;
      m = t - n * p.m_tiles;
    } else {
      m = t / p.n_tiles;
      n = t - m * p.n_tiles;
    }
    k0 = split * p.k_blocks;
    k1 = min(k0 + p.k_blocks, p.k_end);
  }
};

// FORWARD: logits tiles alone; else the three kinds of the backward pass.
template <bool FORWARD, bool FEW>
__global__ void __launch_bounds__(kVocabThreads, 1) vocab_kernel(const __grid_constant__ VocabParams gp) {
  constexpr int kStages = kVocabStages;
  const uint32_t rank = ptx::cluster_ctarank();
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t smem_base = ptx::smem_u32(smem);
  uint8_t* const out_ptr = smem + kStages * kVocabStageBytes;
  uint8_t* const bar_ptr = out_ptr + kVocabOutBytes;
  const uint32_t bar_base = ptx::smem_u32(bar_ptr);
  auto full = [&](int s) { return bar_base + 8u * s; };
  auto empty = [&](int s) { return bar_base + 8u * (kStages + s); };
  auto acc_full = [&](int a) { return bar_base + 8u * (2 * kStages + a); };
  auto acc_empty = [&](int a) { return bar_base + 8u * (2 * kStages + 2 + a); };
  const uint32_t drain_bar = bar_base + 8u * (2 * kStages + 4);
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bar_ptr + 8 * (2 * kStages + 5));
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* const cols = reinterpret_cast<float*>(bar_ptr + kVocabBarBytes);  // [2][3][256]
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
      ptx::mbar_init(acc_empty(a), kVocabEpilogueWarps * 2);
    }
    ptx::mbar_init(drain_bar, 1);
    *abort_flag = 0;
    ptx::fence_mbar_init();
  }
  if (warp == 1) {
    ptx::tmem_alloc_cg<2>(ptx::smem_u32(tmem_slot), 2 * kVocabTile);
    ptx::tmem_relinquish_cg<2>();
  }
  ptx::tcgen05_fence_before_sync();
  __syncthreads();
  ptx::cluster_sync_all();
  ptx::tcgen05_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  pdl_begin();
  auto lead = [&](uint32_t bar) { return ptx::map_to_cta(bar, 0); };
  const int g = (int)blockIdx.x / 2;
  bool timed_out = false;
  int where = 0;

  if (warp == 0) {
    // ---------------- TMA producer ------------------------------------------------------------------
    if (ptx::elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      VocabCursor c;
      for (bool have = c.first(gp, g); have && !timed_out; have = c.next(gp, g)) {
        const VocabProblem& pr = gp.prob[c.i];
        const VocabTileAt at(pr, c.t);
        const int width = FEW ? pr.width : kVocabTile;
        const int a_row = at.m * kVocabTile + (int)rank * 128, b_row = at.n * kVocabTile + (int)rank * (width / 2);
        const uint32_t bytes = kVocabStageBytes + 2 * (width * 128);
        const CUtensorMap* const ma = &gp.map[pr.map_a];
        const CUtensorMap* const mb = &gp.map[pr.map_b];
        for (int kb = at.k0; kb < at.k1; kb += 2) {
          if (!wait_barrier_relaxed(empty(stage), phase ^ 1u, abort_flag)) {
            timed_out = true;
            where = (0 << 16) | stage;
            break;
          }
          const uint32_t a_smem = smem_base + stage * kVocabStageBytes, b_smem = a_smem + kVocabStageBytes / 2, bar = lead(full(stage));
          if (rank == 0) ptx::mbar_arrive_expect_tx(full(stage), bytes);
          auto load = [&](uint32_t dst, const CUtensorMap* tm, int form, int mn, int row0, int rows) {
            if (form == kRows) {
              ptx::tma_load_3d_pair(dst, tm, bar, 0, row0 + mn, kb);
            } else if (form == kCols) {
              ptx::tma_load_3d_pair(dst, tm, bar, 0, row0 + kb * 64, mn / 64);
            } else if (form == kRows2) {
              ptx::tma_load_2d_pair(dst, tm, bar, kb * 64, row0 + mn);
              ptx::tma_load_2d_pair(dst + rows * 128, tm, bar, kb * 64 + 64, row0 + mn);
            } else {
              ptx::tma_load_2d_pair(dst, tm, bar, mn, row0 + kb * 64);
              ptx::tma_load_2d_pair(dst + 16384, tm, bar, mn + 64, row0 + kb * 64);
            }
          };
          load(a_smem, ma, pr.a_form, a_row, pr.a_row0, 128);
          load(b_smem, mb, pr.b_form, b_row, pr.b_row0, width / 2);
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
    // ---------------- MMA issuer (in the pair's first CTA only) ---------------------------------------
    if (rank == 0 && ptx::elect_one()) {
      int stage = 0, it = 0;
      uint32_t phase = 0;
      VocabCursor c;
      for (bool have = c.first(gp, g); have && !timed_out; have = c.next(gp, g), ++it) {
        const VocabProblem& pr = gp.prob[c.i];
        const VocabTileAt at(pr, c.t);
        const int a = it & 1;
        const uint32_t d = tmem_base + (uint32_t)(a * kVocabTile);
        const int width = FEW ? pr.width : kVocabTile;
        const bool a_mn = pr.a_form >= kCols, b_mn = pr.b_form >= kCols;
        const uint32_t idesc = vocab_idesc(a_mn, b_mn, width);
        const uint64_t a_desc0 = vocab_desc(smem_base, a_mn), b_desc0 = vocab_desc(smem_base + kVocabStageBytes / 2, b_mn);
        // 16 elements of K per instruction: 32 bytes of a row, or 16 rows of 128 bytes
        const uint32_t a_step = a_mn ? 2048 >> 4 : 32 >> 4, b_step = b_mn ? 2048 >> 4 : 32 >> 4;
        const uint32_t a_next = a_mn ? 8192 >> 4 : 16384 >> 4, b_next = b_mn ? 8192 >> 4 : (uint32_t)(width / 2 * 128) >> 4;  // second K block
        if (!wait_barrier(acc_empty(a), ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_flag)) {
          timed_out = true;
          where = (1 << 16) | 0x100 | a;
          break;
        }
        for (int kb = at.k0; kb < at.k1; kb += 2) {
          if (!wait_barrier(full(stage), phase, abort_flag)) {
            timed_out = true;
            where = (1 << 16) | stage;
            break;
          }
          ptx::tcgen05_fence_after_sync();
          const uint64_t a_desc = a_desc0 + (uint64_t)(stage * (kVocabStageBytes >> 4));
          const uint64_t b_desc = b_desc0 + (uint64_t)(stage * (kVocabStageBytes >> 4));
#pragma unroll
          for (int j = 0; j < 4; ++j)
            ptx::mma_f16_ss_pair(d, a_desc + (uint64_t)(a_step * j), b_desc + (uint64_t)(b_step * j), idesc, kb != at.k0 || j != 0 ? 1u : 0u);
          if (kb + 1 < at.k1) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              ptx::mma_f16_ss_pair(d, a_desc + (uint64_t)(a_next + a_step * j), b_desc + (uint64_t)(b_next + b_step * j), idesc, 1u);
          }
          ptx::mma_commit_cg<2>(empty(stage));
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
        if (!timed_out) ptx::mma_commit_cg<2>(acc_full(a));
      }
      if (timed_out) {  // wait (bounded) for what was issued before tensor memory is freed
        ptx::mma_commit_cg<2>(drain_bar);
        const long long t0 = clock64();
        while (!ptx::mbar_try_wait(drain_bar, 0) && clock64() - t0 < 400000000ll) {
        }
      }
    }
  } else if (warp >= 4) {
    // ---------------- epilogue ----------------------------------------------------------------------
    const int ew = warp - 4, quarter = warp & 3, half = ew >> 2, e = threadIdx.x - 128;
    uint8_t* const buf = out_ptr + ew * 2048;
    const uint32_t lanes = tmem_base + ((uint32_t)(quarter * 32) << 16);
    int it = 0;
    VocabCursor c;
    for (bool have = c.first(gp, g); have; have = c.next(gp, g), ++it) {
      const VocabProblem& pr = gp.prob[c.i];
      const VocabTileAt at(pr, c.t);
      const int a = it & 1;
      const int row0 = at.m * kVocabTile + (int)rank * 128 + quarter * 32, row = row0 + lane;
      const int col0 = at.n * kVocabTile;
      float* const tile_cols = cols + a * 768;
      // what the tile's columns need: words' biases (forward), or the tokens' lse, gradient and target
      if (FORWARD && !FEW) {
        const int v = col0 + e;
        tile_cols[e] = v >= gp.V ? -INFINITY : (gp.bias ? gp.bias[v] : 0.0f);
      } else if (!FORWARD && pr.kind == kGradZ) {
        const int t = col0 + e;
        float lse = INFINITY, gl = 0.0f;
        int target = -1;
        if (t < gp.T) {  // three loads at once: the gradient's does not wait for the target
          lse = gp.lse[t];
          target = gp.targets[t];
          gl = gp.grad_loss[t];
          if (target < 0 || target >= gp.V) {
            gl = 0.0f;
            lse = INFINITY;  // its probabilities are 0 whatever the caller's lse holds
          } else if (lse == INFINITY) {
            lse = NAN;  // a softmax over an infinite logit has no value
          }
        }
        tile_cols[e] = -lse;
        tile_cols[256 + e] = gl;
        reinterpret_cast<int*>(tile_cols)[512 + e] = target;
      }
      // the row's own, fetched while the products run
      int target = -1;
      float bias = 0.0f;
      if (FORWARD && !FEW) {
        if (row < gp.T) target = gp.targets[row];
      } else if (FORWARD || pr.kind == kGradZ) {
        const int v = gp.v0 + row;
        bias = v >= gp.V ? -INFINITY : (gp.bias ? gp.bias[v] : 0.0f);
      }
      const bool ok = ew != 0 || wait_barrier_warp(acc_full(a), (uint32_t)(it >> 1) & 1u, abort_flag);
      if (vocab_epilogue_sync_or(!ok)) {  // publishes the columns' values, and all eight warps give up together
        timed_out = true;
        where = (3 << 16) | a;
        break;
      }
      ptx::tcgen05_fence_after_sync();
      const uint32_t acc = lanes + (uint32_t)(a * kVocabTile);
      auto release = [&]() {  // the warp has read all it needs from the accumulator
        ptx::tcgen05_fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          if (rank != 0) ptx::mbar_arrive_remote(lead(acc_empty(a)));
          else ptx::mbar_arrive(acc_empty(a));
        }
      };
      // A line (128 bytes) of every lane's row through the warp's staging buffer, 16 rows at a time, and out of it as whole lines, 16
      // bytes a lane and four rows a store.  The swizzle keeps eight lanes on different banks either way.
      auto staged = [&](int r, int piece) { return reinterpret_cast<uint4*>(buf + r * 128 + ((piece ^ (r & 7)) << 4)); };
      auto send = [&](const uint4 (&w)[8], uint8_t* to, size_t pitch, int rows, int bytes, bool add) {  // rows, bytes of a row that exist
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          __syncwarp();
          if ((lane >> 4) == h) {
#pragma unroll
            for (int j = 0; j < 8; ++j) *staged(lane & 15, j) = w[j];
          }
          __syncwarp();
          const int piece = lane & 7;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = 4 * i + (lane >> 3);
            const uint4 v = *staged(r, piece);
            if (16 * h + r < rows && piece * 16 < bytes) {
              uint8_t* const p = to + (size_t)(16 * h + r) * pitch + piece * 16;
              if (add) ptx::red_add_v4(p, v);
              else *reinterpret_cast<uint4*>(p) = v;
            }
          }
        }
      };

      if constexpr (FORWARD && !FEW) {
        const int chunks = row0 < gp.T ? min(8, (gp.V - col0 + 31) / 32) : 0;
        if (half >= chunks) release();
        float top = -INFINITY, sum = 0.0f;
#pragma unroll 1
        for (int ch = half; ch < chunks; ch += 2) {
          uint32_t v[32];
          ptx::tmem_ld_32x32b_x32(acc + (uint32_t)(ch * 32), v);
          ptx::tmem_ld_wait();
          ptx::tmem_ld_regs_ready(v);
          if (ch + 2 >= chunks) release();
          const int hit = target - (col0 + ch * 32), words = gp.V - (col0 + ch * 32);
          if (words < 32) {  // what lies behind the last word is an infinite h times 0, NaN, which no bias takes out
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (j >= words) v[j] = 0u;
          }
          if (hit >= 0 && hit < 32 && target < gp.V) {
            float z = 0.0f;
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (j == hit) z = __uint_as_float(v[j]);
            if (row < gp.T) gp.z_target[row] = gp.bias ? z + gp.bias[target] : z;
          }
          float z[32], most = top;
          const float4* const b4 = reinterpret_cast<const float4*>(tile_cols + ch * 32);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float4 b = b4[j];
            const float2 lo = ptx::unpack_f32x2(ptx::add_f32x2(ptx::pack_u32x2(v[4 * j], v[4 * j + 1]), ptx::pack_f32x2(b.x, b.y)));
            const float2 hi = ptx::unpack_f32x2(ptx::add_f32x2(ptx::pack_u32x2(v[4 * j + 2], v[4 * j + 3]), ptx::pack_f32x2(b.z, b.w)));
            z[4 * j] = lo.x;
            z[4 * j + 1] = lo.y;
            z[4 * j + 2] = hi.x;
            z[4 * j + 3] = hi.y;
            most = fmaxf(most, fmaxf(fmaxf(z[4 * j], z[4 * j + 1]), fmaxf(z[4 * j + 2], z[4 * j + 3])));
          }
          const float base = exp_base(most);
          sum = sum * exp_fast(top - base) + exp_sum(z, base);
          top = most;
        }
        if (row < gp.T) gp.part[(size_t)(2 * at.n + half) * gp.T + row] = make_float2(top, sum);
      } else if constexpr (FORWARD) {
        // lane: word, column: token.  A warp's 32 words of 32 tokens at a time are turned in the staging buffer (lane l's column j
        // goes to row j, place l), so that a lane has a token's 32 logits
        const int chunks = (gp.T + 31) / 32;
        float2* const joined = reinterpret_cast<float2*>(cols);  // [quarter][token]
        if (half >= chunks) release();
#pragma unroll 1
        for (int ch = half; ch < chunks; ch += 2) {
          uint32_t v[32];
          ptx::tmem_ld_32x32b_x32(acc + (uint32_t)(ch * 32), v);
          ptx::tmem_ld_wait();
          ptx::tmem_ld_regs_ready(v);
          if (ch + 2 >= chunks) release();
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = __float_as_uint((row < gp.V ? __uint_as_float(v[j]) : 0.0f) + bias);  // (as above)
          const int t = ch * 32 + lane;
          const int target = t < gp.T ? gp.targets[t] : -1, hit = target - row0;
          float z[32];
#pragma unroll
          for (int h = 0; h < 2; ++h) {  // 16 tokens at a time: rows of 128 bytes
#pragma unroll
            for (int j = 0; j < 16; ++j)
              *reinterpret_cast<uint32_t*>(buf + j * 128 + (((lane >> 2) ^ (j & 7)) << 4) + (lane & 3) * 4) = v[16 * h + j];
            __syncwarp();
            if ((lane >> 4) == h) {
              const uint8_t* const from = buf + (lane & 15) * 128;
#pragma unroll
              for (int j = 0; j < 8; ++j) *reinterpret_cast<uint4*>(&z[4 * j]) = *reinterpret_cast<const uint4*>(from + ((j ^ (lane & 7)) << 4));
              if (hit >= 0 && hit < 32 && target < gp.V)
                gp.z_target[t] = *reinterpret_cast<const float*>(from + (((hit >> 2) ^ (lane & 7)) << 4) + (hit & 3) * 4);
            }
            __syncwarp();
          }
          float most = fmaxf(z[0], z[1]);
#pragma unroll
          for (int j = 2; j < 32; j += 2) most = fmaxf(most, fmaxf(z[j], z[j + 1]));
          joined[quarter * kFewTokens + ch * 32 + lane] = make_float2(most, exp_sum(z, exp_base(most)));
          __syncwarp();
        }
        // the CTA's four quarters of words, joined in order (the next tile's barrier comes before the next writes)
        vocab_epilogue_sync_or(false);
        if (e < gp.T) {
          float2 q[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) q[i] = joined[i * kFewTokens + e];
          const float top = fmaxf(fmaxf(q[0].x, q[1].x), fmaxf(q[2].x, q[3].x)), base = exp_base(top);
          float s = 0.0f;
#pragma unroll
          for (int i = 0; i < 4; ++i) s += q[i].y * exp_fast(q[i].x - base);
          gp.part[(size_t)(2 * at.m + rank) * gp.T + e] = make_float2(top, s);
        }
      } else if (pr.kind == kGradH) {
        const int chunks = row0 < gp.T ? min(8, (gp.D - col0 + 31) / 32) : 0;
        if (half >= chunks) release();
#pragma unroll 1
        for (int ch = half; ch < chunks; ch += 2) {
          uint32_t v[32];
          ptx::tmem_ld_32x32b_x32(acc + (uint32_t)(ch * 32), v);
          ptx::tmem_ld_wait();
          ptx::tmem_ld_regs_ready(v);
          if (ch + 2 >= chunks) release();
          const int c0 = col0 + ch * 32;
          uint8_t* const to = reinterpret_cast<uint8_t*>(gp.slabs + ((size_t)at.split * gp.T + row0) * gp.D + c0);
          uint4 w[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
          send(w, to, (size_t)gp.D * 4, gp.T - row0, (gp.D - c0) * 4, gp.add != 0);
        }
      } else {
        const bool grad_z = pr.kind == kGradZ;
        // (FEW: the tile covers all of g's row, zeros behind its columns)
        const int rows = gp.V - gp.out_v0, width = grad_z ? (FEW ? gp.g_pitch : gp.T) : gp.D;
        // g is formed for all rows of the piece's tiles: the products read whole K blocks of it
        const int chunks = grad_z || row0 < rows ? min(4, (width - col0 + 63) / 64) : 0;
        if (half >= chunks) release();
        uint64_t bias_grad[2] = {0, 0};
        const uint64_t bias2 = ptx::pack_f32x2(bias, bias), log2e2 = ptx::pack_f32x2(kLog2e, kLog2e);
        const int word = gp.v0 + row;
#pragma unroll 1
        for (int ch = half; ch < chunks; ch += 2) {
          uint32_t v[2][32];
          ptx::tmem_ld_32x32b_x32(acc + (uint32_t)(ch * 64), v[0]);
          ptx::tmem_ld_32x32b_x32(acc + (uint32_t)(ch * 64 + 32), v[1]);
          ptx::tmem_ld_wait();
          ptx::tmem_ld_regs_ready(v[0]);
          ptx::tmem_ld_regs_ready(v[1]);
          if (ch + 2 >= chunks) release();
          if (grad_z) {
            const ulonglong2* const lse2 = reinterpret_cast<const ulonglong2*>(tile_cols + ch * 64);  // two columns a word
            const ulonglong2* const gl2 = reinterpret_cast<const ulonglong2*>(tile_cols + 256 + ch * 64);
            const int* const tg = reinterpret_cast<const int*>(tile_cols + 512 + ch * 64);
            const int tokens = gp.T - (col0 + ch * 64);
            if (tokens < 64) {  // behind the last token: an infinite w times 0, NaN, or (FEW) what an earlier tile left
#pragma unroll
              for (int j = 0; j < 64; ++j)
                if (j >= tokens) v[j >> 5][j & 31] = 0u;
            }
            // Two columns an instruction.  A target among the warp's 32 words is rare, so that the comparisons are made where there is
            // one (both: 4,096 x 30,522 x 768 backward 447 -> 437 us).
            // z is rounded as in the forward pass, and lse is no less than the largest z: a probability is never above 1, and
            // p - 1 never has the wrong sign (the scaled form that rounds at lse's size: 441 us, so 446).
            const auto two = [&](uint32_t* x, uint64_t lse, uint64_t w, int k, auto hits, int j) {
              float2 p = ptx::unpack_f32x2(ptx::mul_f32x2(ptx::add_f32x2(ptx::add_f32x2(ptx::pack_u32x2(x[0], x[1]), bias2), lse), log2e2));
              p.x = exp2_fast(p.x);
              p.y = exp2_fast(p.y);
              uint64_t d;
              if constexpr (decltype(hits)::value) {
                const float2 g = ptx::unpack_f32x2(w);
                d = ptx::pack_f32x2(g.x * p.x - (tg[j] == word ? g.x : 0.0f), g.y * p.y - (tg[j + 1] == word ? g.y : 0.0f));
              } else {
                d = ptx::mul_f32x2(w, ptx::pack_f32x2(p.x, p.y));
              }
              bias_grad[k] = ptx::add_f32x2(bias_grad[k], d);
              const float2 f = ptx::unpack_f32x2(d);
              x[0] = __float_as_uint(f.x);
              x[1] = __float_as_uint(f.y);
            };
            const auto all = [&](auto hits) {
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                const ulonglong2 l = lse2[j], g = gl2[j];
                uint32_t* const x = &v[j >> 3][(j & 7) * 4];
                two(x, l.x, g.x, 0, hits, 4 * j);
                two(x + 2, l.y, g.y, 1, hits, 4 * j + 2);
              }
            };
            const uint32_t first = (uint32_t)(gp.v0 + row0);
            if (__any_sync(0xffffffffu, (uint32_t)tg[lane] - first < 32u || (uint32_t)tg[lane + 32] - first < 32u)) all(std::true_type());
            else all(std::false_type());
          }
          const int c0 = col0 + ch * 64;
          uint4 w[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const auto f = [&](int i) { return __uint_as_float(v[j >> 2][8 * (j & 3) + i]); };
            w[j] = make_uint4(pack_bf16(f(0), f(1)), pack_bf16(f(2), f(3)), pack_bf16(f(4), f(5)), pack_bf16(f(6), f(7)));
          }
          if (grad_z)  // whole K blocks: the rows and columns behind the last word and token too
            send(w, reinterpret_cast<uint8_t*>(gp.g_new + (size_t)row0 * gp.g_pitch + c0), (size_t)gp.g_pitch * 2, 32, 128, false);
          else
            send(w, reinterpret_cast<uint8_t*>(gp.grad_w + (size_t)(gp.out_v0 + row0) * gp.D + c0), (size_t)gp.D * 2, rows - row0, (gp.D - c0) * 2, false);
        }
        if (grad_z && gp.part_bias && word < gp.V) {
          const float2 b0 = ptx::unpack_f32x2(bias_grad[0]), b1 = ptx::unpack_f32x2(bias_grad[1]);
          gp.part_bias[(size_t)(2 * at.n + half) * gp.V + word] = (b0.x + b0.y) + (b1.x + b1.y);
        }
      }
    }
  }
  if (timed_out) {
    *abort_flag = 1;
    report_status(gp.ws, QB_ERR_TIMEOUT, where);
  }
  ptx::tcgen05_fence_before_sync();
  __syncthreads();
  ptx::cluster_sync_all();  // the other CTA's MMAs and arrivals reach into this CTA
  if (warp == 1) {
    __syncwarp();
    ptx::tcgen05_fence_after_sync();
    ptx::tmem_dealloc_cg<2>(tmem_base, 2 * kVocabTile);
  }
}

// Joins the tiles' maxima and sums of 32 tokens per block: every warp a share of the tiles, the maximum first (the loads of
// kJoinDepth tiles in flight), then the warps in order.
constexpr int kJoinWarps = 16, kJoinDepth = 8;
__global__ void __launch_bounds__(32 * kJoinWarps) vocab_join_kernel(const float2* part, int parts, const float* z_target, const int32_t* targets,
                                                                     int T, int V, float* loss, float* lse, void* ws) {
  __shared__ float2 joined[kJoinWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = blockIdx.x * 32 + lane;
  pdl_begin();
  float top = -INFINITY, sum = 0.0f;
  for (int i0 = warp; i0 < parts; i0 += kJoinWarps * kJoinDepth) {
    float2 p[kJoinDepth];
#pragma unroll
    for (int d = 0; d < kJoinDepth; ++d) {
      const int i = i0 + d * kJoinWarps;
      p[d] = make_float2(-INFINITY, 0.0f);
      if (i < parts && t < T) p[d] = part[(size_t)i * T + t];
    }
    float most = top;
#pragma unroll
    for (int d = 0; d < kJoinDepth; ++d) most = fmaxf(most, p[d].x);
    const float base = exp_base(most);
    sum *= exp_fast(top - base);
#pragma unroll
    for (int d = 0; d < kJoinDepth; ++d) sum += p[d].y * exp_fast(p[d].x - base);
    top = most;
  }
  joined[warp][lane] = make_float2(top, sum);
  __syncthreads();
  if (warp != 0 || t >= T) return;
  float most = -INFINITY;
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) most = fmaxf(most, joined[w][lane].x);
  const float base = exp_base(most);
  sum = 0.0f;
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) sum += joined[w][lane].y * exp_fast(joined[w][lane].x - base);
  const float log_sum = logf(sum);  // sum >= 1: the maximum's own term
  const int target = targets[t];
  lse[t] = most + log_sum;
  const bool valid = target >= 0 && target < V;
  if (target >= V) report_status(ws, QB_ERR_INVALID, t);
  // the difference of two logits first: lse - z would leave the rounding of lse, of either sign, of a loss near 0
  loss[t] = valid ? (most - z_target[t]) + log_sum : 0.0f;
}

// grad_h = the slabs' sum in bfloat16 (the first `h_blocks` blocks); grad_bias = the tiles' sum (the others).
// A block has 32 groups of four elements times eight warps; with more than four slabs every warp sums every eighth, and the warps'
// sums are joined in order, else every warp takes groups of its own.
__global__ void __launch_bounds__(256) vocab_finish_kernel(const float* slabs, int splits, int64_t n, uint16_t* grad_h, int h_blocks,
                                                           const float* part_bias, int parts, int V, float* grad_bias) {
  __shared__ float4 joined[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_begin();
  if ((int)blockIdx.x >= h_blocks) {
    const int v = ((int)blockIdx.x - h_blocks) * 256 + threadIdx.x;
    if (v >= V) return;
    float s = 0.0f;
#pragma unroll 8
    for (int i = 0; i < parts; ++i) s += part_bias[(size_t)i * V + v];
    grad_bias[v] = s;
    return;
  }
  const bool shared = splits > 4;
  const int64_t i = ((int64_t)blockIdx.x * (shared ? 32 : 256) + (shared ? lane : threadIdx.x)) * 4;  // n is a multiple of 8
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  if (i < n) {
#pragma unroll 8
    for (int s = shared ? warp : 0; s < splits; s += shared ? 8 : 1) {
      const float4 c = *reinterpret_cast<const float4*>(slabs + s * n + i);
      a.x += c.x;
      a.y += c.y;
      a.z += c.z;
      a.w += c.w;
    }
  }
  if (shared) {
    joined[warp][lane] = a;
    __syncthreads();
    if (warp != 0) return;
#pragma unroll
    for (int w = 1; w < 8; ++w) {
      const float4 c = joined[w][lane];
      a.x += c.x;
      a.y += c.y;
      a.z += c.z;
      a.w += c.w;
    }
  }
  if (i < n) *reinterpret_cast<uint2*>(grad_h + i) = make_uint2(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w));
}

// ---- host side -----------------------------------------------------------------------------------
static int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m; }

// How the backward pass cuts its work.
struct VocabPlan {
  int64_t rows;      // words per piece, a multiple of 256
  int64_t pieces;
  int64_t k_split;   // K blocks of a split of grad_h
  int64_t splits;
  int64_t g_bytes, slab_bytes, bias_bytes;
  size_t bytes() const { return (size_t)(1024 + (pieces > 1 ? 2 : 1) * g_bytes + splits * slab_bytes + bias_bytes); }
};
constexpr int64_t kPieceBytes = 48 << 20;  // of g: a launch has enough tiles to level them, and L2 still holds most of what is read again

// Cost of a tile in K blocks: it takes at least as long as its epilogue, about ten (with the K blocks alone 5 tokens x 47,258 x 960
// backward took 91 us, so 83; 300 tokens x 30,522 x 768 74 and 71).
static int64_t vocab_tile_cost(int64_t k_blocks) { return std::max<int64_t>(k_blocks, 10) + 2; }

// Columns of a tile of logits in the backward pass (few tokens: in the forward pass too).
static int64_t vocab_width(int64_t T) { return T <= kFewTokens ? up(T, 32) * 32 : kVocabTile; }

static VocabPlan plan_vocab(int64_t T, int64_t V, int64_t D, int pairs, size_t budget) {
  VocabPlan p;
  const int64_t Tp = up(T, 64) * 64, t_tiles = up(T, 256), d_tiles = up(D, 256), all = up(V, 256) * 256;
  p.slab_bytes = T * D * 4;  // (D is a multiple of 8: slabs begin at multiples of 32 bytes)
  p.bias_bytes = up(2 * t_tiles * V * 4, 1024) * 1024;
  int64_t rows = std::min(all, std::max<int64_t>(256, kPieceBytes / (2 * Tp) / 256 * 256));
  for (;; rows -= 256) {
    p.pieces = up(all, rows);
    p.rows = up(up(V, p.pieces), 256) * 256;
    p.pieces = up(V, p.rows);
    p.g_bytes = up(p.rows * Tp * 2, 1024) * 1024;
    // grad_h's contraction over the piece is split where a tile of it would outlast the launch
    // (blocks of the first piece, whose splits are what is stored and summed; no piece has more)
    const int64_t blocks = up(std::min(p.rows, V), 64), v_tiles = p.rows / 256;
    const int64_t work = t_tiles * d_tiles * blocks + v_tiles * d_tiles * vocab_tile_cost(Tp / 64) +
                         (p.pieces > 1 ? v_tiles * t_tiles * vocab_tile_cost(up(D, 64)) : 0);
    p.k_split = std::min(blocks, std::max<int64_t>(16, work / pairs / 2));
    p.splits = up(blocks, p.k_split);
    p.k_split = up(up(blocks, p.splits), 2) * 2;
    p.splits = up(blocks, p.k_split);
    if (p.bytes() <= budget || rows <= 256) return p;
  }
}

// Deals `tiles` tiles of `cost` over the pairs: each to the least loaded one, as level as they come; contiguous tiles per pair.
static void deal_tiles(VocabProblem& p, int64_t tiles, int64_t cost, int64_t* load, int pairs) {
  int64_t least = load[0], most = load[0];
  for (int g = 1; g < pairs; ++g) {
    least = std::min(least, load[g]);
    most = std::max(most, load[g]);
  }
  if (least == most) {  // nothing dealt yet
    const int64_t each = tiles / pairs, more = tiles - each * pairs;
    for (int g = 0; g <= pairs; ++g) p.start[g] = (int32_t)(g * each + std::min<int64_t>(g, more));
    for (int g = 0; g < pairs; ++g) load[g] += (each + (g < more)) * cost;
    return;
  }
  // The least level at which they all fit, by bisection; the loads above the least one and the costs fit 32 bits, or are taken
  // in units in which they do (host time: 740 divisions of 64 bits took 6 us).
  int64_t unit = 1;
  while ((most - least + cost * (up(tiles, pairs) + 1)) / unit >= (int64_t)1 << 30) unit *= 2;
  const uint32_t c = (uint32_t)std::max<int64_t>(1, cost / unit);
  uint32_t l[kMaxPairs];
  for (int g = 0; g < pairs; ++g) l[g] = (uint32_t)((load[g] - least) / unit);
  uint32_t lo = 0, hi = (uint32_t)((most - least) / unit) + c * (uint32_t)(up(tiles, pairs) + 1);
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2;
    int64_t room = 0;
    for (int g = 0; g < pairs; ++g) room += mid > l[g] ? (mid - l[g]) / c : 0;
    if (room >= tiles) hi = mid;
    else lo = mid + 1;
  }
  int64_t t = 0;
  for (int g = 0; g < pairs; ++g) {
    const int64_t n = std::min<int64_t>(tiles - t, lo > l[g] ? (lo - l[g]) / c : 0);
    p.start[g] = (int32_t)t;
    t += n;
    load[g] += n * cost;
  }
  p.start[pairs] = (int32_t)t;
}

template <bool FORWARD, bool FEW>
static qb_status launch_vocab(const VocabParams& gp, int pairs, cudaStream_t stream) {
  auto kernel = vocab_kernel<FORWARD, FEW>;
  static std::atomic<bool> attr_set[64] = {};
  int dev = 0;
  QB_CUDA_TRY(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
    QB_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kVocabSmemBytes));
    if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
  }
  QB_CUDA_TRY(launch_kernel(kernel, (unsigned)(2 * pairs), kVocabThreads, kVocabSmemBytes, stream, 2, false, gp));
  return QB_OK;
}

// The operand with its rows along M or N, and with its columns along them.
static int32_t rows_form(int64_t cols) { return cols % 64 == 0 ? kRows : kRows2; }
static int32_t cols_form(int64_t cols) { return cols % 64 == 0 ? kCols : kCols2; }
static qb_status operand_map(CUtensorMap* tm, const void* base, int64_t rows, int64_t cols, int64_t box_rows = 128) {
  if (cols % 64 == 0) return make_group_map(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, rows, cols * 2, (int)box_rows, 2);
  return make_matrix_map(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, base, rows, cols, cols * 2, (int)box_rows, 64, CU_TENSOR_MAP_SWIZZLE_128B);
}

static qb_status validate_vocab(const char* who, bool null, const void* h, const void* w, int64_t T, int64_t V, int64_t D) {
  if (null || T <= 0 || V <= 0 || D <= 0 || T > QB_MAX_MN || V > QB_MAX_MN || D > QB_MAX_VOCAB_D || up(T, 256) * up(V, 256) > 1 << 30) {
    set_last_error("%s: null pointer or size out of range (T=%lld V=%lld D=%lld)", who, (long long)T, (long long)V, (long long)D);
    return QB_ERR_INVALID;
  }
  if (D % 8 != 0 || !aligned16(h) || !aligned16(w)) {
    set_last_error("%s: D must be a multiple of 8, matrices 16-byte aligned", who);
    return QB_ERR_ALIGN;
  }
  return QB_OK;
}
static bool aligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

static size_t vocab_forward_bytes(int64_t T, int64_t V) { return (size_t)(1024 + up(T * 4, 1024) * 1024 + 2 * up(V, 256) * T * 8); }

}  // namespace qb

extern "C" size_t qb_vocab_loss_workspace_bytes(int64_t T, int64_t V, int64_t D) {
  using namespace qb;
  if (T <= 0 || V <= 0 || D <= 0 || T > QB_MAX_MN || V > QB_MAX_MN || D > QB_MAX_VOCAB_D) return 0;
  int sms = 148;
  require_sm100(&sms);  // without a device: for a 148-SM part
  const size_t back = plan_vocab(T, V, D, std::min(sms / 2, kMaxPairs), ~(size_t)0).bytes();
  return up(std::max(back, vocab_forward_bytes(T, V)), 256) * 256;
}

extern "C" qb_status qb_vocab_loss(const uint16_t* h, const uint16_t* w, const float* bias, const int32_t* targets, int64_t T, int64_t V,
                                   int64_t D, float* loss, float* lse, void* ws, size_t ws_bytes, void* cuda_stream) {
  using namespace qb;
  qb_status st = validate_vocab("qb_vocab_loss", !h || !w || !targets || !loss || !lse, h, w, T, V, D);
  if (st != QB_OK) return st;
  if (!aligned4(bias) || !aligned4(targets) || !aligned4(loss) || !aligned4(lse)) {
    set_last_error("qb_vocab_loss: bias, targets, loss and lse must be 4-byte aligned");
    return QB_ERR_ALIGN;
  }
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 != 0 || ws_bytes < vocab_forward_bytes(T, V)) {
    set_last_error("qb_vocab_loss: workspace null, not 256-byte aligned or smaller than %zu bytes", vocab_forward_bytes(T, V));
    return QB_ERR_WORKSPACE;
  }
  int sms = 0;
  st = require_sm100(&sms);
  if (st != QB_OK) return st;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  // all tokens of a tile of words one after the other: w is read once, h stays in L2
  const bool few = T <= kFewTokens;
  const int64_t width = vocab_width(T), tiles = up(V, 256) * up(T, 256);
  VocabParams gp = {};
  if ((st = operand_map(&gp.map[kMapHTile], h, T, D, few ? width / 2 : 128)) != QB_OK) return st;
  if ((st = operand_map(&gp.map[kMapW], w, V, D)) != QB_OK) return st;
  char* const scratch = static_cast<char*>(ws) + 1024;
  gp.z_target = reinterpret_cast<float*>(scratch);
  gp.part = reinterpret_cast<float2*>(scratch + up(T * 4, 1024) * 1024);
  gp.T = (int32_t)T;
  gp.V = (int32_t)V;
  gp.D = (int32_t)D;
  gp.bias = bias;
  gp.targets = targets;
  gp.ws = ws;
  gp.count = 1;
  VocabProblem& p = gp.prob[0];
  p.kind = kLogits;
  p.map_a = few ? kMapW : kMapHTile;
  p.map_b = few ? kMapHTile : kMapW;
  p.a_form = p.b_form = rows_form(D);
  p.n_tiles = 1;
  p.m_tiles = few ? 0 : (int32_t)up(T, 256);
  p.width = (int32_t)width;
  p.split_tiles = (int32_t)tiles;
  p.k_blocks = p.k_end = (int32_t)up(D, 64);
  const int pairs = (int)std::min<int64_t>(tiles, std::min(sms / 2, kMaxPairs));
  int64_t load[kMaxPairs] = {};
  deal_tiles(p, tiles, 1, load, pairs);
  if ((st = few ? launch_vocab<true, true>(gp, pairs, stream) : launch_vocab<true, false>(gp, pairs, stream)) != QB_OK) return st;
  QB_CUDA_TRY(launch_kernel(vocab_join_kernel, (unsigned)up(T, 32), 32 * kJoinWarps, 0, stream, 1, false, gp.part, (int)(2 * up(V, 256)), gp.z_target, targets,
                            (int)T, (int)V, loss, lse, ws));
  return QB_OK;
}

extern "C" qb_status qb_vocab_loss_backward(const uint16_t* h, const uint16_t* w, const float* bias, const int32_t* targets,
                                            const float* lse, const float* grad_loss, int64_t T, int64_t V, int64_t D, uint16_t* grad_h,
                                            uint16_t* grad_w, float* grad_bias, void* ws, size_t ws_bytes, void* cuda_stream) {
  using namespace qb;
  qb_status st = validate_vocab("qb_vocab_loss_backward", !h || !w || !targets || !lse || !grad_loss || (!grad_h && !grad_w && !grad_bias), h, w,
                                T, V, D);
  if (st != QB_OK) return st;
  if (!aligned4(bias) || !aligned4(targets) || !aligned4(lse) || !aligned4(grad_loss) || !aligned4(grad_bias) || !aligned16(grad_h) ||
      !aligned16(grad_w)) {
    set_last_error("qb_vocab_loss_backward: vectors must be 4-byte, matrices 16-byte aligned");
    return QB_ERR_ALIGN;
  }
  int sms = 148;
  const qb_status device = require_sm100(&sms);
  const int pairs = std::min(sms / 2, kMaxPairs);
  const VocabPlan plan = plan_vocab(T, V, D, pairs, ws_bytes);
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 != 0 || ws_bytes < plan.bytes()) {
    set_last_error("qb_vocab_loss_backward: workspace null, not 256-byte aligned or smaller than %zu bytes", plan.bytes());
    return QB_ERR_WORKSPACE;
  }
  if (device != QB_OK) return device;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  char* const g0 = static_cast<char*>(ws) + 1024;
  char* const g1 = plan.pieces > 1 ? g0 + plan.g_bytes : g0;
  float* const slabs = reinterpret_cast<float*>(g1 + plan.g_bytes);
  float* const part_bias = reinterpret_cast<float*>(reinterpret_cast<char*>(slabs) + plan.splits * plan.slab_bytes);
  const int64_t Tp = up(T, 64) * 64;
  VocabParams gp = {};
  CUtensorMap g_map[2];
  uint16_t* const g[2] = {reinterpret_cast<uint16_t*>(g0), reinterpret_cast<uint16_t*>(g1)};
  const bool few = T <= kFewTokens;
  const int64_t width = vocab_width(T);
  if ((st = operand_map(&gp.map[kMapH], h, T, D)) != QB_OK) return st;
  if ((st = operand_map(&gp.map[kMapHTile], h, T, D, few ? width / 2 : 128)) != QB_OK) return st;
  if ((st = operand_map(&gp.map[kMapW], w, V, D)) != QB_OK) return st;
  for (int i = 0; i < 2; ++i)
    if ((st = operand_map(&g_map[i], g[i], plan.rows, Tp)) != QB_OK) return st;
  gp.g_pitch = (int32_t)Tp;
  gp.grad_w = grad_w;
  gp.slabs = slabs;
  gp.T = (int32_t)T;
  gp.V = (int32_t)V;
  gp.D = (int32_t)D;
  gp.bias = bias;
  gp.targets = targets;
  gp.lse = lse;
  gp.grad_loss = grad_loss;
  gp.part_bias = grad_bias ? part_bias : nullptr;
  gp.ws = ws;
  const int32_t t_tiles = (int32_t)up(T, 256), d_tiles = (int32_t)up(D, 256);
  for (int64_t i = 0; i <= plan.pieces; ++i) {
    int64_t load[kMaxPairs] = {};
    gp.count = 0;
    const auto add = [&](const VocabProblem& p, int64_t tiles, int64_t cost) {
      gp.prob[gp.count] = p;
      deal_tiles(gp.prob[gp.count++], tiles, cost, load, pairs);
    };
    if (i > 0) {  // the products of the piece whose g the launch before formed
      const int64_t v0 = (i - 1) * plan.rows, rows = std::min(plan.rows, V - v0);
      gp.map[kMapG] = g_map[(i - 1) & 1];
      gp.out_v0 = (int32_t)v0;
      gp.add = i > 1;
      VocabProblem p = {};
      if (grad_h) {
        p.kind = kGradH;
        p.width = kVocabTile;
        p.map_a = kMapG;
        p.map_b = kMapW;
        p.a_form = kCols;
        p.b_form = cols_form(D);
        p.n_tiles = d_tiles;
        p.split_tiles = t_tiles * d_tiles;
        p.k_blocks = (int32_t)plan.k_split;
        // every split of the first piece stores its slab; what a shorter last piece lacks adds nothing
        p.k_end = (int32_t)up(rows, 64);
        p.b_row0 = (int32_t)v0;
        add(p, (int64_t)up(p.k_end, p.k_blocks) * p.split_tiles, vocab_tile_cost(p.k_blocks));
      }
      if (grad_w) {
        p = VocabProblem{};
        p.kind = kGradW;
        p.width = kVocabTile;
        p.map_a = kMapG;
        p.map_b = kMapH;
        p.a_form = kRows;
        p.b_form = cols_form(D);
        p.n_tiles = d_tiles;
        p.split_tiles = (int32_t)up(rows, 256) * d_tiles;
        p.k_blocks = p.k_end = (int32_t)(Tp / 64);
        add(p, p.split_tiles, vocab_tile_cost(p.k_blocks));
      }
    }
    if (i < plan.pieces) {
      const int64_t v0 = i * plan.rows, rows = std::min(plan.rows, V - v0);
      gp.g_new = g[i & 1];
      gp.v0 = (int32_t)v0;
      VocabProblem p = {};
      p.kind = kGradZ;
      p.width = (int32_t)width;
      p.map_a = kMapW;
      p.map_b = kMapHTile;
      p.a_form = p.b_form = rows_form(D);
      p.a_row0 = (int32_t)v0;
      p.n_tiles = t_tiles;
      p.split_tiles = (int32_t)up(rows, 256) * t_tiles;
      p.k_blocks = p.k_end = (int32_t)up(D, 64);
      add(p, p.split_tiles, vocab_tile_cost(p.k_blocks));
    }
    if (gp.count == 0) continue;
    if ((st = few ? launch_vocab<false, true>(gp, pairs, stream) : launch_vocab<false, false>(gp, pairs, stream)) != QB_OK) return st;
  }
  if (grad_h || grad_bias) {
    const int64_t h_blocks = grad_h ? up(T * D, plan.splits > 4 ? 128 : 1024) : 0, b_blocks = grad_bias ? up(V, 256) : 0;
    QB_CUDA_TRY(launch_kernel(vocab_finish_kernel, (unsigned)(h_blocks + b_blocks), 256, 0, stream, 1, false, slabs, (int)plan.splits, T * D, grad_h,
                              (int)h_blocks, part_bias, 2 * t_tiles, (int)V, grad_bias));
  }
  return QB_OK;
}
