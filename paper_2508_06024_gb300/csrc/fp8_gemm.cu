// Grouped product of 8-bit operands (e4m3) with one fp32 scale per block of 128
// on the sm_103a tensor cores.  With A_g the group's rows [M_g, K] and B_g [N, K],
//
//   c[m, n] = sum_b sa[m, b] sb[n / 128, b] sum_{j in block b} qa[m, j] qb[n, j]
//
// The inner sums are tcgen05.mma (kind::f8f6f4) products over one block of K:
// 128 e4m3 values are one 128-byte swizzle row, so a pipeline stage is a block
// and its four MMAs leave the block's unscaled sums in tensor memory.  The scales
// are arbitrary fp32 numbers, so every block's sums leave tensor memory: eight
// warps read them and multiply-add them into fp32 registers with the row's scale
// (a thread's TMEM lane is its row) times the column block's, while the MMAs fill
// the other of two tensor-memory buffers.
//
// CTA layout (384 threads):
//   warp 0       TMA producer
//   warp 1       TMEM allocator and MMA issuer
//   warp 2       scales: the rows' and the column blocks' of each block of K, from
//                global memory to a ring in shared memory
//   warps 4..11  sums: warp w reads TMEM lanes 32 (w % 4) .. +31, and of the
//                tile's two halves of 128 columns the 64 of each that (w - 4) / 4
//                names; at the end of a tile its epilogue.
// The two halves are two column blocks of B, or (SwiGLU) the same block of W1
// and W3, so that a thread holds both factors of its hidden values.  Their
// result is quantised here, from the fp32 values: the two warps that hold a
// row's 128 columns exchange its largest magnitude.
//
// CTA pairs (PAIR): a cluster of two CTAs computes a 256-row tile with
// cta_group::2; each stages its own 128 rows of A and half of the B tile, and
// reads its own 128 rows of sums.  The even CTA issues the MMAs.
//
// Shared K (few tiles, stored sums): with at most half as many tiles as SMs, the 2 to
// 8 CTAs of a cluster divide a tile's K blocks.  Each leaves its sums where its
// operand stages were; after a cluster barrier CTA r adds up the r-th share of the
// rows, in the order of the parts, through distributed shared memory.  One group 4096
// x 14336: 129 rows 53 us -> 25, 300 rows 57 -> 37; 4096 x 4096, 129 rows 20 -> 16.
// Parts of less than MIN_GROUPS groups of blocks cost what they save (1024 x 1024: 14
// us in parts of one group, 12 whole).
//
// What bounds it: a K block of a 128 x 256 tile takes the MMAs 512 clocks, the fp32
// multiply-adds of its sums 256 and reading them about as long; with the waits and
// hand-overs between (two buffers, a warp's registers full of sums) a block takes
// about 930: no unit is full, what is left is latency.  16384 x 14336 x 4096 in 8 groups: 780 us = 2.47 PFLOP/s (a library's
// product without scales 509 us), 850 us once power holds the clocks; experts of
// 14336 x 4096, 1024 tokens: the tensor pipe is busy 50% of the time.
//
// Every wait is bounded as in the bf16 kernel: a wait that gives up sets the
// error word and the CTA's abort flag, waits for copies and MMAs in flight,
// frees its tensor memory and returns.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"
#include "tc_ptx.cuh"

namespace ec2moe {

// bit 0: a bounded wait timed out; bit 1: a group range (offsets) or a scatter
// destination (perm) outside the rows of the call was skipped
__device__ unsigned int g_fp8_error;

namespace {

using namespace tc;

constexpr int BM = 128;   // tile rows of a CTA (MMA M, TMEM lanes)
constexpr int BN = 256;   // tile columns: two halves of 128
constexpr int HALF = 128;
constexpr int BK = FP8_BLOCK;
constexpr int UK = 32;    // K of one tcgen05.mma kind::f8f6f4
constexpr int SUM_WARPS = 8;
constexpr int FIRST_SUM = 4;      // the first warpgroup loads, issues and idles
constexpr int NUM_THREADS = 32 * (FIRST_SUM + SUM_WARPS);
// Registers: 384 threads start with 168 each (64512); the sums' warpgroups take
// what the first one gives up (128 * 40 + 256 * 232 = 64512).  With 56 and 224 the
// quantising modes spilled 130 bytes (experts, Mixtral 8192: 2451 us, now 2356).
constexpr int REGS_FEW = 40, REGS_SUM = 232;
constexpr int MAX_GROUPS = 136;
constexpr int MAX_PIECES = 8;
constexpr int MIN_GROUPS = 2;
constexpr int TMEM_COLS = 512;
// Scales are handed over for SG blocks of K at a time: a wait and a release cost
// about 200 clocks, a block's MMAs 512.
constexpr int SG = 4;
constexpr int RING = 3;              // such groups held
constexpr int RING_GROUP = (BM + 2) * SG;  // floats: [BM rows][SG], then [SG][2 halves]

// What happens to a tile: stored (bf16 or fp32, optionally scattered and scaled
// by row), or put through the activation and quantised.
enum Mode { STORE_BF16 = 0, STORE_F32 = 1, QUANT_GELU = 2, QUANT_SWIGLU = 3 };

struct Params {
  const float* SA;           // [rows, n_kb], pitch sa_pitch
  int sa_pitch;
  int sa_words;              // scales per copy: what the pitch and the address align to
  const float* SB;           // [G, n_nb, n_kb]
  const float* SB2;          // SwiGLU: of W3
  const int32_t* offsets;    // [G + 1], nullptr: one group of all rows
  int G, rows, N, K, n_kb, n_nb;
  int n_tiles_n;
  int pieces;                // CTAs of a cluster that share a tile's K (1: no cluster)
  void* out;                 // STORE: [rows, ldo]; QUANT: e4m3 [rows, N]
  long long ldo;
  float* out_scale;          // QUANT: [rows, ceil(N / 128)], pitch out_scale_pitch
  int out_scale_pitch;
  const int32_t* perm;       // STORE: destination of each row (nullptr: itself)
  const float* row_scale;    // STORE: factor of each destination (nullptr: 1)
  long long timeout;
};

struct TileCoord {
  int g, m_blk, n_blk;
};
// Linear tile order: group-major, then n block, then m block, so CTAs that run
// at the same time share the group's weight tiles and rows in L2.
__device__ __forceinline__ TileCoord decode_tile(int tile, const int* tile_prefix, int n_tiles_n, int& cursor) {
  while (tile >= tile_prefix[cursor + 1] * n_tiles_n) ++cursor;
  const int mt = tile_prefix[cursor + 1] - tile_prefix[cursor];
  const int rem = tile - tile_prefix[cursor] * n_tiles_n;
  return TileCoord{cursor, rem % mt, rem / mt};
}

template <int MODE, bool PAIR>
struct Cfg {
  static constexpr bool QUANT = MODE == QUANT_GELU || MODE == QUANT_SWIGLU;
  static constexpr int TILE_M = PAIR ? 2 * BM : BM;
  static constexpr int B_ROWS = PAIR ? HALF : BN;  // rows of the B tile this CTA stages
  static constexpr int A_BYTES = BM * BK;
  static constexpr int B_BYTES = B_ROWS * BK;
  static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
  static constexpr int STAGES = PAIR ? 5 : 4;
  static constexpr int OUT_COLS = MODE == QUANT_SWIGLU ? HALF : BN;  // columns of the result per tile
  static constexpr int BUFS = TMEM_COLS / BN;
  static constexpr bool PIECES = !QUANT && !PAIR;  // a tile's K can be shared by a cluster
  static constexpr int SUM_PITCH = BN + 4;         // floats of a row of the sums handed over
  static_assert(BM * SUM_PITCH * 4 <= STAGES * STAGE_BYTES || !PIECES, "the sums take the place of the stages");
  static constexpr int N_BARS = 2 * STAGES + 2 * BUFS + 2 * RING + 1;  // full, empty, tfull, tempty, sfull, sempty, drain
  static constexpr int OFF_BARS = STAGES * STAGE_BYTES;
  static constexpr int OFF_SLOT = OFF_BARS + N_BARS * 8;
  static constexpr int OFF_PREFIX = OFF_SLOT + 16;
  static constexpr int OFF_ROW0 = OFF_PREFIX + (MAX_GROUPS + 1) * 4;
  static constexpr int OFF_CNT = OFF_ROW0 + (MAX_GROUPS + 1) * 4;
  static constexpr int OFF_MAX = OFF_CNT + MAX_GROUPS * 4;  // [2 halves of 64][128 rows] magnitudes
  static constexpr int MAX_BYTES = QUANT ? 2 * BM * 4 : 0;
  static constexpr int OFF_RING = (OFF_MAX + MAX_BYTES + 15) / 16 * 16;  // [RING][RING_GROUP]
  static constexpr int STG_ROW = QUANT || !PAIR ? 64 : 128;  // staging per warp: 32 rows of so many bytes
  static constexpr int OFF_DST = OFF_RING + RING * RING_GROUP * 4;  // STORE: [sum warp][32] destination rows, factors
  static constexpr int OFF_STG = (OFF_DST + (QUANT ? 0 : SUM_WARPS * 32 * 8) + 127) / 128 * 128;
  static constexpr int SMEM = 1024 + OFF_STG + SUM_WARPS * 32 * STG_ROW;
  static_assert((OFF_BARS + 2 * STAGES * 8) % 16 == 0 && BUFS == 2, "the buffers' barriers, see the sums");
  static_assert(OFF_BARS % 8 == 0 && SMEM <= 232448, "shared memory per CTA");
};

template <int MODE, bool PAIR>
__global__ void __launch_bounds__(NUM_THREADS, 1)
    fp8_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                    const __grid_constant__ CUtensorMap tmB2, const Params p) {
  using C = Cfg<MODE, PAIR>;
  constexpr int STAGES = C::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sA = smem;
  uint8_t* sB = smem + STAGES * C::A_BYTES;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::OFF_BARS);
  uint64_t* empty = full + STAGES;
  uint64_t* tfull = empty + STAGES;
  uint64_t* tempty = tfull + C::BUFS;
  uint64_t* sfull = tempty + C::BUFS;
  uint64_t* sempty = sfull + RING;
  uint64_t* drain = sempty + RING;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_SLOT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  // what the roles leave in flight when they end: the producer's stages (low half) and the
  // phases that they complete, the lane + 1 of the MMA warp that issued MMAs (in registers
  // of all warps behind their roles they cost the sums 30 bytes of spills)
  volatile uint32_t* in_flight = tmem_slot + 2;
  int* tile_prefix = reinterpret_cast<int*>(smem + C::OFF_PREFIX);
  int* row0 = reinterpret_cast<int*>(smem + C::OFF_ROW0);
  int* row_cnt = reinterpret_cast<int*>(smem + C::OFF_CNT);
  float* s_max = reinterpret_cast<float*>(smem + C::OFF_MAX);
  float* ring = reinterpret_cast<float*>(smem + C::OFF_RING);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
  const bool shared_k = C::PIECES && p.pieces > 1;  // the cluster has one tile, or none
  const int tile_first = PAIR || shared_k ? static_cast<int>(cluster_id_x()) : static_cast<int>(blockIdx.x);
  const int tile_step = PAIR       ? static_cast<int>(cluster_count_x())
                        : shared_k ? 1 << 30
                                   : static_cast<int>(gridDim.x);
  const int piece = shared_k ? static_cast<int>(cluster_ctarank()) : 0;
  // Barrier set-up, TMEM allocation and descriptor prefetch overlap the previous
  // kernel; everything that reads its results comes after pdl_wait.
  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&full[s]), 1);
      mbar_init(smem_u32(&empty[s]), 1);
    }
    for (int b = 0; b < C::BUFS; ++b) {
      mbar_init(smem_u32(&tfull[b]), 1);
      mbar_init(smem_u32(&tempty[b]), PAIR ? 2 * SUM_WARPS : SUM_WARPS);
    }
    for (int r = 0; r < RING; ++r) {
      mbar_init(smem_u32(&sfull[r]), 32);
      mbar_init(smem_u32(&sempty[r]), SUM_WARPS);
    }
    mbar_init(smem_u32(drain), 1);
    *abort_flag = 0;
    in_flight[0] = in_flight[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 0) {
    pdl_wait();
    // Per-group first rows and tile prefix (m tiles), one warp-wide scan.
    scan_group_rows<(MAX_GROUPS + 31) / 32, C::TILE_M>(p.offsets, p.G, p.rows, lane, row0, row_cnt, tile_prefix,
                                                       &g_fp8_error);
  }
  if (warp == 0 && lane == 0) {
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
    if (MODE == QUANT_SWIGLU) tma_prefetch_desc(&tmB2);
  }
  if (warp == 1) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                   "r"(TMEM_COLS)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                   "r"(TMEM_COLS)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  // PAIR: both CTAs' barriers are initialised before either arrives remotely
  if (PAIR) cluster_sync_all();
  tc_fence_after();
  pdl_wait();
  const uint32_t tmem_base = *tmem_slot;
  const int n_tiles = tile_prefix[p.G] * p.n_tiles_n;
  // this CTA's blocks of K: all, or its share in whole groups of SG
  const int n_sg = (p.n_kb + SG - 1) / SG;
  const int kb_first = shared_k ? piece * n_sg / p.pieces * SG : 0;
  const int n_kb = (shared_k && piece + 1 < p.pieces ? (piece + 1) * n_sg / p.pieces * SG : p.n_kb) - kb_first;
  const long long budget = p.timeout;

  if (warp < FIRST_SUM) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_FEW));
    if (warp == 0) {
      // ---------------------------------------------------------------- producer
      const bool issue = elect_one();
      int stage = 0;
      uint32_t phase = 0;
      uint32_t issued = 0, issued_phase = 0;  // bit s: stage s holds a copy, the phase that it completes
      int cursor = 0;
      bool ok = true;
      for (int tile = tile_first; tile < n_tiles && ok; tile += tile_step) {
        const TileCoord tc = decode_tile(tile, tile_prefix, p.n_tiles_n, cursor);
        const int a_row = row0[tc.g] + tc.m_blk * C::TILE_M + static_cast<int>(rank) * BM;
        const int b_row = tc.g * p.N + tc.n_blk * C::OUT_COLS;
        for (int kb = 0; kb < n_kb; ++kb) {
          if (!__all_sync(0xffffffffu,
                          mbar_wait(smem_u32(&empty[stage]), phase ^ 1u, budget, abort_flag, &g_fp8_error))) {
            ok = false;
            break;
          }
          const uint32_t fb = smem_u32(&full[stage]);
          const uint32_t da = smem_u32(sA + stage * C::A_BYTES);
          const uint32_t db = smem_u32(sB + stage * C::B_BYTES);
          const int k = (kb_first + kb) * BK;
          if (!issue) {
          } else if (PAIR) {
            // both halves complete on the even CTA's full barrier; of the B tile
            // the even CTA stages the first half of the columns, the odd CTA the second
            if (rank == 0) mbar_expect_tx(fb, 2 * C::STAGE_BYTES);
            const uint32_t fb0 = rank == 0 ? fb : map_to_rank(fb, 0);
            tma_load_2d_to_pair_bar(da, &tmA, k, a_row, fb0);
            tma_load_2d_to_pair_bar(db, MODE == QUANT_SWIGLU && rank ? &tmB2 : &tmB, k,
                                    b_row + (MODE == QUANT_SWIGLU ? 0 : static_cast<int>(rank) * HALF), fb0);
          } else {
            mbar_expect_tx(fb, C::STAGE_BYTES);
            tma_load_2d(da, &tmA, k, a_row, fb);
            tma_load_2d(db, &tmB, k, b_row, fb);
            tma_load_2d(db + HALF * BK, MODE == QUANT_SWIGLU ? &tmB2 : &tmB, k,
                        b_row + (MODE == QUANT_SWIGLU ? 0 : HALF), fb);
          }
          issued |= 1u << stage;
          issued_phase = (issued_phase & ~(1u << stage)) | (phase << stage);
          if (++stage == STAGES) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      if (lane == 0) in_flight[0] = issued | (issued_phase << 16);
    } else if (warp == 1 && (!PAIR || rank == 0)) {
      // -------------------------------------------------------------- MMA issuer
      const bool issue = elect_one();
      constexpr uint32_t IDESC = idesc_e4m3(C::TILE_M, BN);
      const uint64_t da0 = sdesc_sw128(smem_u32(sA));
      const uint64_t db0 = sdesc_sw128(smem_u32(sB));
      int stage = 0;
      uint32_t phase = 0;
      uint32_t it = 0;  // blocks so far: buffer it & 1, its phase (it >> 1) & 1
      bool ok = true, any = false;
      for (int tile = tile_first; tile < n_tiles && ok; tile += tile_step) {
        for (int kb = 0; kb < n_kb; ++kb, ++it) {
          const uint32_t buf = it & 1u, bph = (it >> 1) & 1u;
          // the operands first: they are there while the buffer is still being read
          const bool there = mbar_wait_strict(smem_u32(&full[stage]), phase, budget, abort_flag, &g_fp8_error);
          if (!__all_sync(0xffffffffu,
                          there && (PAIR ? mbar_wait_cluster(smem_u32(&tempty[buf]), bph ^ 1u, budget, abort_flag, &g_fp8_error)
                                         : mbar_wait(smem_u32(&tempty[buf]), bph ^ 1u, budget, abort_flag, &g_fp8_error)))) {
            ok = false;
            break;
          }
          tc_fence_after();
          // stage-0 descriptors plus the stage offset; each K = 32 step adds 32
          // bytes (2 in the address field, which cannot carry: shared addresses
          // are below 256 KB)
          const uint64_t da = da0 + static_cast<uint64_t>(stage) * (C::A_BYTES >> 4);
          const uint64_t db = db0 + static_cast<uint64_t>(stage) * (C::B_BYTES >> 4);
          const uint32_t d = tmem_base + buf * BN;
          if (issue) {
#pragma unroll
            for (int kk = 0; kk < BK / UK; ++kk) {
              if (PAIR) umma_fp8_pair(d, da + 2 * kk, db + 2 * kk, IDESC, kk ? 1u : 0u);
              else umma_fp8(d, da + 2 * kk, db + 2 * kk, IDESC, kk ? 1u : 0u);
            }
            if (PAIR) {
              umma_commit_pair_mc(smem_u32(&tfull[buf]));
              umma_commit_pair_mc(smem_u32(&empty[stage]));
            } else {
              umma_commit(smem_u32(&tfull[buf]));
              umma_commit(smem_u32(&empty[stage]));
            }
          }
          any = true;
          if (++stage == STAGES) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      if (any && issue) in_flight[1] = lane + 1;
    } else if (warp == 2) {
      // ------------------------------------------------------------------ scales
      // Asynchronous copies, as far ahead as the ring is deep: a row's SG scales at
      // once where they are aligned to that.  A copy takes the load path a turn per
      // row, which the barriers share; copies of single scales held up the sums
      // (16384 x 14336 x 4096: 846 us, without them 717).
      const uint32_t ring0 = smem_u32(ring);
      uint32_t it = 0;
      int cursor = 0;
      bool ok = true;
      for (int tile = tile_first; tile < n_tiles && ok; tile += tile_step) {
        const TileCoord tc = decode_tile(tile, tile_prefix, p.n_tiles_n, cursor);
        const int mg = row_cnt[tc.g];
        const int left = mg - tc.m_blk * C::TILE_M - static_cast<int>(rank) * BM - lane;  // > 32 i: row lane + 32 i exists
        const float* sa = p.SA + (static_cast<long long>(row0[tc.g]) + mg - left) * p.sa_pitch + kb_first;
        // lanes 0 and 1: the tile's two column blocks (one beyond N: the last
        // block's, its columns are not stored)
        int nb = MODE == QUANT_SWIGLU ? tc.n_blk : 2 * tc.n_blk + (lane & 1);
        if (nb >= p.n_nb) nb = p.n_nb - 1;
        const float* sb =
            (MODE == QUANT_SWIGLU && (lane & 1) ? p.SB2 : p.SB) + (static_cast<long long>(tc.g) * p.n_nb + nb) * p.n_kb +
            kb_first;
        for (int kb0 = 0; kb0 < n_kb; kb0 += SG, ++it) {
          const uint32_t slot = it % RING, sph = (it / RING) & 1u;
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sempty[slot]), sph ^ 1u, budget, abort_flag, &g_fp8_error));
          if (!ok) break;
          const uint32_t to = ring0 + slot * (RING_GROUP * 4);
          const int n = n_kb - kb0 < SG ? n_kb - kb0 : SG;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (left <= 32 * i) continue;
            const float* from = sa + static_cast<long long>(32 * i) * p.sa_pitch + kb0;
            const uint32_t at = to + 16 * (lane + 32 * i);
            if (n == SG && p.sa_words == 4) {
              cp_async<16>(at, from);
            } else if (n == SG && p.sa_words == 2) {
              cp_async<8>(at, from);
              cp_async<8>(at + 8, from + 2);
            } else {
              for (int u = 0; u < n; ++u) cp_async<4>(at + 4 * u, from + u);
            }
          }
          if (lane < 2)
            for (int u = 0; u < n; ++u) cp_async<4>(to + 16 * BM + 4 * (2 * u + lane), sb + kb0 + u);
          cp_async_arrive(smem_u32(&sfull[slot]));
        }
      }
      cp_async_wait();  // none in flight when shared memory is released
    }
    if (shared_k) {
      __syncwarp();
      cluster_sync_all();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_SUM));
    // ------------------------------------------------------ sums and epilogue
    const int q = warp & 3;                    // TMEM lane quadrant this warp may read
    const int part = (warp - FIRST_SUM) >> 2;  // which 64 columns of each half
    const int row_in_tile = q * 32 + lane;
    const uint32_t t_row = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + part * 64;
    const uint32_t release0 = PAIR ? map_to_rank(smem_u32(&tempty[0]), 0) : smem_u32(&tempty[0]);
    uint8_t* stg = smem + C::OFF_STG + (warp - FIRST_SUM) * 32 * C::STG_ROW;
    int2* s_dst = reinterpret_cast<int2*>(smem + C::OFF_DST) + (warp - FIRST_SUM) * 32;
    // the buffer in turn: its columns, its barriers (8 bytes apart, pairs aligned
    // to 16) and its phase
    uint32_t t_at = t_row, full_at = smem_u32(&tfull[0]), release_at = release0, bph = 0;
    uint32_t slot = 0, sph = 0;            // of the scales
    bool summed = false, scaled = false;  // the next block's sums, the next group's scales are there
    int cursor = 0;
    bool ok = true;
    for (int tile = tile_first; tile < n_tiles; tile += tile_step) {
      const TileCoord tc = decode_tile(tile, tile_prefix, p.n_tiles_n, cursor);
      const int mg = row_cnt[tc.g];
      const int local = tc.m_blk * C::TILE_M + static_cast<int>(rank) * BM + row_in_tile;
      const bool valid = local < mg;
      const long long row = static_cast<long long>(row0[tc.g]) + local;
      if (!C::QUANT) {
        // where the row goes (-1: nowhere) and its factor, read while the first
        // block is multiplied and kept out of the registers meanwhile
        int dest = valid ? static_cast<int>(row) : -1;
        float sc = 1.0f;
        if (valid && p.perm) {
          dest = p.perm[row];
          if (dest < 0 || dest >= p.rows) {
            atomicOr(&g_fp8_error, 2u);
            dest = -1;
          } else if (p.row_scale) {
            sc = p.row_scale[dest];
          }
        }
        s_dst[lane] = make_int2(dest, __float_as_int(sc));
      }
      float acc[128];
#pragma unroll
      for (int i = 0; i < 128; ++i) acc[i] = 0.0f;
      for (int kb0 = 0; kb0 < n_kb; kb0 += SG) {
        if (!__all_sync(0xffffffffu, scaled)) {
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sfull[slot]), sph, budget, abort_flag, &g_fp8_error));
          if (!ok) break;
        }
        // the group's scales (of rows that do not exist: anything, their sums are
        // not stored)
        const float* scales = ring + slot * RING_GROUP;
        float a[SG];
        *reinterpret_cast<float4*>(a) = *reinterpret_cast<const float4*>(scales + SG * row_in_tile);
        float2 b_next = *reinterpret_cast<const float2*>(scales + SG * BM);
#pragma unroll
        for (int u = 0; u < SG; ++u) {
          if (kb0 + u >= n_kb) break;
          const float2 b = b_next;
          if (!__all_sync(0xffffffffu, summed)) {
            ok = __all_sync(0xffffffffu, mbar_wait(full_at, bph, budget, abort_flag, &g_fp8_error));
            if (!ok) break;
          }
          tc_fence_after();
          // Hands the buffer back and turns to the other one, and asks for what the
          // next block needs: the answers come while this one's sums are added.  An
          // answered wait takes about 100 clocks, the sums of a block 256.
          auto release = [&] {
            tc_fence_before();
            __syncwarp();
            if (PAIR) mbar_arrive_remote_if(lane == 0, release_at);
            else mbar_arrive_if(lane == 0, release_at);
            // both have been used once more after the second
            bph ^= (t_at / BN) & 1u;
            t_at ^= BN;
            full_at ^= 8u;
            release_at ^= 8u;
            summed = mbar_test_wait(full_at, bph);
            if (u + 1 < SG && kb0 + u + 1 < n_kb) {
              b_next = *reinterpret_cast<const float2*>(scales + SG * BM + 2 * (u + 1));
            } else {
              // the group's scales have been read (into registers: b is used below)
              mbar_arrive_if(lane == 0, smem_u32(&sempty[slot]));
              if (++slot == RING) {
                slot = 0;
                sph ^= 1u;
              }
              scaled = mbar_test_wait(smem_u32(&sfull[slot]), sph);
            }
          };
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float r[64];
            tmem_ld64(t_at + h * HALF, r);
            if (h == 1) release();
            const float f = a[u] * (h ? b.y : b.x);
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[h * 64 + i] = fmaf(r[i], f, acc[h * 64 + i]);
          }
        }
        if (!ok) break;
      }
      if (C::QUANT) {
        // the two warps of a lane quadrant meet at named barriers: agree first
        uint32_t all_ok;
        asm volatile(
            "{\n .reg .pred p, r;\n setp.ne.u32 p, %1, 0;\n"
            " bar.red.and.pred r, %2, 64, p;\n selp.u32 %0, 1, 0, r;\n}"
            : "=r"(all_ok)
            : "r"(ok ? 1u : 0u), "r"(1 + q)
            : "memory");
        ok = all_ok != 0;
      }
      if (!ok) break;
      const unsigned vmask = __ballot_sync(0xffffffffu, valid);
      if constexpr (C::QUANT) {
        constexpr int BLOCKS = MODE == QUANT_SWIGLU ? 1 : 2;
#pragma unroll
        for (int h = 0; h < BLOCKS; ++h) {
          const int col0 = tc.n_blk * C::OUT_COLS + h * HALF + part * 64;
          float m = 0.0f;
#pragma unroll
          for (int i = 0; i < 64; ++i) {
            float& v = acc[h * 64 + i];
            v = MODE == QUANT_SWIGLU ? silu_bf16out(v) * acc[64 + i] : gelu_fp8out(v);
            m = fmaxf(m, fabsf(v));
          }
          if (col0 + 64 > p.N) {
            // columns beyond N belong to other weights: not part of the block
            m = 0.0f;
#pragma unroll
            for (int i = 0; i < 64; ++i)
              if (col0 + i < p.N) m = fmaxf(m, fabsf(acc[h * 64 + i]));
          }
          s_max[part * BM + row_in_tile] = m;
          asm volatile("bar.sync %0, 64;" ::"r"(1 + q) : "memory");
          m = fmaxf(m, s_max[(part ^ 1) * BM + row_in_tile]);
          const Fp8Scale f = fp8_scale(m);
          const int nb = tc.n_blk * BLOCKS + h;
          if (valid && part == 0 && nb < p.n_nb) p.out_scale[row * p.out_scale_pitch + nb] = f.scale;
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<U4*>(stg + lane * 64 + ((j ^ ((lane >> 1) & 3)) * 16)) =
                fp8_pack16(&acc[h * 64 + 16 * j], f.inv);
          __syncwarp();
          uint8_t* o = static_cast<uint8_t*>(p.out) + col0;
#pragma unroll 1
          for (int pass = 0; pass < 4; ++pass) {
            const int rr = pass * 8 + (lane >> 2);
            const int seg = lane & 3;
            const U4 x = *reinterpret_cast<const U4*>(stg + rr * 64 + ((seg ^ ((rr >> 1) & 3)) * 16));
            if (((vmask >> rr) & 1u) && col0 + seg * 16 < p.N)
              *reinterpret_cast<U4*>(o + (row - lane + rr) * p.N + seg * 16) = x;
          }
          // the other warp has read this half's magnitudes before they change
          asm volatile("bar.sync %0, 64;" ::"r"(1 + q) : "memory");
        }
      } else if (shared_k) {
        // handed over where the operands were, which have all been multiplied
        float* to = reinterpret_cast<float*>(smem) + row_in_tile * C::SUM_PITCH + part * 64;
#pragma unroll
        for (int i = 0; i < 128; i += 4)
          *reinterpret_cast<float4*>(to + (i >> 6) * HALF + (i & 63)) = make_float4(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
      } else {
        // Slabs of SLAB columns: rounded into the warp's staging rows (16-byte
        // chunks XOR-swizzled by row), then stored as whole row segments.  The
        // storing loop is rolled: this code runs once per tile, and fetching it
        // is what it takes longest for.
        constexpr int ES = MODE == STORE_F32 ? 4 : 2;
        constexpr int SLAB = C::STG_ROW / ES, SEGS = C::STG_ROW / 16;
        constexpr int SHIFT = SEGS == 4 ? 1 : 0;
        const float sc = __int_as_float(s_dst[lane].y);
#pragma unroll
        for (int c = 0; c < 128; c += SLAB) {
          __syncwarp();
#pragma unroll
          for (int j = 0; j < SEGS; ++j) {
            U4 x;
            if (MODE == STORE_F32) {
              const float* v = &acc[c + 4 * j];
              x = U4{__float_as_uint(v[0] * sc), __float_as_uint(v[1] * sc), __float_as_uint(v[2] * sc),
                     __float_as_uint(v[3] * sc)};
            } else {
              const float* v = &acc[(c + 8 * j) & 127];
              x = U4{pack_bf16x2(v[0] * sc, v[1] * sc), pack_bf16x2(v[2] * sc, v[3] * sc),
                     pack_bf16x2(v[4] * sc, v[5] * sc), pack_bf16x2(v[6] * sc, v[7] * sc)};
            }
            *reinterpret_cast<U4*>(stg + lane * C::STG_ROW + ((j ^ ((lane >> SHIFT) & (SEGS - 1))) * 16)) = x;
          }
          __syncwarp();
          const int seg = lane & (SEGS - 1);
          const int col = tc.n_blk * BN + (c >> 6) * HALF + part * 64 + (c & 63) + seg * (16 / ES);
#pragma unroll 1
          for (int rr = lane / SEGS; rr < 32; rr += 32 / SEGS) {
            const U4 x = *reinterpret_cast<const U4*>(stg + rr * C::STG_ROW + ((seg ^ ((rr >> SHIFT) & (SEGS - 1))) * 16));
            const int drow = s_dst[rr].x;
            if (drow >= 0 && col < p.N)
              *reinterpret_cast<U4*>(static_cast<uint8_t*>(p.out) + (drow * p.ldo + col) * ES) = x;
          }
        }
        __syncwarp();
      }
    }
    if (shared_k) {
      // CTA r of the cluster adds and stores rows [r BM / pieces, (r + 1) BM / pieces)
      // of the tile, the pieces in their order.
      __syncwarp();
      cluster_sync_all();
      if (tile_first < n_tiles) {
        int from = 0;
        const TileCoord tc = decode_tile(tile_first, tile_prefix, p.n_tiles_n, from);
        const int2* dst = reinterpret_cast<const int2*>(smem + C::OFF_DST);  // by row: its quadrant's first warp's
        const int row_first = piece * BM / p.pieces, rows = (piece + 1) * BM / p.pieces - row_first;
        const uint32_t sums = smem_u32(smem);
#pragma unroll 1
        for (int i = threadIdx.x - 32 * FIRST_SUM; i < rows * (BN / 4); i += 32 * SUM_WARPS) {
          const int r = row_first + i / (BN / 4), c = i % (BN / 4) * 4;
          const int2 to = dst[r];
          const int col = tc.n_blk * BN + c;
          if (to.x < 0 || col >= p.N) continue;
          const uint32_t at = sums + (r * C::SUM_PITCH + c) * 4;
          float4 part_of[MAX_PIECES];
#pragma unroll
          for (int k = 0; k < MAX_PIECES; ++k)
            if (k < p.pieces) part_of[k] = ld_cluster_v4(map_to_rank(at, k));
          float4 v = part_of[0];
#pragma unroll
          for (int k = 1; k < MAX_PIECES; ++k) {
            if (k >= p.pieces) break;
            v.x += part_of[k].x;
            v.y += part_of[k].y;
            v.z += part_of[k].z;
            v.w += part_of[k].w;
          }
          const float sc = __int_as_float(to.y);
          const long long o = to.x * p.ldo + col;
          if (MODE == STORE_F32)
            *reinterpret_cast<float4*>(static_cast<float*>(p.out) + o) = make_float4(v.x * sc, v.y * sc, v.z * sc, v.w * sc);
          else
            *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + o) =
                make_uint2(pack_bf16x2(v.x * sc, v.y * sc), pack_bf16x2(v.z * sc, v.w * sc));
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  // PAIR: the even CTA's MMAs read both CTAs' shared memory and write both CTAs' TMEM;
  // neither is released before both CTAs are done with them, nor, where a wait of either
  // gave up, before what is in flight has ended.
  if (PAIR) {
    if (threadIdx.x == 0) abort_pair(abort_flag, rank);
    __syncwarp();
    cluster_sync_all();
  }
  if (*abort_flag) {  // no warp waits any more: the same in all of them, and in the pair
    if (warp == 0) {
      const uint32_t copies = in_flight[0];
      if (rank == 0) {
        drain_copies(smem_u32(full), copies & 0xffffu, copies >> 16);
      } else if (copies) {
        // the odd CTA's copies complete on the even one's barriers, which has waited only
        // for those that it expected
        wait_for_remote_copies();
      }
    } else if (warp == 1 && in_flight[1] == lane + 1u) {
      // the thread that issued the MMAs: a commit covers its own
      if (PAIR) umma_commit_pair(smem_u32(drain));
      else umma_commit(smem_u32(drain));
      mbar_drain(smem_u32(drain), 0, DRAIN_CYCLES);
    }
    __syncthreads();
    __syncwarp();
    if (PAIR) cluster_sync_all();
  }
  // shared K: no CTA ends while its sums are read
  if (shared_k) cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    if (PAIR)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS)
                   : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS)
                   : "memory");
  }
}

// ------------------------------------------------------------------ host side
// Tiles of a call at most: every group that has rows may end inside one.
long long max_tiles(const Fp8GemmArgs& a, int tile_m, int out_cols) {
  const long long live = a.rows < a.G ? a.rows : a.G;
  return (a.rows + live * (tile_m - 1)) / tile_m * ((a.N + out_cols - 1) / out_cols);
}

// Among how many CTAs a tile's K is divided: as many as give every cluster a place
// at once, and each CTA MIN_GROUPS groups of SG blocks.
int k_pieces(const void* kfn, int smem, long long tiles, int n_kb) {
  long long n = tiles > 0 ? sm_count() / tiles : 1;
  if (n > MAX_PIECES) n = MAX_PIECES;
  if (n > n_kb / (MIN_GROUPS * SG)) n = n_kb / (MIN_GROUPS * SG);
  while (n > 1 && tiles > max_clusters(kfn, NUM_THREADS, smem, static_cast<int>(n))) --n;
  return n > 1 ? static_cast<int>(n) : 1;
}

template <int MODE, bool PAIR>
cudaError_t launch_cfg(const Fp8GemmArgs& a, cudaStream_t s) {
  using C = Cfg<MODE, PAIR>;
  const void* kfn = reinterpret_cast<const void*>(fp8_gemm_kernel<MODE, PAIR>);
  cudaError_t e = ensure_smem_attr(kfn, C::SMEM);
  if (e != cudaSuccess) return e;
  CUtensorMap mA, mB, mB2;
  const long long b_rows = static_cast<long long>(a.G) * a.N;
  if (!make_tensor_map_u8(&mA, a.A, a.rows, a.K, BM)) return cudaErrorInvalidValue;
  if (!make_tensor_map_u8(&mB, a.B, b_rows, a.K, HALF)) return cudaErrorInvalidValue;
  mB2 = mB;
  if (MODE == QUANT_SWIGLU && !make_tensor_map_u8(&mB2, a.B2, b_rows, a.K, HALF)) return cudaErrorInvalidValue;
  Params p;
  p.SA = a.SA;
  p.sa_pitch = a.sa_pitch > 0 ? a.sa_pitch : (a.K + BK - 1) / BK;
  p.sa_words = 1;
  for (int w = 4; w > 1 && p.sa_words == 1; w /= 2)
    if (p.sa_pitch % w == 0 && reinterpret_cast<uintptr_t>(a.SA) % (4 * w) == 0) p.sa_words = w;
  p.SB = a.SB;
  p.SB2 = a.SB2;
  p.offsets = a.offsets;
  p.G = a.G;
  p.rows = a.rows;
  p.N = a.N;
  p.K = a.K;
  p.n_kb = (a.K + BK - 1) / BK;
  p.n_nb = (a.N + HALF - 1) / HALF;
  p.n_tiles_n = (a.N + C::OUT_COLS - 1) / C::OUT_COLS;
  p.out = a.out;
  p.ldo = a.ldo;
  p.out_scale = a.out_scale;
  p.out_scale_pitch = a.out_scale_pitch;
  p.perm = a.perm;
  p.row_scale = a.row_scale;
  p.timeout = a.timeout_cycles;
  p.pieces = 1;
  const long long tiles = max_tiles(a, C::TILE_M, C::OUT_COLS);
  KernelScope ks(a.name, s);
  if (PAIR) {
    int clusters = max_clusters(kfn, NUM_THREADS, C::SMEM, 2);
    if (clusters < 1) return cudaErrorInvalidConfiguration;
    if (tiles < clusters) clusters = static_cast<int>(tiles);
    e = launch_cluster(fp8_gemm_kernel<MODE, PAIR>, clusters, 2, NUM_THREADS, (size_t)C::SMEM, s, mA, mB, mB2, p);
  } else if (int pieces = C::PIECES ? k_pieces(kfn, C::SMEM, tiles, p.n_kb) : 1; pieces > 1) {
    p.pieces = pieces;
    e = launch_cluster(fp8_gemm_kernel<MODE, PAIR>, static_cast<int>(tiles), pieces, NUM_THREADS, (size_t)C::SMEM, s, mA,
                       mB, mB2, p);
  } else {
    const int grid = static_cast<int>(tiles < sm_count() ? tiles : sm_count());
    e = launch_kernel(fp8_gemm_kernel<MODE, PAIR>, dim3(grid), dim3(NUM_THREADS), (size_t)C::SMEM, s, mA, mB, mB2, p);
  }
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

// 256-row tiles on CTA pairs where they waste at most a tenth more rows than 128-row
// tiles.  Several groups end inside a tile each, on average half of one, however
// even their expected rows: six experts of 341 rows where 256 were expected took 455
// us in pairs, 367 in single tiles.  Not where clusters can share K instead.
template <int MODE>
bool use_pairs(const Fp8GemmArgs& a) {
  using C = Cfg<MODE, false>;
  if (C::PIECES && 2 * max_tiles(a, C::TILE_M, C::OUT_COLS) <= sm_count()) return false;
  if (a.G > 1) {
    const long long per = a.rows / a.G;
    return 10 * (per + BM) <= 11 * (per + BM / 2);
  }
  const long long pad1 = (a.rows + BM - 1) / BM * BM, pad2 = (a.rows + 2 * BM - 1) / (2 * BM) * (2 * BM);
  return 10 * pad2 <= 11 * pad1;
}

template <int MODE>
cudaError_t launch_mode(const Fp8GemmArgs& a, cudaStream_t s) {
  return use_pairs<MODE>(a) ? launch_cfg<MODE, true>(a, s) : launch_cfg<MODE, false>(a, s);
}

}  // namespace

cudaError_t launch_gemm_fp8(const Fp8GemmArgs& a, int epi, cudaStream_t s) {
  if (a.G < 1 || a.G > MAX_GROUPS || a.N % 16 != 0 || a.K % 16 != 0) return cudaErrorInvalidValue;
  switch (epi) {
    case EPI_STORE: return a.out_bf16 ? launch_mode<STORE_BF16>(a, s) : launch_mode<STORE_F32>(a, s);
    case EPI_GELU: return launch_mode<QUANT_GELU>(a, s);
    case EPI_SWIGLU: return launch_mode<QUANT_SWIGLU>(a, s);
  }
  return cudaErrorInvalidValue;
}

cudaError_t read_fp8_error(unsigned int* word) {
  unsigned int zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(word, g_fp8_error, sizeof(unsigned int));
  if (e != cudaSuccess) return e;
  return cudaMemcpyToSymbol(g_fp8_error, &zero, sizeof(unsigned int));
}

}  // namespace ec2moe
