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
// (a thread's TMEM lane is its row) times the column block's, two per
// instruction, while the MMAs fill the other of two tensor-memory buffers.
//
// CTA layout (320 threads):
//   warp 0      TMA producer
//   warp 1      TMEM allocator and MMA issuer
//   warps 2..9  sums: warp w reads TMEM lanes 32 (w % 4) .. +31, and of the
//               tile's two halves of 128 columns the 64 of each that (w - 2) / 4
//               names; at the end of a tile its epilogue.
// The two halves are two column blocks of B, or (SwiGLU) the same block of W1
// and W3, so that a thread holds both factors of its hidden values.  Their
// result is quantised here, from the fp32 values: the two warps that hold a
// row's 128 columns exchange its largest magnitude.
//
// CTA pairs (PAIR): a cluster of two CTAs computes a 256-row tile with
// cta_group::2; each stages its own 128 rows of A and half of the B tile, and
// reads its own 128 rows of sums.  The even CTA issues the MMAs.
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
constexpr int NUM_THREADS = 64 + 32 * SUM_WARPS;
constexpr int MAX_GROUPS = 136;
constexpr int TMEM_COLS = 2 * BN;

// What happens to a tile: stored (bf16 or fp32, optionally scattered and scaled
// by row), or put through the activation and quantised.
enum Mode { STORE_BF16 = 0, STORE_F32 = 1, QUANT_GELU = 2, QUANT_SWIGLU = 3 };

struct Params {
  const float* SA;           // [rows, n_kb]
  const float* SB;           // [G, n_nb, n_kb]
  const float* SB2;          // SwiGLU: of W3
  const int32_t* offsets;    // [G + 1], nullptr: one group of all rows
  int G, rows, N, K, n_kb, n_nb;
  int n_tiles_n;
  void* out;                 // STORE: [rows, ldo]; QUANT: e4m3 [rows, N]
  long long ldo;
  float* out_scale;          // QUANT: [rows, ceil(N / 128)]
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
  static constexpr int B_ROWS = PAIR ? BN / 2 : BN;  // rows of the B tile this CTA stages
  static constexpr int A_BYTES = BM * BK;
  static constexpr int B_BYTES = B_ROWS * BK;
  static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
  static constexpr int STAGES = PAIR ? 6 : 4;
  static constexpr int OUT_COLS = MODE == QUANT_SWIGLU ? HALF : BN;  // columns of the result per tile
  static constexpr int N_BARS = 2 * STAGES + 5;  // full, empty, tfull[2], tempty[2], drain
  static constexpr int OFF_BARS = STAGES * STAGE_BYTES;
  static constexpr int OFF_SLOT = OFF_BARS + N_BARS * 8;
  static constexpr int OFF_PREFIX = OFF_SLOT + 16;
  static constexpr int OFF_ROW0 = OFF_PREFIX + (MAX_GROUPS + 1) * 4;
  static constexpr int OFF_MAX = OFF_ROW0 + (MAX_GROUPS + 1) * 4;  // [2 halves of 64][128 rows] magnitudes
  static constexpr int MAX_BYTES = QUANT ? 2 * BM * 4 : 0;
  // staging per warp: 32 rows of 128 bytes (STORE) or 64 bytes (QUANT)
  static constexpr int STG_ROW = QUANT ? 64 : 128;
  static constexpr int OFF_STG = (OFF_MAX + MAX_BYTES + 127) / 128 * 128;
  static constexpr int SMEM = 1024 + OFF_STG + SUM_WARPS * 32 * STG_ROW;
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
  uint64_t* tempty = tfull + 2;
  uint64_t* drain = tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_SLOT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* tile_prefix = reinterpret_cast<int*>(smem + C::OFF_PREFIX);
  int* row0 = reinterpret_cast<int*>(smem + C::OFF_ROW0);
  float* s_max = reinterpret_cast<float*>(smem + C::OFF_MAX);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
  const int tile_first = PAIR ? static_cast<int>(cluster_id_x()) : static_cast<int>(blockIdx.x);
  const int tile_step = PAIR ? static_cast<int>(cluster_count_x()) : static_cast<int>(gridDim.x);
  // Barrier set-up, TMEM allocation and descriptor prefetch overlap the previous
  // kernel; everything that reads its results comes after pdl_wait.
  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&full[s]), 1);
      mbar_init(smem_u32(&empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&tfull[b]), 1);
      mbar_init(smem_u32(&tempty[b]), PAIR ? 2 * SUM_WARPS : SUM_WARPS);
    }
    mbar_init(smem_u32(drain), 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 0) {
    pdl_wait();
    // Per-group first rows and tile prefix (m tiles), one warp-wide scan.
    warp_exclusive_scan<(MAX_GROUPS + 31) / 32>(
        p.G, lane,
        [&](int g) {
          int r0 = 0, mg = p.rows;
          if (p.offsets) {
            r0 = p.offsets[g];
            mg = p.offsets[g + 1] - r0;
            if (r0 < 0 || mg < 0 || static_cast<long long>(r0) + mg > p.rows) {
              // not a range of this call's rows: the group is skipped
              atomicOr(&g_fp8_error, 2u);
              r0 = 0;
              mg = 0;
            }
          }
          row0[g] = r0;
          return (mg + C::TILE_M - 1) / C::TILE_M;
        },
        tile_prefix);
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
  const int n_kb = p.n_kb;
  const long long budget = p.timeout;

  if (warp == 0) {
    // ---------------------------------------------------------------- producer
    const bool issue = elect_one();
    int stage = 0;
    uint32_t phase = 0;
    uint32_t issued = 0;  // bit s: stage s holds a copy the consumer has not released
    uint32_t issued_phase = 0;
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
        if (!issue) {
        } else if (PAIR) {
          // both halves complete on the even CTA's full barrier; of the B tile
          // the even CTA stages the first half of the columns, the odd CTA the second
          if (rank == 0) mbar_expect_tx(fb, 2 * C::STAGE_BYTES);
          const uint32_t fb0 = rank == 0 ? fb : map_to_rank(fb, 0);
          tma_load_2d_to_pair_bar(da, &tmA, kb * BK, a_row, fb0);
          const CUtensorMap* tb = (MODE == QUANT_SWIGLU && rank) ? &tmB2 : &tmB;
          tma_load_2d_to_pair_bar(db, tb, kb * BK,
                                  b_row + (MODE == QUANT_SWIGLU ? 0 : static_cast<int>(rank) * HALF), fb0);
        } else {
          mbar_expect_tx(fb, C::STAGE_BYTES);
          tma_load_2d(da, &tmA, kb * BK, a_row, fb);
          tma_load_2d(db, &tmB, kb * BK, b_row, fb);
          tma_load_2d(db + HALF * BK, MODE == QUANT_SWIGLU ? &tmB2 : &tmB, kb * BK,
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
    if (!ok || *abort_flag) {
      // Let every copy this CTA started land before shared memory is released.
      if (PAIR && rank != 0) {
        // its copies complete on the even CTA's barriers: wait a fixed time
        if (issued) {
          const unsigned long long t0 = globaltimer_ns();
          while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
        }
      } else {
        for (int s = 0; s < STAGES; ++s)
          if (issued & (1u << s)) mbar_drain(smem_u32(&full[s]), (issued_phase >> s) & 1u, DRAIN_CYCLES);
      }
    }
  } else if (warp == 1) {
    if (!PAIR || rank == 0) {
      // -------------------------------------------------------------- MMA issuer
      const bool issue = elect_one();
      constexpr uint32_t IDESC = idesc_e4m3(C::TILE_M, BN);
      const uint64_t da0 = sdesc_sw128(smem_u32(sA));
      const uint64_t db0 = sdesc_sw128(smem_u32(sB));
      int stage = 0;
      uint32_t phase = 0;
      uint32_t it = 0;  // blocks so far: buffer it & 1, phase (it >> 1) & 1
      bool ok = true, any = false;
      for (int tile = tile_first; tile < n_tiles && ok; tile += tile_step) {
        for (int kb = 0; kb < n_kb; ++kb, ++it) {
          const uint32_t buf = it & 1u, bph = (it >> 1) & 1u;
          const bool freed =
              PAIR ? mbar_wait_cluster(smem_u32(&tempty[buf]), bph ^ 1u, budget, abort_flag, &g_fp8_error)
                   : mbar_wait(smem_u32(&tempty[buf]), bph ^ 1u, budget, abort_flag, &g_fp8_error);
          if (!__all_sync(0xffffffffu, freed && mbar_wait(smem_u32(&full[stage]), phase, budget, abort_flag,
                                                          &g_fp8_error))) {
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
              umma_commit_pair_mc(smem_u32(&empty[stage]));
              umma_commit_pair_mc(smem_u32(&tfull[buf]));
            } else {
              umma_commit(smem_u32(&empty[stage]));
              umma_commit(smem_u32(&tfull[buf]));
            }
          }
          any = true;
          if (++stage == STAGES) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      if ((!ok || *abort_flag) && any && issue) {
        // All MMAs issued so far must finish before TMEM is freed.
        if (PAIR) umma_commit_pair(smem_u32(drain));
        else umma_commit(smem_u32(drain));
        mbar_drain(smem_u32(drain), 0, DRAIN_CYCLES);
      }
    }
  } else {
    // ------------------------------------------------------ sums and epilogue
    const int q = warp & 3;              // TMEM lane quadrant this warp may read
    const int part = (warp - 2) >> 2;    // which 64 columns of each half
    const int row_in_tile = q * 32 + lane;
    const uint32_t t_row = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + part * 64;
    const uint32_t release0 = PAIR ? map_to_rank(smem_u32(&tempty[0]), 0) : smem_u32(&tempty[0]);
    uint8_t* stg = smem + C::OFF_STG + (warp - 2) * 32 * C::STG_ROW;
    uint32_t it = 0;
    int cursor = 0;
    bool ok = true;
    for (int tile = tile_first; tile < n_tiles; tile += tile_step) {
      const TileCoord tc = decode_tile(tile, tile_prefix, p.n_tiles_n, cursor);
      const int mg = p.offsets ? p.offsets[tc.g + 1] - p.offsets[tc.g] : p.rows;
      const int local = tc.m_blk * C::TILE_M + static_cast<int>(rank) * BM + row_in_tile;
      const bool valid = local < mg;
      const long long row = static_cast<long long>(row0[tc.g]) + local;
      const float* sa = p.SA + row * n_kb;
      // the scales of the two halves' column blocks (a half beyond N: the last
      // block's, its columns are not stored)
      const int nb0 = MODE == QUANT_SWIGLU ? tc.n_blk : 2 * tc.n_blk;
      const int nb1 = MODE == QUANT_SWIGLU ? tc.n_blk : (2 * tc.n_blk + 1 < p.n_nb ? 2 * tc.n_blk + 1 : nb0);
      const float* sb0 = p.SB + (static_cast<long long>(tc.g) * p.n_nb + nb0) * n_kb;
      const float* sb1 =
          (MODE == QUANT_SWIGLU ? p.SB2 : p.SB) + (static_cast<long long>(tc.g) * p.n_nb + nb1) * n_kb;
      uint64_t acc[2][32];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[h][i] = 0;
      // scales one block ahead
      float a_next = valid ? sa[0] : 0.0f, b0_next = sb0[0], b1_next = sb1[0];
      for (int kb = 0; kb < n_kb && ok; ++kb, ++it) {
        const uint32_t buf = it & 1u, bph = (it >> 1) & 1u;
        const float f0 = a_next * b0_next, f1 = a_next * b1_next;
        if (kb + 1 < n_kb) {
          a_next = valid ? sa[kb + 1] : 0.0f;
          b0_next = sb0[kb + 1];
          b1_next = sb1[kb + 1];
        }
        const uint64_t ff[2] = {f32x2(f0, f0), f32x2(f1, f1)};
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&tfull[buf]), bph, budget, abort_flag, &g_fp8_error));
        if (!ok) break;
        tc_fence_after();
        const uint32_t t0 = t_row + buf * BN;
        // pieces of 16 columns, one in flight while the one before is added
        uint32_t r[2][16];
        tmem_ld16_nw(t0, r[0]);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          tmem_wait_for16(r[c & 1]);
          if (c + 1 < 8) tmem_ld16_nw(t0 + ((c + 1) >> 2) * HALF + ((c + 1) & 3) * 16, r[(c + 1) & 1]);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            acc[c >> 2][(c & 3) * 8 + i] =
                f32x2_fma(f32x2_bits(r[c & 1][2 * i], r[c & 1][2 * i + 1]), ff[c >> 2], acc[c >> 2][(c & 3) * 8 + i]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR) mbar_arrive_remote(release0 + 8 * buf);
          else mbar_arrive(release0 + 8 * buf);
        }
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
          float v[64];
          float m = 0.0f;
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float2 u = f32x2_get(acc[h][i]);
            if (MODE == QUANT_SWIGLU) {
              const float2 w = f32x2_get(acc[1][i]);
              u.x = silu_bf16out(u.x) * w.x;
              u.y = silu_bf16out(u.y) * w.y;
            } else {
              u.x = gelu_erf(u.x);
              u.y = gelu_erf(u.y);
            }
            v[2 * i] = u.x;
            v[2 * i + 1] = u.y;
            // columns beyond N belong to other weights: not part of the block
            if (col0 + 2 * i < p.N) m = fmaxf(m, fmaxf(fabsf(u.x), fabsf(u.y)));
          }
          s_max[part * BM + row_in_tile] = m;
          asm volatile("bar.sync %0, 64;" ::"r"(1 + q) : "memory");
          m = fmaxf(m, s_max[(part ^ 1) * BM + row_in_tile]);
          const Fp8Scale f = fp8_scale(m);
          const int nb = tc.n_blk * BLOCKS + h;
          if (valid && part == 0 && nb < p.n_nb) p.out_scale[row * p.n_nb + nb] = f.scale;
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<U4*>(stg + lane * 64 + ((j ^ ((lane >> 1) & 3)) * 16)) = fp8_pack16(v + 16 * j, f.inv);
          __syncwarp();
          uint8_t* o = static_cast<uint8_t*>(p.out) + col0;
#pragma unroll
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
      } else {
        constexpr int ES = MODE == STORE_F32 ? 4 : 2;
        constexpr int SLAB = 128 / ES;  // columns of one 128-byte row segment
        long long dest = row;
        float sc = 1.0f;
        bool put = valid;
        if (valid && p.perm) {
          dest = p.perm[row];
          if (dest < 0 || dest >= p.rows) {
            atomicOr(&g_fp8_error, 2u);
            put = false;
            dest = 0;
          } else if (p.row_scale) {
            sc = p.row_scale[dest];
          }
        }
        const unsigned pmask = __ballot_sync(0xffffffffu, put);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int sl = 0; sl < 64 / SLAB; ++sl) {
            const int col0 = tc.n_blk * BN + h * HALF + part * 64 + sl * SLAB;
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              U4 x;
              uint32_t w[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                if (MODE == STORE_F32) {
                  const float2 u = f32x2_get(acc[h][sl * 16 + j * 2 + (i >> 1)]);
                  w[i] = __float_as_uint((i & 1 ? u.y : u.x) * sc);
                } else {
                  const float2 u = f32x2_get(acc[h][(j * 4 + i) & 31]);
                  w[i] = pack_bf16x2(u.x * sc, u.y * sc);
                }
              }
              x = U4{w[0], w[1], w[2], w[3]};
              *reinterpret_cast<U4*>(stg + lane * 128 + ((j ^ (lane & 7)) * 16)) = x;
            }
            __syncwarp();
            const int seg = lane & 7;
            const int col = col0 + seg * (16 / ES);
#pragma unroll
            for (int pass = 0; pass < 8; ++pass) {
              const int rr = pass * 4 + (lane >> 3);
              const U4 x = *reinterpret_cast<const U4*>(stg + rr * 128 + ((seg ^ (rr & 7)) * 16));
              const long long drow = __shfl_sync(0xffffffffu, dest, rr);
              if (((pmask >> rr) & 1u) && col < p.N)
                *reinterpret_cast<U4*>(static_cast<uint8_t*>(p.out) + (drow * p.ldo + col) * ES) = x;
            }
          }
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  // PAIR: the even CTA's MMAs write both CTAs' TMEM; neither releases its
  // columns before both are done with them
  if (PAIR) cluster_sync_all();
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
  p.perm = a.perm;
  p.row_scale = a.row_scale;
  p.timeout = a.timeout_cycles;
  const long long tiles = (static_cast<long long>(a.rows) / C::TILE_M + a.G) * p.n_tiles_n;
  KernelScope ks(a.name, s);
  if (PAIR) {
    int clusters = max_clusters(kfn, NUM_THREADS, C::SMEM, 2);
    if (clusters < 1) return cudaErrorInvalidConfiguration;
    if (tiles < clusters) clusters = static_cast<int>(tiles);
    e = launch_cluster(fp8_gemm_kernel<MODE, PAIR>, clusters, 2, NUM_THREADS, (size_t)C::SMEM, s, mA, mB, mB2, p);
  } else {
    const int grid = static_cast<int>(tiles < sm_count() ? tiles : sm_count());
    e = launch_kernel(fp8_gemm_kernel<MODE, PAIR>, dim3(grid), dim3(NUM_THREADS), (size_t)C::SMEM, s, mA, mB, mB2, p);
  }
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

// 256-row tiles on CTA pairs where the expected rows per group waste at most a
// tenth more rows in them than in 128-row tiles.
bool use_pairs(const Fp8GemmArgs& a) {
  const long long per = a.rows / (a.g_active > 0 ? a.g_active : a.G);
  if (per < 2 * BM) return false;
  const long long pad1 = (per + BM - 1) / BM * BM, pad2 = (per + 2 * BM - 1) / (2 * BM) * (2 * BM);
  return 10 * pad2 <= 11 * pad1;
}

template <int MODE>
cudaError_t launch_mode(const Fp8GemmArgs& a, cudaStream_t s) {
  return use_pairs(a) ? launch_cfg<MODE, true>(a, s) : launch_cfg<MODE, false>(a, s);
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
