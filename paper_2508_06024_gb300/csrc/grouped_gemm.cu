// Products grouped by expert on bf16 operands and their gradients, on the sm_103a
// tensor cores.  Group g owns the rows [offsets[g], offsets[g + 1]) of the row
// matrices and the weights B_g [N, K]:
//
//   FWD    C_g  = A_g  B_g^T   [rows, N]   sum over K
//   DGRAD  dA_g = dC_g B_g     [rows, K]   sum over N
//   WGRAD  dB_g = dC_g^T A_g   [N, K]      sum over the group's rows
//
// One kernel, whose operands differ in which axis is contiguous in memory: the
// sum's (K-major: A and B of FWD, dC of DGRAD) or the result's (MN-major: B of
// DGRAD, both of WGRAD).  tcgen05.mma reads either from 128-byte swizzled shared
// memory, so nothing is transposed on the way: a K-major tile is rows of 64 sum
// elements, an MN-major one chunks of 64 result elements by 64 sum rows.
//
// CTA layout:
//   warp 0       TMA producer
//   warp 1       TMEM allocator and MMA issuer
//   warp 2       (WGRAD) zeroes the sum rows of a stage behind the group's end
//   16 warps     epilogue: warp w reads TMEM lanes 32 (w % 4) .. +31; the four
//                warps of a lane quadrant share the tile's columns and stage
//                slabs of 128-byte row segments for the stores
// CTA pairs: a cluster of two CTAs computes a 256-row tile with cta_group::2; each
// stages its own 128 rows of the M operand and half of the N operand.  The even
// CTA issues the MMAs.
//
// Ragged sums (WGRAD): a group's last 64-row block may hold rows of the next
// group, in both operands, and 0 times an infinity there would be NaN.  The MMAs
// stop at the 16-row step that holds the last row, and warp 2 overwrites that
// step's other rows with zeros once the block has landed, well before the MMAs
// get to it: such a block completes on a barrier of its own (tland), and warp 2's
// arrival takes the place of the copies' on the stage's barrier.  In a pair the
// odd CTA's warp 2 reports to the even one's (tpeer), which arrives for both.
//
// Sums: the tensor core adds into its fp32 accumulator without rounding to
// nearest, so sums are kept short: after SEG blocks of 64 (4 for fp32 results, 128
// for bf16 ones) the accumulator is handed over and added to fp32 registers of
// the epilogue, while the next segment fills the other one.
//
// Split sums: where there are fewer tiles than CTA pairs the sum is cut into
// ranges; each writes fp32 partial results to the workspace and a second kernel
// adds them in order.
//
// Every wait is bounded: a wait that gives up sets the error word and the CTA's
// abort flag, waits for copies and MMAs in flight, frees its tensor memory and
// returns.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <mutex>
#include <type_traits>

#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"
#include "tc_ptx.cuh"

namespace ec2moe {

// bit 0: a bounded wait timed out; bit 1: a group range (offsets) or a scatter
// destination (perm) outside the rows of the call was skipped
__device__ unsigned int g_grouped_error;

namespace {

using namespace tc;

constexpr int BM = 128;  // tile rows of a CTA (MMA M, TMEM lanes)
constexpr int BK = 64;   // sum elements per stage
constexpr int UK = 16;   // sum elements of one tcgen05.mma kind::f16
constexpr int CHUNK = 64 * BK * 2;  // bytes of an MN-major chunk: 64 sum rows of 128 bytes
constexpr int EPI_WARPS = 16;
constexpr int MAX_GROUPS = 136;
constexpr int SHORT_ROWS = 32;  // rows of the small box that short tiles' A operand comes in

enum Form { FWD = 0, DGRAD = 1, WGRAD = 2 };

struct Params {
  const int32_t* offsets;  // [G + 1], nullptr: one group of all rows
  int G, rows;
  int M, N, K;             // of the tile's product: M only for WGRAD, K for FWD and DGRAD
  int tiles_m, tiles_n;    // tiles_m: WGRAD
  int split;               // ranges of the sum
  int seg;                 // blocks per segment
  const int32_t* perm;     // destination of each row (nullptr: itself); not with split > 1
  void* out;               // split > 1: fp32 [split][...], dense
  long long ldo;
  long long part_stride;   // elements between two ranges' partial results
  int accumulate;
  long long timeout;
};

template <int FORM, bool F32, bool PAIR, int BN>
struct Cfg {
  static constexpr bool A_MN = FORM == WGRAD, B_MN = FORM != FWD;
  static constexpr int TILE_M = PAIR ? 2 * BM : BM;
  static constexpr int B_ROWS = PAIR ? BN / 2 : BN;  // columns of the tile whose operand this CTA stages
  static constexpr int A_BYTES = BM * BK * 2;
  static constexpr int B_BYTES = B_ROWS * BK * 2;
  static constexpr int STAGE_BYTES = A_BYTES + B_BYTES;
  static constexpr int STAGES = 196608 / STAGE_BYTES;
  static constexpr int FIRST_EPI = FORM == WGRAD ? 3 : 2;
  static constexpr int THREADS = 32 * (FIRST_EPI + EPI_WARPS);
  static constexpr int CPT = BN / 4;                 // columns per epilogue thread
  static constexpr int SLAB = F32 ? 32 : 64;         // columns of a staged slab: 128 bytes
  static constexpr int CW = SLAB / 4;                // of which a warp stages so many
  static constexpr int N_SLABS = BN / SLAB;
  static constexpr int TMEM_COLS = 2 * BN;
  // full, empty, tland, tpeer [STAGES]; tfull, tempty [2]; drain
  static constexpr int N_BARS = 4 * STAGES + 5;
  static constexpr int OFF_BARS = STAGES * STAGE_BYTES;
  static constexpr int OFF_SLOT = OFF_BARS + N_BARS * 8;
  static constexpr int OFF_PREFIX = OFF_SLOT + 24;
  static constexpr int OFF_ROW0 = OFF_PREFIX + (MAX_GROUPS + 1) * 4;
  static constexpr int OFF_CNT = OFF_ROW0 + MAX_GROUPS * 4;
  static constexpr int OFF_STG = (OFF_CNT + MAX_GROUPS * 4 + 127) / 128 * 128;
  static constexpr int STG_BYTES = 2 * 4 * 32 * 128;  // two slabs of 32 rows per lane quadrant
  static constexpr int SMEM = 1024 + OFF_STG + STG_BYTES;
  static_assert(BN == 128 || BN == 256, "two accumulators are a power of two of TMEM columns");
  static_assert(STAGES <= 16 && OFF_BARS % 8 == 0 && SMEM <= 232448, "shared memory per CTA");
};

struct Tile {
  int g, m, n, ks;   // group, row and column of the tile, range of the sum
  int kb0, kb1;      // its blocks
  int len;           // length of the whole sum
};

template <int FORM>
__device__ __forceinline__ Tile decode(const Params& p, int unit, const int* prefix, const int* cnt, int& cursor) {
  Tile t;
  t.ks = unit % p.split;
  const int tile = unit / p.split;
  if (FORM == WGRAD) {
    const int per = p.tiles_m * p.tiles_n;
    t.g = tile / per;
    const int rem = tile - t.g * per;
    t.m = rem % p.tiles_m;
    t.n = rem / p.tiles_m;
    t.len = cnt[t.g];
  } else {
    while (tile >= prefix[cursor + 1] * p.tiles_n) ++cursor;
    const int mt = prefix[cursor + 1] - prefix[cursor];
    const int rem = tile - prefix[cursor] * p.tiles_n;
    t.g = cursor;
    t.m = rem % mt;
    t.n = rem / mt;
    t.len = p.K;
  }
  const int n_kb = (t.len + BK - 1) / BK;
  const int per_split = (n_kb + p.split - 1) / p.split;
  t.kb0 = min(t.ks * per_split, n_kb);
  t.kb1 = min(t.kb0 + per_split, n_kb);
  return t;
}

// MN-major operand tile: chunks of 64 result elements (128 bytes, swizzled) by 64
// sum rows, CHUNK bytes apart (leading offset, bits 16-29); 8 sum rows are 1024
// bytes (stride offset, bits 32-45).  Other fields as sdesc_sw128.
__device__ __forceinline__ uint64_t sdesc_mn(uint32_t saddr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(CHUNK >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}

// A copy whose completion is counted on `bar`: this CTA's, or (TO_PAIR) a
// shared::cluster address that may be the pair's even CTA's.
template <bool TO_PAIR>
__device__ __forceinline__ void load_2d(uint32_t dst, const CUtensorMap* tm, int x, int y, uint32_t bar) {
  if (TO_PAIR) tma_load_2d_to_pair_bar(dst, tm, x, y, bar);
  else tma_load_2d(dst, tm, x, y, bar);
}
template <bool TO_PAIR>
__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar) {
  if (TO_PAIR)
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, "
        "%3, %4}], [%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], "
        "[%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void arrive_cluster(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// Bytes of A that arrive for `held` rows of a CTA's 128: a whole box, or short ones.
__device__ __forceinline__ int a_boxes(int held) { return held <= 0 ? 0 : (min(held, BM) + SHORT_ROWS - 1) / SHORT_ROWS; }

// What the roles share.
struct Shared {
  uint8_t *sA, *sB, *stg;
  uint64_t *full, *empty, *tland, *tpeer, *tfull, *tempty, *drain;
  volatile int* abort_flag;
  // what the roles leave in flight when they end: [0] the producer's stages (low half)
  // and the phases that they complete, [1] the same of those that complete on tland, [2]
  // the lane + 1 of the MMA warp that issued MMAs
  volatile uint32_t* in_flight;
  int *prefix, *row0, *cnt;
};

template <int FORM, bool F32, bool PAIR, int BN>
__global__ void __launch_bounds__((Cfg<FORM, F32, PAIR, BN>::THREADS), 1)
    grouped_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmShort,
                        const __grid_constant__ CUtensorMap tmB, const Params p) {
  using C = Cfg<FORM, F32, PAIR, BN>;
  constexpr int STAGES = C::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Shared sh;
  sh.sA = smem;
  sh.sB = smem + STAGES * C::A_BYTES;
  sh.stg = smem + C::OFF_STG;
  sh.full = reinterpret_cast<uint64_t*>(smem + C::OFF_BARS);
  sh.empty = sh.full + STAGES;
  sh.tland = sh.empty + STAGES;
  sh.tpeer = sh.tland + STAGES;
  sh.tfull = sh.tpeer + STAGES;
  sh.tempty = sh.tfull + 2;
  sh.drain = sh.tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_SLOT);
  sh.abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  sh.in_flight = tmem_slot + 2;
  sh.prefix = reinterpret_cast<int*>(smem + C::OFF_PREFIX);
  sh.row0 = reinterpret_cast<int*>(smem + C::OFF_ROW0);
  sh.cnt = reinterpret_cast<int*>(smem + C::OFF_CNT);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
  const int unit_first = PAIR ? static_cast<int>(cluster_id_x()) : static_cast<int>(blockIdx.x);
  const int unit_step = PAIR ? static_cast<int>(cluster_count_x()) : static_cast<int>(gridDim.x);
  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&sh.full[s]), 1);
      mbar_init(smem_u32(&sh.empty[s]), 1);
      mbar_init(smem_u32(&sh.tland[s]), 1);
      mbar_init(smem_u32(&sh.tpeer[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&sh.tfull[b]), 1);
      mbar_init(smem_u32(&sh.tempty[b]), PAIR ? 2 * EPI_WARPS : EPI_WARPS);
    }
    mbar_init(smem_u32(sh.drain), 1);
    *sh.abort_flag = 0;
    sh.in_flight[0] = sh.in_flight[1] = sh.in_flight[2] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 0) {
    pdl_wait();
    scan_group_rows<(MAX_GROUPS + 31) / 32, C::TILE_M>(p.offsets, p.G, p.rows, lane, sh.row0, sh.cnt, sh.prefix,
                                                       &g_grouped_error);
    if (lane == 0) {
      tma_prefetch_desc(&tmA);
      tma_prefetch_desc(&tmB);
    }
  }
  if (warp == 1) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                   "r"(C::TMEM_COLS)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                   "r"(C::TMEM_COLS)
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
  const int n_units = (FORM == WGRAD ? p.G * p.tiles_m : sh.prefix[p.G]) * p.tiles_n * p.split;
  const long long budget = p.timeout;

  if (warp == 0) {
    // ---------------------------------------------------------------- producer
    const bool issue = elect_one();
    int stage = 0;
    uint32_t phase = 0;
    uint32_t issued = 0, issued_phase = 0;  // bit s: stage s holds a copy, the phase that it completes
    uint32_t tailed = 0, tail_phase = 0;    // the same for copies that complete on tland; tail_phase: its next
    uint32_t tailed_phase = 0;
    int cursor = 0;
    bool ok = true;
    for (int unit = unit_first; unit < n_units && ok; unit += unit_step) {
      const Tile t = decode<FORM>(p, unit, sh.prefix, sh.cnt, cursor);
      const int r0 = sh.row0[t.g], n_rows = sh.cnt[t.g];
      const int m0 = t.m * C::TILE_M + static_cast<int>(rank) * BM;
      const int n0 = t.n * BN + static_cast<int>(rank) * C::B_ROWS;
      // boxes of A: of this CTA, of the pair
      const int mine = C::A_MN ? 0 : a_boxes(n_rows - m0);
      const int both = C::A_MN ? 0 : PAIR ? a_boxes(n_rows - t.m * C::TILE_M) + a_boxes(n_rows - t.m * C::TILE_M - BM) : mine;
      for (int kb = t.kb0; kb < t.kb1; ++kb) {
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.empty[stage]), phase ^ 1u, budget, sh.abort_flag, &g_grouped_error))) {
          ok = false;
          break;
        }
        const int k0 = kb * BK;
        const bool tail = FORM == WGRAD && (t.len - k0 < BK) && (t.len % UK != 0);
        if (issue) {
          const uint32_t da = smem_u32(sh.sA + stage * C::A_BYTES), db = smem_u32(sh.sB + stage * C::B_BYTES);
          if (FORM == WGRAD) {
            uint32_t bar;
            if (tail) {
              bar = smem_u32(&sh.tland[stage]);
              mbar_expect_tx(bar, C::STAGE_BYTES);
            } else {
              bar = smem_u32(&sh.full[stage]);
              if (rank == 0) mbar_expect_tx(bar, (PAIR ? 2 : 1) * C::STAGE_BYTES);
              else bar = map_to_rank(bar, 0);
            }
#pragma unroll
            for (int c = 0; c < BM / 64; ++c) {
              if (PAIR && !tail) load_2d<true>(da + c * CHUNK, &tmA, m0 + c * 64, r0 + k0, bar);
              else load_2d<false>(da + c * CHUNK, &tmA, m0 + c * 64, r0 + k0, bar);
            }
#pragma unroll
            for (int c = 0; c < C::B_ROWS / 64; ++c) {
              if (PAIR && !tail) load_2d<true>(db + c * CHUNK, &tmB, n0 + c * 64, r0 + k0, bar);
              else load_2d<false>(db + c * CHUNK, &tmB, n0 + c * 64, r0 + k0, bar);
            }
          } else {
            uint32_t bar = smem_u32(&sh.full[stage]);
            if (rank == 0) mbar_expect_tx(bar, (PAIR ? 2 : 1) * C::B_BYTES + both * (SHORT_ROWS * BK * 2));
            else bar = map_to_rank(bar, 0);
            if (mine == BM / SHORT_ROWS) {
              load_2d<PAIR>(da, &tmA, k0, r0 + m0, bar);
            } else {
              for (int b = 0; b < mine; ++b)
                load_2d<PAIR>(da + b * (SHORT_ROWS * BK * 2), &tmShort, k0, r0 + m0 + b * SHORT_ROWS, bar);
            }
            if (FORM == FWD) {
              load_3d<PAIR>(db, &tmB, k0, n0, t.g, bar);
            } else {
#pragma unroll
              for (int c = 0; c < C::B_ROWS / 64; ++c) load_3d<PAIR>(db + c * CHUNK, &tmB, n0 + c * 64, k0, t.g, bar);
            }
          }
        }
        const uint32_t bit = 1u << stage;
        if (tail) {
          issued &= ~bit;
          tailed |= bit;
          tailed_phase = (tailed_phase & ~bit) | (tail_phase & bit);
          tail_phase ^= bit;
        } else {
          tailed &= ~bit;
          issued |= bit;
          issued_phase = (issued_phase & ~bit) | (phase << stage);
        }
        if (++stage == STAGES) {
          stage = 0;
          phase ^= 1u;
        }
      }
    }
    if (lane == 0) {
      sh.in_flight[0] = issued | (issued_phase << 16);
      sh.in_flight[1] = tailed | (tailed_phase << 16);
    }
  } else if (warp == 1) {
    if (!PAIR || rank == 0) {
      // -------------------------------------------------------------- MMA issuer
      const bool issue = elect_one();
      constexpr uint32_t IDESC =
          idesc_bf16(C::TILE_M, BN) | (C::A_MN ? 1u << 15 : 0u) | (C::B_MN ? 1u << 16 : 0u);
      // the address field's step per 16 sum elements: 32 bytes of a row, or 16 rows
      constexpr uint64_t STEP_A = C::A_MN ? 16 * 128 / 16 : 2, STEP_B = C::B_MN ? 16 * 128 / 16 : 2;
      const uint64_t da0 = C::A_MN ? sdesc_mn(smem_u32(sh.sA)) : sdesc_sw128(smem_u32(sh.sA));
      const uint64_t db0 = C::B_MN ? sdesc_mn(smem_u32(sh.sB)) : sdesc_sw128(smem_u32(sh.sB));
      int stage = 0;
      uint32_t phase = 0;
      uint32_t it = 0;  // segments so far: accumulator it & 1
      int cursor = 0;
      bool ok = true, any = false;
      for (int unit = unit_first; unit < n_units && ok; unit += unit_step) {
        const Tile t = decode<FORM>(p, unit, sh.prefix, sh.cnt, cursor);
        for (int s0 = t.kb0; s0 < t.kb1 && ok; s0 += p.seg, ++it) {
          const uint32_t acc = it & 1u, acc_phase = (it >> 1) & 1u;
          const uint32_t tempty = smem_u32(&sh.tempty[acc]);
          const bool freed = PAIR ? mbar_wait_cluster(tempty, acc_phase ^ 1u, budget, sh.abort_flag, &g_grouped_error)
                                  : mbar_wait(tempty, acc_phase ^ 1u, budget, sh.abort_flag, &g_grouped_error);
          if (!__all_sync(0xffffffffu, freed)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t d = tmem_base + acc * BN;
          const int s1 = min(s0 + p.seg, t.kb1);
          for (int kb = s0; kb < s1; ++kb) {
            const uint32_t fb = smem_u32(&sh.full[stage]);
            const bool there = FORM == WGRAD && PAIR
                                   ? mbar_wait_cluster(fb, phase, budget, sh.abort_flag, &g_grouped_error)
                                   : mbar_wait(fb, phase, budget, sh.abort_flag, &g_grouped_error);
            if (!__all_sync(0xffffffffu, there)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint64_t da = da0 + static_cast<uint64_t>(stage) * (C::A_BYTES >> 4);
            const uint64_t db = db0 + static_cast<uint64_t>(stage) * (C::B_BYTES >> 4);
            const int left = t.len - kb * BK;
            if (issue) {
#pragma unroll
              for (int kk = 0; kk < BK / UK; ++kk) {
                if (FORM == WGRAD && kk * UK >= left) break;
                const uint32_t add = kb != s0 || kk != 0 ? 1u : 0u;
                if (PAIR) umma_bf16_pair(d, da + kk * STEP_A, db + kk * STEP_B, IDESC, add);
                else umma_bf16(d, da + kk * STEP_A, db + kk * STEP_B, IDESC, add);
              }
              if (PAIR) umma_commit_pair_mc(smem_u32(&sh.empty[stage]));
              else umma_commit(smem_u32(&sh.empty[stage]));
            }
            any = true;
            if (++stage == STAGES) {
              stage = 0;
              phase ^= 1u;
            }
          }
          if (ok && issue) {
            if (PAIR) umma_commit_pair_mc(smem_u32(&sh.tfull[acc]));
            else umma_commit(smem_u32(&sh.tfull[acc]));
          }
        }
      }
      if (any && issue) sh.in_flight[2] = lane + 1;
    }
  } else if (FORM == WGRAD && warp == 2) {
    // ------------------------------------------------- rows behind a group's end
    uint32_t blocks = 0;      // so far
    uint32_t tail_phase = 0;  // bit s: phase of stage s's tland and tpeer
    int cursor = 0;
    bool ok = true;
    for (int unit = unit_first; unit < n_units && ok; unit += unit_step) {
      const Tile t = decode<FORM>(p, unit, sh.prefix, sh.cnt, cursor);
      blocks += static_cast<uint32_t>(t.kb1 - t.kb0);
      const int left = t.len - (t.kb1 - 1) * BK;
      if (t.kb1 <= t.kb0 || left >= BK || left % UK == 0) continue;
      const uint32_t stage = (blocks - 1) % STAGES, bit = 1u << stage;
      const uint32_t ph = (tail_phase & bit) ? 1u : 0u;
      tail_phase ^= bit;
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.tland[stage]), ph, budget, sh.abort_flag, &g_grouped_error))) {
        ok = false;
        break;
      }
      // rows [left, end) of every chunk: 8 lanes per 128-byte row (the swizzle
      // permutes within a row)
      const int end = (left + UK - 1) / UK * UK;
      for (int r = left + (lane >> 3); r < end; r += 4) {
        const int at = r * 128 + (lane & 7) * 16;
#pragma unroll
        for (int c = 0; c < BM / 64; ++c)
          *reinterpret_cast<U4*>(sh.sA + stage * C::A_BYTES + c * CHUNK + at) = U4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < C::B_ROWS / 64; ++c)
          *reinterpret_cast<U4*>(sh.sB + stage * C::B_BYTES + c * CHUNK + at) = U4{0, 0, 0, 0};
      }
      asm volatile("fence.proxy.async;" ::: "memory");
      __syncwarp();
      if (PAIR && rank != 0) {
        if (lane == 0) arrive_cluster(map_to_rank(smem_u32(&sh.tpeer[stage]), 0));
        continue;
      }
      if (PAIR && !__all_sync(0xffffffffu, mbar_wait_cluster(smem_u32(&sh.tpeer[stage]), ph, budget, sh.abort_flag,
                                                             &g_grouped_error))) {
        ok = false;
        break;
      }
      if (lane == 0) arrive_cluster(smem_u32(&sh.full[stage]));
    }
  } else {
    // ---------------------------------------------------------------- epilogue
    const int q = warp & 3;                        // TMEM lane quadrant this warp may access
    const int part = (warp - C::FIRST_EPI) >> 2;   // which part of a slab's columns
    uint8_t* stg = sh.stg + q * (32 * 128);
    using OutT = typename std::conditional<F32, float, __nv_bfloat16>::type;
    constexpr int VEC = 16 / sizeof(OutT);         // columns of a 16-byte store
    uint32_t it = 0;
    int cursor = 0;
    for (int unit = unit_first; unit < n_units; unit += unit_step) {
      const Tile t = decode<FORM>(p, unit, sh.prefix, sh.cnt, cursor);
      const int local = t.m * C::TILE_M + static_cast<int>(rank) * BM + q * 32 + lane;  // row of the group, or of dB_g
      bool valid;
      long long dest;
      if (FORM == WGRAD) {
        if (t.kb0 >= t.kb1 && (p.split > 1 || p.accumulate)) continue;  // nothing to add
        valid = local < p.M;
        dest = static_cast<long long>(t.g) * p.M + local;
      } else {
        valid = local < sh.cnt[t.g];
        dest = sh.row0[t.g] + local;
        if (t.kb0 >= t.kb1) continue;  // an empty range of a split sum
        if (valid && p.perm) {
          dest = p.perm[dest];
          if (dest < 0 || dest >= p.rows) {
            atomicOr(&g_grouped_error, 2u);
            valid = false;
            dest = 0;
          }
        }
      }
      float v[C::CPT];
      bool ok = true;
      if (t.kb0 >= t.kb1) {
#pragma unroll
        for (int i = 0; i < C::CPT; ++i) v[i] = 0.0f;
      }
      for (int s0 = t.kb0; s0 < t.kb1; s0 += p.seg, ++it) {
        const uint32_t acc = it & 1u, acc_phase = (it >> 1) & 1u;
        if (!__all_sync(0xffffffffu,
                        mbar_wait(smem_u32(&sh.tfull[acc]), acc_phase, budget, sh.abort_flag, &g_grouped_error))) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t at = tmem_base + acc * BN + (static_cast<uint32_t>(q * 32) << 16) + part * C::CW;
        if (s0 == t.kb0) {
          uint32_t r[C::CPT];
#pragma unroll
          for (int sl = 0; sl < C::N_SLABS; ++sl) {
            if (F32) tmem_ld8_nw(at + sl * C::SLAB, r + sl * C::CW);
            else tmem_ld16_nw(at + sl * C::SLAB, r + sl * C::CW);
          }
          tmem_wait();
#pragma unroll
          for (int i = 0; i < C::CPT; ++i) v[i] = __uint_as_float(r[i]);
        } else {
#pragma unroll
          for (int sl = 0; sl < C::N_SLABS; ++sl) {
            uint32_t r[C::CW];
            if (F32) tmem_ld8_nw(at + sl * C::SLAB, r);
            else tmem_ld16_nw(at + sl * C::SLAB, r);
            tmem_wait();
#pragma unroll
            for (int i = 0; i < C::CW; ++i) v[sl * C::CW + i] += __uint_as_float(r[i]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          // PAIR: both CTAs release the accumulator on the even CTA's barrier
          if (PAIR) mbar_arrive_remote(map_to_rank(smem_u32(&sh.tempty[acc]), 0));
          else mbar_arrive(smem_u32(&sh.tempty[acc]));
        }
      }
      {
        // the quadrant's four warps take the same path (they meet at named barriers)
        uint32_t all_ok;
        asm volatile(
            "{\n .reg .pred p, r;\n setp.ne.u32 p, %1, 0;\n"
            " bar.red.and.pred r, %2, 128, p;\n selp.u32 %0, 1, 0, r;\n}"
            : "=r"(all_ok)
            : "r"(ok ? 1u : 0u), "r"(1 + q)
            : "memory");
        if (!all_ok) break;
      }
      OutT* out = static_cast<OutT*>(p.out) + t.ks * p.part_stride;
      const int seg = lane & 7;
#pragma unroll
      for (int sl = 0; sl < C::N_SLABS; ++sl) {
        uint8_t* slab = stg + (sl & 1) * (4 * 32 * 128);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float* w = v + sl * C::CW + j * VEC;
          U4 q4;
          if constexpr (F32)
            q4 = U4{__float_as_uint(w[0]), __float_as_uint(w[1]), __float_as_uint(w[2]), __float_as_uint(w[3])};
          else
            q4 = U4{pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]), pack_bf16x2(w[4], w[5]), pack_bf16x2(w[6], w[7])};
          *reinterpret_cast<U4*>(slab + lane * 128 + (((2 * part + j) ^ (lane & 7)) * 16)) = q4;
        }
        asm volatile("bar.sync %0, 128;" ::"r"(1 + q) : "memory");
        const int col = t.n * BN + sl * C::SLAB + seg * VEC;
#pragma unroll
        for (int pass = 0; pass < 2; ++pass) {
          const int rr = part * 8 + pass * 4 + (lane >> 3);
          const bool rvalid = __shfl_sync(0xffffffffu, valid ? 1 : 0, rr) != 0;
          const long long drow = __shfl_sync(0xffffffffu, dest, rr);
          U4 q4 = *reinterpret_cast<const U4*>(slab + rr * 128 + ((seg ^ (rr & 7)) * 16));
          if (rvalid && col < p.N) {
            U4* to = reinterpret_cast<U4*>(out + drow * p.ldo + col);
            if (F32 && FORM == WGRAD && p.accumulate) {
              const float4 o = *reinterpret_cast<const float4*>(to);
              q4 = U4{__float_as_uint(__uint_as_float(q4.x) + o.x), __float_as_uint(__uint_as_float(q4.y) + o.y),
                      __float_as_uint(__uint_as_float(q4.z) + o.z), __float_as_uint(__uint_as_float(q4.w) + o.w)};
            }
            *to = q4;
          }
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  // PAIR: the even CTA's MMAs read both CTAs' shared memory and write both CTAs' TMEM;
  // neither is released before both CTAs are done with them, nor, where a wait of either
  // gave up, before what is in flight has ended
  if (PAIR) {
    if (threadIdx.x == 0) abort_pair(sh.abort_flag, rank);
    __syncwarp();
    cluster_sync_all();
  }
  if (*sh.abort_flag) {  // no warp waits any more: the same in all of them, and in the pair
    if (warp == 0) {
      const uint32_t copies = sh.in_flight[0], tails = sh.in_flight[1];
      if (rank == 0) drain_copies(smem_u32(sh.full), copies & 0xffffu, copies >> 16);
      else if (copies) wait_for_remote_copies();
      drain_copies(smem_u32(sh.tland), tails & 0xffffu, tails >> 16);
    } else if (warp == 1 && sh.in_flight[2] == lane + 1u) {
      // the thread that issued the MMAs: a commit covers its own
      if (PAIR) umma_commit_pair(smem_u32(sh.drain));
      else umma_commit(smem_u32(sh.drain));
      mbar_drain(smem_u32(sh.drain), 0, DRAIN_CYCLES);
    }
    __syncthreads();
    __syncwarp();
    if (PAIR) cluster_sync_all();
  }
  if (warp == 1) {
    tc_fence_after();
    if (PAIR)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::TMEM_COLS)
                   : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::TMEM_COLS)
                   : "memory");
  }
}

// ------------------------------------------------------------------ split sums
struct JoinParams {
  const int32_t* offsets;
  int G, rows, N;         // N: columns of the result
  int split;
  int wgrad_rows;         // WGRAD: rows of a group's result (0: FWD, DGRAD)
  const float* part;
  long long part_stride;
  const int32_t* perm;
  void* out;
  long long ldo;
  int accumulate;
};

// out = part[0] + part[1] + ..: rows of the groups (through perm) or the groups' dB.
template <bool F32>
__global__ void __launch_bounds__(256) grouped_join_kernel(const JoinParams p) {
  pdl_trigger();
  pdl_wait();
  __shared__ int row0[MAX_GROUPS], cnt[MAX_GROUPS], prefix[MAX_GROUPS + 1];
  if (threadIdx.x < 32)
    scan_group_rows<(MAX_GROUPS + 31) / 32, 1>(p.offsets, p.G, p.rows, threadIdx.x, row0, cnt, prefix, nullptr);
  __syncthreads();
  const int quads = p.N / 4;
  const long long n_rows = p.wgrad_rows ? static_cast<long long>(p.G) * p.wgrad_rows : prefix[p.G];
  const long long n = n_rows * quads;
  for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < n; i += 256LL * gridDim.x) {
    const long long r = i / quads;
    const int col = static_cast<int>(i - r * quads) * 4;
    long long src = r, dest = r;
    int ranges = p.split;
    if (p.wgrad_rows) {
      const int n_kb = (cnt[r / p.wgrad_rows] + BK - 1) / BK;
      const int per = (n_kb + p.split - 1) / p.split;
      ranges = per ? (n_kb + per - 1) / per : 0;
      if (ranges == 0 && p.accumulate) continue;
    } else {
      int lo = 0, hi = p.G;  // prefix[lo] <= r < prefix[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (prefix[mid] <= r) lo = mid;
        else hi = mid;
      }
      src = row0[lo] + (r - prefix[lo]);
      dest = p.perm ? p.perm[src] : src;
      if (dest < 0 || dest >= p.rows) {
        atomicOr(&g_grouped_error, 2u);
        continue;
      }
    }
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float* from = p.part + src * p.N + col;
    for (int s = 0; s < ranges; ++s) {
      const float4 x = *reinterpret_cast<const float4*>(from + s * p.part_stride);
      v = make_float4(v.x + x.x, v.y + x.y, v.z + x.z, v.w + x.w);
    }
    if (F32) {
      float4* to = reinterpret_cast<float4*>(static_cast<float*>(p.out) + dest * p.ldo + col);
      if (p.accumulate) {
        const float4 o = *to;
        v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
      }
      *to = v;
    } else {
      *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + dest * p.ldo + col) =
          make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    }
  }
}

// ------------------------------------------------------------------ host side
PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
  });
  return fn;
}

// bf16 [mats, rows, cols], rows `ld` elements apart (matrices dense), box 64 columns x
// box_rows rows of one matrix, 128-byte swizzle, zero fill out of bounds.  mats = 0: a
// two-dimensional map.
bool encode(CUtensorMap* m, const void* ptr, int mats, long long rows, long long cols, long long ld, int box_rows) {
  auto fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(mats)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(ld) * 2 * rows};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_rows), 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, mats ? 3 : 2, const_cast<void*>(ptr), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a call is cut: columns per tile, ranges of the sum.
struct Plan {
  int bn, split;
};

// `tiles_m` tiles of 256 rows (an estimate for ragged rows), `cols` columns, sums of
// `n_kb` blocks; out_elems: elements of the result.
Plan make_plan(double tiles_m, int cols, long long n_kb, double out_elems, int clusters) {
  (void)out_elems;
  (void)tiles_m;
  (void)cols;
  (void)n_kb;
  (void)clusters;
  return Plan{256, 1};
}

Plan plan_of(int form, int G, int rows, int N, int K) {
  const int clusters = sm_count() / 2;
  if (form == WGRAD) {
    const double tiles = static_cast<double>(G) * ((N + 255) / 256);
    return make_plan(tiles, K, (rows / G + BK - 1) / BK, static_cast<double>(G) * N * K, clusters);
  }
  const int cols = form == FWD ? N : K;
  const double tiles = rows / 256.0 + (G < rows ? G : rows) * (G > 1 ? 0.5 : 1.0);
  return make_plan(tiles, cols, ((form == FWD ? K : N) + BK - 1) / BK, static_cast<double>(rows) * cols, clusters);
}

template <int FORM, bool F32, int BN>
cudaError_t launch(const GroupedArgs& a, const Plan& plan, cudaStream_t s) {
  constexpr bool PAIR = true;
  using C = Cfg<FORM, F32, PAIR, BN>;
  const void* kfn = reinterpret_cast<const void*>(grouped_gemm_kernel<FORM, F32, PAIR, BN>);
  cudaError_t e = ensure_smem_attr(kfn, C::SMEM);
  if (e != cudaSuccess) return e;
  CUtensorMap mA, mShort, mB;
  bool good;
  if (FORM == WGRAD) {
    good = encode(&mA, a.X, 0, a.rows, a.N, a.ldx, 64) && encode(&mB, a.W, 0, a.rows, a.K, a.ldw, 64);
    mShort = mA;
  } else {
    const int depth = FORM == FWD ? a.K : a.N;
    good = encode(&mA, a.X, 0, a.rows, depth, a.ldx, BM) && encode(&mShort, a.X, 0, a.rows, depth, a.ldx, SHORT_ROWS) &&
           encode(&mB, a.W, a.G, a.N, a.K, a.K, FORM == FWD ? C::B_ROWS : BK);
  }
  if (!good) return cudaErrorInvalidValue;
  Params p{};
  p.offsets = a.offsets;
  p.G = a.G;
  p.rows = a.rows;
  p.M = a.N;
  p.N = FORM == FWD ? a.N : a.K;
  p.K = FORM == FWD ? a.K : a.N;
  p.tiles_m = (a.N + C::TILE_M - 1) / C::TILE_M;
  p.tiles_n = (p.N + BN - 1) / BN;
  p.split = plan.split;
  p.seg = F32 ? 4 : 128;
  p.perm = plan.split > 1 ? nullptr : a.perm;
  p.out = plan.split > 1 ? a.workspace : a.out;
  p.ldo = plan.split > 1 ? p.N : a.ldo;
  p.part_stride = plan.split > 1 ? (FORM == WGRAD ? static_cast<long long>(a.G) * a.N : a.rows) * static_cast<long long>(p.N) : 0;
  p.accumulate = plan.split > 1 ? 0 : a.accumulate;
  p.timeout = a.timeout_cycles;
  long long units = (FORM == WGRAD ? static_cast<long long>(a.G) * p.tiles_m : a.rows / C::TILE_M + a.G) * p.tiles_n * p.split;
  int clusters = max_clusters(kfn, C::THREADS, C::SMEM, 2);
  if (clusters < 1) return cudaErrorInvalidConfiguration;
  if (units < clusters) clusters = static_cast<int>(units < 1 ? 1 : units);
  {
    KernelScope ks(a.name, s);
    e = launch_cluster(grouped_gemm_kernel<FORM, F32, PAIR, BN>, clusters, 2, C::THREADS, (size_t)C::SMEM, s, mA, mShort, mB, p);
    if (e != cudaSuccess) return e;
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (plan.split == 1) return cudaSuccess;
  JoinParams j{};
  j.offsets = a.offsets;
  j.G = a.G;
  j.rows = a.rows;
  j.N = p.N;
  j.split = plan.split;
  j.wgrad_rows = FORM == WGRAD ? a.N : 0;
  j.part = static_cast<const float*>(a.workspace);
  j.part_stride = p.part_stride;
  j.perm = a.perm;
  j.out = a.out;
  j.ldo = a.ldo;
  j.accumulate = a.accumulate;
  const long long quads = p.part_stride / 4;
  const long long most = 8LL * sm_count();
  const long long grid = (quads + 255) / 256 < most ? (quads + 255) / 256 : most;
  KernelScope ks("grouped_join", s);
  e = a.out_bf16 ? launch_kernel(grouped_join_kernel<false>, dim3(static_cast<unsigned>(grid)), dim3(256), 0, s, j)
                 : launch_kernel(grouped_join_kernel<true>, dim3(static_cast<unsigned>(grid)), dim3(256), 0, s, j);
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

template <int FORM>
cudaError_t launch_form(const GroupedArgs& a, cudaStream_t s) {
  const Plan plan = plan_of(FORM, a.G, a.rows, a.N, a.K);
  const bool f32 = !a.out_bf16 || plan.split > 1;
  if (plan.bn == 256) return f32 ? launch<FORM, true, 256>(a, plan, s) : launch<FORM, false, 256>(a, plan, s);
  return f32 ? launch<FORM, true, 128>(a, plan, s) : launch<FORM, false, 128>(a, plan, s);
}

}  // namespace

size_t grouped_bytes(int form, int G, int rows, int N, int K) {
  const Plan plan = plan_of(form, G, rows, N, K);
  if (plan.split == 1) return 0;
  const size_t out = form == GROUPED_WGRAD ? static_cast<size_t>(G) * N * K
                                           : static_cast<size_t>(rows) * (form == GROUPED_FWD ? N : K);
  return plan.split * out * 4;
}

cudaError_t launch_grouped(const GroupedArgs& a, int form, cudaStream_t s) {
  if (form == GROUPED_FWD) return launch_form<FWD>(a, s);
  if (form == GROUPED_DGRAD) return launch_form<DGRAD>(a, s);
  return launch_form<WGRAD>(a, s);
}

cudaError_t read_grouped_error(unsigned int* word) {
  unsigned int zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(word, g_grouped_error, sizeof(unsigned int));
  if (e != cudaSuccess) return e;
  return cudaMemcpyToSymbol(g_grouped_error, &zero, sizeof(unsigned int));
}

}  // namespace ec2moe
