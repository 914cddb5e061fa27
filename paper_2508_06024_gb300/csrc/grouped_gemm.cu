// Products grouped by expert on bf16 operands and their gradients, on the sm_103a
// tensor cores.  Group g owns the rows [offsets[g], offsets[g + 1]) of the row
// matrices and the weights B_g [N, K]:
//
//   FWD    C_g  = A_g  B_g^T   [rows, N]   sum over K
//   DGRAD  dA_g = dC_g B_g     [rows, K]   sum over N
//   WGRAD  dB_g = dC_g^T A_g   [N, K]      sum over the group's rows
//
// One kernel.  The result's columns (contiguous in memory) are on the MMA's M side,
// 256 of them per CTA pair (cta_group::2, 128 per CTA), its rows on the N side: a
// group's rows are padded to multiples of 32 only.  A warp reads 32 consecutive
// columns (its TMEM lanes): an fp32 row of theirs is a whole line and is stored from
// registers, bf16 ones are transposed by stmatrix on the way.  The operands differ in which axis is contiguous:
// the sum's (K-major: B of FWD, A of FWD, dC of DGRAD) or the result's (MN-major: B of
// DGRAD, both of WGRAD).  tcgen05.mma reads either from 128-byte swizzled shared
// memory, so nothing is transposed on the way: a K-major tile is rows of 64 sum
// elements, an MN-major one chunks of 64 result elements by 64 sum rows.
//
// CTA layout:
//   warp 0       TMA producer
//   warp 1       TMEM allocator and MMA issuer (the even CTA's)
//   warps 2, 3   (WGRAD) zero the sum rows of a stage behind the group's end
//   16 warps     epilogue: warp w reads TMEM lanes 32 (w % 4) .. +31, every fourth
//                block of 16 result rows
//
// Ragged sums (WGRAD): a group's last 64-row block may hold rows of the next
// group, in both operands, and 0 times an infinity there would be NaN.  The MMAs
// stop at the 16-row step that holds the last row, and warp 2 or 3 overwrites that
// step's other rows with zeros once the block has landed, well before the MMAs
// get to it: such a block completes on a barrier of its own (tland), and the warp's
// arrival takes the place of the copies' on the stage's barrier.  The odd CTA's
// warp reports to the even one's (tpeer), which arrives for both.
//
// Sums: the tensor core adds into its fp32 accumulator without rounding to
// nearest, so sums are kept short: after `seg` blocks of 64 (8 for fp32 results, 128
// for bf16 ones) the accumulator is handed over and added to fp32 registers of
// the epilogue, while the next segment fills the other one.
//
// Split sums: where there are fewer tiles than CTA pairs the sum is cut into
// ranges.  Up to 4 are a cluster's pairs (CLUSTER): each pair leaves its sums where its
// operands were, and after a cluster barrier every pair adds up its share of the
// rows through distributed shared memory, in the order of the ranges.  More ranges
// write fp32 partial results to the workspace and a second kernel adds them in order.
//
// What bounds it: the tensor pipe for long sums and many rows, 91% busy (forward) and 90%
// (weights) of a 4096-row capture with 2 experts of 14336 x 4096; 16384 rows of 8 of them
// take 1163, 1200 and 1240 us back to back, under the power cap (forward, rows' gradient,
// weights' gradient; 1.65, 1.60 and 1.55 PFLOP/s), one call on a rested card 1052, 1109 and
// 1145 (1.83, 1.74 and 1.68).  With a few rows per expert the
// weights' bytes (32 rows of these experts: 142 us, 6.6 TB/s), for their gradient the
// result's (256 rows: 175 us, 5.4 TB/s; fp32 332 us, 5.7).  Short calls have about 6 us of
// launch, prologue and hand-overs around their blocks.
//
// Every wait is bounded: a wait that gives up sets the error word and the CTA's
// abort flag, waits for copies and MMAs in flight, frees its tensor memory and
// returns.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <mutex>

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

constexpr int BM = 128;  // columns of the result per CTA (MMA M is 256 over the pair)
constexpr int BN = 256;  // most rows of the result per tile (MMA N)
constexpr int BK = 64;   // sum elements per stage
constexpr int UK = 16;   // sum elements of one tcgen05.mma kind::f16
constexpr int CHUNK = 64 * BK * 2;  // bytes of an MN-major chunk: 64 sum rows of 128 bytes
constexpr int EPI_WARPS = 16;
constexpr int MAX_GROUPS = 128;
constexpr int BOX = 16;  // rows of the small box that short tiles' rows come in
// Tiles along the rows that are walked together (16384 rows of 8 experts of 14336 x 4096,
// gradient of the weights: 4 to 12 alike, 64 5% slower).
constexpr int BAND = 8;

enum Form { FWD = 0, DGRAD = 1, WGRAD = 2 };

// n / d for 0 <= n < 2^31 by a multiplication: with m = ceil(2^(32 + s) / d), s = ceil(log2 d)
// - 1, the quotient is floor(n m / 2^(32 + s)) (Granlund & Montgomery, 1994).  Every warp
// takes four quotients per tile; as divisions they were most of a short tile's
// instructions.
struct FastDiv {
  uint32_t m, s;
  __device__ __forceinline__ int operator()(int n) const {
    return m ? static_cast<int>(__umulhi(static_cast<uint32_t>(n), m) >> s) : n;
  }
};
FastDiv fast_div(int d) {
  if (d == 1) return FastDiv{0, 0};
  uint32_t s = 0;
  while ((1LL << (s + 1)) < d) ++s;
  const uint64_t m = ((1ULL << (32 + s)) + d - 1) / d;
  return FastDiv{static_cast<uint32_t>(m), s};
}

struct Params {
  const int32_t* offsets;  // [G + 1], nullptr: one group of all rows
  int G, rows;
  int cols;                // of the result
  int out_rows;            // WGRAD: rows of a group's result
  int depth;               // FWD, DGRAD: length of the sums
  int tiles_c, tiles_r;    // tiles along the columns; WGRAD: along the rows
  FastDiv by_split, by_group, by_band;  // ranges; WGRAD: tiles of a group; tiles of a band
  int split;               // ranges of the sum
  int out_bf16;            // CLUSTER: type of the result
  int seg;                 // blocks per segment
  const int32_t* perm;     // destination of each row (nullptr: itself); not with ranges in the workspace
  void* out;               // ranges in the workspace: fp32 [split][...], dense
  long long ldo;
  long long part_stride;   // elements between two ranges' partial results
  int accumulate;
  long long timeout;
};

constexpr int A_BYTES = BM * BK * 2;      // M side per CTA and stage
constexpr int B_BYTES = BN / 2 * BK * 2;  // N side, at most
constexpr int MAX_STAGES = 7;
// bf16 results: the last stage's place is where they are transposed, two blocks of 16
// rows x 64 bytes for every epilogue warp
__host__ __device__ constexpr int stages(bool f32) { return f32 ? MAX_STAGES : MAX_STAGES - 1; }
constexpr int STG_BLOCK = 16 * 64;
constexpr int OFF_STG = (MAX_STAGES - 1) * (A_BYTES + B_BYTES);
static_assert(2 * EPI_WARPS * STG_BLOCK <= A_BYTES + B_BYTES, "the blocks take the place of a stage");
constexpr int TMEM_COLS = 2 * BN;
// full, empty, tland, tpeer [MAX_STAGES]; tfull, tempty [2]; drain
constexpr int N_BARS = 4 * MAX_STAGES + 5;
constexpr int OFF_BARS = MAX_STAGES * (A_BYTES + B_BYTES);
constexpr int OFF_SLOT = OFF_BARS + N_BARS * 8;
constexpr int OFF_PREFIX = OFF_SLOT + 24;
constexpr int OFF_ROW0 = OFF_PREFIX + (MAX_GROUPS + 1) * 4;
constexpr int OFF_CNT = OFF_ROW0 + MAX_GROUPS * 4;
constexpr int SMEM = 1024 + OFF_CNT + MAX_GROUPS * 4;
static_assert(MAX_STAGES <= 16 && OFF_BARS % 8 == 0 && SMEM <= 232448, "shared memory per CTA");
constexpr int MAX_PAIRS = 4;  // of a cluster
static_assert(BN * BM * 4 <= OFF_BARS, "the sums take the operands' place");
constexpr int FIRST_EPI = 4;  // the first warpgroup loads, issues and zeroes
constexpr int THREADS = 32 * (FIRST_EPI + EPI_WARPS);
// Registers: 640 threads start with 96 each (61440); the epilogue takes what the first
// warpgroup gives up (128 * 56 + 512 * 104 = 60416).
constexpr int REGS_FEW = 56, REGS_EPI = 104;

struct Tile {
  int g, c, r0, n;   // group, column tile, first row (of the group, or of dB_g), rows
  int nn;            // rows that the MMAs compute: a multiple of 32
  int ks;            // range of the sum
  int kb0, kb1;      // its blocks
  int len;           // length of the whole sum
};

// Unit order: group, band of row tiles, column tile, row tile of the band, range.
// CTA pairs that run at the same time share the weights of a column tile and the
// band's rows in L2.
template <int FORM>
__device__ __forceinline__ Tile decode(const Params& p, int unit, const int* prefix, const int* cnt, int& cursor) {
  Tile t;
  int rem = p.by_split(unit);
  t.ks = unit - rem * p.split;
  int tiles_r, n_rows;
  if (FORM == WGRAD) {
    t.g = p.by_group(rem);
    rem -= t.g * (p.tiles_r * p.tiles_c);
    tiles_r = p.tiles_r;
    n_rows = p.out_rows;
    t.len = cnt[t.g];
  } else {
    while (rem >= prefix[cursor + 1] * p.tiles_c) ++cursor;
    t.g = cursor;
    rem -= prefix[cursor] * p.tiles_c;
    tiles_r = prefix[cursor + 1] - prefix[cursor];
    n_rows = cnt[t.g];
    t.len = p.depth;
  }
  const int band = p.by_band(rem);
  const int wide = min(BAND, tiles_r - band * BAND);
  rem -= band * (BAND * p.tiles_c);
  t.c = wide == BAND ? rem / BAND : rem / wide;
  t.r0 = (band * BAND + rem - t.c * wide) * BN;
  t.n = min(BN, n_rows - t.r0);
  t.nn = (t.n + 31) & ~31;
  const int n_kb = (t.len + BK - 1) / BK;
  const int per_split = p.by_split(n_kb + p.split - 1);
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

// As tma_load_2d_to_pair_bar, from a three-dimensional map.
__device__ __forceinline__ void load_3d_to_pair_bar(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, "
      "%3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void arrive_cluster(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// 16 TMEM lanes x 16 columns of 32-bit words, issue only: thread t receives, for each 8
// columns, those at 2 (t % 4) and the next of lane t / 4 and of lane t / 4 + 8: the layout
// of an 8 x 8 matrix's fragments.
__device__ __forceinline__ void tmem_ld_16x16_nw(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
// Waits for the TMEM loads so far; what they brought is used behind it, for the compiler
// too (a wait alone names no register).
template <int N>
__device__ __forceinline__ void tmem_wait_for(uint32_t* r) {
  tmem_wait();
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}
// Four 8 x 8 matrices of 16-bit elements, stored transposed: thread t names row t % 8 of
// matrix t / 8 (16 bytes).
__device__ __forceinline__ void store_4_transposed(uint32_t saddr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(saddr), "r"(a), "r"(b), "r"(c),
               "r"(d)
               : "memory");
}

// Arrives on the barrier at shared address `bar` in both CTAs of the pair whose even CTA
// has rank `lead` in the cluster, once the pair's MMAs issued so far have completed.
__device__ __forceinline__ void commit_to_pair(uint32_t bar, uint32_t lead) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
      "h"(static_cast<uint16_t>(0x3u << lead))
      : "memory");
}

// What the roles share.
struct Shared {
  uint8_t *sA, *sB;
  uint64_t *full, *empty, *tland, *tpeer, *tfull, *tempty, *drain;
  volatile int* abort_flag;
  // what the roles leave in flight when they end: [0] the producer's stages (low half)
  // and the phases that they complete, [1] the same of those that complete on tland, [2]
  // the lane + 1 of the MMA warp that issued MMAs
  volatile uint32_t* in_flight;
  int *prefix, *row0, *cnt;
};

template <int FORM>
__device__ __forceinline__ Tile decode_any(const Params& p, int unit, const int* prefix, const int* cnt) {
  int cursor = 0;
  return decode<FORM>(p, unit, prefix, cnt, cursor);
}

// CLUSTER: this CTA's columns of its pair's share of the tile's rows, from the sums that
// the pairs' CTAs of the same rank left at `sums` ([row][BM] fp32).  A warp takes a row.
template <int FORM>
__device__ __forceinline__ void join_ranges(const Params& p, const Tile& t, const Shared& sh, uint32_t sums, uint32_t cta) {
  const int warp = (threadIdx.x >> 5) - FIRST_EPI, lane = threadIdx.x & 31;
  const int piece = static_cast<int>(cta >> 1), share = (t.n + p.split - 1) / p.split;
  const int end = min(t.n, (piece + 1) * share);
  if (FORM == WGRAD && p.accumulate && t.len == 0) return;  // as it was, the sign of a zero too
  const int col = (t.c * 2 + static_cast<int>(cta & 1u)) * BM + lane * 4;
  uint32_t from[MAX_PAIRS];
#pragma unroll
  for (int s = 0; s < MAX_PAIRS; ++s) from[s] = map_to_rank(sums, s < p.split ? 2 * s + (cta & 1u) : cta) + lane * 16;
  for (int r = piece * share + warp; r < end; r += EPI_WARPS) {
    long long d = t.r0 + r;
    if (FORM == WGRAD) {
      d += static_cast<long long>(t.g) * p.out_rows;
    } else {
      d += sh.row0[t.g];
      if (p.perm) {
        d = p.perm[d];
        if (d < 0 || d >= p.rows) {
          if (lane == 0) atomicOr(&g_grouped_error, 2u);
          continue;
        }
      }
    }
    float4 x[MAX_PAIRS];
#pragma unroll
    for (int s = 0; s < MAX_PAIRS; ++s)
      if (s < p.split) x[s] = ld_cluster_v4(from[s] + r * (BM * 4));
    float4 v = x[0];
#pragma unroll
    for (int s = 1; s < MAX_PAIRS; ++s)
      if (s < p.split) v = make_float4(v.x + x[s].x, v.y + x[s].y, v.z + x[s].z, v.w + x[s].w);
    if (col >= p.cols) continue;
    if (p.out_bf16) {
      *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + d * p.ldo + col) =
          make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    } else {
      float4* to = reinterpret_cast<float4*>(static_cast<float*>(p.out) + d * p.ldo + col);
      if (FORM == WGRAD && p.accumulate) {
        const float4 o = *to;
        v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
      }
      *to = v;
    }
  }
}

template <int FORM, bool F32, bool PERM, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, 1)
    grouped_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                        const __grid_constant__ CUtensorMap tmBox, const Params p) {
  constexpr bool A_MN = FORM != FWD, B_MN = FORM == WGRAD;
  constexpr int STAGES = stages(F32);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Shared sh;
  sh.sA = smem;
  sh.sB = smem + STAGES * A_BYTES;
  sh.full = reinterpret_cast<uint64_t*>(smem + OFF_BARS);
  sh.empty = sh.full + STAGES;
  sh.tland = sh.empty + STAGES;
  sh.tpeer = sh.tland + STAGES;
  sh.tfull = sh.tpeer + STAGES;
  sh.tempty = sh.tfull + 2;
  sh.drain = sh.tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + OFF_SLOT);
  sh.abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  sh.in_flight = tmem_slot + 2;
  sh.prefix = reinterpret_cast<int*>(smem + OFF_PREFIX);
  sh.row0 = reinterpret_cast<int*>(smem + OFF_ROW0);
  sh.cnt = reinterpret_cast<int*>(smem + OFF_CNT);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  static_assert(!CLUSTER || (F32 && !PERM), "the ranges' sums are fp32 and have their own way out");
  // Rank in the CTA pair, the even CTA's rank in the cluster.  CLUSTER: the cluster has one
  // tile, or none, and each of its pairs a range.
  const uint32_t cta = cluster_ctarank();
  const uint32_t rank = cta & 1u, lead = CLUSTER ? cta & ~1u : 0u;
  const int unit_first = static_cast<int>(cluster_id_x()) * (CLUSTER ? p.split : 1) + (CLUSTER ? static_cast<int>(cta >> 1) : 0);
  const int unit_step = CLUSTER ? 1 << 29 : static_cast<int>(cluster_count_x());
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
      mbar_init(smem_u32(&sh.tempty[b]), 2 * EPI_WARPS);
    }
    mbar_init(smem_u32(sh.drain), 1);
    *sh.abort_flag = 0;
    sh.in_flight[0] = sh.in_flight[1] = sh.in_flight[2] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 0) {
    pdl_wait();
    scan_group_rows<(MAX_GROUPS + 31) / 32, BN>(p.offsets, p.G, p.rows, lane, sh.row0, sh.cnt, sh.prefix, &g_grouped_error);
  }
  if (warp == 2 && lane == 0) {
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
    if (FORM != WGRAD) tma_prefetch_desc(&tmBox);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  // both CTAs' barriers are initialised before either arrives remotely
  cluster_sync_all();
  tc_fence_after();
  pdl_wait();
  const uint32_t tmem_base = *tmem_slot;
  const int n_units = (FORM == WGRAD ? p.G * p.tiles_r : sh.prefix[p.G]) * p.tiles_c * p.split;
  const long long budget = p.timeout;

  if (warp < FIRST_EPI) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_FEW));
    if (warp == 0) {
      // ---------------------------------------------------------------- producer
      const bool issue = elect_one();
      int stage = 0;
      uint32_t phase = 0;
      uint32_t issued = 0, issued_phase = 0;  // bit s: stage s holds a copy, the phase that it completes
      uint32_t tailed = 0, tailed_phase = 0;  // the same for copies that complete on tland
      uint32_t tail_phase = 0;                // tland's next phase
      int cursor = 0;
      bool ok = true;
      for (int unit = unit_first; unit < n_units && ok; unit += unit_step) {
        const Tile t = decode<FORM>(p, unit, sh.prefix, sh.cnt, cursor);
        const int row0 = sh.row0[t.g];
        const int c0 = t.c * 2 * BM + static_cast<int>(rank) * BM;  // this CTA's columns
        const int half = t.nn / 2;                                  // and its half of the rows
        const int r0 = t.r0 + static_cast<int>(rank) * half;
        const int b_bytes = B_MN ? (half + 63) / 64 * CHUNK : half * BK * 2;
        for (int kb = t.kb0; kb < t.kb1; ++kb) {
          if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&sh.empty[stage]), phase ^ 1u, budget, sh.abort_flag, &g_grouped_error))) {
            ok = false;
            break;
          }
          const int k0 = kb * BK;
          const bool tail = FORM == WGRAD && t.len - k0 < BK && t.len % UK != 0;
          if (issue) {
            const uint32_t da = smem_u32(sh.sA + stage * A_BYTES), db = smem_u32(sh.sB + stage * B_BYTES);
            if (FORM == WGRAD && tail) {
              const uint32_t bar = smem_u32(&sh.tland[stage]);
              mbar_expect_tx(bar, A_BYTES + b_bytes);
              for (int c = 0; c < BM / 64; ++c) tma_load_2d(da + c * CHUNK, &tmA, c0 + c * 64, row0 + k0, bar);
              for (int c = 0; c * 64 < half; ++c) tma_load_2d(db + c * CHUNK, &tmB, r0 + c * 64, row0 + k0, bar);
            } else {
              uint32_t bar = smem_u32(&sh.full[stage]);
              // both CTAs' copies complete on the even CTA's barrier
              if (rank == 0) mbar_expect_tx(bar, 2 * (A_BYTES + b_bytes));
              else bar = map_to_rank(bar, lead);
              if (FORM == WGRAD) {
#pragma unroll
                for (int c = 0; c < BM / 64; ++c) tma_load_2d_to_pair_bar(da + c * CHUNK, &tmA, c0 + c * 64, row0 + k0, bar);
                for (int c = 0; c * 64 < half; ++c) tma_load_2d_to_pair_bar(db + c * CHUNK, &tmB, r0 + c * 64, row0 + k0, bar);
              } else {
                if (FORM == FWD) {
                  load_3d_to_pair_bar(da, &tmA, k0, c0, t.g, bar);
                } else {
#pragma unroll
                  for (int c = 0; c < BM / 64; ++c) load_3d_to_pair_bar(da + c * CHUNK, &tmA, c0 + c * 64, k0, t.g, bar);
                }
                if (half == BN / 2) {
                  tma_load_2d_to_pair_bar(db, &tmB, k0, row0 + r0, bar);
                } else {
                  for (int b = 0; b < half; b += BOX) tma_load_2d_to_pair_bar(db + b * (BK * 2), &tmBox, k0, row0 + r0 + b, bar);
                }
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
      if (rank == 0) {
        // -------------------------------------------------------------- MMA issuer
        const bool issue = elect_one();
        constexpr uint32_t IDESC0 = idesc_bf16(2 * BM, 0) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u);
        // the address field's step per 16 sum elements: 32 bytes of a row, or 16 rows
        constexpr uint64_t STEP_A = A_MN ? 16 * 128 / 16 : 2, STEP_B = B_MN ? 16 * 128 / 16 : 2;
        const uint64_t da0 = A_MN ? sdesc_mn(smem_u32(sh.sA)) : sdesc_sw128(smem_u32(sh.sA));
        const uint64_t db0 = B_MN ? sdesc_mn(smem_u32(sh.sB)) : sdesc_sw128(smem_u32(sh.sB));
        int stage = 0;
        uint32_t phase = 0;
        uint32_t it = 0;  // segments so far: accumulator it & 1
        int cursor = 0;
        bool ok = true, any = false;
        for (int unit = unit_first; unit < n_units && ok; unit += unit_step) {
          const Tile t = decode<FORM>(p, unit, sh.prefix, sh.cnt, cursor);
          const uint32_t idesc = IDESC0 | (static_cast<uint32_t>(t.nn >> 3) << 17);
          for (int s0 = t.kb0; s0 < t.kb1 && ok; s0 += p.seg, ++it) {
            const uint32_t acc = it & 1u, acc_phase = (it >> 1) & 1u;
            if (!__all_sync(0xffffffffu, mbar_wait_cluster(smem_u32(&sh.tempty[acc]), acc_phase ^ 1u, budget, sh.abort_flag,
                                                           &g_grouped_error))) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint32_t d = tmem_base + acc * BN;
            const int s1 = min(s0 + p.seg, t.kb1);
            for (int kb = s0; kb < s1; ++kb) {
              const uint32_t fb = smem_u32(&sh.full[stage]);
              const bool there = FORM == WGRAD ? mbar_wait_cluster(fb, phase, budget, sh.abort_flag, &g_grouped_error)
                                               : mbar_wait(fb, phase, budget, sh.abort_flag, &g_grouped_error);
              if (!__all_sync(0xffffffffu, there)) {
                ok = false;
                break;
              }
              tc_fence_after();
              const uint64_t da = da0 + static_cast<uint64_t>(stage) * (A_BYTES >> 4);
              const uint64_t db = db0 + static_cast<uint64_t>(stage) * (B_BYTES >> 4);
              const int left = t.len - kb * BK;
              if (issue) {
#pragma unroll
                for (int kk = 0; kk < BK / UK; ++kk) {
                  if (FORM == WGRAD && kk * UK >= left) break;
                  umma_bf16_pair(d, da + kk * STEP_A, db + kk * STEP_B, idesc, kb != s0 || kk != 0 ? 1u : 0u);
                }
                commit_to_pair(smem_u32(&sh.empty[stage]), lead);
              }
              any = true;
              if (++stage == STAGES) {
                stage = 0;
                phase ^= 1u;
              }
            }
            if (ok && issue) commit_to_pair(smem_u32(&sh.tfull[acc]), lead);
          }
        }
        if (any && issue) sh.in_flight[2] = lane + 1;
      }
    } else {
      if (FORM == WGRAD) {
        // ------------------------------------------------- rows behind a group's end
        // The two warps share the stages, even and odd ones: a block's zeroes, fence and
        // hand-over between the CTAs take about as long as a short unit.  Every such block of
        // a stage is one warp's, so that it has seen a phase of the stage's barriers before the
        // next one can begin: a phase's parity alone does not tell it from the one before.
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
          if ((stage & 1u) != static_cast<uint32_t>(warp - 2)) continue;
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
            for (int c = 0; c < BM / 64; ++c) *reinterpret_cast<U4*>(sh.sA + stage * A_BYTES + c * CHUNK + at) = U4{0, 0, 0, 0};
            for (int c = 0; c * 64 < t.nn / 2; ++c)
              *reinterpret_cast<U4*>(sh.sB + stage * B_BYTES + c * CHUNK + at) = U4{0, 0, 0, 0};
          }
          asm volatile("fence.proxy.async;" ::: "memory");
          __syncwarp();
          if (rank != 0) {
            if (lane == 0) arrive_cluster(map_to_rank(smem_u32(&sh.tpeer[stage]), lead));
            continue;
          }
          if (!__all_sync(0xffffffffu,
                          mbar_wait_cluster(smem_u32(&sh.tpeer[stage]), ph, budget, sh.abort_flag, &g_grouped_error))) {
            ok = false;
            break;
          }
          if (lane == 0) arrive_cluster(smem_u32(&sh.full[stage]));
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_EPI));
    // ---------------------------------------------------------------- epilogue
    // A warp has 32 result columns (its TMEM lanes) and the blocks of 16 rows part, part +
    // 4, part + 8, part + 12.  fp32: a thread's column is its TMEM lane.  bf16: fragments of
    // 8 x 8 matrices, 8 columns by 8 rows.
    const int q = warp & 3;
    const int part = (warp - FIRST_EPI) >> 2;
    constexpr int NB = BN / 64;  // blocks of a warp
    uint32_t it = 0;
    int cursor = 0;
    auto load_block = [&](uint32_t lanes, int b, uint32_t* r) {
      if constexpr (F32) {
        tmem_ld16_nw(lanes + b * 64, r);
      } else {
        tmem_ld_16x16_nw(lanes + b * 64, r);
        tmem_ld_16x16_nw(lanes + b * 64 + (16u << 16), r + 8);
      }
    };
    for (int unit = unit_first; unit < n_units; unit += unit_step) {
      const Tile t = decode<FORM>(p, unit, sh.prefix, sh.cnt, cursor);
      if (!CLUSTER && t.kb0 >= t.kb1 && (FORM != WGRAD || p.split > 1 || p.accumulate)) continue;  // nothing to add
      const int first = FORM == WGRAD ? t.r0 : sh.row0[t.g] + t.r0;
      // With a perm: destinations (-1: none).  fp32: lane l those of the rows l % 16 of the
      // warp's blocks l / 16 and 2 + l / 16.  bf16: of the rows l / 4 and 8 + l / 4 of each block.
      int dst[NB][2];
      if constexpr (PERM) {
#pragma unroll
        for (int b = 0; b < (F32 ? 1 : NB); ++b) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int r = F32 ? (part + 4 * (2 * h + (lane >> 4))) * 16 + (lane & 15) : (part + 4 * b) * 16 + 8 * h + (lane >> 2);
            dst[b][h] = r < t.n ? p.perm[first + r] : -1;
            if (r < t.n && (dst[b][h] < 0 || dst[b][h] >= p.rows)) {
              atomicOr(&g_grouped_error, 2u);
              dst[b][h] = -1;
            }
          }
        }
      }
      float v[NB][16];
      bool ok = true;
      // the first segment comes straight into the sums, those behind it are added
      auto arrived = [&] {
        const bool here = __all_sync(0xffffffffu, mbar_wait_strict(smem_u32(&sh.tfull[it & 1u]), (it >> 1) & 1u, budget,
                                                                   sh.abort_flag, &g_grouped_error));
        tc_fence_after();
        return here;
      };
      auto release = [&] {
        tc_fence_before();
        __syncwarp();
        // both CTAs release the accumulator on the even CTA's barrier
        if (lane == 0) mbar_arrive_remote(map_to_rank(smem_u32(&sh.tempty[it & 1u]), lead));
        ++it;
      };
      const uint32_t lanes = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + part * 16;
      if (t.kb0 < t.kb1) {
        ok = arrived();
        if (!ok) break;
        uint32_t r[NB][16];
#pragma unroll
        for (int b = 0; b < NB; ++b) load_block(lanes + (it & 1u) * BN, b, r[b]);
        tmem_wait_for<NB * 16>(&r[0][0]);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) v[b][i] = __uint_as_float(r[b][i]);
        release();
      } else {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) v[b][i] = 0.0f;
      }
#pragma unroll 1
      for (int s0 = t.kb0 + p.seg; s0 < t.kb1; s0 += p.seg) {
        ok = arrived();
        if (!ok) break;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          uint32_t r[16];
          load_block(lanes + (it & 1u) * BN, b, r);
          tmem_wait_for<16>(r);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[b][i] += __uint_as_float(r[i]);
        }
        release();
      }
      if (!ok) break;
      const int col0 = t.c * 2 * BM + static_cast<int>(rank) * BM + q * 32;
      if constexpr (CLUSTER) {
        // the operands' place is free: the last MMAs have read them
        float* sums = reinterpret_cast<float*>(smem) + q * 32 + lane;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if ((part + 4 * b) * 16 >= t.n) break;  // the whole warp
#pragma unroll
          for (int i = 0; i < 16; ++i) sums[((part + 4 * b) * 16 + i) * BM] = v[b][i];
        }
      } else if constexpr (F32) {
        const int col = col0 + lane;
        const bool held = col < p.cols;
        float* out = static_cast<float*>(p.out) + t.ks * p.part_stride + col;
        if (FORM == WGRAD) out += static_cast<long long>(t.g) * p.out_rows * p.ldo;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if ((part + 4 * b) * 16 >= t.n) break;  // the whole warp
          // a row of the warp: 128 contiguous bytes
          if constexpr (PERM) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int d = __shfl_sync(0xffffffffu, dst[0][b >> 1], (b & 1) * 16 + i);
              if (d >= 0 && held) out[d * p.ldo] = v[b][i];
            }
            continue;
          }
          float* to = out + (first + (part + 4 * b) * 16) * p.ldo;
          const int n = held ? t.n - (part + 4 * b) * 16 : 0;
#pragma unroll
          for (int i = 0; i < 16; i += 4, to += 4 * p.ldo) {
            if (FORM == WGRAD && p.accumulate) {
              float o[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) o[j] = i + j < n ? to[j * p.ldo] : 0.0f;
#pragma unroll
              for (int j = 0; j < 4; ++j) v[b][i + j] += o[j];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (i + j < n) to[j * p.ldo] = v[b][i + j];
          }
        }
      } else {
        // A block of 16 rows x 32 columns is transposed through shared memory (rows of 64
        // bytes, their 16-byte pieces permuted so that no side meets a bank twice) and
        // stored 8 rows at a time, 16 bytes per lane.  Packed in registers and stored two
        // columns per lane, a tile took 600 instructions per warp: 211 us for 256 rows of 8
        // experts of 14336 x 4096.
        const uint32_t stg = smem_u32(smem + OFF_STG) + (warp - FIRST_EPI) * 2 * STG_BLOCK;
        const uint32_t put = stg + (lane & 7) * 64 + (((lane >> 3) ^ ((lane >> 1) & 3)) * 16);
        const uint32_t get = stg + (lane >> 2) * 64 + (((lane & 3) ^ ((lane >> 3) & 3)) * 16);
        const bool held = col0 + (lane & 3) * 8 < p.cols;
        // packed at once, which leaves half the registers (16384 rows of 8 experts of 4096 x
        // 512, forward: 58 us without it, 50 with it)
        uint32_t w[NB][8];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 8; ++i) w[b][i] = pack_bf16x2(v[b][2 * i], v[b][2 * i + 1]);
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + col0 + (lane & 3) * 8;
        if (FORM == WGRAD) out += static_cast<long long>(t.g) * p.out_rows * p.ldo;
        const int r0 = part * 16 + (lane >> 2);
        if (!PERM) out += (first + r0) * p.ldo;
        const long long step = p.ldo * 8;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if ((part + 4 * b) * 16 >= t.n) break;  // the whole warp
#pragma unroll
          for (int k = 0; k < 2; ++k)  // 8 rows each
            store_4_transposed(put + (b & 1) * STG_BLOCK + k * 512, w[b][2 * k], w[b][2 * k + 1], w[b][2 * k + 4],
                               w[b][2 * k + 5]);
          __syncwarp();
          U4 o[2];
#pragma unroll
          for (int h = 0; h < 2; ++h)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(o[h].x), "=r"(o[h].y), "=r"(o[h].z), "=r"(o[h].w)
                         : "r"(get + (b & 1) * STG_BLOCK + h * 512)
                         : "memory");
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if constexpr (PERM) {
              if (held && dst[b][h] >= 0) *reinterpret_cast<U4*>(out + dst[b][h] * p.ldo) = o[h];
            } else {
              if (held && r0 + 64 * b + 8 * h < t.n) *reinterpret_cast<U4*>(out + (8 * b + h) * step) = o[h];
            }
          }
        }
        __syncwarp();
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  // the even CTA's MMAs read both CTAs' shared memory and write both CTAs' TMEM;
  // neither is released before both CTAs are done with them, nor, where a wait of either
  // gave up, before what is in flight has ended
  if (CLUSTER) {
    // all of the cluster agree: they meet at further barriers
    if (threadIdx.x < 2 * p.split && threadIdx.x != cta && *sh.abort_flag)
      asm volatile("st.shared::cluster.s32 [%0], 1;" ::"r"(
                       map_to_rank(smem_u32(const_cast<int*>(sh.abort_flag)), threadIdx.x))
                   : "memory");
  } else if (threadIdx.x == 0) {
    abort_pair(sh.abort_flag, rank);
  }
  __syncwarp();
  cluster_sync_all();
  if (*sh.abort_flag) {  // no warp waits any more: the same in all of them, and in the pair
    if (warp == 0) {
      const uint32_t copies = sh.in_flight[0], tails = sh.in_flight[1];
      if (rank == 0) drain_copies(smem_u32(sh.full), copies & 0xffffu, copies >> 16);
      else if (copies) wait_for_remote_copies();
      drain_copies(smem_u32(sh.tland), tails & 0xffffu, tails >> 16);
    } else if (warp == 1 && sh.in_flight[2] == lane + 1u) {
      // the thread that issued the MMAs: a commit covers its own
      umma_commit_pair(smem_u32(sh.drain));
      mbar_drain(smem_u32(sh.drain), 0, DRAIN_CYCLES);
    }
    __syncthreads();
    __syncwarp();
    cluster_sync_all();
  } else if (CLUSTER && warp >= FIRST_EPI && unit_first < n_units) {
    join_ranges<FORM>(p, decode_any<FORM>(p, unit_first, sh.prefix, sh.cnt), sh, smem_u32(smem), cta);
  }
  if (CLUSTER) {  // no CTA ends while another reads its sums
    __syncwarp();
    cluster_sync_all();
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
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

// How a call's sums are cut.
struct Plan {
  int split;     // ranges
  bool cluster;  // the pairs of a cluster each
};

template <int FORM>
int clusters_of(int split) {
  auto kernel = grouped_gemm_kernel<FORM, true, false, true>;
  const void* kfn = reinterpret_cast<const void*>(kernel);
  return ensure_smem_attr(kfn, SMEM) == cudaSuccess ? max_clusters(kfn, THREADS, SMEM, 2 * split) : 0;
}

// The least of
//   waves * blocks of a range * 0.27 us, or what HBM needs if that is more,
//   + for ranges in a cluster 2 us, for ranges in the workspace 4.6 us and the partial
//   results' way there and back
// (0.27 us: a block of 64 of one tile at full clock; the others fitted to 700 x 512 x
// 4096 in the workspace: one range 27 us, four 19, seven 17; 700 x 4096 x 4096: 27, two 41;
// the gradient of 512 x 4096 weights over 8191 rows: 48, two 40, four 45; 32 rows of 8
// experts of 4096 x 14336, bound by HBM: 139, two 160).  Ragged rows: the tiles are
// expected ones.
Plan plan_of(int form, int G, int rows, int N, int K) {
  const int pairs = sm_count() / 2;
  const int cols = form == FWD ? N : K;
  const double tiles_c = (cols + 2 * BM - 1) / (2 * BM);
  const int held = G < rows ? G : rows;  // groups with rows, at most
  double tiles, out, bytes;
  int n_kb;
  if (form == WGRAD) {
    tiles = tiles_c * G * ((N + BN - 1) / BN);
    out = static_cast<double>(G) * N * K;
    n_kb = rows < G ? 1 : (rows / G + BK - 1) / BK;  // fewer rows than groups: those with one have a block
    bytes = 2.0 * rows * (static_cast<double>(N) + K) + 2.0 * out;
  } else {
    tiles = tiles_c * (rows < held * BN ? held : rows / BN + 0.5 * held);
    out = static_cast<double>(rows) * cols;
    n_kb = ((form == FWD ? K : N) + BK - 1) / BK;
    bytes = 2.0 * rows * (static_cast<double>(N) + K) + 2.0 * held * N * static_cast<double>(K);
  }
  const double hbm = bytes / 6.4e6;  // us
  Plan best{1, false};
  double least = 0.0;
  for (int s = 1; s <= GROUPED_MAX_SPLIT && (s == 1 || s * 4 <= n_kb); ++s) {
    const int per = (n_kb + s - 1) / s;
    if ((n_kb + per - 1) / per != s) continue;  // no empty range (FWD, DGRAD)
    for (int cluster = 0; cluster < 2; ++cluster) {
      if (cluster && (s == 1 || s > MAX_PAIRS || tiles * s > pairs)) continue;
      int at_once = pairs / s;
      if (cluster) at_once = form == FWD ? clusters_of<FWD>(s) : form == DGRAD ? clusters_of<DGRAD>(s) : clusters_of<WGRAD>(s);
      if (cluster && at_once < 1) continue;
      const double waves = cluster ? ceil(tiles / at_once) : ceil(tiles * s / pairs);
      const double mma = waves * per * 0.27;
      const double us = (mma > hbm ? mma : hbm) + (s == 1 ? 0.0 : cluster ? 2.0 : 4.6 + s * out * 8.0 / 5e6);
      if (least == 0.0 || us < least) {
        best = Plan{s, cluster != 0};
        least = us;
      }
    }
  }
  return best;
}

template <int FORM, bool F32, bool PERM, bool CLUSTER>
cudaError_t launch(const GroupedArgs& a, int split, cudaStream_t s) {
  auto kernel = grouped_gemm_kernel<FORM, F32, PERM, CLUSTER>;
  const void* kfn = reinterpret_cast<const void*>(kernel);
  cudaError_t e = ensure_smem_attr(kfn, SMEM);
  if (e != cudaSuccess) return e;
  CUtensorMap mA, mB, mBox;
  bool good;
  if (FORM == WGRAD) {
    good = encode(&mA, a.W, 0, a.rows, a.K, a.ldw, BK) && encode(&mB, a.X, 0, a.rows, a.N, a.ldx, BK);
    mBox = mB;
  } else {
    const int depth = FORM == FWD ? a.K : a.N;
    good = encode(&mA, a.W, a.G, a.N, a.K, a.K, FORM == FWD ? BM : BK) &&
           encode(&mB, a.X, 0, a.rows, depth, a.ldx, BN / 2) && encode(&mBox, a.X, 0, a.rows, depth, a.ldx, BOX);
  }
  if (!good) return cudaErrorInvalidValue;
  const bool parts = split > 1 && !CLUSTER;
  Params p{};
  p.offsets = a.offsets;
  p.G = a.G;
  p.rows = a.rows;
  p.cols = FORM == FWD ? a.N : a.K;
  p.out_rows = a.N;
  p.depth = FORM == FWD ? a.K : a.N;
  p.tiles_c = (p.cols + 2 * BM - 1) / (2 * BM);
  p.tiles_r = (a.N + BN - 1) / BN;
  p.split = split;
  p.by_split = fast_div(split);
  p.by_group = fast_div(p.tiles_r * p.tiles_c);
  p.by_band = fast_div(BAND * p.tiles_c);
  p.out_bf16 = a.out_bf16;
  p.seg = F32 ? 8 : 128;
  p.perm = parts ? nullptr : a.perm;
  p.out = parts ? a.workspace : a.out;
  p.ldo = parts ? p.cols : a.ldo;
  p.part_stride = parts ? (FORM == WGRAD ? static_cast<long long>(a.G) * a.N : a.rows) * static_cast<long long>(p.cols) : 0;
  p.accumulate = parts ? 0 : a.accumulate;
  p.timeout = a.timeout_cycles;
  const long long row_tiles = FORM == WGRAD ? static_cast<long long>(a.G) * p.tiles_r : a.rows / BN + a.G;
  const long long units = row_tiles * p.tiles_c * p.split;
  int clusters;
  if (CLUSTER) {
    clusters = static_cast<int>(units / split);  // one tile each, at most
  } else {
    clusters = max_clusters(kfn, THREADS, SMEM, 2);
    if (clusters < 1) return cudaErrorInvalidConfiguration;
    if (units < clusters) clusters = static_cast<int>(units);
  }
  {
    KernelScope ks(a.name, s);
    e = launch_cluster(kernel, clusters, CLUSTER ? 2 * split : 2, THREADS, (size_t)SMEM, s, mA, mB, mBox, p);
    if (e != cudaSuccess) return e;
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (!parts) return cudaSuccess;
  JoinParams j{};
  j.offsets = a.offsets;
  j.G = a.G;
  j.rows = a.rows;
  j.N = p.cols;
  j.split = split;
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
  if (plan.cluster) return launch<FORM, true, false, true>(a, plan.split, s);
  if (plan.split > 1) return launch<FORM, true, false, false>(a, plan.split, s);
  if constexpr (FORM != WGRAD) {
    if (a.perm) return a.out_bf16 ? launch<FORM, false, true, false>(a, 1, s) : launch<FORM, true, true, false>(a, 1, s);
  }
  return a.out_bf16 ? launch<FORM, false, false, false>(a, 1, s) : launch<FORM, true, false, false>(a, 1, s);
}

}  // namespace

size_t grouped_bytes(int form, int G, int rows, int N, int K) {
  const Plan plan = plan_of(form, G, rows, N, K);
  if (plan.split == 1 || plan.cluster) return 0;
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
