// The grouped product of 8-bit operands for groups of few rows: the weights on
// the MMA's M side (128 weight rows fill the TMEM lanes), a group's rows on its N
// side, ROWS at a time.
//
// Such calls are bounded by streaming the weights of the groups that hold rows
// once.  All their K blocks, tile after tile, form one line that is cut into as
// many equal pieces as there are CTAs, one per SM, wherever the cuts fall
// (experts of 14336 x 4096, 2 rows: 14336 blocks, 94 or 95 per CTA; whole tiles
// would be 2.9 waves, run as 3).  A stage carries a block of 16 KB of weights and
// the group's rows; about 180 KB are in flight per SM.  The scaled sums of a CTA's
// part of a tile go to the workspace in fp32, and a second kernel adds the parts
// of each tile in order: to the output (optionally scattered and scaled by row),
// or through the activation, quantised again.
//
// CTA (256 threads): warp 0 loads, warp 1 issues the MMAs, warp 2 copies scales
// ahead, warps 4..7 add every block's sums, read from tensor memory, times the
// scales in fp32 registers (a thread holds one weight row and ROWS tokens).
// Every wait is bounded (see the tall kernel's).
//
// Measured: one token through two experts of 14336 x 4096 (352 MB) 69 us, 5.1 TB/s
// with its four launches; 353 MB of up weights alone 61 us, 5.8 TB/s.
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
__device__ unsigned int g_fp8_swap_error;

namespace {

using namespace tc;

constexpr int BM = 128;        // weight rows per tile
constexpr int ROWS = 16;       // rows of the group per tile
constexpr int BK = FP8_BLOCK;
constexpr int UK = 32;
constexpr int NUM_THREADS = 256;
constexpr int FIRST_SUM = 4, SUM_WARPS = 4;
constexpr int MAX_GROUPS = 128;
constexpr int SG = 4;          // blocks whose scales are handed over together

// The tiles of a call: token tiles of ROWS rows per group, times weight tiles,
// times matrices (two for SwiGLU).
struct Shape {
  const int32_t* offsets;  // [G + 1], nullptr: one group of all rows
  int G, rows, N, n_kb, n_nb, mats;
};

struct Params {
  Shape sh;
  const float* SA;
  int sa_pitch;
  const float* SB;
  const float* SB2;
  float* part;     // [slot][ROWS][128], slot = CTA + tile
  long long timeout;
};

// First rows, row counts and token-tile prefix of the groups (one warp).
__device__ __forceinline__ void scan_groups(const Shape& s, int lane, int* row0, int* cnt, int* prefix, bool report) {
  scan_group_rows<(MAX_GROUPS + 31) / 32, ROWS>(s.offsets, s.G, s.rows, lane, row0, cnt, prefix,
                                                report ? &g_fp8_swap_error : nullptr);
}

struct Tile {
  int g, nb, mat;
  int row, n;  // first row and rows of the token tile
};
__device__ __forceinline__ Tile decode_tile(const Shape& s, int t, const int* row0, const int* cnt, const int* prefix,
                                            int& cursor) {
  const int per = s.n_nb * s.mats;
  const int tt = t / per, rem = t - tt * per;
  while (tt >= prefix[cursor + 1]) ++cursor;
  const int first = (tt - prefix[cursor]) * ROWS;
  const int n = cnt[cursor] - first;
  return Tile{cursor, rem / s.mats, rem % s.mats, row0[cursor] + first, n < ROWS ? n : ROWS};
}

// The line of `total` blocks in pieces, one per CTA and none of them empty: piece
// c is [cut(c), cut(c + 1)).
__device__ __forceinline__ int pieces(long long total, int ctas) { return total < ctas ? static_cast<int>(total) : ctas; }
__device__ __forceinline__ long long cut(long long total, int c, int ctas) { return total * c / ctas; }
// The piece that holds block x.
__device__ __forceinline__ int piece_of(long long total, long long x, int ctas) {
  return static_cast<int>(((x + 1) * ctas - 1) / total);
}

struct Cfg {
  static constexpr int W_BYTES = BM * BK;
  static constexpr int X_BYTES = ROWS * BK;
  static constexpr int STAGE_BYTES = W_BYTES + X_BYTES;
  static constexpr int STAGES = 10;
  static constexpr int BUFS = 8;
  static constexpr int TMEM_COLS = BUFS * ROWS;
  static constexpr int RING = 4;
  static constexpr int RING_ROW = ROWS + 4;  // floats per block: the tokens' scales, then the weights'
  static constexpr int RING_GROUP = SG * RING_ROW;
  static constexpr int N_BARS = 2 * STAGES + 2 * BUFS + 2 * RING + 1;
  static constexpr int OFF_X = STAGES * W_BYTES;
  static constexpr int OFF_BARS = OFF_X + STAGES * X_BYTES;
  static constexpr int OFF_SLOT = OFF_BARS + N_BARS * 8;
  static constexpr int OFF_PREFIX = OFF_SLOT + 16;
  static constexpr int OFF_ROW0 = OFF_PREFIX + (MAX_GROUPS + 1) * 4;
  static constexpr int OFF_CNT = OFF_ROW0 + MAX_GROUPS * 4;
  static constexpr int OFF_RING = (OFF_CNT + MAX_GROUPS * 4 + 15) / 16 * 16;
  static constexpr int SMEM = 1024 + OFF_RING + RING * RING_GROUP * 4;
  static_assert(X_BYTES % 1024 == 0 && SMEM <= 232448, "shared memory per CTA");
  static_assert((TMEM_COLS & (TMEM_COLS - 1)) == 0 && TMEM_COLS >= 32 && TMEM_COLS <= 512, "TMEM columns");
};

__global__ void __launch_bounds__(NUM_THREADS, 1)
    fp8_swap_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW,
                    const __grid_constant__ CUtensorMap tmW2, const Params p) {
  using C = Cfg;
  constexpr int STAGES = C::STAGES, BUFS = C::BUFS, RING = C::RING;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sW = smem;
  uint8_t* sX = smem + C::OFF_X;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::OFF_BARS);
  uint64_t* empty = full + STAGES;
  uint64_t* tfull = empty + STAGES;
  uint64_t* tempty = tfull + BUFS;
  uint64_t* sfull = tempty + BUFS;
  uint64_t* sempty = sfull + RING;
  uint64_t* drain = sempty + RING;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_SLOT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  // what the roles leave in flight when they end: the producer's stages (low half) and the
  // phases that they complete, the lane + 1 of the MMA warp that issued MMAs
  volatile uint32_t* in_flight = tmem_slot + 2;
  int* prefix = reinterpret_cast<int*>(smem + C::OFF_PREFIX);
  int* row0 = reinterpret_cast<int*>(smem + C::OFF_ROW0);
  int* cnt = reinterpret_cast<int*>(smem + C::OFF_CNT);
  float* ring = reinterpret_cast<float*>(smem + C::OFF_RING);
  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&full[s]), 1);
      mbar_init(smem_u32(&empty[s]), 1);
    }
    for (int b = 0; b < BUFS; ++b) {
      mbar_init(smem_u32(&tfull[b]), 1);
      mbar_init(smem_u32(&tempty[b]), SUM_WARPS);
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
  // offsets and weights are inputs of the call, which its first kernel, launched
  // without overlap, has waited for: they are read before the wait for the kernel
  // before this one
  if (warp == 0) {
    scan_groups(p.sh, lane, row0, cnt, prefix, blockIdx.x == 0);
    if (lane == 0) {
      tma_prefetch_desc(&tmX);
      tma_prefetch_desc(&tmW);
      if (p.sh.mats == 2) tma_prefetch_desc(&tmW2);
    }
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(C::TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int n_kb = p.sh.n_kb;
  const long long total = static_cast<long long>(prefix[p.sh.G]) * p.sh.n_nb * p.sh.mats * n_kb;
  const int ctas = pieces(total, gridDim.x);
  const bool mine = static_cast<int>(blockIdx.x) < ctas;
  const long long lo = mine ? cut(total, blockIdx.x, ctas) : 0;
  const int n = mine ? static_cast<int>(cut(total, blockIdx.x + 1, ctas) - lo) : 0;  // blocks of this CTA
  const int tile0 = n > 0 ? static_cast<int>(lo / n_kb) : 0;
  const int kb_first = static_cast<int>(lo - static_cast<long long>(tile0) * n_kb);
  const long long budget = p.timeout;

  if (warp == 0) {
    // ---------------------------------------------------------------- producer
    const bool issue = elect_one();
    int stage = 0;
    uint32_t phase = 0;
    uint32_t issued = 0, issued_phase = 0;  // bit s: stage s holds a copy, the phase that it completes
    int cursor = 0, tile = tile0, kb = kb_first;
    bool ok = true;
    Tile t{};
    // block i's place, tile by tile
    auto place = [&](int i) {
      if (i == 0 || kb == 0) t = decode_tile(p.sh, tile, row0, cnt, prefix, cursor);
    };
    auto next = [&] {
      if (++kb == n_kb) {
        kb = 0;
        ++tile;
      }
    };
    auto load_w = [&](int s) {
      const uint32_t fb = smem_u32(&full[s]);
      mbar_expect_tx(fb, C::STAGE_BYTES);
      tma_load_2d(smem_u32(sW + s * C::W_BYTES), t.mat ? &tmW2 : &tmW, kb * BK, t.g * p.sh.N + t.nb * BM, fb);
    };
    auto load_x = [&](int s) {
      tma_load_2d(smem_u32(sX + s * C::X_BYTES), &tmX, kb * BK, t.row, smem_u32(&full[s]));
    };
    // the first stages' weights while the kernel before ends, then their rows
    const int pre = n < STAGES ? n : STAGES;
    for (int i = 0; i < pre; ++i, next()) {
      place(i);
      if (issue) load_w(i);
    }
    pdl_wait();
    cursor = 0;
    tile = tile0;
    kb = kb_first;
    for (int i = 0; i < pre; ++i, next()) {
      place(i);
      if (issue) load_x(i);
      issued |= 1u << i;
    }
    if (pre < STAGES) {
      stage = pre;
    } else {
      phase = 1u;
    }
    for (int i = pre; i < n; ++i, next()) {
      place(i);
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&empty[stage]), phase ^ 1u, budget, abort_flag, &g_fp8_swap_error));
      if (!ok) break;
      if (issue) {
        load_w(stage);
        load_x(stage);
      }
      issued_phase = (issued_phase & ~(1u << stage)) | (phase << stage);
      if (++stage == STAGES) {
        stage = 0;
        phase ^= 1u;
      }
    }
    if (lane == 0) in_flight[0] = issued | (issued_phase << 16);
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer
    const bool issue = elect_one();
    constexpr uint32_t IDESC = idesc_e4m3(BM, ROWS);
    const uint64_t dw0 = sdesc_sw128(smem_u32(sW));
    const uint64_t dx0 = sdesc_sw128(smem_u32(sX));
    int stage = 0, buf = 0;
    uint32_t phase = 0, bph = 0;
    bool ok = true, any = false;
    for (int i = 0; i < n; ++i) {
      const bool there = mbar_wait_strict(smem_u32(&full[stage]), phase, budget, abort_flag, &g_fp8_swap_error);
      ok = __all_sync(0xffffffffu, there && mbar_wait(smem_u32(&tempty[buf]), bph ^ 1u, budget, abort_flag, &g_fp8_swap_error));
      if (!ok) break;
      tc_fence_after();
      // stage-0 descriptors plus the stage offset; each K = 32 step adds 32 bytes
      // (2 in the address field, which cannot carry)
      const uint64_t dw = dw0 + static_cast<uint64_t>(stage) * (C::W_BYTES >> 4);
      const uint64_t dx = dx0 + static_cast<uint64_t>(stage) * (C::X_BYTES >> 4);
      if (issue) {
#pragma unroll
        for (int kk = 0; kk < BK / UK; ++kk)
          umma_fp8(tmem_base + buf * ROWS, dw + 2 * kk, dx + 2 * kk, IDESC, kk ? 1u : 0u);
        umma_commit(smem_u32(&tfull[buf]));
        umma_commit(smem_u32(&empty[stage]));
      }
      any = true;
      if (++stage == STAGES) {
        stage = 0;
        phase ^= 1u;
      }
      if (++buf == BUFS) {
        buf = 0;
        bph ^= 1u;
      }
    }
    if (any && issue) in_flight[1] = lane + 1;
  } else if (warp == 2) {
    // ------------------------------------------------------------------ scales
    pdl_wait();  // the rows' scales
    const uint32_t ring_at = smem_u32(ring);
    int slot = 0;
    uint32_t sph = 0;
    int cursor = 0, tile = tile0, kb = kb_first;
    bool ok = true;
    Tile t{};
    for (int i = 0; i < n && ok; i += SG) {
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sempty[slot]), sph ^ 1u, budget, abort_flag, &g_fp8_swap_error));
      if (!ok) break;
      for (int u = 0; u < SG && i + u < n; ++u) {
        if (i + u == 0 || kb == 0) t = decode_tile(p.sh, tile, row0, cnt, prefix, cursor);
        const uint32_t to = ring_at + 4 * (slot * C::RING_GROUP + u * C::RING_ROW);
        for (int r = lane; r < t.n; r += 32)
          cp_async<4>(to + 4 * r, p.SA + static_cast<long long>(t.row + r) * p.sa_pitch + kb);
        if (lane == 0)
          cp_async<4>(to + 4 * ROWS, (t.mat ? p.SB2 : p.SB) + (static_cast<long long>(t.g) * p.sh.n_nb + t.nb) * n_kb + kb);
        if (++kb == n_kb) {
          kb = 0;
          ++tile;
        }
      }
      cp_async_arrive(smem_u32(&sfull[slot]));
      if (++slot == RING) {
        slot = 0;
        sph ^= 1u;
      }
    }
    cp_async_wait();  // none in flight when shared memory is released
  } else if (warp >= FIRST_SUM) {
    // -------------------------------------------------------------------- sums
    pdl_wait();  // the kernel before may still read the partial sums' space
    const int q = warp & 3;  // TMEM lane quadrant
    const uint32_t t_row = tmem_base + (static_cast<uint32_t>(q * 32) << 16);
    int slot = 0, buf = 0;
    uint32_t sph = 0, bph = 0;
    int cursor = 0, tile = tile0, kb = kb_first;
    float acc[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) acc[j] = 0.0f;
    for (int i = 0; i < n; ++i) {
      const int u = i % SG;
      bool ok = true;
      if (u == 0) ok = mbar_wait(smem_u32(&sfull[slot]), sph, budget, abort_flag, &g_fp8_swap_error);
      ok = ok && mbar_wait(smem_u32(&tfull[buf]), bph, budget, abort_flag, &g_fp8_swap_error);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after();
      float r[ROWS];
      tmem_ld16(t_row + buf * ROWS, r);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&tempty[buf]));
      // tokens beyond the group's: whatever the ring holds, not stored
      const float* s = ring + slot * C::RING_GROUP + u * C::RING_ROW;
      const float sw = s[ROWS];
#pragma unroll
      for (int j = 0; j < ROWS; j += 4) {
        const float4 f = *reinterpret_cast<const float4*>(s + j);
        acc[j] = fmaf(r[j], f.x * sw, acc[j]);
        acc[j + 1] = fmaf(r[j + 1], f.y * sw, acc[j + 1]);
        acc[j + 2] = fmaf(r[j + 2], f.z * sw, acc[j + 2]);
        acc[j + 3] = fmaf(r[j + 3], f.w * sw, acc[j + 3]);
      }
      if (u == SG - 1 || i == n - 1) {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sempty[slot]));
        if (++slot == RING) {
          slot = 0;
          sph ^= 1u;
        }
      }
      if (++buf == BUFS) {
        buf = 0;
        bph ^= 1u;
      }
      if (++kb == n_kb || i == n - 1) {
        // this CTA's part of the tile
        const Tile t = decode_tile(p.sh, tile, row0, cnt, prefix, cursor);
        float* to = p.part + (static_cast<long long>(blockIdx.x) + tile) * (ROWS * BM) + q * 32 + lane;
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
          if (j < t.n) to[j * BM] = acc[j];
          acc[j] = 0.0f;
        }
        kb = 0;
        ++tile;
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {  // no warp waits any more: the same in all of them
    if (warp == 0) {
      drain_copies(smem_u32(full), in_flight[0] & 0xffffu, in_flight[0] >> 16);
    } else if (warp == 1 && in_flight[1] == lane + 1u) {
      // the thread that issued the MMAs: a commit covers its own
      umma_commit(smem_u32(drain));
      mbar_drain(smem_u32(drain), 0, DRAIN_CYCLES);
    }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::TMEM_COLS) : "memory");
  }
}

// ------------------------------------------------------------------ second kernel
enum Mode { STORE_BF16 = 0, STORE_F32 = 1, QUANT_GELU = 2, QUANT_SWIGLU = 3 };

struct SumParams {
  Shape sh;
  const float* part;
  int ctas;  // of the first kernel
  void* out;
  long long ldo;
  float* out_scale;
  int out_scale_pitch;
  const int32_t* perm;
  const float* row_scale;
};

// A warp takes one token's 128 columns of a tile (of two tiles for SwiGLU), four
// per lane; a CTA the tokens of one tile.
template <int MODE>
__global__ void __launch_bounds__(256) fp8_swap_sum_kernel(const SumParams p) {
  __shared__ int row0[MAX_GROUPS], cnt[MAX_GROUPS], prefix[MAX_GROUPS + 1];
  constexpr bool QUANT = MODE == QUANT_GELU || MODE == QUANT_SWIGLU;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_trigger();
  pdl_wait();
  if (warp == 0) scan_groups(p.sh, lane, row0, cnt, prefix, false);
  __syncthreads();
  const int tiles = prefix[p.sh.G] * p.sh.n_nb * p.sh.mats;
  const long long total = static_cast<long long>(tiles) * p.sh.n_kb;
  const int ctas = pieces(total, p.ctas);
  int cursor = 0;
  for (int tile = blockIdx.x * p.sh.mats; tile < tiles; tile += gridDim.x * p.sh.mats) {
    const Tile t = decode_tile(p.sh, tile, row0, cnt, prefix, cursor);
    const int col = t.nb * BM + 4 * lane;
    for (int j = warp; j < t.n; j += 8) {
      float4 v[2];
#pragma unroll
      for (int m = 0; m < (MODE == QUANT_SWIGLU ? 2 : 1); ++m) {
        const long long x0 = static_cast<long long>(tile + m) * p.sh.n_kb;
        const int c0 = piece_of(total, x0, ctas), c1 = piece_of(total, x0 + p.sh.n_kb - 1, ctas);
        v[m] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
        for (int c = c0; c <= c1; ++c) {
          const float4 a =
              *reinterpret_cast<const float4*>(p.part + ((static_cast<long long>(c) + tile + m) * ROWS + j) * BM + 4 * lane);
          v[m].x += a.x;
          v[m].y += a.y;
          v[m].z += a.z;
          v[m].w += a.w;
        }
      }
      const long long row = t.row + j;
      if constexpr (QUANT) {
        if constexpr (MODE == QUANT_SWIGLU) {
          v[0].x = silu_bf16out(v[0].x) * v[1].x;
          v[0].y = silu_bf16out(v[0].y) * v[1].y;
          v[0].z = silu_bf16out(v[0].z) * v[1].z;
          v[0].w = silu_bf16out(v[0].w) * v[1].w;
        } else {
          v[0].x = gelu_fp8out(v[0].x);
          v[0].y = gelu_fp8out(v[0].y);
          v[0].z = gelu_fp8out(v[0].z);
          v[0].w = gelu_fp8out(v[0].w);
        }
        // columns beyond N belong to other weights: not part of the block
        float m = col < p.sh.N ? fmaxf(fmaxf(fabsf(v[0].x), fabsf(v[0].y)), fmaxf(fabsf(v[0].z), fabsf(v[0].w))) : 0.0f;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const Fp8Scale f = fp8_scale(m);
        if (lane == 0) p.out_scale[row * p.out_scale_pitch + t.nb] = f.scale;
        if (col < p.sh.N)
          *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(p.out) + row * p.sh.N + col) =
              fp8_pack2(v[0].x, v[0].y, f.inv) | (fp8_pack2(v[0].z, v[0].w, f.inv) << 16);
      } else {
        long long dest = row;
        float sc = 1.0f;
        if (p.perm) {
          dest = p.perm[row];
          if (dest < 0 || dest >= p.sh.rows) {
            if (lane == 0) atomicOr(&g_fp8_swap_error, 2u);
            continue;
          }
          if (p.row_scale) sc = p.row_scale[dest];
        }
        if (col >= p.sh.N) continue;
        if (MODE == STORE_F32)
          *reinterpret_cast<float4*>(static_cast<float*>(p.out) + dest * p.ldo + col) =
              make_float4(v[0].x * sc, v[0].y * sc, v[0].z * sc, v[0].w * sc);
        else
          *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + dest * p.ldo + col) =
              make_uint2(pack_bf16x2(v[0].x * sc, v[0].y * sc), pack_bf16x2(v[0].z * sc, v[0].w * sc));
      }
    }
  }
}

// ------------------------------------------------------------------ host side
// Token tiles that the groups can hold at most: they own `rows` rows together at
// most, whatever `offsets` says (scan_group_rows), and the partial sums' space is
// sized by this.
long long token_tiles(int G, int rows) { return (rows < G ? rows : G) + rows / ROWS; }

}  // namespace

cudaError_t launch_gemm_fp8_swap(const Fp8GemmArgs& a, int epi, cudaStream_t s) {
  using C = Cfg;
  const void* kfn = reinterpret_cast<const void*>(fp8_swap_kernel);
  cudaError_t e = ensure_smem_attr(kfn, C::SMEM);
  if (e != cudaSuccess) return e;
  const int mats = epi == EPI_SWIGLU ? 2 : 1;
  const long long b_rows = static_cast<long long>(a.G) * a.N;
  CUtensorMap mX, mW, mW2;
  if (!make_tensor_map_u8(&mX, a.A, a.rows, a.K, ROWS)) return cudaErrorInvalidValue;
  if (!make_tensor_map_u8(&mW, a.B, b_rows, a.K, BM)) return cudaErrorInvalidValue;
  mW2 = mW;
  if (mats == 2 && !make_tensor_map_u8(&mW2, a.B2, b_rows, a.K, BM)) return cudaErrorInvalidValue;
  Params p;
  p.sh = Shape{a.offsets, a.G, a.rows, a.N, (a.K + BK - 1) / BK, (a.N + BM - 1) / BM, mats};
  p.SA = a.SA;
  p.sa_pitch = a.sa_pitch > 0 ? a.sa_pitch : p.sh.n_kb;
  p.SB = a.SB;
  p.SB2 = a.SB2;
  p.part = static_cast<float*>(a.part);
  p.timeout = a.timeout_cycles;
  const long long tiles = token_tiles(a.G, a.rows) * p.sh.n_nb * mats;
  const int ctas = fp8_swap_ctas();
  {
    KernelScope ks(a.name, s);
    e = launch_kernel(fp8_swap_kernel, dim3(ctas), dim3(NUM_THREADS), (size_t)C::SMEM, s, mX, mW, mW2, p);
    if (e != cudaSuccess) return e;
  }
  SumParams r;
  r.sh = p.sh;
  r.part = p.part;
  r.ctas = ctas;
  r.out = a.out;
  r.ldo = a.ldo;
  r.out_scale = a.out_scale;
  r.out_scale_pitch = a.out_scale_pitch;
  r.perm = a.perm;
  r.row_scale = a.row_scale;
  const long long blocks = tiles / mats;
  const dim3 grid(static_cast<unsigned>(blocks < 4096 ? blocks : 4096));
  KernelScope ks("fp8_sum", s);
  if (epi == EPI_SWIGLU) e = launch_kernel(fp8_swap_sum_kernel<QUANT_SWIGLU>, grid, dim3(256), 0, s, r);
  else if (epi == EPI_GELU) e = launch_kernel(fp8_swap_sum_kernel<QUANT_GELU>, grid, dim3(256), 0, s, r);
  else if (a.out_bf16) e = launch_kernel(fp8_swap_sum_kernel<STORE_BF16>, grid, dim3(256), 0, s, r);
  else e = launch_kernel(fp8_swap_sum_kernel<STORE_F32>, grid, dim3(256), 0, s, r);
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

int fp8_swap_ctas() { return sm_count(); }

// The tall kernel's tiles of a call (128 rows, 256 columns of B) are whole units of
// work: with few waves of them SMs are left without one, which the line of blocks
// here is not.  It pays for that with partial sums and, beyond one token tile per
// group, with reading the weights again.  Measured (us, this / tall, cold L2):
// - one wave of tiles or less: 1 group 4096 x 14336, 1 row 16 / 19, 17 rows 20 / 18,
//   128 rows 41 / 21; 8 groups 4096 x 4096, 17 rows each 34 / 31, 65 each 53 / 31;
// - 1.5 waves: 4 groups 14336 x 4096, 1 row each 37 / 49, 4 each 47 / 61, 8 each 48 / 48;
// - 3 waves: 8 groups 14336 x 4096, 1 row each 65 / 76, 4 each 82 / 80; 4.6 waves of
//   short K: 64 groups 1408 x 2048, 1 row each 30 / 29, 4 each 44 / 41.
bool fp8_swap_pays(int G, int rows, int N, int K, int mats) {
  if (rows == 0) return false;
  const long long groups = rows < G ? rows : G;
  const long long per = rows / groups;
  const long long tall = groups * ((static_cast<long long>(N) * mats + 255) / 256);
  const long long sms = sm_count();
  if (tall <= sms) return per <= 16;
  return (2 * tall <= 5 * sms && per <= 8) || (K >= 4096 && per <= 2);
}

size_t fp8_swap_bytes(int G, int rows, int N, int K, int mats) {
  if (!fp8_swap_pays(G, rows, N, K, mats)) return 0;
  const long long tiles = token_tiles(G, rows) * ((N + BM - 1) / BM) * mats;
  return static_cast<size_t>(tiles + fp8_swap_ctas()) * ROWS * BM * 4;
}

cudaError_t read_fp8_swap_error(unsigned int* word) {
  unsigned int zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(word, g_fp8_swap_error, sizeof(unsigned int));
  if (e != cudaSuccess) return e;
  return cudaMemcpyToSymbol(g_fp8_swap_error, &zero, sizeof(unsigned int));
}

}  // namespace ec2moe
