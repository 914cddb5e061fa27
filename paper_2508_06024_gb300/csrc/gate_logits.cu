// The gate's logits in fp32 accuracy, [T, E + K]: X W_local^T + b_local, then
// X W_global^T + b_global (Eq. 5 and 6 before their softmaxes), as training and
// tuning of the gate need them.
//
// bf16 activations: every fp32 gate row is split exactly into three bf16 terms
// (w = w0 + w1 + w2, the rest below 2^-24 |w|) whose products with a bf16 value
// are exact in fp32.  Up to 128 gate rows one kernel multiplies 128-token tiles by
// all three, X w0 into a tensor-memory accumulator of its own.  The tensor core adds
// without rounding to nearest, so sums are kept short: every 256 columns of d_model
// the accumulators are added to fp32 registers while the next segment fills the other
// ones.  Few tokens: a cluster of CTAs shares a tile's columns and adds its parts, in
// order, through distributed shared memory.  What bounds long batches is the stream of X and, per
// tile, of the split rows (16 + 30 KB a 64-column block for 72 gate rows).
//   warp 0 loads (TMA), warp 1 issues the MMAs, warps 2..5 drain; every wait is
//   bounded.
// A result that is not finite says nothing: with an infinity in X (or a weight beyond
// bf16's range) terms of both signs, and terms of 0, give NaN where the definition has
// an infinity.  Such results are computed again from X and the fp32 gate rows.
// More gate rows are a grouped-GEMM product of the terms in ranges of K, which a
// last kernel adds in fp32 with the bias; fp32 activations take the fp32-accurate
// GEMM.
//
// Measured: 16384 x 2048, 72 rows: 22.5 us for 72 MB (floor 10.7), of which the
// split takes 3 before the product can start; 1024 x 768, 64 rows: 10 us, two
// launches.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "common.cuh"
#include "internal.h"
#include "tc_ptx.cuh"

namespace ec2moe {

__device__ unsigned int g_logits_error;  // bit 0: a bounded wait timed out

namespace {

using namespace tc;

constexpr int RANGE = 512;  // columns of X that the grouped GEMM sums on the tensor core

// Gate row o (local rows, then global ones) of length d.
__device__ __forceinline__ const float* gate_row(const float* W_local, const float* W_global, int E, int d, int o) {
  return o < E ? W_local + static_cast<size_t>(o) * d : W_global + static_cast<size_t>(o - E) * d;
}

__device__ __forceinline__ bool finite(float v) { return fabsf(v) < INFINITY; }

// What the gate's logits are made of.
struct Source {
  const __nv_bfloat16* X;
  const float* W_local;
  const float* W_global;
  const float* b_local;
  const float* b_global;
  int E, O, d;
};
// Computes again, in 64 bits, the results that are not finite of those that a warp
// stored: out[i], the logit i % O of token t0 + i / O, for i = first + lane, first + lane +
// step, ... below n.  Kept out of line: few calls come here, and short ones are mostly
// fetching their code.
__device__ __noinline__ void mend_not_finite(const Source& src, float* out, long long n, long long first, int step,
                                             long long t0) {
  const int lane = threadIdx.x & 31;
  long long row = -1;  // the token asked for last
  bool row_nan = false;
  for (long long i0 = first; i0 < n; i0 += step) {
    uint32_t m = __ballot_sync(0xffffffffu, i0 + lane < n && !finite(out[i0 + lane]));
    for (; m; m &= m - 1) {
      const long long i = i0 + __ffs(m) - 1, t = t0 + i / src.O;
      const int o = static_cast<int>(i % src.O);
      const __nv_bfloat16* x = src.X + t * src.d;
      if (t != row) {
        bool nan = false;
        for (int c = 8 * lane; c < src.d; c += 256) {
          float v[8];
          load8(x + c, v);
#pragma unroll
          for (int u = 0; u < 8; ++u) nan |= isnan(v[u]);
        }
        row = t;
        row_nan = __any_sync(0xffffffffu, nan);
      }
      if (row_nan) continue;  // so are its logits, as they stand
      const float* w = gate_row(src.W_local, src.W_global, src.E, src.d, o);
      double s = 0.0;
      for (int c = 4 * lane; c < src.d; c += 128) {
        const uint2 xv = *reinterpret_cast<const uint2*>(x + c);
        const float4 wv = *reinterpret_cast<const float4*>(w + c);
        s += static_cast<double>(bf16_lo(xv.x)) * wv.x;
        s += static_cast<double>(bf16_hi(xv.x)) * wv.y;
        s += static_cast<double>(bf16_lo(xv.y)) * wv.z;
        s += static_cast<double>(bf16_hi(xv.y)) * wv.w;
      }
#pragma unroll
      for (int j = 16; j > 0; j >>= 1) s += __shfl_xor_sync(0xffffffffu, s, j);
      if (lane == 0) out[i] = static_cast<float>(s + (o < src.E ? src.b_local[o] : src.b_global[o - src.E]));
    }
  }
}

// terms[j * pad + o][c] = term j of gate row o, 0 for O <= o < pad; four columns per
// thread.
__global__ void __launch_bounds__(256) logits_split_kernel(const float* W_local, const float* W_global, int E, int O,
                                                           int pad, int d, __nv_bfloat16* terms) {
  pdl_trigger();
  pdl_wait();
  const long long i = (blockIdx.x * 256LL + threadIdx.x) * 4;
  if (i >= static_cast<long long>(pad) * d) return;
  const int o = static_cast<int>(i / d), c = static_cast<int>(i % d);
  float4 w = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (o < O) w = *reinterpret_cast<const float4*>(gate_row(W_local, W_global, E, d, o) + c);
  float v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    const uint32_t lo = pack_bf16x2(v[0], v[1]), hi = pack_bf16x2(v[2], v[3]);
    *reinterpret_cast<uint2*>(terms + (static_cast<size_t>(j) * pad + o) * d + c) = make_uint2(lo, hi);
    v[0] -= bf16_lo(lo);
    v[1] -= bf16_hi(lo);
    v[2] -= bf16_lo(hi);
    v[3] -= bf16_hi(hi);
  }
}

// rows[o] = gate row o for o < O, 0 for O <= o < N: the local and the global rows
// as one matrix of the GEMM's row count.
__global__ void __launch_bounds__(256) logits_rows_kernel(const float* W_local, const float* W_global, int E, int O,
                                                          int N, int d, float* rows) {
  pdl_trigger();
  pdl_wait();
  const long long i = (blockIdx.x * 256LL + threadIdx.x) * 4;
  if (i >= static_cast<long long>(N) * d) return;
  const int o = static_cast<int>(i / d), c = static_cast<int>(i % d);
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (o < O) v = *reinterpret_cast<const float4*>(gate_row(W_local, W_global, E, d, o) + c);
  *reinterpret_cast<float4*>(rows + i) = v;
}

// logits[t][o] = bias + the sum over ranges and terms of part[range][t][term * O + o] (pitch N).
// src.X: the activations where the sums are of terms (nullptr: they are the products' own).
__global__ void __launch_bounds__(256) logits_sum_kernel(const float* part, int ranges, int terms, int N, int T,
                                                         const __grid_constant__ Source src, float* logits) {
  pdl_trigger();
  pdl_wait();
  const int O = src.O;
  const long long n = static_cast<long long>(T) * O, i = blockIdx.x * 256LL + threadIdx.x;
  bool all = true;
  if (i < n) {
    const long long t = i / O;
    const int o = static_cast<int>(i - t * O);
    float v = o < src.E ? src.b_local[o] : src.b_global[o - src.E];
    for (int j = terms - 1; j >= 0; --j)
      for (int r = 0; r < ranges; ++r) v += part[(static_cast<long long>(r) * T + t) * N + j * O + o];
    logits[i] = v;
    all = finite(v);
  }
  if (__any_sync(0xffffffffu, !all) && src.X) {
    const long long first = i - (threadIdx.x & 31);
    mend_not_finite(src, logits, first + 32 < n ? first + 32 : n, first, 32, 0);
  }
}

// ------------------------------------------------------------- the fused kernel
constexpr int BM = 128;       // tokens per tile
constexpr int BK = 64;        // columns per stage: one 128-byte swizzle row of bf16
constexpr int SEG = 4;        // stages summed in tensor memory
constexpr int LG_THREADS = 192;
constexpr int MAX_STAGES = 8;
constexpr int ACC_COLS = 128;   // TMEM columns of an accumulator; two per buffer, two buffers
constexpr int MAX_CLUSTER = 8;
constexpr int MAX_ROWS = 128;   // gate rows

struct LgParams {
  const float* b_local;
  const float* b_global;
  float* logits;
  Source src;
  int T, E, O, pad, nk, cs, stages, pitch;
  long long timeout;
};
__host__ __device__ constexpr int lg_stage_bytes(int pad) { return BM * BK * 2 + 3 * pad * BK * 2; }
// stages, then the tile of sums, biases, barriers, TMEM slot
int lg_smem(int pad, int pitch, int stages) {
  return 1024 + stages * lg_stage_bytes(pad) + BM * pitch * 4 + MAX_ROWS * 4 + (2 * MAX_STAGES + 5) * 8 + 16;
}

template <int NB>  // blocks of 16 gate rows
__global__ void __launch_bounds__(LG_THREADS, 1)
    logits_tc_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW,
                     const __grid_constant__ LgParams p) {
  // up to 80 gate rows the three terms are one MMA of 3 pad <= 240 columns, with an
  // accumulator each (16384 x 2048, 72 rows: 26.6 -> 20.5 us)
  constexpr bool WIDE = NB <= 5;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int S = p.stages, stage_bytes = lg_stage_bytes(p.pad);
  float* tile_out = reinterpret_cast<float*>(smem + S * stage_bytes);  // [BM][pitch]
  float* bias = tile_out + BM * p.pitch;
  uint64_t* full = reinterpret_cast<uint64_t*>(bias + MAX_ROWS);
  uint64_t* empty = full + MAX_STAGES;
  uint64_t* tfull = empty + MAX_STAGES;
  uint64_t* tempty = tfull + 2;
  uint64_t* drain = tempty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  // what the roles leave in flight when they end: the producer's stages (low half) and the
  // phases that they complete, the lane + 1 of the MMA warp that issued MMAs
  volatile uint32_t* in_flight = tmem_slot + 2;
  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const int cs = p.cs;
  const int rank = cs > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int n_tiles = (p.T + BM - 1) / BM;
  // a cluster of cs > 1 CTAs has one tile, a CTA alone every gridDim-th
  const int tile_first = cs > 1 ? static_cast<int>(cluster_id_x()) : static_cast<int>(blockIdx.x);
  const int tile_step = cs > 1 ? n_tiles : static_cast<int>(gridDim.x);
  const int kb0 = rank * p.nk / cs, kb1 = (rank + 1) * p.nk / cs;  // this CTA's blocks of d_model
  const long long budget = p.timeout;
  pdl_trigger();
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(smem_u32(&full[s]), 1);
      mbar_init(smem_u32(&empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&tfull[b]), 1);
      mbar_init(smem_u32(&tempty[b]), 4);
    }
    mbar_init(smem_u32(drain), 1);
    *abort_flag = 0;
    in_flight[0] = in_flight[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  for (int o = threadIdx.x; o < p.O; o += LG_THREADS) bias[o] = o < p.E ? p.b_local[o] : p.b_global[o - p.E];
  if (warp == 0 && lane == 0) {
    tma_prefetch_desc(&tmX);
    tma_prefetch_desc(&tmW);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    // ---------------------------------------------------------------- producer
    // X is the caller's: its boxes of the first stages go out before the wait for
    // the split rows, which the kernel before makes.
    const bool issue = elect_one();
    const uint32_t bytes = static_cast<uint32_t>(stage_bytes);
    const int my_tiles = tile_first < n_tiles ? (n_tiles - 1 - tile_first) / tile_step + 1 : 0;
    const int per_tile = kb1 - kb0, total = my_tiles * per_tile;
    const int pre = total < S ? total : S;
    auto load_x = [&](int c, int s) {
      const uint32_t fb = smem_u32(&full[s]);
      mbar_expect_tx(fb, bytes);
      tma_load_2d(smem_u32(smem + s * stage_bytes), &tmX, (kb0 + c % per_tile) * BK,
                  (tile_first + c / per_tile * tile_step) * BM, fb);
    };
    auto load_w = [&](int c, int s) {
      for (int j = 0; j < 3; ++j)
        tma_load_2d(smem_u32(smem + s * stage_bytes + BM * BK * 2 + j * p.pad * BK * 2), &tmW,
                    (kb0 + c % per_tile) * BK, j * p.pad, smem_u32(&full[s]));
    };
    if (issue)
      for (int c = 0; c < pre; ++c) load_x(c, c);
    pdl_wait();
    if (issue)
      for (int c = 0; c < pre; ++c) load_w(c, c);
    // bit s: stage s holds a copy, the phase that it completes
    uint32_t issued = pre ? (1u << pre) - 1u : 0u, issued_phase = 0;
    int stage = pre == S ? 0 : pre;
    uint32_t phase = pre == S ? 1u : 0u;
    bool ok = true;
    for (int c = pre; c < total; ++c) {
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&empty[stage]), phase ^ 1u, budget, abort_flag, &g_logits_error));
      if (!ok) break;
      if (issue) {
        load_x(c, stage);
        load_w(c, stage);
      }
      issued_phase = (issued_phase & ~(1u << stage)) | (phase << stage);
      if (++stage == S) {
        stage = 0;
        phase ^= 1u;
      }
    }
    if (lane == 0) in_flight[0] = issued | (issued_phase << 16);
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer
    const bool issue = elect_one();
    const uint32_t idesc = idesc_bf16(BM, WIDE ? 3 * p.pad : p.pad);
    int stage = 0;
    uint32_t phase = 0, it = 0;  // segments so far: buffer it & 1, its phase (it >> 1) & 1
    bool ok = true, any = false;
    for (int tile = tile_first; tile < n_tiles && ok; tile += tile_step) {
      for (int seg = kb0; seg < kb1 && ok; seg += SEG, ++it) {
        const uint32_t buf = it & 1u, bph = (it >> 1) & 1u;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&tempty[buf]), bph ^ 1u, budget, abort_flag, &g_logits_error));
        if (!ok) break;
        tc_fence_after();
        // X w0, and where three terms are too wide for one MMA X w1 + X w2
        const uint32_t d0 = tmem_base + buf * 2 * ACC_COLS, d1 = d0 + ACC_COLS;
        for (int kb = seg; kb < kb1 && kb < seg + SEG; ++kb) {
          ok = __all_sync(0xffffffffu, mbar_wait_strict(smem_u32(&full[stage]), phase, budget, abort_flag, &g_logits_error));
          if (!ok) break;
          tc_fence_after();
          const uint32_t at = smem_u32(smem + stage * stage_bytes);
          const uint64_t dx = sdesc_sw128(at);
          const uint64_t dw = sdesc_sw128(at + BM * BK * 2);
          const uint64_t term = static_cast<uint64_t>(p.pad * BK * 2 >> 4);
          if (issue) {
#pragma unroll
            for (int kk = 0; kk < BK / 16; ++kk) {
              const uint32_t more = kb != seg || kk ? 1u : 0u;
              umma_bf16(d0, dx + 2 * kk, dw + 2 * kk, idesc, more);
              if (WIDE) continue;
              umma_bf16(d1, dx + 2 * kk, dw + term + 2 * kk, idesc, more);
              umma_bf16(d1, dx + 2 * kk, dw + 2 * term + 2 * kk, idesc, 1u);
            }
            umma_commit(smem_u32(&empty[stage]));
          }
          any = true;
          if (++stage == S) {
            stage = 0;
            phase ^= 1u;
          }
        }
        if (ok && issue) umma_commit(smem_u32(&tfull[buf]));
      }
    }
    if (any && issue) in_flight[1] = lane + 1;
  } else {
    // -------------------------------------------------------------------- drain
    const int q = warp & 3;
    const int row = q * 32 + lane;
    const uint32_t t_row = tmem_base + (static_cast<uint32_t>(q * 32) << 16);
    uint32_t it = 0;
    bool ok = true;
    for (int tile = tile_first; tile < n_tiles; tile += tile_step) {
      float acc[NB][16];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[b][j] = 0.0f;
      for (int seg = kb0; seg < kb1 && ok; seg += SEG, ++it) {
        const uint32_t buf = it & 1u, bph = (it >> 1) & 1u;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&tfull[buf]), bph, budget, abort_flag, &g_logits_error));
        if (!ok) break;
        tc_fence_after();
        const uint32_t t0 = t_row + buf * 2 * ACC_COLS;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          uint32_t v0[16], v1[16], v2[16];
          tmem_ld16_nw(t0 + b * 16, v0);
          tmem_ld16_nw(t0 + (WIDE ? p.pad : ACC_COLS) + b * 16, v1);
          if (WIDE) tmem_ld16_nw(t0 + 2 * p.pad + b * 16, v2);
          tmem_wait();
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float small = WIDE ? __uint_as_float(v1[j]) + __uint_as_float(v2[j]) : __uint_as_float(v1[j]);
            acc[b][j] += __uint_as_float(v0[j]) + small;
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&tempty[buf]));
      }
      float* to = tile_out + row * p.pitch;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int o = b * 16 + j;
          if (o < p.O) to[o] = cs > 1 ? acc[b][j] : acc[b][j] + bias[o];
        }
      if (cs > 1) break;
      // the tile's rows are one piece of the result
      asm volatile("bar.sync 1, 128;" ::: "memory");
      const int n = (p.T - tile * BM < BM ? p.T - tile * BM : BM) * p.O;
      float* out = p.logits + static_cast<long long>(tile) * BM * p.O;
      int r = (threadIdx.x - 64) / p.O, c = (threadIdx.x - 64) - r * p.O;
      const int dr = 128 / p.O, dc = 128 - dr * p.O;
      bool all = true;  // results are finite
#pragma unroll 4
      for (int i = threadIdx.x - 64; i < n; i += 128) {
        const float v = tile_out[r * p.pitch + c];
        out[i] = v;
        all &= finite(v);
        r += dr;
        c += dc;
        if (c >= p.O) {
          c -= p.O;
          ++r;
        }
      }
      if (__any_sync(0xffffffffu, !all))
        mend_not_finite(p.src, out, n, threadIdx.x - 64 - lane, 128, static_cast<long long>(tile) * BM);
      asm volatile("bar.sync 1, 128;" ::: "memory");
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
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512) : "memory");
  }
  if (cs == 1) return;
  // CTA r of the cluster adds up and writes the rows [r BM / cs, (r + 1) BM / cs)
  cluster_sync_all();
  if (tile_first < n_tiles) {
    const int rows = BM / cs, first = rank * rows;
    const int left = p.T - tile_first * BM - first;
    const int n = (left < rows ? left : rows) * p.O;
    float* out = p.logits + (static_cast<long long>(tile_first) * BM + first) * p.O;
    bool all = true;  // results are finite
    for (int i = threadIdx.x; i < n; i += LG_THREADS) {
      const int r = i / p.O, c = i - r * p.O;
      const uint32_t at = smem_u32(tile_out + (first + r) * p.pitch + c);
      float part[MAX_CLUSTER];
#pragma unroll
      for (int k = 0; k < MAX_CLUSTER; ++k)
        if (k < cs) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(part[k]) : "r"(map_to_rank(at, k)) : "memory");
      float v = bias[c];
#pragma unroll
      for (int k = 0; k < MAX_CLUSTER; ++k)
        if (k < cs) v += part[k];
      out[i] = v;
      all &= finite(v);
    }
    if (__any_sync(0xffffffffu, !all))
      mend_not_finite(p.src, out, n, threadIdx.x - lane, LG_THREADS, static_cast<long long>(tile_first) * BM + first);
  }
  cluster_sync_all();  // no CTA ends while its sums are read
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

struct Plan {
  int O, pad, N, ranges;
  bool fused;
  size_t rows, total;  // bytes of the prepared gate rows, and with the partial sums
};
Plan make_plan(int T, int d, int E, int K, bool bf16) {
  Plan p;
  p.O = E + (K > 1 ? K : 0);
  p.fused = bf16 && p.O <= MAX_ROWS;
  p.pad = p.fused ? (p.O + 15) / 16 * 16 : p.O;
  p.N = bf16 ? (3 * p.O + 31) / 32 * 32 : (p.O + 7) / 8 * 8;
  p.ranges = 1;
  if (bf16) {
    // the count of non-empty ranges that the GEMM derives from this request
    const int nk = (d + 63) / 64, want = (d + RANGE - 1) / RANGE, per = (nk + want - 1) / want;
    p.ranges = (nk + per - 1) / per;
  }
  p.rows = align256(static_cast<size_t>(bf16 ? 3 * p.pad : p.N) * d * (bf16 ? 2 : 4));
  p.total = p.rows + (p.fused ? 0 : align256(static_cast<size_t>(p.ranges) * T * p.N * 4));
  return p;
}

template <int NB>
cudaError_t launch_fused_nb(const LgParams& p, const CUtensorMap& mX, const CUtensorMap& mW, int smem, cudaStream_t s) {
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(logits_tc_kernel<NB>), smem);
  if (e != cudaSuccess) return e;
  const int tiles = (p.T + BM - 1) / BM;
  KernelScope ks("logits_gemm", s);
  if (p.cs > 1) return launch_cluster(logits_tc_kernel<NB>, tiles, p.cs, LG_THREADS, (size_t)smem, s, mX, mW, p);
  const int grid = tiles < sm_count() ? tiles : sm_count();
  return launch_kernel(logits_tc_kernel<NB>, dim3(grid), dim3(LG_THREADS), (size_t)smem, s, mX, mW, p);
}

cudaError_t launch_fused(const LogitsArgs& a, const Plan& plan, cudaStream_t s) {
  LgParams p;
  p.b_local = a.b_local;
  p.b_global = a.b_global;
  p.logits = a.logits;
  p.src = Source{static_cast<const __nv_bfloat16*>(a.X), a.W_local, a.W_global, a.b_local, a.b_global, a.E, plan.O, a.d};
  p.T = a.T;
  p.E = a.E;
  p.O = plan.O;
  p.pad = plan.pad;
  p.nk = (a.d + BK - 1) / BK;
  p.pitch = plan.O | 1;
  p.timeout = a.timeout_cycles;
  p.stages = MAX_STAGES;
  while (p.stages > 2 && lg_smem(p.pad, p.pitch, p.stages) > 232448) --p.stages;
  // as many CTAs to a tile as leave every CTA an SM
  const int tiles = (a.T + BM - 1) / BM;
  p.cs = 1;
  while (p.cs < MAX_CLUSTER && 2 * p.cs <= p.nk && 2LL * p.cs * tiles <= sm_count()) p.cs *= 2;
  CUtensorMap mX, mW;
  if (!make_tensor_map_bf16(&mX, a.X, a.T, a.d, BM)) return cudaErrorInvalidValue;
  if (!make_tensor_map_bf16(&mW, a.workspace, 3LL * p.pad, a.d, p.pad)) return cudaErrorInvalidValue;
  const int smem = lg_smem(p.pad, p.pitch, p.stages);
  const int nb = p.pad / 16;
  cudaError_t e = nb == 1   ? launch_fused_nb<1>(p, mX, mW, smem, s)
                  : nb <= 2 ? launch_fused_nb<2>(p, mX, mW, smem, s)
                  : nb <= 5 ? launch_fused_nb<5>(p, mX, mW, smem, s)
                            : launch_fused_nb<8>(p, mX, mW, smem, s);
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

}  // namespace

size_t gate_logits_bytes(int T, int d, int E, int K, bool bf16) { return make_plan(T, d, E, K, bf16).total; }

cudaError_t launch_gate_logits(const LogitsArgs& a, bool bf16, cudaStream_t s) {
  const Plan p = make_plan(a.T, a.d, a.E, a.K, bf16);
  void* rows = a.workspace;
  float* part = reinterpret_cast<float*>(static_cast<uint8_t*>(a.workspace) + p.rows);
  const long long items = static_cast<long long>(bf16 ? p.pad : p.N) * a.d / 4;
  cudaError_t e;
  {
    KernelScope ks("logits_prep", s);
    const dim3 grid(static_cast<unsigned>((items + 255) / 256));
    e = bf16 ? launch_kernel(logits_split_kernel, grid, dim3(256), 0, s, a.W_local, a.W_global, a.E, p.O,
                             p.pad, a.d, static_cast<__nv_bfloat16*>(rows))
             : launch_kernel(logits_rows_kernel, grid, dim3(256), 0, s, a.W_local, a.W_global, a.E, p.O, p.N,
                             a.d, static_cast<float*>(rows));
    if (e != cudaSuccess) return e;
  }
  if (p.fused) return launch_fused(a, p, s);
  GemmArgs g{};
  g.self_row_base = -1;
  g.timeout_cycles = a.timeout_cycles;
  g.name = "logits_gemm";
  g.A = a.X;
  g.a_rows = a.T;
  g.B = rows;
  g.b_rows = bf16 ? 3LL * p.O : p.O;
  g.G = 1;
  g.M = a.T;
  g.N = p.N;
  g.K = a.d;
  g.max_rows = a.T;
  if (bf16) {
    g.split_k = p.ranges;
    g.partial = part;
    g.part_rows = a.T;
    e = launch_gemm_tc(g, EPI_PARTIAL, s);
  } else {
    g.out = part;
    g.ldo = p.N;
    plain_next_launch();  // this GEMM takes its B for weights, which nothing writes while it runs
    e = launch_gemm_f32(g, EPI_STORE, s);
  }
  if (e != cudaSuccess) return e;
  KernelScope ks("logits_sum", s);
  e = launch_kernel(logits_sum_kernel, dim3(static_cast<unsigned>((static_cast<long long>(a.T) * p.O + 255) / 256)), dim3(256), 0,
                    s, part, p.ranges, bf16 ? 3 : 1, p.N, a.T,
                    Source{bf16 ? static_cast<const __nv_bfloat16*>(a.X) : nullptr, a.W_local, a.W_global, a.b_local, a.b_global,
                           a.E, p.O, a.d},
                    a.logits);
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

cudaError_t read_logits_error(unsigned int* word) {
  unsigned int zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(word, g_logits_error, sizeof(unsigned int));
  if (e != cudaSuccess) return e;
  return cudaMemcpyToSymbol(g_logits_error, &zero, sizeof(unsigned int));
}

}  // namespace ec2moe
