// Root-mean-square norm of the rows in front of a layer, with the residual's
// addition, and its gradient.
//
//   h = x + residual,  rstd = 1 / sqrt(mean h^2 + eps),  y = h rstd w
//
// h is the fp32 sum: y and its quantisation are taken from it, not from the h
// that is stored rounded.  y is stored in 16 or 32 bits, and/or quantised to e4m3
// with a scale per 128 columns by quantize_rows' rule (fp8.cuh).  With g = dy w and xhat = h rstd the gradient is
//
//   dx = rstd (g - xhat mean(g xhat)) + dh,   dw = sum over rows of dy xhat.
//
// Bounded by HBM.  A CTA per SM is divided into teams of whole warps, a row to a
// team at a time: a thread holds up to 4 x 8 of its columns (16 consecutive threads:
// one 128-column block of the quantisation).  Each team has a ring of rows in shared
// memory, filled by bulk copies that its first thread issues as soon as the team has
// read a row, so rows keep arriving while others are reduced and stored.  Every
// operand is read once, and H or dx may take an operand's place.  The gradient's
// threads keep their columns' share of dw over all their rows; a second kernel adds
// up the CTAs' shares in a fixed order.  Short calls take a CTA per row, without the
// ring (300 x 4096: 5.4 us, with it 8).
//
// Measured: 16384 x 4096 bf16 with residual and 8-bit rows 100 us (6.0 TB/s; with plain
// loads, a row in registers, 133), its gradient 88 us (6.1 TB/s), fp32 160 us (6.7 TB/s);
// 16384 x 2048, gradient, 50 us, of which 4 are the second kernel.  Rows stored by bulk
// copies from the ring were slower (111), as were stores that leave L2 first.
//
// Every wait for a row is bounded: one that gives up sets the error word, the team
// waits for its copies in flight and ends.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"
#include "tc_ptx.cuh"

namespace ec2moe {

// bit 0: a bounded wait timed out
__device__ unsigned int g_norm_error;

namespace {

using namespace tc;

constexpr int PER = 8;        // columns per thread and step: 16 bytes of bf16
constexpr int MAX_WARPS = 32;
constexpr int LANES = FP8_BLOCK / PER;  // threads of a block of the quantisation

// Sum over the tpr threads (whole warps) of a row; every thread gets it.  The
// warps' sums are added in order.
__device__ __forceinline__ float row_sum(float v, int tpr, float* s_sum) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (tpr == 32) return v;
  const int warp = threadIdx.x >> 5, per = tpr >> 5;
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s_sum[warp] = v;
  __syncthreads();
  const int first = warp / per * per;
  float t = 0.0f;
  for (int i = 0; i < per; ++i) t += s_sum[first + i];
  return t;
}

// e4m3's ties.  From 2^-6 on its values have 3 bits behind the leading one, so a quotient at a tie
// has 0x80000 in its bits 0-19; below, its steps are 2^-9 throughout, as between 2^-6 and 2^-5, so
// there the same goes for the quotient plus 2^-6.
constexpr float NORMAL = 0x1p-6f;  // e4m3's least value with a leading one
__device__ __forceinline__ float subnormal_shift(float q) { return fabsf(q) < NORMAL ? NORMAL : 0.0f; }
// Where bits 0-19 lie from a tie's, times 2^12: 0 .. 14 for TIE_UNITS = 7 units of the last place below
// it to 7 above.
constexpr uint32_t TIE_UNITS = 7;
constexpr uint32_t BESIDE_TIE = 2 * TIE_UNITS << 12;
__device__ __forceinline__ uint32_t beside_tie(float z) { return __float_as_uint(z) * 4096u + ((0x80000u + TIE_UNITS) << 12); }
// v = |a b| as the 24 bits of its fp32 rounding p and the rounding error e, exact in fp32: v 2^(47 - k),
// k the exponent of p, an integer of 48 bits.
__device__ __forceinline__ int exponent(float p) { return static_cast<int>(__float_as_uint(p) >> 23) - 127; }
__device__ __forceinline__ float product_error(float a, float b) {
  const float p = a * b;
  return copysignf(1.0f, p) * fmaf(a, b, -p);
}
__device__ __forceinline__ long long product_bits(float p, float e) {
  // 2^(47 - k) in two factors, each within fp32's range
  const int k = exponent(p);
  const float part = e * __uint_as_float(static_cast<uint32_t>(127 - k) << 23) * 0x1p47f;
  return (static_cast<long long>((__float_as_uint(p) & 0x7fffffu) | 0x800000u) << 24) + static_cast<int>(part);
}
// A quotient q beside a tie, moved to the side of it where 448 |h w| / most lies, most = m + m_error the
// block's largest |h w|: the signs of integers of 53 bits at most, 448 = 7 2^6 and a tie having 5 bits.
__device__ __forceinline__ float decide_tie(float q, float h, float w, float m, float m_error) {
  const float shift = subnormal_shift(q), z = fabsf(q) + shift;
  const float tie = __uint_as_float(__float_as_uint(z) + TIE_UNITS - (beside_tie(z) >> 12)) - shift;
  const float p = fabsf(h * w);
  const uint32_t bits = __float_as_uint(tie);
  const int up = exponent(p) - exponent(tie) - exponent(m) + 10;  // 1 to 3: the two are next to each other
  const long long there = 7 * product_bits(p, product_error(h, w)) << up;
  const long long at = static_cast<long long>(((bits & 0x7fffffu) | 0x800000u) >> 19) * product_bits(m, m_error);
  const uint32_t r = there > at ? bits + 1u : there < at ? bits - 1u : bits;
  return copysignf(__uint_as_float(r), q);
}

// A chunk of PER columns of a row: y = h rstd w, stored and quantised.  The 16 lanes
// of a block of 128 columns call it together, `mine` where the chunk is inside the row.
// rstd is in a value and in its block's largest alike: what e4m3 rounds is 448 h w over
// the largest |h w|.  The fp32 quotient is within 7 2^-24 of itself (4 for the fast division's 2 units,
// one each for the two products, the largest's and the last): beside a tie, whose mantissa is 31/16 at
// most, 6.8 units of its last place (below 2^-6, shifted: 4).  Where it is further from a tie its
// rounding is right; a warp that holds another one, one in 270, decides that by exact
// products (as integers: 64-bit floats took 9 us more for 16384 x 4096).  Returns the
// block's largest |y|.
template <typename TX, typename TY>
__device__ __forceinline__ float finish_chunk(const NormArgs& a, long long row, int c, bool mine, float rstd, const float* h,
                                              const float* w) {
  if (mine && a.H) store8(static_cast<TX*>(a.H) + row * a.cols + c * PER, h);
  if (mine && a.Y) {
    float y[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) y[j] = h[j] * rstd * w[j];
    store8(static_cast<TY*>(a.Y) + row * a.cols + c * PER, y);
  }
  if (!a.Q) return 0.0f;
  float q[PER];
  float m = 0.0f;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    q[j] = h[j] * w[j];  // 0 where the chunk is not inside the row
    m = fmaxf(m, fabsf(q[j]));
  }
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float most = m * rstd;
  const bool plain = most >= 0x1p-96f && most < INFINITY && m < 0x1p100f && m > 0x1p-80f;
  if (!__all_sync(0xffffffffu, plain || !mine)) {
    // blocks of zeros or next to them, infinities and NaN: fp8_scale's rule on y itself
    float z = 0.0f;
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (mine) z = fmaxf(z, fabsf(h[j] * rstd * w[j]));
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) z = fmaxf(z, __shfl_xor_sync(0xffffffffu, z, o));
    if (!plain) {
      most = z;
      const float inv = fp8_scale(z).inv;
#pragma unroll
      for (int j = 0; j < PER; ++j) q[j] = h[j] * rstd * w[j] * inv;
    }
  }
  uint32_t nearest = 0xffffffffu;
  float least = INFINITY;
  if (plain && mine) {
    const float inv = __fdividef(448.0f, m);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      q[j] *= inv;
      nearest = min(nearest, beside_tie(q[j]));
      least = fminf(least, fabsf(q[j]));
    }
  }
  // first whether the warp holds one next to a normal tie or any below the normal range, then which
  if (__any_sync(0xffffffffu, nearest <= BESIDE_TIE || least < NORMAL)) {
    nearest = 0xffffffffu;
    if (plain && mine) {
#pragma unroll
      for (int j = 0; j < PER; ++j) nearest = min(nearest, beside_tie(fabsf(q[j]) + subnormal_shift(q[j])));
    }
    if (__any_sync(0xffffffffu, nearest <= BESIDE_TIE)) {
      float m_error = -INFINITY;  // of the largest of those that round to m
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (fabsf(h[j] * w[j]) == m) m_error = fmaxf(m_error, product_error(h[j], w[j]));
#pragma unroll
      for (int o = 1; o < LANES; o <<= 1) m_error = fmaxf(m_error, __shfl_xor_sync(0xffffffffu, m_error, o));
      if (nearest <= BESIDE_TIE) {
#pragma unroll
        for (int j = 0; j < PER; ++j)
          if (beside_tie(fabsf(q[j]) + subnormal_shift(q[j])) <= BESIDE_TIE) q[j] = decide_tie(q[j], h[j], w[j], m, m_error);
      }
    }
  }
  if (!mine) return most;
  const uint32_t q0 = fp8_pack2(q[0], q[1], 1.0f) | (fp8_pack2(q[2], q[3], 1.0f) << 16);
  const uint32_t q1 = fp8_pack2(q[4], q[5], 1.0f) | (fp8_pack2(q[6], q[7], 1.0f) << 16);
  *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.Q) + row * a.cols + c * PER) = make_uint2(q0, q1);
  return most;
}

__device__ __forceinline__ float rstd_of(float sum, const NormArgs& a) {
  return __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(sum, static_cast<float>(a.cols)) + a.eps));
}

// Short calls: a row per CTA, a chunk per thread.
template <typename TX, typename TY>
__global__ void __launch_bounds__(1024) rmsnorm_kernel(const NormArgs a) {
  pdl_trigger();
  pdl_wait();
  __shared__ float s_sum[MAX_WARPS];
  const int c = threadIdx.x;
  const long long row = blockIdx.x;
  const bool mine = c < a.cols / PER;
  float h[PER] = {}, w[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) w[j] = 1.0f;
  if (mine) {
    load8(static_cast<const TX*>(a.X) + row * a.ld + c * PER, h);
    if (a.weight) load8(a.weight + c * PER, w);
    if (a.residual) {
      float r[PER];
      load8(static_cast<const TX*>(a.residual) + row * a.ld + c * PER, r);
#pragma unroll
      for (int j = 0; j < PER; ++j) h[j] += r[j];
    }
  }
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < PER; ++j) sum = fmaf(h[j], h[j], sum);
  sum = row_sum(sum, blockDim.x, s_sum);
  const float rstd = rstd_of(sum, a);
  if (c == 0 && a.rstd) a.rstd[row] = rstd;
  const float most = finish_chunk<TX, TY>(a, row, c, mine, rstd, h, w);
  if (a.Q && mine && c % LANES == 0) a.scale[row * ((a.cols + FP8_BLOCK - 1) / FP8_BLOCK) + c / LANES] = fp8_scale(most).scale;
}

// ------------------------------------------------------------- rows through a ring
constexpr int NCH = 4;            // chunks per thread
constexpr int RING_THREADS = 512;
constexpr int MAX_TEAMS = RING_THREADS / 32;
constexpr int MAX_DEPTH = 4;
constexpr int RING_BYTES = 208 * 1024;

struct Ring {
  int tpr, teams, depth;  // threads of a team, teams of a CTA, rows of a team's ring
  int bytes;              // of a row's operands
  int grid;
  int smem;
};

// At least two rows per team where they fit: one arrives while the other is worked on.
// Calls with a team for every row (2001 x 768 fp32, gradient: 10.2 -> 9.4 us) have one.
Ring ring_of(int rows, int cols, int bytes) {
  Ring r;
  r.tpr = ((cols / PER + NCH - 1) / NCH + 31) / 32 * 32;
  r.bytes = bytes;
  r.teams = RING_THREADS / r.tpr;
  const int one = RING_BYTES / bytes < r.teams ? RING_BYTES / bytes : r.teams;  // teams with one row each
  if (rows <= one * sm_count()) {
    r.teams = (rows + sm_count() - 1) / sm_count();
    r.depth = 1;
  } else {
    while (r.teams > 1 && r.teams * 2 * bytes > RING_BYTES) --r.teams;
    r.depth = RING_BYTES / (r.teams * bytes);
    r.depth = r.depth < 1 ? 1 : r.depth > MAX_DEPTH ? MAX_DEPTH : r.depth;
  }
  const long long units = (static_cast<long long>(rows) + r.teams - 1) / r.teams;
  r.grid = units < sm_count() ? static_cast<int>(units) : sm_count();
  r.smem = r.teams * r.depth * bytes;
  return r;
}

// Copy of `bytes` (a multiple of 16, both addresses too) counted on `bar`.
__device__ __forceinline__ void copy_row(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

// What a team's warps tell each other about a row; two rows' worth, so that one
// barrier per row is enough.
struct TeamSums {
  float sum[2][MAX_WARPS];
  int ok[2][MAX_WARPS];
};

// Sum over the team, in the warps' order; false where any of its warps gave up.
// Every thread of the team is through with the row before the barrier.
__device__ __forceinline__ bool team_sum(float& v, bool ok, int tpr, int team, int turn, TeamSums& s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  ok = __all_sync(0xffffffffu, ok);
  if (tpr == 32) return ok;
  const int warp = threadIdx.x >> 5, per = tpr >> 5, first = team * per;
  if ((threadIdx.x & 31) == 0) {
    s.sum[turn][warp] = v;
    s.ok[turn][warp] = ok;
  }
  asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(tpr) : "memory");
  v = 0.0f;
  ok = true;
  for (int i = 0; i < per; ++i) {
    v += s.sum[turn][first + i];
    ok = ok && s.ok[turn][first + i] != 0;
  }
  return ok;
}
__device__ __forceinline__ void team_sync(int tpr, int team) {
  if (tpr == 32) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(tpr) : "memory");
}

// The copies that a team has in flight when it ends: of `row` and the rows behind it
// that are fetched, in the ring from place d on.
__device__ __forceinline__ void drain_ring(uint64_t* full, int d, uint32_t phase, int depth, long long row, long long step,
                                           long long rows) {
  const long long t0 = clock64();
  for (int i = 0; i < depth && row < rows; ++i, row += step) {
    mbar_drain(smem_u32(&full[d]), phase, DRAIN_CYCLES - (clock64() - t0));
    if (++d == depth) {
      d = 0;
      phase ^= 1u;
    }
  }
}

template <typename TX, typename TY>
__global__ void __launch_bounds__(RING_THREADS, 1) rmsnorm_ring_kernel(const NormArgs a, const Ring g) {
  pdl_trigger();
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ uint64_t full[MAX_TEAMS][MAX_DEPTH];
  __shared__ TeamSums sums;
  const int t = threadIdx.x % g.tpr, team = threadIdx.x / g.tpr;
  const int n_chunks = a.cols / PER;
  if (t == 0) {
    for (int d = 0; d < g.depth; ++d) mbar_init(smem_u32(&full[team][d]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  team_sync(g.tpr, team);
  pdl_wait();
  uint8_t* mine_ring = ring + static_cast<size_t>(team) * g.depth * g.bytes;
  const int part = a.cols * static_cast<int>(sizeof(TX));
  const long long step = static_cast<long long>(gridDim.x) * g.teams;
  const long long first = static_cast<long long>(blockIdx.x) * g.teams + team;
  auto fetch = [&](long long row, int d) {
    const uint32_t bar = smem_u32(&full[team][d]), dst = smem_u32(mine_ring + d * g.bytes);
    mbar_expect_tx(bar, g.bytes);
    copy_row(dst, static_cast<const TX*>(a.X) + row * a.ld, part, bar);
    if (a.residual) copy_row(dst + part, static_cast<const TX*>(a.residual) + row * a.ld, part, bar);
  };
  if (t == 0)
    for (int d = 0; d < g.depth; ++d)
      if (first + d * step < a.rows) fetch(first + d * step, d);
  float w[NCH][PER];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
#pragma unroll
    for (int j = 0; j < PER; ++j) w[i][j] = 1.0f;
    if (a.weight && i * g.tpr + t < n_chunks) load8(a.weight + (i * g.tpr + t) * PER, w[i]);
  }
  const int n_kb = (a.cols + FP8_BLOCK - 1) / FP8_BLOCK;
  int d = 0, turn = 0;
  uint32_t phase = 0;
  volatile int no_abort = 0;
  long long row = first;
  for (; row < a.rows; row += step) {
    bool ok = mbar_wait_strict(smem_u32(&full[team][d]), phase, a.timeout_cycles, &no_abort, &g_norm_error);
    const TX* x = reinterpret_cast<const TX*>(mine_ring + d * g.bytes);
    const TX* res = x + a.cols;
    float h[NCH][PER];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = i * g.tpr + t;
#pragma unroll
      for (int j = 0; j < PER; ++j) h[i][j] = 0.0f;
      if (c < n_chunks) {
        load8(x + c * PER, h[i]);
        if (a.residual) {
          float r[PER];
          load8(res + c * PER, r);
#pragma unroll
          for (int j = 0; j < PER; ++j) h[i][j] += r[j];
        }
      }
#pragma unroll
      for (int j = 0; j < PER; ++j) sum = fmaf(h[i][j], h[i][j], sum);
    }
    ok = team_sum(sum, ok, g.tpr, team, turn, sums);
    if (!ok) break;
    if (t == 0 && row + g.depth * step < a.rows) fetch(row + g.depth * step, d);
    const float rstd = rstd_of(sum, a);
    if (t == 0 && a.rstd) a.rstd[row] = rstd;
    // lane i of a block's 16 keeps chunk i's scale: one division for all of them
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      if (i * g.tpr >= n_chunks) break;  // the whole row
      const float v = finish_chunk<TX, TY>(a, row, i * g.tpr + t, i * g.tpr + t < n_chunks, rstd, h[i], w[i]);
      if (t % LANES == i) most = v;
    }
    if (a.Q && t % LANES < NCH) {
      const int c = t % LANES * g.tpr + t / LANES * LANES;  // the block's first chunk
      if (c < n_chunks) a.scale[row * n_kb + c / LANES] = fp8_scale(most).scale;
    }
    turn ^= 1;
    if (++d == g.depth) {
      d = 0;
      phase ^= 1u;
    }
  }
  // after a timeout: the copies of this row and those behind it
  if (row < a.rows && t == 0) drain_ring(&full[team][0], d, phase, g.depth, row, step, a.rows);
}

template <typename TX, typename TY>
__global__ void __launch_bounds__(RING_THREADS, 1) rmsnorm_backward_kernel(const NormBackArgs a, const Ring g) {
  pdl_trigger();
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ uint64_t full[MAX_TEAMS][MAX_DEPTH];
  __shared__ TeamSums sums;
  const int t = threadIdx.x % g.tpr, team = threadIdx.x / g.tpr;
  const int n_chunks = a.cols / PER;
  if (t == 0) {
    for (int d = 0; d < g.depth; ++d) mbar_init(smem_u32(&full[team][d]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  team_sync(g.tpr, team);
  pdl_wait();
  uint8_t* mine_ring = ring + static_cast<size_t>(team) * g.depth * g.bytes;
  const int part_y = a.cols * static_cast<int>(sizeof(TY)), part_x = a.cols * static_cast<int>(sizeof(TX));
  const long long step = static_cast<long long>(gridDim.x) * g.teams;
  const long long first = static_cast<long long>(blockIdx.x) * g.teams + team;
  auto fetch = [&](long long row, int d) {
    const uint32_t bar = smem_u32(&full[team][d]), dst = smem_u32(mine_ring + d * g.bytes);
    mbar_expect_tx(bar, g.bytes);
    copy_row(dst, static_cast<const TY*>(a.dY) + row * a.ld, part_y, bar);
    copy_row(dst + part_y, static_cast<const TX*>(a.H) + row * a.cols, part_x, bar);
    if (a.dH) copy_row(dst + part_y + part_x, static_cast<const TX*>(a.dH) + row * a.cols, part_x, bar);
  };
  if (t == 0)
    for (int d = 0; d < g.depth; ++d)
      if (first + d * step < a.rows) fetch(first + d * step, d);
  float w[NCH][PER], dw[NCH][PER] = {};
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
#pragma unroll
    for (int j = 0; j < PER; ++j) w[i][j] = 1.0f;
    if (a.weight && i * g.tpr + t < n_chunks) load8(a.weight + (i * g.tpr + t) * PER, w[i]);
  }
  int d = 0, turn = 0;
  uint32_t phase = 0;
  volatile int no_abort = 0;
  long long row = first;
  for (; row < a.rows; row += step) {
    const float rstd = a.rstd[row];
    bool ok = mbar_wait_strict(smem_u32(&full[team][d]), phase, a.timeout_cycles, &no_abort, &g_norm_error);
    const TY* dy = reinterpret_cast<const TY*>(mine_ring + d * g.bytes);
    const TX* h = reinterpret_cast<const TX*>(mine_ring + d * g.bytes + part_y);
    const TX* dh = h + a.cols;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = i * g.tpr + t;
      if (c < n_chunks) {
        float y[PER], x[PER];
        load8(dy + c * PER, y);
        load8(h + c * PER, x);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
          x[j] *= rstd;
          dw[i][j] = fmaf(y[j], x[j], dw[i][j]);
          sum = fmaf(y[j] * w[i][j], x[j], sum);
        }
      }
    }
    ok = team_sum(sum, ok, g.tpr, team, turn, sums);
    if (!ok) break;
    const float mean = __fdiv_rn(sum, static_cast<float>(a.cols));
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = i * g.tpr + t;
      if (c < n_chunks) {
        float y[PER], x[PER];
        load8(dy + c * PER, y);
        load8(h + c * PER, x);
#pragma unroll
        for (int j = 0; j < PER; ++j) y[j] = rstd * fmaf(-(x[j] * rstd), mean, y[j] * w[i][j]);
        if (a.dH) {
          load8(dh + c * PER, x);
#pragma unroll
          for (int j = 0; j < PER; ++j) y[j] += x[j];
        }
        store8(static_cast<TX*>(a.dX) + row * a.cols + c * PER, y);
      }
    }
    team_sync(g.tpr, team);  // the row is read
    if (t == 0 && row + g.depth * step < a.rows) fetch(row + g.depth * step, d);
    turn ^= 1;
    if (++d == g.depth) {
      d = 0;
      phase ^= 1u;
    }
  }
  if (row < a.rows && t == 0) drain_ring(&full[team][0], d, phase, g.depth, row, step, a.rows);
  if (!a.d_weight) return;
  // the teams' shares, where the rows were, added in order
  __syncthreads();
  float* s_dw = reinterpret_cast<float*>(ring);
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = i * g.tpr + t;
    if (c < n_chunks) store8(s_dw + team * a.cols + c * PER, dw[i]);
  }
  __syncthreads();
  for (int c = threadIdx.x * 4; c < a.cols; c += blockDim.x * 4) {
    float4 v = *reinterpret_cast<const float4*>(s_dw + c);
    for (int r = 1; r < g.teams; ++r) {
      const float4 o = *reinterpret_cast<const float4*>(s_dw + r * a.cols + c);
      v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
    }
    *reinterpret_cast<float4*>(a.partial + static_cast<long long>(blockIdx.x) * a.cols + c) = v;
  }
}

// out[c] = sum of partial[0 .. n)[c]: 32 columns per CTA, its warps take every 32nd row
// (so that the few rows are fetched at once), their sums are added in order.
__global__ void __launch_bounds__(1024) dweight_sum_kernel(const float* partial, int n, int cols, float* out,
                                                           int accumulate) {
  pdl_trigger();
  pdl_wait();
  __shared__ float s[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  float v = 0.0f;
  if (c < cols) {
#pragma unroll 8
    for (int r = warp; r < n; r += 32) v += partial[static_cast<long long>(r) * cols + c];
  }
  s[warp][lane] = v;
  __syncthreads();
  // warp w adds up column w
  v = s[lane][warp];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (lane == 0 && blockIdx.x * 32 + warp < cols) {
    float* to = out + blockIdx.x * 32 + warp;
    *to = accumulate ? *to + v : v;
  }
}

template <typename TX, typename TY>
cudaError_t forward(const NormArgs& a, cudaStream_t s) {
  KernelScope ks("rmsnorm", s);
  cudaError_t e;
  if (a.cols / PER <= 1024 && a.rows < 2 * sm_count()) {
    const int threads = (a.cols / PER + 31) / 32 * 32;
    e = launch_kernel(rmsnorm_kernel<TX, TY>, dim3(a.rows), dim3(threads), 0, s, a);
  } else {
    const Ring g = ring_of(a.rows, a.cols, a.cols * static_cast<int>(sizeof(TX)) * (a.residual ? 2 : 1));
    auto kernel = rmsnorm_ring_kernel<TX, TY>;
    e = ensure_smem_attr(reinterpret_cast<const void*>(kernel), g.smem);
    if (e != cudaSuccess) return e;
    e = launch_kernel(kernel, dim3(g.grid), dim3(g.tpr * g.teams), g.smem, s, a, g);
  }
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

template <typename TX, typename TY>
cudaError_t backward(const NormBackArgs& a, cudaStream_t s) {
  const Ring g = ring_of(a.rows, a.cols, a.cols * static_cast<int>(sizeof(TY) + sizeof(TX) * (a.dH ? 2 : 1)));
  const int dw_bytes = g.teams * a.cols * 4;
  const int smem = g.smem > dw_bytes ? g.smem : dw_bytes;
  auto kernel = rmsnorm_backward_kernel<TX, TY>;
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(kernel), smem);
  if (e != cudaSuccess) return e;
  {
    KernelScope ks("rmsnorm_backward", s);
    e = launch_kernel(kernel, dim3(g.grid), dim3(g.tpr * g.teams), smem, s, a, g);
    if (e != cudaSuccess) return e;
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (!a.d_weight) return cudaSuccess;
  KernelScope ks("rmsnorm_dweight", s);
  e = launch_kernel(dweight_sum_kernel, dim3((a.cols + 31) / 32), dim3(1024), 0, s, a.partial, g.grid, a.cols, a.d_weight,
                    a.accumulate);
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

}  // namespace

size_t norm_backward_bytes(int rows, int cols) {
  return static_cast<size_t>(rows < sm_count() ? rows : sm_count()) * cols * 4;  // a share per CTA
}

cudaError_t launch_rmsnorm(const NormArgs& a, bool bf16, bool y_bf16, cudaStream_t s) {
  if (bf16) return y_bf16 ? forward<__nv_bfloat16, __nv_bfloat16>(a, s) : forward<__nv_bfloat16, float>(a, s);
  return y_bf16 ? forward<float, __nv_bfloat16>(a, s) : forward<float, float>(a, s);
}

cudaError_t launch_rmsnorm_backward(const NormBackArgs& a, bool bf16, bool y_bf16, cudaStream_t s) {
  if (bf16) return y_bf16 ? backward<__nv_bfloat16, __nv_bfloat16>(a, s) : backward<__nv_bfloat16, float>(a, s);
  return y_bf16 ? backward<float, __nv_bfloat16>(a, s) : backward<float, float>(a, s);
}

cudaError_t read_norm_error(unsigned int* word) {
  unsigned int zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(word, g_norm_error, sizeof(unsigned int));
  if (e != cudaSuccess) return e;
  return cudaMemcpyToSymbol(g_norm_error, &zero, sizeof(unsigned int));
}

}  // namespace ec2moe
