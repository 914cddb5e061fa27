// Root-mean-square norm of the rows in front of a layer, with the residual's
// addition, and its gradient.
//
//   h = x + residual,  rstd = 1 / sqrt(mean h^2 + eps),  y = h rstd w
//
// h is the fp32 sum: y and its quantisation are taken from it, not from the h
// that is stored rounded.  y is stored in 16 or 32 bits, and/or quantised to e4m3
// with a scale per 128 columns by quantize_rows' rule (fp8.cuh), from the fp32
// value.  With g = dy w and xhat = h rstd the gradient is
//
//   dx = rstd (g - xhat mean(g xhat)) + dh,   dw = sum over rows of dy xhat.
//
// A row is held in registers by its threads, 8 columns at a time (16 consecutive
// threads: one 128-column block of the quantisation), so every operand is read
// once and h or dx may take an operand's place.  The gradient's threads keep
// their columns' share of dw over all their rows; a second kernel adds up the
// CTAs' shares in a fixed order.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"

namespace ec2moe {

namespace {

constexpr int PER = 8;        // columns per thread and step: 16 bytes of bf16
constexpr int MAX_WARPS = 32;

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

template <typename TX, typename TY, int NCH>
__global__ void __launch_bounds__(NCH == 1 ? 1024 : 512) rmsnorm_kernel(const NormArgs a, int tpr) {
  pdl_trigger();
  pdl_wait();
  __shared__ float s_sum[MAX_WARPS];
  const int rpb = blockDim.x / tpr;
  const int t = threadIdx.x % tpr;
  const long long row = static_cast<long long>(blockIdx.x) * rpb + threadIdx.x / tpr;
  const bool in = row < a.rows;
  const int n_chunks = a.cols / PER;
  const TX* x = static_cast<const TX*>(a.X) + row * a.ld;
  const TX* res = static_cast<const TX*>(a.residual) + row * a.ld;
  float h[NCH][PER];
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = i * tpr + t;
#pragma unroll
    for (int j = 0; j < PER; ++j) h[i][j] = 0.0f;
    if (in && c < n_chunks) load8(x + c * PER, h[i]);
  }
  if (a.residual) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = i * tpr + t;
      if (in && c < n_chunks) {
        float r[PER];
        load8(res + c * PER, r);
#pragma unroll
        for (int j = 0; j < PER; ++j) h[i][j] += r[j];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int j = 0; j < PER; ++j) sum = fmaf(h[i][j], h[i][j], sum);
  sum = row_sum(sum, tpr, s_sum);
  const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fdiv_rn(sum, static_cast<float>(a.cols)) + a.eps));
  if (in && t == 0 && a.rstd) a.rstd[row] = rstd;
  const int n_kb = (a.cols + FP8_BLOCK - 1) / FP8_BLOCK;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = i * tpr + t;
    if (i * tpr >= n_chunks) break;  // the whole row
    const bool mine = in && c < n_chunks;
    if (mine && a.H) store8(static_cast<TX*>(a.H) + row * a.cols + c * PER, h[i]);
    float w[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) w[j] = 1.0f;
    if (mine && a.weight) load8(a.weight + c * PER, w);
#pragma unroll
    for (int j = 0; j < PER; ++j) h[i][j] = h[i][j] * rstd * w[j];
    if (mine && a.Y) store8(static_cast<TY*>(a.Y) + row * a.cols + c * PER, h[i]);
    if (a.Q) {
      float m = 0.0f;
      if (mine) {
#pragma unroll
        for (int j = 0; j < PER; ++j) m = fmaxf(m, fabsf(h[i][j]));
      }
#pragma unroll
      for (int o = 1; o < FP8_BLOCK / PER; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      if (mine) {
        const Fp8Scale f = fp8_scale(m);
        const uint32_t lo = fp8_pack2(h[i][0], h[i][1], f.inv) | (fp8_pack2(h[i][2], h[i][3], f.inv) << 16);
        const uint32_t hi = fp8_pack2(h[i][4], h[i][5], f.inv) | (fp8_pack2(h[i][6], h[i][7], f.inv) << 16);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(a.Q) + row * a.cols + c * PER) = make_uint2(lo, hi);
        if (c % (FP8_BLOCK / PER) == 0) a.scale[row * n_kb + c / (FP8_BLOCK / PER)] = f.scale;
      }
    }
  }
}

template <typename TX, typename TY, int NCH>
__global__ void __launch_bounds__(512) rmsnorm_backward_kernel(const NormBackArgs a, int tpr) {
  pdl_trigger();
  pdl_wait();
  extern __shared__ float s_dw[];  // [rows of the CTA - 1][cols]
  __shared__ float s_sum[MAX_WARPS];
  const int rpb = blockDim.x / tpr;
  const int t = threadIdx.x % tpr, mine_row = threadIdx.x / tpr;
  const int n_chunks = a.cols / PER;
  float dw[NCH][PER] = {};
  const long long step = static_cast<long long>(gridDim.x) * rpb;
  for (long long first = static_cast<long long>(blockIdx.x) * rpb; first < a.rows; first += step) {
    const long long row = first + mine_row;
    const bool in = row < a.rows;
    const float rstd = in ? a.rstd[row] : 0.0f;
    float g[NCH][PER], xh[NCH][PER];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = i * tpr + t;
#pragma unroll
      for (int j = 0; j < PER; ++j) g[i][j] = xh[i][j] = 0.0f;
      if (in && c < n_chunks) {
        load8(static_cast<const TY*>(a.dY) + row * a.ld + c * PER, g[i]);
        load8(static_cast<const TX*>(a.H) + row * a.cols + c * PER, xh[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = i * tpr + t;
      float w[PER];
#pragma unroll
      for (int j = 0; j < PER; ++j) w[j] = 1.0f;
      if (c < n_chunks && a.weight) load8(a.weight + c * PER, w);
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        xh[i][j] *= rstd;
        dw[i][j] = fmaf(g[i][j], xh[i][j], dw[i][j]);
        g[i][j] *= w[j];
        sum = fmaf(g[i][j], xh[i][j], sum);
      }
    }
    const float mean = __fdiv_rn(row_sum(sum, tpr, s_sum), static_cast<float>(a.cols));
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = i * tpr + t;
      if (!in || c >= n_chunks) continue;
      float d[PER];
#pragma unroll
      for (int j = 0; j < PER; ++j) d[j] = rstd * (g[i][j] - xh[i][j] * mean);
      if (a.dH) {
        float r[PER];
        load8(static_cast<const TX*>(a.dH) + row * a.cols + c * PER, r);
#pragma unroll
        for (int j = 0; j < PER; ++j) d[j] += r[j];
      }
      store8(static_cast<TX*>(a.dX) + row * a.cols + c * PER, d);
    }
  }
  if (!a.d_weight) return;
  // the CTA's rows' shares, in order, then one share per CTA
  __syncthreads();
  if (mine_row > 0) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = i * tpr + t;
      if (c < n_chunks) store8(s_dw + (mine_row - 1) * a.cols + c * PER, dw[i]);
    }
  }
  __syncthreads();
  if (mine_row == 0) {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = i * tpr + t;
      if (c >= n_chunks) continue;
      for (int r = 0; r + 1 < rpb; ++r) {
        float o[PER];
        load8(s_dw + r * a.cols + c * PER, o);
#pragma unroll
        for (int j = 0; j < PER; ++j) dw[i][j] += o[j];
      }
      store8(a.partial + static_cast<long long>(blockIdx.x) * a.cols + c * PER, dw[i]);
    }
  }
}

// out[c] = sum of partial[0 .. n)[c]: 32 columns per CTA, its warps take every
// eighth row, their sums are added in order.
__global__ void __launch_bounds__(256) dweight_sum_kernel(const float* partial, int n, int cols, float* out) {
  pdl_trigger();
  pdl_wait();
  __shared__ float s[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  float v = 0.0f;
  if (c < cols) {
#pragma unroll 8
    for (int r = warp; r < n; r += 8) v += partial[static_cast<long long>(r) * cols + c];
  }
  s[warp][lane] = v;
  __syncthreads();
  if (warp == 0 && c < cols) {
#pragma unroll
    for (int w = 1; w < 8; ++w) v += s[w][lane];
    out[c] = v;
  }
}

int round_warps(int threads) { return (threads + 31) / 32 * 32; }

template <typename TX, typename TY>
cudaError_t forward(const NormArgs& a, cudaStream_t s) {
  const int n_chunks = a.cols / PER;
  KernelScope ks("rmsnorm", s);
  const bool one = n_chunks <= 1024 && a.rows < 2 * sm_count();
  const int tpr = round_warps(one ? n_chunks : (n_chunks + 3) / 4);
  int rpb = one ? 1 : 256 / tpr;
  if (rpb < 1) rpb = 1;
  const unsigned grid = static_cast<unsigned>((static_cast<long long>(a.rows) + rpb - 1) / rpb);
  cudaError_t e = one ? launch_kernel(rmsnorm_kernel<TX, TY, 1>, dim3(grid), dim3(tpr * rpb), 0, s, a, tpr)
                      : launch_kernel(rmsnorm_kernel<TX, TY, 4>, dim3(grid), dim3(tpr * rpb), 0, s, a, tpr);
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

struct BackShape {
  int tpr, rpb, grid;
};
BackShape back_shape(int rows, int cols) {
  BackShape b;
  b.tpr = round_warps((cols / PER + 3) / 4);
  b.rpb = 256 / b.tpr < 1 ? 1 : 256 / b.tpr;
  const long long units = (static_cast<long long>(rows) + b.rpb - 1) / b.rpb;
  const long long most = 2LL * sm_count();
  b.grid = static_cast<int>(units < most ? units : most);
  return b;
}

template <typename TX, typename TY>
cudaError_t backward(const NormBackArgs& a, cudaStream_t s) {
  const BackShape b = back_shape(a.rows, a.cols);
  const size_t smem = static_cast<size_t>(b.rpb - 1) * a.cols * 4;  // at most 7 rows of 1024
  {
    KernelScope ks("rmsnorm_backward", s);
    cudaError_t e = launch_kernel(rmsnorm_backward_kernel<TX, TY, 4>, dim3(b.grid), dim3(b.tpr * b.rpb), smem, s, a, b.tpr);
    if (e != cudaSuccess) return e;
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (!a.d_weight) return cudaSuccess;
  KernelScope ks("rmsnorm_dweight", s);
  cudaError_t e = launch_kernel(dweight_sum_kernel, dim3((a.cols + 31) / 32), dim3(256), 0, s, a.partial, b.grid, a.cols,
                                a.d_weight);
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

}  // namespace

size_t norm_backward_bytes(int rows, int cols) { return static_cast<size_t>(back_shape(rows, cols).grid) * cols * 4; }

cudaError_t launch_rmsnorm(const NormArgs& a, bool bf16, bool y_bf16, cudaStream_t s) {
  if (bf16) return y_bf16 ? forward<__nv_bfloat16, __nv_bfloat16>(a, s) : forward<__nv_bfloat16, float>(a, s);
  return y_bf16 ? forward<float, __nv_bfloat16>(a, s) : forward<float, float>(a, s);
}

cudaError_t launch_rmsnorm_backward(const NormBackArgs& a, bool bf16, bool y_bf16, cudaStream_t s) {
  if (bf16) return y_bf16 ? backward<__nv_bfloat16, __nv_bfloat16>(a, s) : backward<__nv_bfloat16, float>(a, s);
  return y_bf16 ? backward<float, __nv_bfloat16>(a, s) : backward<float, float>(a, s);
}

}  // namespace ec2moe
