// Quantisation to 8-bit floating point (e4m3) with one fp32 scale for each block
// of 128 columns: of one row (activations) or of 128 rows (weights).
//
//   a = max(2^-96, max |x| over the block),  s = a / 448,  q = e4m3(x * (448 / a))
//
// 448 is e4m3's largest value, so nothing saturates; the two quotients are
// rounded once to fp32 each and the product once to fp32 and once to e4m3 (to
// nearest, ties to even).  The floor on a keeps 448 / a finite and makes a block
// of zeros an ordinary one.  A NaN element becomes e4m3's NaN and leaves its
// block alone; an infinite element makes the scale infinite and the block's
// products with it NaN, as the sum over them is in any precision.
//
// Rows can be written straight into expert order: row t goes to the rows
// inv_perm[t k .. t k + k - 1], so the k copies of an activation row are made
// from one read of it and at one byte per element.
//
// Bounded by HBM: 16384 x 2048 bf16 to six copies, 275 MB, 40.8 us (6.7 TB/s, 0.99
// of a copy's rate) in the kernel and 45 us with its launch; short calls by the
// launch (64 x 4096: 5 us).
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"

namespace ec2moe {

// nonzero: a placement outside the rows of the call was skipped
__device__ unsigned int g_quant_error;

namespace {

constexpr int PER = 16;                      // elements per thread: one 16-byte store
constexpr int LANES = FP8_BLOCK / PER;       // threads per 128-column block

template <typename T>
__device__ __forceinline__ void load16(const T* p, float* v) {
  load8(p, v);
  load8(p + 8, v + 8);
}

__device__ __forceinline__ float absmax16(const float* v) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < PER; ++i) m = fmaxf(m, fabsf(v[i]));
  return m;
}

// One block of a row per LANES threads.
template <typename T>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T* X, long long ld, int rows, int cols, int n_kb,
                                                            const int32_t* inv_perm, int k, uint8_t* Q, float* S) {
  pdl_trigger();
  pdl_wait();
  const uint32_t unit = blockIdx.x * (256u / LANES) + threadIdx.x / LANES;  // below 2^31 + 32
  const int part = threadIdx.x % LANES;
  const long long row = unit / static_cast<uint32_t>(n_kb);
  const int kb = static_cast<int>(unit - static_cast<uint32_t>(row) * n_kb);
  const int col = kb * FP8_BLOCK + part * PER;
  const bool in = row < rows;
  const bool mine = in && col < cols;
  float v[PER] = {};
  if (mine) load16(X + row * ld + col, v);
  float m = absmax16(v);
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (!in) return;
  const Fp8Scale f = fp8_scale(m);
  const U4 q = fp8_pack16(v, f.inv);
  if (!inv_perm) {
    if (mine) *reinterpret_cast<U4*>(Q + row * cols + col) = q;
    if (part == 0) S[row * n_kb + kb] = f.scale;
    return;
  }
  const long long n = static_cast<long long>(rows) * k;
  for (int s = 0; s < k; ++s) {
    const long long dst = inv_perm[row * k + s];
    if (dst < 0 || dst >= n) {
      if (dst != -1 && part == 0) atomicOr(&g_quant_error, 1u);  // -1: an entry that routing skipped
      continue;
    }
    if (mine) *reinterpret_cast<U4*>(Q + dst * cols + col) = q;
    if (part == 0) S[dst * n_kb + kb] = f.scale;
  }
}

// One 128 x 128 block of a weight matrix per CTA.
template <typename T>
__global__ void __launch_bounds__(256) quantize_blocks_kernel(const T* X, long long ld, int rows, int cols, int n_rb,
                                                              int n_kb, uint8_t* Q, float* S) {
  pdl_trigger();
  pdl_wait();
  constexpr int ROWS_PER_PASS = 256 / LANES;
  constexpr int PASSES = FP8_BLOCK / ROWS_PER_PASS;
  __shared__ float warp_max[8];
  const long long unit = blockIdx.x;
  const int kb = static_cast<int>(unit % n_kb);
  const long long rest = unit / n_kb;
  const int rb = static_cast<int>(rest % n_rb);
  const long long row0 = (rest / n_rb) * rows;  // the matrix's first row
  const int part = threadIdx.x % LANES;
  const int col = kb * FP8_BLOCK + part * PER;
  float v[PASSES][PER] = {};
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int r = rb * FP8_BLOCK + i * ROWS_PER_PASS + threadIdx.x / LANES;
    if (r < rows && col < cols) load16(X + (row0 + r) * ld + col, v[i]);
  }
#pragma unroll
  for (int i = 0; i < PASSES; ++i) m = fmaxf(m, absmax16(v[i]));
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (threadIdx.x % 32 == 0) warp_max[threadIdx.x / 32] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, warp_max[i]);
  const Fp8Scale f = fp8_scale(m);
  if (threadIdx.x == 0) S[unit] = f.scale;
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int r = rb * FP8_BLOCK + i * ROWS_PER_PASS + threadIdx.x / LANES;
    if (r < rows && col < cols) *reinterpret_cast<U4*>(Q + (row0 + r) * cols + col) = fp8_pack16(v[i], f.inv);
  }
}

template <typename T>
cudaError_t launch(const QuantArgs& a, cudaStream_t s) {
  const int n_kb = (a.cols + FP8_BLOCK - 1) / FP8_BLOCK;
  const T* X = static_cast<const T*>(a.X);
  uint8_t* Q = static_cast<uint8_t*>(a.Q);
  KernelScope ks(a.block_rows == 1 ? "quantize_rows" : "quantize_blocks", s);
  cudaError_t e;
  if (a.block_rows == 1) {
    const int rows = a.n_mats * a.rows;
    const long long threads = static_cast<long long>(rows) * n_kb * LANES;
    e = launch_kernel(quantize_rows_kernel<T>, dim3(static_cast<unsigned>((threads + 255) / 256)), dim3(256), 0, s, X,
                      a.ld, rows, a.cols, n_kb, a.inv_perm, a.k, Q, a.scale);
  } else {
    const int n_rb = (a.rows + FP8_BLOCK - 1) / FP8_BLOCK;
    e = launch_kernel(quantize_blocks_kernel<T>, dim3(static_cast<unsigned>((long long)a.n_mats * n_rb * n_kb)),
                      dim3(256), 0, s, X, a.ld, a.rows, a.cols, n_rb, n_kb, Q, a.scale);
  }
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_quantize(const QuantArgs& a, bool bf16, cudaStream_t s) {
  return bf16 ? launch<__nv_bfloat16>(a, s) : launch<float>(a, s);
}

cudaError_t read_quant_error(unsigned int* word) {
  unsigned int zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(word, g_quant_error, sizeof(unsigned int));
  if (e != cudaSuccess) return e;
  return cudaMemcpyToSymbol(g_quant_error, &zero, sizeof(unsigned int));
}

}  // namespace ec2moe
