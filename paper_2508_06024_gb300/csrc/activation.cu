// The experts' activation on its own, with each row's gate weight, and its
// gradient: what a training step does between the up and the down products.
//
//   a = SiLU(u) v  or  GELU(u) (exact erf form),   h = s a
//
// with s the gate weight of the row's slot.  SiLU(u) = u p with p = 1 / (1 + e^-u),
// SiLU'(u) = p (1 + u (1 - p)); GELU(u) = u P(u) with P the normal distribution,
// GELU'(u) = P(u) + u e^(-u^2 / 2) / sqrt(2 pi).  P is taken from the fitted erfc of the 8-bit
// experts (2.8e-8 at most, fp8.cuh): erff bound the kernel by its instructions (98304 x
// 1408 GELU: 169 us, now 115; gradient 256, 206).  The gradient computes h again (the
// weights' gradient needs it, and it costs no read) and the gate weight's, the row's sum
// of dh a.
//
// Bounded by HBM.  A row is walked by `tpr` threads (whole warps), 8 columns each
// at a time.  SwiGLU, 98304 x 1408 bf16: 124 us (6.7 TB/s), gradient 270 us (6.1 TB/s);
// 1554 x 14336, gradient: 47 us (5.7 TB/s; 3.4 waves of CTAs of one row each).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "common.cuh"
#include "fp8.cuh"
#include "internal.h"

namespace ec2moe {

// nonzero: a slot outside the rows of the call was skipped
__device__ unsigned int g_act_error;

namespace {

constexpr int PER = 8;
constexpr int THREADS = 256;

// 8 elements as they lie in memory: fetched ahead, widened when they are used.
template <typename T>
struct Raw8 {
  U4 w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Raw8<T> fetch8(const T* p) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) r.w[i] = reinterpret_cast<const U4*>(p)[i];
  return r;
}
__device__ __forceinline__ void widen8(const Raw8<__nv_bfloat16>& r, float* v) {
  const U4& q = r.w[0];
  v[0] = bf16_lo(q.x); v[1] = bf16_hi(q.x); v[2] = bf16_lo(q.y); v[3] = bf16_hi(q.y);
  v[4] = bf16_lo(q.z); v[5] = bf16_hi(q.z); v[6] = bf16_lo(q.w); v[7] = bf16_hi(q.w);
}
__device__ __forceinline__ void widen8(const Raw8<float>& r, float* v) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    v[4 * i + 0] = __uint_as_float(r.w[i].x);
    v[4 * i + 1] = __uint_as_float(r.w[i].y);
    v[4 * i + 2] = __uint_as_float(r.w[i].z);
    v[4 * i + 3] = __uint_as_float(r.w[i].w);
  }
}

__device__ __forceinline__ float sigmoid(float u) { return __fdividef(1.0f, 1.0f + __expf(-u)); }

// P(u), with e = e^(-u^2 / 2).
__device__ __forceinline__ float normal(float u, float e) {
  const float tail = 0.5f * erfc_fit(fabsf(u), e);
  return u < 0.0f ? tail : 1.0f - tail;
}

// The row's slot, or -1 (reported) where perm names none of the call's rows.
__device__ __forceinline__ int slot_of(const ActArgs& a, long long row, int t) {
  if (!a.perm) return static_cast<int>(row);
  const int slot = a.perm[row];
  if (slot >= 0 && slot < a.rows) return slot;
  if (t == 0) atomicOr(&g_act_error, 1u);
  return -1;
}

template <typename T, bool GLU>
__global__ void __launch_bounds__(THREADS) activation_kernel(const ActArgs a, int tpr) {
  pdl_trigger();
  pdl_wait();
  const int t = threadIdx.x % tpr;
  const long long row = static_cast<long long>(blockIdx.x) * (THREADS / tpr) + threadIdx.x / tpr;
  if (row >= a.rows) return;
  const int slot = slot_of(a, row, t);
  if (slot < 0) return;
  const float w = a.row_scale ? a.row_scale[slot] : 1.0f;
  const T* u = static_cast<const T*>(a.U) + row * a.ld;
  const T* v = static_cast<const T*>(a.V) + row * a.ld;
  T* h = static_cast<T*>(a.H) + row * a.cols;
#pragma unroll 2
  for (int c = t * PER; c < a.cols; c += tpr * PER) {
    float x[PER], y[PER];
    load8(u + c, x);
    if (GLU) load8(v + c, y);
#pragma unroll
    for (int j = 0; j < PER; ++j) x[j] = GLU ? x[j] * sigmoid(x[j]) * y[j] * w : x[j] * normal(x[j], gauss(x[j])) * w;
    store8(h + c, x);
  }
}

template <typename T, bool GLU>
__global__ void __launch_bounds__(THREADS, sizeof(T) == 2 ? 4 : 3) activation_backward_kernel(const ActArgs a, int tpr) {
  pdl_trigger();
  pdl_wait();
  __shared__ float s_sum[THREADS / 32];
  const int t = threadIdx.x % tpr;
  const long long row = static_cast<long long>(blockIdx.x) * (THREADS / tpr) + threadIdx.x / tpr;
  const bool in = row < a.rows;
  const int slot = in ? slot_of(a, row, t) : -1;
  float sum = 0.0f;
  if (slot >= 0) {
    const float w = a.row_scale ? a.row_scale[slot] : 1.0f;
    const T* u = static_cast<const T*>(a.U) + row * a.ld;
    const T* v = static_cast<const T*>(a.V) + row * a.ld;
    const T* dh = static_cast<const T*>(a.dH) + row * a.cols;
    T* du = static_cast<T*>(a.dU) + row * a.ld;
    T* dv = static_cast<T*>(a.dV) + row * a.ld;
    T* h = static_cast<T*>(a.H) + row * a.cols;
    // the next chunk's operands are on their way while this one's are used
    Raw8<T> nu{}, nv{}, ng{};
    if (t * PER < a.cols) {
      nu = fetch8(u + t * PER);
      if (GLU) nv = fetch8(v + t * PER);
      ng = fetch8(dh + t * PER);
    }
#pragma unroll 1
    for (int c = t * PER; c < a.cols; c += tpr * PER) {
      float x[PER], y[PER], g[PER], o[PER];
      widen8(nu, x);
      if (GLU) widen8(nv, y);
      widen8(ng, g);
      const int next = c + tpr * PER;
      if (next < a.cols) {
        nu = fetch8(u + next);
        if (GLU) nv = fetch8(v + next);
        ng = fetch8(dh + next);
      }
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        const float gw = g[j] * w;
        if (GLU) {
          const float p = sigmoid(x[j]), s = x[j] * p, act = s * y[j];
          sum = fmaf(g[j], act, sum);
          o[j] = act * w;
          x[j] = gw * y[j] * (p * (1.0f + x[j] * (1.0f - p)));
          y[j] = gw * s;
        } else {
          const float e = gauss(x[j]), P = normal(x[j], e), act = x[j] * P;
          sum = fmaf(g[j], act, sum);
          o[j] = act * w;
          x[j] = gw * (P + x[j] * e * 0.3989422804014327f);
        }
      }
      store8(du + c, x);
      if (GLU) store8(dv + c, y);
      if (a.H) store8(h + c, o);
    }
  }
  if (!a.d_row_scale) return;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  const int warp = threadIdx.x >> 5, per = tpr >> 5;
  if ((threadIdx.x & 31) == 0) s_sum[warp] = sum;
  __syncthreads();
  if (t == 0 && slot >= 0) {
    for (int i = 1; i < per; ++i) sum += s_sum[warp + i];
    a.d_row_scale[slot] = sum;
  }
}

template <typename T, bool GLU>
cudaError_t launch(const ActArgs& a, bool back, cudaStream_t s) {
  int tpr = 32;
  while (tpr < THREADS && a.cols > tpr * PER * 4) tpr *= 2;
  const int rpb = THREADS / tpr;
  const unsigned grid = static_cast<unsigned>((static_cast<long long>(a.rows) + rpb - 1) / rpb);
  KernelScope ks(back ? "activation_backward" : "activation", s);
  cudaError_t e = back ? launch_kernel(activation_backward_kernel<T, GLU>, dim3(grid), dim3(THREADS), 0, s, a, tpr)
                       : launch_kernel(activation_kernel<T, GLU>, dim3(grid), dim3(THREADS), 0, s, a, tpr);
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_activation(const ActArgs& a, bool bf16, bool glu, bool back, cudaStream_t s) {
  if (bf16) return glu ? launch<__nv_bfloat16, true>(a, back, s) : launch<__nv_bfloat16, false>(a, back, s);
  return glu ? launch<float, true>(a, back, s) : launch<float, false>(a, back, s);
}

cudaError_t read_act_error(unsigned int* word) {
  unsigned int zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(word, g_act_error, sizeof(unsigned int));
  if (e != cudaSuccess) return e;
  return cudaMemcpyToSymbol(g_act_error, &zero, sizeof(unsigned int));
}

}  // namespace ec2moe
