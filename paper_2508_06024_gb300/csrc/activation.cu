// The experts' activation on its own, with each row's gate weight, and its
// gradient: what a training step does between the up and the down products.
//
//   a = SiLU(u) v  or  GELU(u) (exact erf form),   h = s a
//
// with s the gate weight of the row's slot.  SiLU(u) = u p with p = 1 / (1 + e^-u),
// SiLU'(u) = p (1 + u (1 - p)); GELU(u) = u P(u) with P the normal distribution,
// GELU'(u) = P(u) + u e^(-u^2 / 2) / sqrt(2 pi).  P is taken from the fitted erfc of the 8-bit
// experts (2.8e-8 at most, fp8.cuh): erff bound the kernel by its instructions (98304 x
// 1408 GELU: 169 us, now 103; gradient 256, 199).  The gradient computes h again (the
// weights' gradient needs it, and it costs no read) and the gate weight's, the row's sum
// of dh a.
//
// Bounded by HBM.  A row is walked by `tpr` threads (whole warps), 8 columns each
// at a time.  SwiGLU, 98304 x 1408 bf16: 124 us (6.7 TB/s), gradient 270 us (6.1 TB/s);
// 1554 x 14336, gradient: 47 us (5.7 TB/s; 2.6 waves of CTAs of one row each, four to an SM).
// GELU is bound by its instructions (floors of 82 and 163).
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
static_assert(ACT_MAX_COLS <= 0x7fffffff - THREADS * PER, "the step behind the last column");

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

// 1 / (1 + e^-u).  Of bf16 rows through the fast exponential and division, whose error (2e-6 of the
// result at |u| = 12) is far below the result's rounding; of fp32 rows to fp32's own accuracy
// (49152 x 1408: 128 us and 248 for the gradient, through the fast ones 127 and 244).
template <typename T>
__device__ __forceinline__ float sigmoid(float u) {
  if constexpr (sizeof(T) == 2) return __fdividef(1.0f, 1.0f + __expf(-u));
  return __fdiv_rn(1.0f, 1.0f + expf(-u));
}

// GELU is computed two columns at a time, its products and sums as pairs (f32x2): with the
// other half of the instructions the same rows take 115 us, the gradient 206.
__device__ __forceinline__ unsigned long long bits2(float2 v) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(v.x), "f"(v.y));
  return r;
}
__device__ __forceinline__ float2 floats2(unsigned long long r) {
  float2 v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(r));
  return v;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
  return floats2(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
  return floats2(r);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
// e^(-u^2 / 2), and with it P(u) = erfc(-u / sqrt 2) / 2.
__device__ __forceinline__ float2 gauss2(float2 u) {
  const float2 q = mul2(mul2(u, u), both(GAUSS));
  float2 e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(q.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(q.y));
  return e;
}
__device__ __forceinline__ float2 normal2(float2 u, float2 e) {
  const float2 d = fma2(make_float2(fabsf(u.x), fabsf(u.y)), both(ERFC_T), both(1.0f));
  float2 t;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t.x) : "f"(d.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t.y) : "f"(d.y));
  float2 q = fma2(t, both(0.5f * ERFC_6), both(0.5f * ERFC_5));
  q = fma2(t, q, both(0.5f * ERFC_4));
  q = fma2(t, q, both(0.5f * ERFC_3));
  q = fma2(t, q, both(0.5f * ERFC_2));
  q = fma2(t, q, both(0.5f * ERFC_1));
  q = mul2(mul2(q, t), e);
  return make_float2(u.x < 0.0f ? q.x : 1.0f - q.x, u.y < 0.0f ? q.y : 1.0f - q.y);
}

// The row's slot, or -1 (reported) where perm names none of the call's rows.
__device__ __forceinline__ int slot_of(const ActArgs& a, long long row, int t) {
  if (!a.perm) return static_cast<int>(row);
  const int slot = a.perm[row];
  if (slot >= 0 && slot < a.rows) return slot;
  if (t == 0) atomicOr(&g_act_error, 1u);
  return -1;
}

// As many warps as an SM holds and a chunk at a time (two of them unrolled: GELU as above 109 us).
template <typename T, bool GLU>
__global__ void __launch_bounds__(THREADS, 8) activation_kernel(const ActArgs a, int tpr) {
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
#pragma unroll 1
  for (int c = t * PER; c < a.cols; c += tpr * PER) {
    float x[PER], y[PER];
    load8(u + c, x);
    if (GLU) load8(v + c, y);
#pragma unroll
    for (int j = 0; j < PER; j += 2) {
      if (GLU) {
        x[j] = x[j] * sigmoid<T>(x[j]) * y[j] * w;
        x[j + 1] = x[j + 1] * sigmoid<T>(x[j + 1]) * y[j + 1] * w;
      } else {
        const float2 u = make_float2(x[j], x[j + 1]), r = mul2(mul2(u, normal2(u, gauss2(u))), both(w));
        x[j] = r.x;
        x[j + 1] = r.y;
      }
    }
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
      if constexpr (GLU) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
          const float gw = g[j] * w, p = sigmoid<T>(x[j]), s = x[j] * p, act = s * y[j];
          sum = fmaf(g[j], act, sum);
          o[j] = act * w;
          x[j] = gw * y[j] * (p * (1.0f + x[j] * (1.0f - p)));
          y[j] = gw * s;
        }
      } else {
#pragma unroll
        for (int j = 0; j < PER; j += 2) {
          const float2 u = make_float2(x[j], x[j + 1]), e = gauss2(u), P = normal2(u, e), act = mul2(u, P);
          sum = fmaf(g[j + 1], act.y, fmaf(g[j], act.x, sum));
          const float2 h2 = mul2(act, both(w)), d = fma2(mul2(u, e), both(0.3989422804014327f), P);
          const float2 du2 = mul2(mul2(make_float2(g[j], g[j + 1]), both(w)), d);
          o[j] = h2.x;
          o[j + 1] = h2.y;
          x[j] = du2.x;
          x[j + 1] = du2.y;
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
