// The gate's logits in fp32 accuracy, [T, E + K]: X W_local^T + b_local, then
// X W_global^T + b_global (Eq. 5 and 6 before their softmaxes), as training and
// tuning of the gate need them.
//
// bf16 activations: every fp32 gate row is split exactly into three bf16 terms
// (w = w0 + w1 + w2, the rest below 2^-24 |w|) whose products with a bf16 value
// are exact in fp32; the three terms are rows of one tensor-core product.  The
// tensor core adds without rounding to nearest, so K is cut into ranges whose
// sums a last kernel adds in fp32 with the bias.  fp32 activations take the
// fp32-accurate GEMM.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "common.cuh"
#include "internal.h"

namespace ec2moe {
namespace {

constexpr int RANGE = 512;  // columns of X summed on the tensor core

// Gate row o (local rows, then global ones) of length d.
__device__ __forceinline__ const float* gate_row(const float* W_local, const float* W_global, int E, int d, int o) {
  return o < E ? W_local + static_cast<size_t>(o) * d : W_global + static_cast<size_t>(o - E) * d;
}

// terms[j * O + o][c] = term j of gate row o; four columns per thread.
__global__ void __launch_bounds__(256) logits_split_kernel(const float* W_local, const float* W_global, int E, int O,
                                                           int d, __nv_bfloat16* terms) {
  pdl_trigger();
  pdl_wait();
  const long long i = (blockIdx.x * 256LL + threadIdx.x) * 4;
  if (i >= static_cast<long long>(O) * d) return;
  const int o = static_cast<int>(i / d), c = static_cast<int>(i % d);
  const float4 w = *reinterpret_cast<const float4*>(gate_row(W_local, W_global, E, d, o) + c);
  float v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    const uint32_t lo = pack_bf16x2(v[0], v[1]), hi = pack_bf16x2(v[2], v[3]);
    *reinterpret_cast<uint2*>(terms + (static_cast<size_t>(j) * O + o) * d + c) = make_uint2(lo, hi);
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
__global__ void __launch_bounds__(256) logits_sum_kernel(const float* part, int ranges, int terms, int N, int T, int E,
                                                         int O, const float* b_local, const float* b_global,
                                                         float* logits) {
  pdl_trigger();
  pdl_wait();
  const long long i = blockIdx.x * 256LL + threadIdx.x;
  if (i >= static_cast<long long>(T) * O) return;
  const long long t = i / O;
  const int o = static_cast<int>(i - t * O);
  float v = o < E ? b_local[o] : b_global[o - E];
  for (int j = terms - 1; j >= 0; --j)
    for (int r = 0; r < ranges; ++r) v += part[(static_cast<long long>(r) * T + t) * N + j * O + o];
  logits[i] = v;
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

struct Plan {
  int O, N, ranges;
  size_t rows, total;  // bytes of the prepared gate rows, and with the partial sums
};
Plan make_plan(int T, int d, int E, int K, bool bf16) {
  Plan p;
  p.O = E + (K > 1 ? K : 0);
  p.N = bf16 ? (3 * p.O + 31) / 32 * 32 : (p.O + 7) / 8 * 8;
  p.ranges = 1;
  if (bf16) {
    // the count of non-empty ranges that the GEMM derives from this request
    const int nk = (d + 63) / 64, want = (d + RANGE - 1) / RANGE, per = (nk + want - 1) / want;
    p.ranges = (nk + per - 1) / per;
  }
  p.rows = align256(static_cast<size_t>(bf16 ? 3 * p.O : p.N) * d * (bf16 ? 2 : 4));
  p.total = p.rows + align256(static_cast<size_t>(p.ranges) * T * p.N * 4);
  return p;
}

}  // namespace

size_t gate_logits_bytes(int T, int d, int E, int K, bool bf16) { return make_plan(T, d, E, K, bf16).total; }

cudaError_t launch_gate_logits(const LogitsArgs& a, bool bf16, cudaStream_t s) {
  const Plan p = make_plan(a.T, a.d, a.E, a.K, bf16);
  void* rows = a.workspace;
  float* part = reinterpret_cast<float*>(static_cast<uint8_t*>(a.workspace) + p.rows);
  const long long items = static_cast<long long>(bf16 ? p.O : p.N) * a.d / 4;
  cudaError_t e;
  {
    KernelScope ks("logits_prep", s);
    const dim3 grid(static_cast<unsigned>((items + 255) / 256));
    e = bf16 ? launch_kernel(logits_split_kernel, grid, dim3(256), 0, s, a.W_local, a.W_global, a.E, p.O, a.d,
                             static_cast<__nv_bfloat16*>(rows))
             : launch_kernel(logits_rows_kernel, grid, dim3(256), 0, s, a.W_local, a.W_global, a.E, p.O, p.N,
                             a.d, static_cast<float*>(rows));
    if (e != cudaSuccess) return e;
  }
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
                    s, part, p.ranges, bf16 ? 3 : 1, p.N, a.T, a.E, p.O, a.b_local, a.b_global, a.logits);
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

}  // namespace ec2moe
