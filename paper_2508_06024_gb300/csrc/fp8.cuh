// Device helpers of the 8-bit floating point path: the scale of a block, the
// conversion of its values, and the tcgen05 forms of 8-bit operands.
#pragma once

#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "tc_ptx.cuh"

namespace ec2moe {

constexpr int FP8_BLOCK = 128;  // columns that share a scale

struct Fp8Scale {
  float scale;  // what a stored value is multiplied by
  float inv;    // what a value is multiplied by before it is stored
};
// Scale of a block whose largest magnitude is m: 448 (e4m3's largest value)
// stands for m, and for 2^-96 where m is smaller.
__device__ __forceinline__ Fp8Scale fp8_scale(float m) {
  const float a = fmaxf(m, 0x1p-96f);
  return Fp8Scale{__fdiv_rn(a, 448.0f), __fdiv_rn(448.0f, a)};
}

// First rows, row counts and the prefix of token tiles of TILE rows of G <= 32 CHUNKS
// groups, from `offsets` (nullptr: one group of all rows).  One warp.  A range that is
// not inside [0, rows] owns no rows; where there is one, ranges behind it may go over
// the same rows again, so a group that starts before the end of one before it owns none
// either: groups never own more than `rows` rows together, which grids and workspaces
// are sized by.  err (nullptr: not reported): bit 1 is set when a range is skipped.
template <int CHUNKS, int TILE>
__device__ __forceinline__ void scan_group_rows(const int32_t* offsets, int G, int rows, int lane, int* row0, int* cnt,
                                                int* prefix, unsigned int* err) {
  int first[CHUNKS], n[CHUNKS];
  bool bad = false;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int g = c * 32 + lane;
    first[c] = 0;
    n[c] = g < G ? rows : 0;
    if (offsets && g < G) {
      const int a = offsets[g], b = offsets[g + 1];
      const bool in = a >= 0 && a <= b && b <= rows;
      first[c] = in ? a : 0;
      n[c] = in ? b - a : 0;
      bad |= !in;
    }
  }
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
    if (c * 32 + lane < G) {
      row0[c * 32 + lane] = first[c];
      cnt[c * 32 + lane] = n[c];
    }
  // ranges that are all in place do not decrease, so they cannot overlap
  if (__any_sync(0xffffffffu, bad)) {
    if (err && lane == 0) atomicOr(err, 2u);
    int reach = 0;  // where the groups before end
#pragma unroll 1
    for (int g = lane; g - lane < G; g += 32) {
      const int from = g < G ? row0[g] : 0, rows_of = g < G ? cnt[g] : 0;
      int end = rows_of > 0 ? from + rows_of : 0;
#pragma unroll 1
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, end, o);
        if (lane >= o) end = max(end, y);
      }
      int before = __shfl_up_sync(0xffffffffu, end, 1);
      before = lane == 0 ? reach : max(before, reach);
      if (g < G && from < before) cnt[g] = 0;
      reach = max(reach, __shfl_sync(0xffffffffu, end, 31));
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) n[c] = c * 32 + lane < G ? cnt[c * 32 + lane] : 0;
  }
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) n[c] = (n[c] + TILE - 1) / TILE;
  warp_exclusive_scan(G, lane, n, prefix);
}

// Two values, scaled, as e4m3 (lo in the low byte).
__device__ __forceinline__ uint32_t fp8_pack2(float lo, float hi, float inv) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo * inv, hi * inv), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ U4 fp8_pack16(const float* v, float inv) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = fp8_pack2(v[4 * i], v[4 * i + 1], inv) | (fp8_pack2(v[4 * i + 2], v[4 * i + 3], inv) << 16);
  return U4{w[0], w[1], w[2], w[3]};
}

// GELU(u) = u Phi(u) = max(u, 0) - |u| erfc(|u| / sqrt 2) / 2 to fp32's own rounding:
// erfc(x) = (c1 t + .. + c6 t^6) e^(-x^2), t = 1 / (1 + 0.4 x), the form of Abramowitz &
// Stegun 7.1.26 with one term more, fitted here to the least largest error (Lawson's
// weights): 2.8e-8, which with the roundings is 2.5e-7 at most.  Shorter forms move
// hidden values over the e4m3 roundings' ties: with 7.1.28 (3e-7) fp32 experts of
// 768 x 3072 were 6e-5 off (median of twelve inputs), with this and with the exact
// form about 1e-5.  Half the exact
// form's instructions (Switch sizes, 4096 rows: 56 us, 66).
__device__ __forceinline__ float gelu_fp8out(float u) {
  const float x = fabsf(u);
  float t, e;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(fmaf(x, 0.4f * 0.70710678118654752f, 1.0f)));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(u * u * (-0.5f * 1.4426950408889634f)));
  float q = fmaf(t, -0.200259726f, 0.709149296f);
  q = fmaf(t, q, -0.370911135f);
  q = fmaf(t, q, 0.468276749f);
  q = fmaf(t, q, 0.16182253f);
  q = fmaf(t, q, 0.231922259f);
  return fmaf(-0.5f * x, q * t * e, fmaxf(u, 0.0f));
}

namespace tc {

// 32 lanes x 64 columns of fp32 TMEM words: thread i of the warp receives the
// columns from taddr's of TMEM lane (quadrant base + i).  Loads and wait are one
// statement, so nothing that reads the values is moved before the wait.
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%64];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
      "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%65];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=&f"(v[0]), "=&f"(v[1]), "=&f"(v[2]), "=&f"(v[3]), "=&f"(v[4]), "=&f"(v[5]), "=&f"(v[6]), "=&f"(v[7]),
        "=&f"(v[8]), "=&f"(v[9]), "=&f"(v[10]), "=&f"(v[11]), "=&f"(v[12]), "=&f"(v[13]), "=&f"(v[14]), "=&f"(v[15]),
        "=&f"(v[16]), "=&f"(v[17]), "=&f"(v[18]), "=&f"(v[19]), "=&f"(v[20]), "=&f"(v[21]), "=&f"(v[22]), "=&f"(v[23]),
        "=&f"(v[24]), "=&f"(v[25]), "=&f"(v[26]), "=&f"(v[27]), "=&f"(v[28]), "=&f"(v[29]), "=&f"(v[30]), "=&f"(v[31]),
        "=&f"(v[32]), "=&f"(v[33]), "=&f"(v[34]), "=&f"(v[35]), "=&f"(v[36]), "=&f"(v[37]), "=&f"(v[38]), "=&f"(v[39]),
        "=&f"(v[40]), "=&f"(v[41]), "=&f"(v[42]), "=&f"(v[43]), "=&f"(v[44]), "=&f"(v[45]), "=&f"(v[46]), "=&f"(v[47]),
        "=&f"(v[48]), "=&f"(v[49]), "=&f"(v[50]), "=&f"(v[51]), "=&f"(v[52]), "=&f"(v[53]), "=&f"(v[54]), "=&f"(v[55]),
        "=&f"(v[56]), "=&f"(v[57]), "=&f"(v[58]), "=&f"(v[59]), "=&f"(v[60]), "=&f"(v[61]), "=&f"(v[62]), "=&f"(v[63])
      : "r"(taddr), "r"(taddr + 32)
      : "memory");
}

// Asynchronous copy of 4, 8 or 16 bytes to shared memory; cp_async_arrive counts
// one arrival on the barrier once the calling thread's copies so far have landed.
template <int BYTES>
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Arrive under a predicate, without a branch.
__device__ __forceinline__ void mbar_arrive_if(bool on, uint32_t bar) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\t@p mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}\n" ::"r"(
                   bar),
               "r"(static_cast<uint32_t>(on))
               : "memory");
}
__device__ __forceinline__ void mbar_arrive_remote_if(bool on, uint32_t cluster_addr) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\t@p mbarrier.arrive.shared::cluster.b64 _, [%0];\n\t}\n" ::"r"(
                   cluster_addr),
               "r"(static_cast<uint32_t>(on))
               : "memory");
}

// Instruction descriptor of tcgen05.mma kind::f8f6f4: fp32 accumulator (bits 4-5
// = 1), A and B e4m3 (bits 7-9 and 10-12 = 0), both K-major, N >> 3 in bits
// 17-22, M >> 4 in bits 24-28.
__host__ __device__ constexpr uint32_t idesc_e4m3(int m, int n) {
  return (1u << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}
__device__ __forceinline__ void umma_fp8(uint32_t d_tmem, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d_tmem),
      "l"(da), "l"(db), "r"(idesc), "r"(accum)
      : "memory");
}
// Over a CTA pair, M = 256 (see umma_bf16_pair).
__device__ __forceinline__ void umma_fp8_pair(uint32_t d_tmem, uint64_t da, uint64_t db, uint32_t idesc,
                                              uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d_tmem),
      "l"(da), "l"(db), "r"(idesc), "r"(accum)
      : "memory");
}

}  // namespace tc
}  // namespace ec2moe
