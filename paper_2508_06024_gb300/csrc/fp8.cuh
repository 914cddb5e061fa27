// Device helpers of the 8-bit floating point path: the scale of a block, the
// conversion of its values, and the tcgen05 forms of 8-bit operands.
#pragma once

#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"

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

// Packed pairs of fp32 (one instruction for two multiply-adds).
__device__ __forceinline__ uint64_t f32x2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ uint64_t f32x2_bits(uint32_t lo, uint32_t hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ float2 f32x2_get(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t f32x2_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t f32x2_mul(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

namespace tc {

// tcgen05.wait::ld, with the 16 registers that the loads fill as operands, so
// that nothing which reads them is moved before it.
__device__ __forceinline__ void tmem_wait_for16(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
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
