// What the attention kernels on the 5th-generation tensor cores share: descriptors of their operands, the product with P in tensor memory, masks as bits.
#pragma once
#include "paged_scores.cuh"

namespace hs {
namespace {

// MN-major 16-bit operand with the 128-byte swizzle: atoms of 64 (MN, contiguous) x 8 (K) elements.
__device__ __forceinline__ uint64_t umma_desc_mnmajor_sw128(uint32_t smem_addr, uint32_t lbo, uint32_t sbo) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((smem_addr & 0x3ffffu) >> 4);
  d |= static_cast<uint64_t>(lbo >> 4) << 16;
  d |= static_cast<uint64_t>(sbo >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}
// D[tmem] (+)= A[tmem] * B[smem]^T
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Instruction descriptor of a product of 16-bit operands (both bf16, or both fp16) with fp32 sums.
template <bool F16>
__host__ __device__ constexpr uint32_t idesc_16(int M, int N) {
  const uint32_t bf16 = umma_idesc_bf16_f32(M, N);
  return F16 ? bf16 & ~((1u << 7) | (1u << 10)) : bf16;
}

// The n lowest bits (all for n >= 32, none for n <= 0).
__device__ __forceinline__ uint32_t first_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

}  // namespace
}  // namespace hs
