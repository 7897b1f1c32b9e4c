// The product of many tokens with 4-bit weights (gemm_w4.cu).
#pragma once

#include "linear_internal.cuh"
#include "w4.cuh"

namespace fgq {
namespace w4 {

// Eight codes of a word as four pairs of fp16 whole numbers: in the low bits of 1024's fp16 a nibble n is 1024 + n, four bits up 1024 + 16 n.
__device__ __forceinline__ uint32_t h2_sub(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t h2_mul(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// ... times the pair `s` of a scale.
__device__ __forceinline__ uint4 scaled_codes(uint32_t w, uint32_t s) {
  const uint32_t v = w >> 8;
  const uint32_t a = h2_sub((w & 0x000f000fu) | 0x64006400u, 0x64086408u);
  const uint32_t b = Operand<__half>::fma2((w & 0x00f000f0u) | 0x64006400u, 0x2c002c00u, 0xd480d480u);  // / 16 - 72
  const uint32_t c = h2_sub((v & 0x000f000fu) | 0x64006400u, 0x64086408u);
  const uint32_t d = Operand<__half>::fma2((v & 0x00f000f0u) | 0x64006400u, 0x2c002c00u, 0xd480d480u);
  return make_uint4(h2_mul(a, s), h2_mul(b, s), h2_mul(c, s), h2_mul(d, s));
}

// How a product is laid out: tile of tokens, splits of K, bytes of its partial sums.
struct ManyPlan {
  size_t part_bytes;
  int bn, splits, parts;
};
ManyPlan plan_many(int P, int parts, int ct, int M);

// x16: fp16 tokens, each in `plan.parts` rows that add up to it, `pitch` elements apart (16-byte aligned rows), written or older than the kernel before; scale: what each is
// multiplied by at the end, or nullptr (1); wexp: the exponent of each row's largest scale, for all rows of the weights' tiles.
fgq_status launch_many(const ManyPlan& plan, const Matrix& w, const int* wexp, const void* x16, int64_t pitch, int K, const float* scale,
                       int P, int M, float* part, const float* bias, void* y, int ytype, cudaStream_t s);

}  // namespace w4
}  // namespace fgq
