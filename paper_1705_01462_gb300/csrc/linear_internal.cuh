// What the 8-bit linear layers' translation units share.
#pragma once

#include "decoder_internal.cuh"

namespace fgq {

// How the product of many tokens is laid out: tile of tokens, splits of K, bytes of its partial sums, and elements
// of an fp16 operand row (whole K-tiles; zero past K).
struct GemmPlan {
  int64_t pitch;
  size_t part_bytes;
  int bn, splits;
};
GemmPlan plan_gemm_w8a8(int P, int K, int M);

// The product on the tensor cores of fp16 operands x16 [P][pitch] and w16 [M][pitch] that the kernel before has
// written; `part` is a temporary of plan.part_bytes.
fgq_status launch_gemm_w8a8(const GemmPlan& plan, const void* x16, const void* w16, float* part, const float* scale,
                            int P, const float* wscale, int M, const float* bias, void* y, int ytype, cudaStream_t s);

__device__ __forceinline__ void store_typed(void* y, int type, int64_t at, float v) {
  if (type == FGQ_F32)
    static_cast<float*>(y)[at] = v;
  else if (type == FGQ_BF16)
    static_cast<__nv_bfloat16*>(y)[at] = __float2bfloat16_rn(v);
  else
    static_cast<__half*>(y)[at] = __float2half_rn(v);
}

}  // namespace fgq
