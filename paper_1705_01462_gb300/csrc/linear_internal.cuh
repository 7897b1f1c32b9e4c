// What the 8-bit linear layers' translation units share.
#pragma once

#include "decoder_internal.cuh"

namespace fgq {

// Elements of a row of fp16 codes, as gemm_w8a8.cu reads them: whole K-tiles.
inline int64_t gemm_w8a8_pitch(int K) { return ((int64_t)K + 63) / 64 * 64; }

// The product on the tensor cores.  Tokens as int8 q [P][K], or as fp16 rows x16 of `pitch` elements
// (gemm_w8a8_pitch, zero past K).
fgq_status launch_gemm_w8a8(const int8_t* q, const void* x16, int64_t pitch, const float* scale, int P, int K,
                            const int8_t* wq, const float* wscale, int M, const float* bias, void* y, int ytype,
                            cudaStream_t s);

__device__ __forceinline__ void store_typed(void* y, int type, int64_t at, float v) {
  if (type == FGQ_F32)
    static_cast<float*>(y)[at] = v;
  else if (type == FGQ_BF16)
    static_cast<__nv_bfloat16*>(y)[at] = __float2bfloat16_rn(v);
  else
    static_cast<__half*>(y)[at] = __float2half_rn(v);
}

}  // namespace fgq
