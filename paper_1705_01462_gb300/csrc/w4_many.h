// The product of many tokens with 4-bit weights (gemm_w4.cu).
#pragma once

#include <type_traits>

#include "linear_internal.cuh"
#include "w4.cuh"

namespace fgq {
namespace w4 {

// Eight codes of a word as four pairs of fp16 whole numbers, a known way with 4-bit weights: in the low bits of 1024's fp16 a nibble n is 1024 + n,
// four bits up 1024 + 16 n.
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

// A token as fp16 rows, by a block of 256: fp16 as they are; bf16 times 2^(14 - e), 2^e <= the row's largest magnitude < 2^(e + 1); fp32 so
// scaled in two rows beside one another, the second what the first's rounding leaves (within 2^-22 of a value, 2^-39 of the largest).
// A row with NaN or Inf: its scale is NaN, and so are its outputs.
template <typename T, bool VEC>
__device__ __forceinline__ void token_row(const T* __restrict__ row, int K, __half* to, int64_t pitch, float* scale) {
  constexpr bool SCALED = !std::is_same<T, __half>::value, TWO = std::is_same<T, float>::value;
  __shared__ float red[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float mul0 = 1.0f, mul1 = 1.0f;
  if (SCALED) {
    float mx = 0.0f;
    if (VEC) {
      for (int k = 8 * threadIdx.x; k < K; k += 2048) {
        Raw8<T> v;
        v.load(row + k);
        float lo, hi;
        v.extremes(lo, hi);
        mx = max_nan(mx, max_nan(-lo, hi));
      }
    } else {
      for (int k = threadIdx.x; k < K; k += 256) mx = max_nan(mx, fabsf(to_float(row[k])));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = max_nan(mx, __shfl_xor_sync(FULL_MASK, mx, o));
    if (lane == 0) red[warp] = mx;
    __syncthreads();
    mx = red[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mx = max_nan(mx, red[i]);
    int e = (int)(__float_as_uint(mx) >> 23 & 255u) - 127;
    if (e < -126) e = -126;
    const bool bad = nonfinite(mx);
    if (threadIdx.x == 0) *scale = bad ? __uint_as_float(0x7fc00000u) : pow2f(e - 14);
    mul0 = bad ? 0.0f : pow2f((14 - e) / 2);
    mul1 = bad ? 0.0f : pow2f((14 - e) - (14 - e) / 2);
    if (bad) {
      for (int64_t k = threadIdx.x; k < pitch * (TWO ? 2 : 1); k += 256) to[k] = __float2half_rn(0.0f);
      return;
    }
  } else if (threadIdx.x == 0) {
    *scale = 1.0f;
  }
  if (VEC) {
    for (int k = 8 * threadIdx.x; k < pitch; k += 2048) {
      Raw8<T> v;
      v.zero();
      if (k < K) v.load(row + k);
      float f[8];
      v.unpack(f);
      if (SCALED) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = f[i] * mul0 * mul1;
      }
      store8(to + k, f);
      if (TWO) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] -= __half2float(__float2half_rn(f[i]));
        store8(to + pitch + k, f);
      }
    }
  } else {
    for (int64_t k = threadIdx.x; k < pitch; k += 256) {
      const float f = k < K ? to_float(row[k]) * mul0 * mul1 : 0.0f;
      const __half h = __float2half_rn(f);
      to[k] = h;
      if (TWO) to[pitch + k] = __float2half_rn(f - __half2float(h));
    }
  }
}

// How a product is laid out: tile of tokens, splits of K, bytes of its partial sums.
struct ManyPlan {
  size_t part_bytes;
  int bn, splits, parts;
};
ManyPlan plan_many(int P, int parts, int ct, int M);

// x16: fp16 tokens, each in `plan.parts` rows that add up to it, `pitch` elements apart (16-byte aligned rows), written or older than
// the kernel before; scale: what each is multiplied by at the end, or nullptr (1); wexp: the exponent of each row's largest scale, for all rows of the weights' tiles.
fgq_status launch_many(const ManyPlan& plan, const Matrix& w, const int* wexp, const void* x16, int64_t pitch, int K, const float* scale,
                       int P, int M, float* part, const float* bias, void* y, int ytype, cudaStream_t s);

// The experts' layers of many tokens: choices sorted by expert, in units of up to `cap` (32, 64, 128 or 256).
struct ExpertsMany {
  Matrix gate, up, down;
  const Unit* units;
  const Choice* choices;
  const int* nunits;  // units, choices
  int K, F, A, cap, most_units;
  void* tmp;  // experts_many_bytes of it
  float* z;   // out, [choice][K]
};
size_t experts_many_bytes(int type, int A, int K, int F);
fgq_status launch_experts_many(const ExpertsMany& a, const void* x, int type, int64_t ldx, cudaStream_t s);

}  // namespace w4
}  // namespace fgq
