// The experts' layers of many tokens with 4-bit weights: tokens as rows in the order of their experts, the products of gemm_w4.cuh for
// a unit of up to 32, 64, 128 or 256 of them and 128 rows of gate, up or down, and the hidden values between them.  Bound as those products are, by
// codes to operands, once for each unit of an expert: 128 tokens of 2 of 8 experts, 4096 -> 14336, 436 us for 110 of bytes
// (hidden values take two rows of fp16, and down's sums leave the tensor memory every 256 columns).
#include "gemm_w4.cuh"

namespace fgq {
namespace w4 {
namespace {

inline size_t up256(size_t v) { return (v + 255) & ~size_t(255); }
// rows of fp16 that a token takes: fp32 two; a hidden value, which is fp32 whatever the tokens are, takes two
int token_parts(int type) { return type == FGQ_F32 ? 2 : 1; }
constexpr int HIDDEN_PARTS = 2;

// Row `place` of x16: the token of that choice.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) gather_kernel(const T* __restrict__ x, int K, int64_t ldx, const Choice* choices, const int* nunits,
                                                     __half* dst, int64_t pitch, float* scale) {
  pdl_wait();
  pdl_trigger();  // from here on the kernel after may read the units
  const int64_t at = blockIdx.x;
  if (at >= __ldcg(nunits + 1)) return;
  token_row<T, VEC>(x + __ldcg(&choices[at].token) * ldx, K, dst + at * pitch * (std::is_same<T, float>::value ? 2 : 1), pitch, scale + at);
}

// h = silu(g) u as two rows of fp16 that add up to it (within 2^-22 of a value, 2^-39 of the largest), after a power of two that takes a
// choice's largest to 2^14; a block a choice, twice over its values.
__global__ void __launch_bounds__(256) hidden_kernel(const float* g, const float* u, int F, const int* nunits, __half* dst, int64_t pitch,
                                                     float* scale) {
  __shared__ float red[8];
  pdl_wait();
  pdl_trigger();
  const int64_t at = blockIdx.x;
  if (at >= __ldcg(nunits + 1)) return;
  const float *gr = g + at * F, *ur = u + at * F;
  __half* to = dst + at * pitch * HIDDEN_PARTS;
  auto value = [&](int k) {
    const float v = __ldcg(gr + k);
    return v / (1.0f + expf(-v)) * __ldcg(ur + k);
  };
  float mx = 0.0f;
#pragma unroll 4
  for (int k = threadIdx.x; k < F; k += 256) mx = max_nan(mx, fabsf(value(k)));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mx = max_nan(mx, __shfl_xor_sync(FULL_MASK, mx, o));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = mx;
  __syncthreads();
  mx = red[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) mx = max_nan(mx, red[i]);
  const bool bad = nonfinite(mx);
  const int e = max((int)(__float_as_uint(mx) >> 23 & 255u) - 127, -126);
  if (threadIdx.x == 0) scale[at] = bad ? __uint_as_float(0x7fc00000u) : pow2f(e - 14);
  const float up = bad ? 0.0f : pow2f((14 - e) / 2), up2 = pow2f((14 - e) - (14 - e) / 2);  // past fp32's largest for tiny ones
#pragma unroll 4
  for (int k = threadIdx.x; k < pitch; k += 256) {
    const float v = k < F && !bad ? value(k) * up * up2 : 0.0f;
    const __half h = __float2half_rn(v);
    to[k] = h;
    to[pitch + k] = __float2half_rn(v - __half2float(h));
  }
}

template <int PARTS>
fgq_status launch_unit_products(const G4Args& a, int bn, int grid, cudaStream_t s) {
  // two smaller blocks an SM where there are tiles for them: one works while the other begins or ends.  us so and with one: 32 experts 4096
  // -> 1024, 4 a token, 128 tokens 136 and 169; but 8 experts 2048 -> 1024, 2 a token 49 and 40
  if (bn == 64) return grid >= 2 * device_sms() ? launch_g4<64, PARTS, true, 8>(a, grid, s) : launch_g4<64, PARTS, true, 16>(a, grid, s);
  return bn == 128 ? launch_g4<128, PARTS, true, 16>(a, grid, s) : launch_g4<256, PARTS, true, 16>(a, grid, s);
}
fgq_status launch_products(const ExpertsMany& e, const Matrix& w, const Matrix* up, const __half* x16, int64_t pitch, const float* scale,
                           int parts, int M, float* y, float* y_up, cudaStream_t s) {
  G4Args a;
  memset(&a, 0, sizeof a);
  a.w = w;
  a.scale = scale;
  a.y = y;
  a.err = device_error_word();
  const int64_t lim_us = debug_wait_limit_us();
  a.timeout_ns = lim_us < 0 ? G4_TIMEOUT_NS : (uint64_t)lim_us * 1000u;
  a.P = e.A;
  a.M = M;
  a.ytype = FGQ_F32;
  a.mtiles = (int)(((int64_t)M + G4_BM - 1) / G4_BM);
  a.matrices = 1;
  if (up) a.up = *up, a.y_up = y_up, a.matrices = 2;
  a.units = e.units;
  a.nunits = e.nunits;
  const int rows = e.cap * parts, bn = rows < 64 ? 64 : (rows > 256 ? 256 : rows);
  a.tiles = rows / bn + (rows < bn);
  const int64_t tiles = (int64_t)a.mtiles * a.matrices * a.tiles * e.most_units;
  if (tiles > INT32_MAX) return FGQ_ERR_UNSUPPORTED;
  if (!make_map_2d(&a.x_map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, x16, (uint64_t)pitch, (uint64_t)e.A * parts, (uint64_t)pitch * 2, 64, (uint32_t)bn,
                   CU_TENSOR_MAP_SWIZZLE_128B))
    return FGQ_ERR_CUDA;
  return parts == 2 ? launch_unit_products<2>(a, bn, (int)tiles, s) : launch_unit_products<1>(a, bn, (int)tiles, s);
}

template <typename T>
fgq_status launch_gather(const ExpertsMany& a, const void* x, int type, int64_t ldx, __half* dst, int64_t pitch, float* scale, cudaStream_t s) {
  const bool vec = a.K % 8 == 0 && aligned(x, 16) && stride16(ldx, type);
  const T* xt = static_cast<const T*>(x);
  return after_launch(launch_pdl(vec ? gather_kernel<T, true> : gather_kernel<T, false>, dim3(a.A), dim3(256), 0, s, xt, a.K, ldx, a.choices,
                                 a.nunits, dst, pitch, scale));
}

struct Layout {
  int64_t kp, fp;
  size_t x, g, h, s;
};
Layout layout(int type, int A, int K, int F) {
  const int64_t kp = copied_pitch(K), fp = copied_pitch(F);
  return {kp, fp, up256((size_t)A * token_parts(type) * kp * 2), up256((size_t)A * F * 4), up256((size_t)A * HIDDEN_PARTS * fp * 2),
          up256((size_t)A * 4)};
}

}  // namespace

size_t experts_many_bytes(int type, int A, int K, int F) {
  const Layout l = layout(type, A, K, F);
  return l.x + 2 * l.g + l.h + 2 * l.s;
}

fgq_status launch_experts_many(const ExpertsMany& a, const void* x, int type, int64_t ldx, cudaStream_t s) {
  const Layout l = layout(type, a.A, a.K, a.F);
  uint8_t* at = static_cast<uint8_t*>(a.tmp);
  auto take = [&](size_t n) {
    uint8_t* p = at;
    at += n;
    return p;
  };
  __half* x16 = reinterpret_cast<__half*>(take(l.x));
  float* g = reinterpret_cast<float*>(take(l.g));
  float* u = reinterpret_cast<float*>(take(l.g));
  __half* h16 = reinterpret_cast<__half*>(take(l.h));
  float* xs = reinterpret_cast<float*>(take(l.s));
  float* hs = reinterpret_cast<float*>(take(l.s));
  fgq_status st = type == FGQ_F32 ? launch_gather<float>(a, x, type, ldx, x16, l.kp, xs, s)
                                  : (type == FGQ_BF16 ? launch_gather<__nv_bfloat16>(a, x, type, ldx, x16, l.kp, xs, s)
                                                      : launch_gather<__half>(a, x, type, ldx, x16, l.kp, xs, s));
  if (st == FGQ_OK) st = launch_products(a, a.gate, &a.up, x16, l.kp, xs, token_parts(type), a.F, g, u, s);
  if (st == FGQ_OK)
    st = after_launch(launch_pdl(hidden_kernel, dim3(a.A), dim3(256), 0, s, static_cast<const float*>(g), static_cast<const float*>(u), a.F,
                                 a.nunits, h16, l.fp, hs));
  if (st == FGQ_OK) st = launch_products(a, a.down, nullptr, h16, l.fp, hs, HIDDEN_PARTS, a.K, a.z, nullptr, s);
  return st;
}

}  // namespace w4
}  // namespace fgq
