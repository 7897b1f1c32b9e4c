// Linear layers of many tokens with 4-bit weights: launches, and the sums of a split K.
#include "gemm_w4.cuh"

namespace fgq {
namespace w4 {
namespace {

// y from the splits' sums: a thread one channel of G4_JOIN tokens, so that their loads are in flight together.
constexpr int G4_JOIN = 4;
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ G4Args a) {
  const int64_t n = (int64_t)a.P * a.M;
  const int m = blockIdx.x * 256 + threadIdx.x;
  pdl_wait();
  if (m >= a.M) return;
  const float sw = pow2f(__ldcg(a.wexp + m) - 12), bias = a.bias ? __ldg(a.bias + m) : 0.0f;
  for (int64_t p = (int64_t)blockIdx.y * G4_JOIN; p < a.P; p += (int64_t)gridDim.y * G4_JOIN) {
    float v[G4_JOIN] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 2
    for (int s = 0; s < a.splits; ++s)
#pragma unroll
      for (int i = 0; i < G4_JOIN; ++i)
        if (p + i < a.P) v[i] += __ldcg(a.part + s * n + (p + i) * a.M + m);
#pragma unroll
    for (int i = 0; i < G4_JOIN; ++i)
      if (p + i < a.P) store_typed(a.y, a.ytype, (p + i) * a.M + m, fmaf(v[i], (a.scale ? __ldcg(a.scale + p + i) : 1.0f) * sw, bias));
  }
}

template <int PARTS>
fgq_status launch_g4_tile(const G4Args& a, int bn, int grid, cudaStream_t s) {
  if (bn == 256) return launch_g4<256, PARTS, false, 16>(a, grid, s);
  return bn == 128 ? launch_g4<128, PARTS, false, 16>(a, grid, s) : launch_g4<64, PARTS, false, 16>(a, grid, s);
}

}  // namespace

ManyPlan plan_many(int P, int parts, int ct, int M) {
  ManyPlan g;
  g.parts = parts;
  const int64_t rows = (int64_t)P * parts;
  const int64_t sms = device_sms(), mt = ((int64_t)M + G4_BM - 1) / G4_BM;
  g.bn = rows <= 64 ? 64 : (rows <= 128 || mt * ((rows + 255) / 256) * 2 <= sms ? 128 : 256);
  // K split over blocks where there are fewer tiles than half the SMs, four tile columns each at least
  const int64_t tiles = mt * ((rows + g.bn - 1) / g.bn), by_k = ct / 4;
  int64_t splits = sms / tiles < by_k ? sms / tiles : by_k;
  g.splits = (int)(splits < 1 ? 1 : (splits > 16 ? 16 : splits));
  g.part_bytes = g.splits > 1 ? (size_t)g.splits * P * M * 4 : 0;
  return g;
}

fgq_status launch_many(const ManyPlan& plan, const Matrix& w, const int* wexp, const void* x16, int64_t pitch, int K, const float* scale,
                       int P, int M, float* part, const float* bias, void* y, int ytype, cudaStream_t s) {
  G4Args a;
  memset(&a, 0, sizeof a);
  a.w = w;
  a.scale = scale;
  a.wexp = wexp;
  a.bias = bias;
  a.y = y;
  a.part = plan.splits > 1 ? part : nullptr;
  a.err = device_error_word();
  const int64_t lim_us = debug_wait_limit_us();
  a.timeout_ns = lim_us < 0 ? G4_TIMEOUT_NS : (uint64_t)lim_us * 1000u;
  a.P = P;
  a.M = M;
  a.ytype = ytype;
  a.mtiles = (int)(((int64_t)M + G4_BM - 1) / G4_BM);
  const int64_t rows = (int64_t)P * plan.parts;
  a.ptiles = (int)((rows + plan.bn - 1) / plan.bn);
  a.splits = plan.splits;
  const int64_t tiles = (int64_t)a.mtiles * a.ptiles * a.splits;
  if (tiles > INT32_MAX) return FGQ_ERR_UNSUPPORTED;
  if (!make_map_2d(&a.x_map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, x16, (uint64_t)K, (uint64_t)rows, (uint64_t)pitch * 2, 64,
                   (uint32_t)plan.bn, CU_TENSOR_MAP_SWIZZLE_128B))
    return FGQ_ERR_CUDA;
  const int grid = (int)tiles;
  fgq_status st = plan.parts == 2 ? launch_g4_tile<2>(a, plan.bn, grid, s) : launch_g4_tile<1>(a, plan.bn, grid, s);
  if (st == FGQ_OK && a.part) {
    const int turns = (P + G4_JOIN - 1) / G4_JOIN;
    const dim3 jg((unsigned)((M + 255) / 256), (unsigned)(turns < 65535 ? turns : 65535));
    st = after_launch(launch_pdl(join_kernel, jg, dim3(256), 0, s, a));
  }
  return st;
}

}  // namespace w4
}  // namespace fgq
