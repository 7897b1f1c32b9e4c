// 8-bit integer product for many tokens on the tensor cores (tcgen05).
//
// int8 operands as fp16 (exact; sm_103a's integer tensor rate is far below its fp16 rate), fp32
// accumulators in tensor memory: sums are exact below 2^24.  Output channels are the M = 128 rows of a
// tile (TMEM lanes), tokens its BN columns, K-tiles of 64.  Both operands are fp16 rows in global memory
// (codes expanded once per call), brought by TMA boxes with the 128-byte swizzle into a ring.
// Warp roles (one block per SM, persistent over tiles):
//   warps 0-7  epilogue: warp w reads TMEM lanes 32 (w % 4) .. (channels), columns BN / 2 (w / 4) .. (tokens),
//              applies scales and bias and stores runs of 32 channels;
//   warp 8     TMEM allocation and the MMA issuer;
//   warp 9     TMA producer.
// Two accumulators: the epilogue of a tile overlaps the MMAs of the next.  Few tiles split K over blocks
// (fp32 partial sums, joined with scales and bias by a second kernel).
// Every wait is bounded; on expiry FGQ_ERR_TIMEOUT is recorded, each role leaves its loop, copies and
// MMAs in flight are waited for, and TMEM is freed.
#include <cstring>

#include "linear_internal.cuh"
#include "tc_common.cuh"

namespace fgq {
namespace {

using namespace dec;
using tc::make_map_2d;

constexpr int GW_BM = 128, GW_KT = 64;
constexpr int GW_EPI_WARPS = 8, GW_MMA_WARP = 8, GW_TMA_WARP = 9;
constexpr int GW_THREADS = 320;
constexpr uint64_t GW_TIMEOUT_NS = 1000000000ull;  // 1 s per wait
constexpr uint32_t GW_BAR_EPI = 1;

template <int BN>
struct GwCfg {
  static constexpr int A_BYTES = GW_BM * GW_KT * 2, B_BYTES = BN * GW_KT * 2, STAGE = A_BYTES + B_BYTES;
  static constexpr int STAGES = BN == 256 ? 4 : 6;
  static constexpr int COLS = 2 * BN < 32 ? 32 : 2 * BN;  // TMEM columns: two accumulators
  static constexpr int SMEM = 1024 + STAGES * STAGE + 8 * (2 * STAGES + 5) + 16;
};
static_assert(GwCfg<256>::SMEM <= 232448, "shared memory budget");

struct GwArgs {
  CUtensorMap w_map, x_map;
  const float* scale;
  const float* wscale;
  const float* bias;
  void* y;
  float* part;  // [splits][P][M] partial sums, or nullptr
  unsigned int* err;
  uint64_t timeout_ns;
  int P, M, ktiles, mtiles, ptiles, splits, ytype;
};

template <int BN>
__global__ void __launch_bounds__(GW_THREADS, 1) gemm_w8a8_kernel(const __grid_constant__ GwArgs a) {
  using C = GwCfg<BN>;
  constexpr int S = C::STAGES;
  extern __shared__ uint8_t smem_gw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_gw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S * C::STAGE);
  uint64_t* empty = full + S;
  uint64_t* acc_full = empty + S;
  uint64_t* acc_empty = acc_full + 2;
  uint64_t* drain_bar = acc_empty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain_bar + 1);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint64_t tmo = a.timeout_ns;

  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], GW_EPI_WARPS);
    }
    mbar_init(drain_bar, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == GW_MMA_WARP) {
    tmem_alloc(tmem_slot, C::COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();  // operands, scales and partial sums are those of the kernels before
  const int ntiles = a.mtiles * a.ptiles * a.splits;
  const int my_tiles = (ntiles - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
  // tile -> channels, tokens, K-tiles [k0, k1): neighbours share tokens
  auto coords = [&](int tl, int& m0, int& p0, int& sp, int& k0, int& k1) {
    int id = (int)blockIdx.x + tl * (int)gridDim.x;
    m0 = (id % a.mtiles) * GW_BM;
    id /= a.mtiles;
    sp = id % a.splits;
    p0 = (id / a.splits) * BN;
    k0 = (int)((int64_t)a.ktiles * sp / a.splits);
    k1 = (int)((int64_t)a.ktiles * (sp + 1) / a.splits);
  };
  auto fail = [&]() {
    *abort_flag = 1;
    record_error(a.err, FGQ_ERR_TIMEOUT);
  };

  if (warp == GW_TMA_WARP && lane == 0) {
    int j = 0;
    bool ok = true;
    for (int tl = 0; tl < my_tiles && ok; ++tl) {
      int m0, p0, sp, k0, k1;
      coords(tl, m0, p0, sp, k0, k1);
      for (int kt = k0; kt < k1; ++kt, ++j) {
        const int st = j % S;
        if (!mbar_wait_timed(&empty[st], ((j / S) & 1) ^ 1, tmo, abort_flag, 0)) {
          ok = false;
          break;
        }
        uint8_t* A = smem + st * C::STAGE;
        mbar_arrive_expect_tx(&full[st], C::STAGE);
        tma_load_2d(smem_u32(A), &a.w_map, kt * GW_KT, m0, &full[st]);
        tma_load_2d(smem_u32(A + C::A_BYTES), &a.x_map, kt * GW_KT, p0, &full[st]);
      }
    }
    if (!ok && !*abort_flag) fail();
    // boxes that the MMA issuer did not consume may still be in flight
    for (int i = j - S < 0 ? 0 : j - S; i < j; ++i) mbar_wait_bounded(&full[i % S], (i / S) & 1, 1u << 16);
  }

  if (warp == GW_MMA_WARP && lane == 0) {
    const uint32_t idesc = idesc_f16_f32(GW_BM, BN);
    int j = 0;
    bool ok = true;
    for (int tl = 0; tl < my_tiles && ok; ++tl) {
      int m0, p0, sp, k0, k1;
      coords(tl, m0, p0, sp, k0, k1);
      const int b = tl & 1;
      if (!mbar_wait_timed(&acc_empty[b], ((tl >> 1) & 1) ^ 1, tmo, abort_flag, 0)) {
        ok = false;
        break;
      }
      tc_fence_after();
      for (int kt = k0; kt < k1; ++kt, ++j) {
        const int st = j % S;
        if (!mbar_wait_timed(&full[st], (j / S) & 1, tmo, abort_flag, 0)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t A = smem_u32(smem + st * C::STAGE);
        const uint64_t ad = sdesc_k_sw128(A), bd = sdesc_k_sw128(A + C::A_BYTES);
#pragma unroll
        for (int s = 0; s < 4; ++s) mma_f16(tmem + (uint32_t)(b * BN), ad + 2 * s, bd + 2 * s, idesc, (kt > k0 || s > 0) ? 1u : 0u);
        mma_commit(&empty[st]);
      }
      if (ok) mma_commit(&acc_full[b]);
    }
    if (!ok && !*abort_flag) fail();
    mma_commit(drain_bar);
    mbar_wait_bounded(drain_bar, 0, 1u << 20);
  }

  if (warp < GW_EPI_WARPS) {
    const int quarter = warp & 3, half = warp >> 2;
    const int t = 32 * quarter + lane;
    for (int tl = 0; tl < my_tiles; ++tl) {
      int m0, p0, sp, k0, k1;
      coords(tl, m0, p0, sp, k0, k1);
      const int b = tl & 1;
      const bool ok = mbar_wait_warp(&acc_full[b], (tl >> 1) & 1, tmo, abort_flag);
      if (!ok && lane == 0 && !*abort_flag) fail();
      if (named_bar_or(GW_BAR_EPI, 32 * GW_EPI_WARPS, !ok)) break;
      tc_fence_after();
      const int m = m0 + t;
      const bool mok = m < a.M;
      const float sw = mok ? __ldg(a.wscale + m) : 0.0f;
      const float bias = mok && a.bias ? __ldg(a.bias + m) : 0.0f;
      const uint32_t ta = tmem + ((uint32_t)(32 * quarter) << 16) + (uint32_t)(b * BN + half * (BN / 2));
      const int pw = p0 + half * (BN / 2);
#pragma unroll 1
      for (int c = 0; c < BN / 2; c += 32) {
        uint32_t r[32];
        tmem_ld32(ta + c, r);
        tmem_ld_wait_regs(r);
        if (c + 32 == BN / 2) {  // this warp has the whole accumulator: free it
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&acc_empty[b]);
        }
        if (!mok) continue;
        if (a.part) {
          float* dst = a.part + ((int64_t)sp * a.P + pw + c) * a.M + m;
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (pw + c + i < a.P) dst[(int64_t)i * a.M] = __uint_as_float(r[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const int p = pw + c + i;
            if (p < a.P)
              store_typed(a.y, a.ytype, (int64_t)p * a.M + m, fmaf(__uint_as_float(r[i]), __ldg(a.scale + p) * sw, bias));
          }
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == GW_MMA_WARP) {
    tc_fence_after();
    tmem_dealloc(tmem, C::COLS);
  }
}

// int8 rows [rows][K] as fp16 rows of `pitch` elements (a multiple of 64), zero past K: eight a thread.
__device__ __forceinline__ void expand8(const int8_t* src, int K, int64_t pitch, bool vec, __half* dst, int64_t i) {
  const int64_t row = i / (pitch / 8);
  const int k = (int)(i - row * (pitch / 8)) * 8;
  float v[8];
  if (vec) {  // K a multiple of 8, 8-byte aligned rows
    const uint2 w = k < K ? __ldg(reinterpret_cast<const uint2*>(src + row * K + k)) : make_uint2(0u, 0u);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)(int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = k + e < K ? (float)__ldg(src + row * K + k + e) : 0.0f;
  }
  store8(dst + row * pitch + k, v);
}

__global__ void __launch_bounds__(256) expand_kernel(const int8_t* __restrict__ w, int64_t w8, __half* __restrict__ w16,
                                                     const int8_t* __restrict__ q, int64_t q8, __half* __restrict__ q16,
                                                     int K, int64_t pitch, int w_vec, int q_vec) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < w8 + q8; i += (int64_t)gridDim.x * 256) {
    if (i < w8)
      expand8(w, K, pitch, w_vec, w16, i);
    else
      expand8(q, K, pitch, q_vec, q16, i - w8);
  }
}

__global__ void __launch_bounds__(256) join_splits_kernel(const __grid_constant__ GwArgs a) {
  const int64_t n = (int64_t)a.P * a.M;
  pdl_wait();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float v = 0.0f;
    for (int s = 0; s < a.splits; ++s) v += a.part[s * n + i];
    const int p = (int)(i / a.M), m = (int)(i - (int64_t)p * a.M);
    store_typed(a.y, a.ytype, i, fmaf(v, __ldg(a.scale + p) * __ldg(a.wscale + m), a.bias ? __ldg(a.bias + m) : 0.0f));
  }
}

template <int BN>
fgq_status launch_gw(const GwArgs& a, int grid, cudaStream_t s) {
  if (!tc::smem_attr_once<gemm_w8a8_kernel<BN>>(GwCfg<BN>::SMEM)) return FGQ_ERR_CUDA;
  return after_launch(launch_pdl(gemm_w8a8_kernel<BN>, dim3(grid), dim3(GW_THREADS), GwCfg<BN>::SMEM, s, a));
}

}  // namespace

fgq_status launch_gemm_w8a8(const int8_t* q, const void* x16, int64_t pitch, const float* scale, int P, int K,
                            const int8_t* wq, const float* wscale, int M, const float* bias, void* y, int ytype,
                            cudaStream_t s) {
  const int sms = device_sms();
  pitch = gemm_w8a8_pitch(K);
  GwArgs a;
  memset(&a, 0, sizeof a);
  a.scale = scale;
  a.wscale = wscale;
  a.bias = bias;
  a.y = y;
  a.err = device_error_word();
  const int64_t lim_us = debug_wait_limit_us();
  a.timeout_ns = lim_us < 0 ? GW_TIMEOUT_NS : (uint64_t)lim_us * 1000u;
  a.P = P;
  a.M = M;
  a.ytype = ytype;
  a.ktiles = (int)(pitch / GW_KT);
  a.mtiles = (M + GW_BM - 1) / GW_BM;
  // token columns of a tile: narrower ones where the wide ones leave SMs idle
  int BN = 256;
  while (BN > 64 && (int64_t)a.mtiles * ((P + BN - 1) / BN) < sms) BN /= 2;
  a.ptiles = (P + BN - 1) / BN;
  const int64_t tiles = (int64_t)a.mtiles * a.ptiles;
  // K split over blocks where there are fewer tiles than half the SMs, 8 K-tiles each at least
  a.splits = 1;
  while (tiles * (a.splits * 2) <= sms && a.ktiles >= 16 * a.splits && a.splits < 16) a.splits *= 2;
  if (tiles * a.splits > INT32_MAX) return FGQ_ERR_UNSUPPORTED;

  const size_t w_bytes = (size_t)M * pitch * 2, q_bytes = q ? (size_t)P * pitch * 2 : 0;
  const size_t part_bytes = a.splits > 1 ? (size_t)a.splits * P * M * 4 : 0;
  uint8_t* tmp = static_cast<uint8_t*>(scratch_alloc(w_bytes + q_bytes + part_bytes, s));
  if (!tmp) return FGQ_ERR_CUDA;
  __half* w16 = reinterpret_cast<__half*>(tmp);
  __half* q16 = reinterpret_cast<__half*>(tmp + w_bytes);
  if (a.splits > 1) a.part = reinterpret_cast<float*>(tmp + w_bytes + q_bytes);
  const int64_t w8 = (int64_t)M * pitch / 8, q8 = q ? (int64_t)P * pitch / 8 : 0;
  const int64_t eb = (w8 + q8 + 255) / 256, most = (int64_t)sms * 32;
  expand_kernel<<<(unsigned)(eb < most ? eb : most), 256, 0, s>>>(wq, w8, w16, q, q8, q16, K, pitch,
                                                                   K % 8 == 0 && aligned(wq, 8), K % 8 == 0 && aligned(q, 8));
  fgq_status st = after_launch();
  if (st == FGQ_OK &&
      (!make_map_2d(&a.w_map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, w16, (uint64_t)pitch, (uint64_t)M, (uint64_t)pitch * 2,
                    GW_KT, GW_BM, CU_TENSOR_MAP_SWIZZLE_128B) ||
       !make_map_2d(&a.x_map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, q ? q16 : x16, (uint64_t)pitch, (uint64_t)P,
                    (uint64_t)pitch * 2, GW_KT, (uint32_t)BN, CU_TENSOR_MAP_SWIZZLE_128B)))
    st = FGQ_ERR_CUDA;
  const int grid = (int)(tiles * a.splits < sms ? tiles * a.splits : sms);
  if (st == FGQ_OK)
    st = BN == 256 ? launch_gw<256>(a, grid, s) : BN == 128 ? launch_gw<128>(a, grid, s) : launch_gw<64>(a, grid, s);
  if (st == FGQ_OK && a.splits > 1) {
    const int64_t jb = ((int64_t)P * M + 255) / 256;
    st = after_launch(launch_pdl(join_splits_kernel, dim3((unsigned)(jb < most ? jb : most)), dim3(256), 0, s, a));
  }
  if (cudaFreeAsync(tmp, s) != cudaSuccess && st == FGQ_OK) st = FGQ_ERR_CUDA;
  return st;
}

}  // namespace fgq
