// 8-bit integer product for many tokens on the tensor cores (tcgen05, pairs of SMs).
//
// int8 operands as fp16 (exact; sm_103a's integer tensor rate is far below its fp16 rate), fp32
// accumulators in tensor memory: sums are exact below 2^24.  A pair of blocks (cta_group::2) takes a tile of
// 256 output channels and BN tokens: each block holds the operand rows of its 128 channels and of half of the
// tokens, and its SM's 128 channels x BN tokens of the accumulator.  Alone, a block reads 12 KB of shared
// memory and is sent 12 KB for an MMA of 128 clocks (128 x 256 x 16), 192 bytes a clock of the 128 there are; in a
// pair it is 8 and 8.  Both operands are fp16 rows in global memory (codes expanded once per call), brought
// by TMA boxes with the 128-byte swizzle into a ring of K-tiles of 64.
// Warp roles (one block per SM, persistent over tiles):
//   warps 0-7  epilogue: warp w reads TMEM lanes 32 (w % 4) .. (channels), columns BN / 2 (w / 4) .. (tokens),
//              applies scales and bias and stores runs of 32 channels;
//   warp 8     TMEM allocation; in the pair's first block the MMA issuer;
//   warp 9     TMA producer of the block's own boxes, which count on the first block's barrier (the loads' cta_group::2
//              form), so that one wait covers both blocks' operands.
// Two accumulators: the epilogue of a tile overlaps the MMAs of the next.  Few tiles split K over pairs
// (fp32 partial sums, joined with scales and bias by a second kernel).
// 4096 tokens, 4096 -> 8192, bf16: 175 us for the layer, 20 of them quantization and expansion, where the products
// alone are due 148; at 2048 tokens, 4096 -> 4096 (49 us) the tensor pipe is active 59% of the time: 128 tiles on
// 76 pairs are two waves.
// Every wait is bounded; on expiry FGQ_ERR_TIMEOUT is recorded and each role leaves its loop.  Nothing is on its way to a block that
// leaves: both blocks wait for every arrival that the MMAs' commits make on their barriers, and meet before TMEM is freed.  After
// an expiry in either they know by then how far each came, wait for the arrivals that there are and the first one for boxes that
// no MMA has read, and meet again.
#include <cstring>

#include "linear_internal.cuh"
#include "tc_common.cuh"

namespace fgq {
namespace {

using namespace dec;
using tc::make_map_2d;

constexpr int GW_BM = 128, GW_KT = 64;  // channels of a block; a pair has twice as many
constexpr int GW_EPI_WARPS = 8, GW_MMA_WARP = 8, GW_TMA_WARP = 9;
constexpr int GW_THREADS = 320;
constexpr uint64_t GW_TIMEOUT_NS = 1000000000ull;  // 1 s per wait
constexpr uint32_t GW_BAR_EPI = 1;

template <int BN>
struct GwCfg {
  static constexpr int A_BYTES = GW_BM * GW_KT * 2, B_BYTES = BN / 2 * GW_KT * 2, STAGE = A_BYTES + B_BYTES;
  static constexpr int STAGES = BN == 256 ? 6 : 8;
  static constexpr int COLS = 2 * BN;  // TMEM columns: two accumulators
  static constexpr int SMEM = 1024 + STAGES * STAGE + 8 * (2 * STAGES + 5) + 32;
};
static_assert(GwCfg<256>::SMEM <= 232448 && GwCfg<128>::SMEM <= 232448, "shared memory budget");

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

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// Shared address `p` of this block as that of the cluster's block `rank`, and an arrival on a barrier there.
__device__ __forceinline__ uint32_t map_rank(const void* p, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// A word at this block's shared address `p`, in the cluster's block `rank`.
__device__ __forceinline__ uint32_t ld_cluster_u32(const uint32_t* p, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(map_rank(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ void st_cluster_u32(const uint32_t* p, uint32_t rank, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_rank(p, rank)), "r"(v) : "memory");
}
// A box into this block's shared memory whose bytes count on a barrier of the pair, `bar` in either block.
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const void* map, int c0, int c1, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], "
      "[%4];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar)
      : "memory");
}
// Bytes that a phase of this block's barrier expects and that were never sent for.
__device__ __forceinline__ void mbar_forgo_tx(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
// mbar_wait_timed for arrivals from the other block, polling: a thread that try_wait has suspended is not woken by
// them (a K-tile took its whole microsecond).
__device__ __forceinline__ bool mbar_wait_cluster(uint64_t* bar, uint32_t parity, uint64_t timeout_ns, volatile uint32_t* abort) {
  auto test = [&]() {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
  };
  if (test()) return true;
  if (timeout_ns == 0) return false;
  const uint64_t t0 = globaltimer_ns();
  for (uint32_t i = 1; i < (1u << 30); ++i) {
    if (test()) return true;
    if ((i & 255u) == 0 && (*abort || globaltimer_ns() - t0 > timeout_ns)) return false;
  }
  return false;
}

// ---- tcgen05, pairs of blocks
__device__ __forceinline__ void tmem_alloc2(uint32_t* slot, uint32_t ncols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(ncols)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc2(uint32_t taddr, uint32_t ncols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
// D (+)= A B^T over the pair: descriptors name the same offsets in both blocks.
__device__ __forceinline__ void mma_f16_pair(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// One arrival on the barrier at this offset in both blocks once the MMAs issued so far are complete.
__device__ __forceinline__ void mma_commit_pair(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
      "h"((uint16_t)3)
      : "memory");
}

// The first `live` of 32 values, one a row of M elements.
template <typename T>
__device__ __forceinline__ void store_column(T* y, int M, int live, const uint32_t (&r)[32]) {
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (i < live) from_float(__uint_as_float(r[i]), y[(int64_t)i * M]);
}

template <int BN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(GW_THREADS, 1)
    gemm_w8a8_kernel(const __grid_constant__ GwArgs a) {
  using C = GwCfg<BN>;
  constexpr int S = C::STAGES;
  extern __shared__ uint8_t smem_gw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_gw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S * C::STAGE);  // first block: both blocks' boxes have arrived
  uint64_t* empty = full + S;     // the MMAs have read them (both blocks)
  uint64_t* acc_full = empty + S;     // an accumulator is complete (both blocks)
  uint64_t* acc_empty = acc_full + 2;  // first block: both blocks' epilogues have read it
  uint64_t* drain_bar = acc_empty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain_bar + 1);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  uint32_t* came = tmem_slot + 2;  // K-tiles asked for by this block; first block: K-tiles, and tiles, that MMAs were committed for
  uint32_t* other_failed = came + 3;  // written by the other block
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const uint64_t tmo = a.timeout_ns;

  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], 2 * GW_EPI_WARPS);
    }
    mbar_init(drain_bar, 1);
    *abort_flag = 0;
    *other_failed = 0;
    fence_mbar_init();
  }
  if (warp == GW_MMA_WARP) tmem_alloc2(tmem_slot, C::COLS);
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // both blocks' barriers are there
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();  // operands, scales and partial sums are those of the kernels before
  const int ntiles = a.mtiles * a.ptiles * a.splits, pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1;
  const int my_tiles = (ntiles - pair + pairs - 1) / pairs;
  // tile -> channels, tokens, K-tiles [k0, k1): neighbours share tokens
  auto coords = [&](int tl, int& m0, int& p0, int& sp, int& k0, int& k1) {
    int id = pair + tl * pairs;
    m0 = (id % a.mtiles) * 2 * GW_BM;
    id /= a.mtiles;
    sp = id % a.splits;
    p0 = (id / a.splits) * BN;
    k0 = (int)((int64_t)a.ktiles * sp / a.splits);
    k1 = (int)((int64_t)a.ktiles * (sp + 1) / a.splits);
  };
  auto fail = [&]() {
    *abort_flag = 1;
    st_cluster_u32(other_failed, rank ^ 1u, 1u);
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
        if (!mbar_wait_cluster(&empty[st], ((j / S) & 1) ^ 1, tmo, abort_flag)) {
          ok = false;
          break;
        }
        uint8_t* A = smem + st * C::STAGE;
        // the second block's bytes may come before they are expected: the phase lasts until this arrival
        if (rank == 0) mbar_arrive_expect_tx(&full[st], 2 * C::STAGE);
        const uint32_t bar = map_rank(&full[st], 0);
        tma_load_2d_pair(smem_u32(A), &a.w_map, kt * GW_KT, m0 + GW_BM * (int)rank, bar);
        tma_load_2d_pair(smem_u32(A + C::A_BYTES), &a.x_map, kt * GW_KT, p0 + BN / 2 * (int)rank, bar);
      }
    }
    came[0] = (uint32_t)j;
    // the commits of the last K-tiles: those before them were waited for, those of tiles are by the epilogue
    for (int i = j - S < 0 ? 0 : j - S; i < j && ok; ++i) ok = mbar_wait_cluster(&empty[i % S], (i / S) & 1, tmo, abort_flag);
    if (!ok && !*abort_flag) fail();
  }

  if (warp == GW_MMA_WARP && rank == 0) {  // converged, an elected lane issues: a divergent one takes 100 clocks an MMA
    const uint32_t idesc = idesc_f16_f32(2 * GW_BM, BN);
    int j = 0, tl = 0;
    bool ok = true;
    for (; tl < my_tiles; ++tl) {
      int m0, p0, sp, k0, k1;
      coords(tl, m0, p0, sp, k0, k1);
      const int b = tl & 1;
      ok = __all_sync(FULL_MASK, mbar_wait_cluster(&acc_empty[b], ((tl >> 1) & 1) ^ 1, tmo, abort_flag));
      if (!ok) break;
      tc_fence_after();
      for (int kt = k0; kt < k1; ++kt, ++j) {
        const int st = j % S;
        ok = __all_sync(FULL_MASK, mbar_wait_cluster(&full[st], (j / S) & 1, tmo, abort_flag));
        if (!ok) break;
        tc_fence_after();
        const uint32_t A = smem_u32(smem + st * C::STAGE);
        const uint64_t ad = sdesc_k_sw128(A), bd = sdesc_k_sw128(A + C::A_BYTES);
        if (elect_one()) {
#pragma unroll
          for (int s = 0; s < 4; ++s)
            mma_f16_pair(tmem + (uint32_t)(b * BN), ad + 2 * s, bd + 2 * s, idesc, (kt > k0 || s > 0) ? 1u : 0u);
          mma_commit_pair(&empty[st]);
        }
      }
      if (!ok) break;
      if (elect_one()) mma_commit_pair(&acc_full[b]);
    }
    if (!ok && lane == 0 && !*abort_flag) fail();
    if (!ok && elect_one()) mma_commit_pair(drain_bar);
    if (lane == 0) {
      came[1] = (uint32_t)j;
      came[2] = (uint32_t)tl;
    }
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
      const int m = m0 + GW_BM * (int)rank + t;
      const bool mok = m < a.M;
      const float sw = mok ? __ldg(a.wscale + m) : 0.0f;
      const float bias = mok && a.bias ? __ldg(a.bias + m) : 0.0f;
      const uint32_t ta = tmem + ((uint32_t)(32 * quarter) << 16) + (uint32_t)(b * BN + half * (BN / 2));
      const int pw = p0 + half * (BN / 2);
#pragma unroll 1
      for (int c = 0; c < BN / 2; c += 32) {
        uint32_t r[32];
        tmem_ld32(ta + c, r);
        // the 32 tokens' scales, one a lane (by now the quantizer has written them: no read-only path)
        const float sx = pw + c + lane < a.P ? a.scale[pw + c + lane] : 0.0f;
        tmem_ld_wait_regs(r);
        if (c + 32 == BN / 2 && tl + 2 < my_tiles) {  // this warp has the whole accumulator: free it for the tile after next
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(map_rank(&acc_empty[b], 0));
        }
        const int live = mok ? a.P - (pw + c) : 0;  // tokens of these 32 that there are
        if (a.part) {
          float* dst = a.part + ((int64_t)sp * a.P + pw + c) * a.M + m;
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (i < live) dst[(int64_t)i * a.M] = __uint_as_float(r[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            r[i] = __float_as_uint(fmaf(__uint_as_float(r[i]), __shfl_sync(FULL_MASK, sx, i) * sw, bias));
          const int64_t at = (int64_t)(pw + c) * a.M + m;
          if (a.ytype == FGQ_F32)
            store_column(static_cast<float*>(a.y) + at, a.M, live, r);
          else if (a.ytype == FGQ_BF16)
            store_column(static_cast<__nv_bfloat16*>(a.y) + at, a.M, live, r);
          else
            store_column(static_cast<__half*>(a.y) + at, a.M, live, r);
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync();  // both blocks' counts and failures are there
  const bool failed = *abort_flag != 0 || *reinterpret_cast<volatile uint32_t*>(other_failed) != 0;  // the same in both
  if (failed && warp == GW_TMA_WARP && lane == 0) {
    auto drain = [](uint64_t* bar, int phase) { mbar_wait_bounded(bar, (uint32_t)phase & 1u, 1u << 20); };
    const int done = (int)ld_cluster_u32(came + 1, 0), tiles = (int)ld_cluster_u32(came + 2, 0);
    for (int i = done > S ? done - S : 0; i < done; ++i) drain(&empty[i % S], i / S);
    for (int i = tiles > 2 ? tiles - 2 : 0; i < tiles; ++i) drain(&acc_full[i & 1], i >> 1);
    if (tiles < my_tiles) drain(drain_bar, 0);
    if (rank == 0) {  // boxes that no MMA has read, S at most as each follows a commit S K-tiles back
      const int mine = (int)came[0], other = (int)ld_cluster_u32(came, 1);
      for (int i = done; i < (mine > other ? mine : other); ++i) {
        if (i >= mine)
          mbar_arrive_expect_tx(&full[i % S], C::STAGE);
        else if (i >= other)
          mbar_forgo_tx(&full[i % S], C::STAGE);
        drain(&full[i % S], i / S);
      }
    }
  }
  if (failed) cluster_sync();  // and nothing is on its way to either
  if (warp == GW_MMA_WARP) {
    tc_fence_after();
    tmem_dealloc2(tmem, C::COLS);
  }
}

// y from the splits' sums: a thread one channel of GW_JOIN tokens, so that their loads are in flight together (512 x 4096,
// two splits: the whole product 39.0 us with one token a thread, 36.8 with four).
constexpr int GW_JOIN = 4;
__global__ void __launch_bounds__(256) join_splits_kernel(const __grid_constant__ GwArgs a) {
  const int64_t n = (int64_t)a.P * a.M;
  const int m = blockIdx.x * 256 + threadIdx.x;
  pdl_wait();
  if (m >= a.M) return;
  const float sw = __ldg(a.wscale + m), bias = a.bias ? __ldg(a.bias + m) : 0.0f;
  for (int64_t p = (int64_t)blockIdx.y * GW_JOIN; p < a.P; p += (int64_t)gridDim.y * GW_JOIN) {
    float v[GW_JOIN] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 2
    for (int s = 0; s < a.splits; ++s)
#pragma unroll
      for (int i = 0; i < GW_JOIN; ++i)
        if (p + i < a.P) v[i] += a.part[s * n + (p + i) * a.M + m];
#pragma unroll
    for (int i = 0; i < GW_JOIN; ++i)
      if (p + i < a.P) store_typed(a.y, a.ytype, (p + i) * a.M + m, fmaf(v[i], a.scale[p + i] * sw, bias));
  }
}

template <int BN>
fgq_status launch_gw(const GwArgs& a, int grid, cudaStream_t s) {
  if (!tc::smem_attr_once<gemm_w8a8_kernel<BN>>(GwCfg<BN>::SMEM)) return FGQ_ERR_CUDA;
  return after_launch(launch_pdl(gemm_w8a8_kernel<BN>, dim3(grid), dim3(GW_THREADS), GwCfg<BN>::SMEM, s, a));
}

}  // namespace

GemmPlan plan_gemm_w8a8(int P, int K, int M) {
  GemmPlan g;
  g.pitch = ((int64_t)K + GW_KT - 1) / GW_KT * GW_KT;
  // 128 tokens a tile also where pairs remain for twice as many tiles: an MMA then reads half as much again of shared
  // memory for its arithmetic, but K is split less or not at all (1000 tokens, 1024 -> 2048: 16.7 us, and 22.7 with
  // 256; 4096 tokens, 512 -> 512: 14.5 and 18.4; 300 tokens, 8192 -> 2048: 31.4 and 33.2)
  const int64_t tiles256 = (int64_t)((M + 2 * GW_BM - 1) / (2 * GW_BM)) * ((P + 255) / 256);
  g.bn = P > 128 && tiles256 * 2 > device_sms() / 2 ? 256 : 128;
  // K split over pairs where there are fewer tiles than half of them, 8 K-tiles each at least
  const int64_t tiles = (int64_t)((M + 2 * GW_BM - 1) / (2 * GW_BM)) * ((P + g.bn - 1) / g.bn), pairs = device_sms() / 2;
  const int64_t by_k = g.pitch / GW_KT / 8;
  int64_t splits = pairs / tiles < by_k ? pairs / tiles : by_k;
  g.splits = (int)(splits < 1 ? 1 : (splits > 16 ? 16 : splits));
  g.part_bytes = g.splits > 1 ? (size_t)g.splits * P * M * 4 : 0;
  return g;
}

fgq_status launch_gemm_w8a8(const GemmPlan& plan, const void* x16, const void* w16, float* part, const float* scale,
                            int P, const float* wscale, int M, const float* bias, void* y, int ytype, cudaStream_t s) {
  GwArgs a;
  memset(&a, 0, sizeof a);
  a.scale = scale;
  a.wscale = wscale;
  a.bias = bias;
  a.y = y;
  a.part = plan.splits > 1 ? part : nullptr;
  a.err = device_error_word();
  const int64_t lim_us = debug_wait_limit_us();
  a.timeout_ns = lim_us < 0 ? GW_TIMEOUT_NS : (uint64_t)lim_us * 1000u;
  a.P = P;
  a.M = M;
  a.ytype = ytype;
  a.ktiles = (int)(plan.pitch / GW_KT);
  a.mtiles = (M + 2 * GW_BM - 1) / (2 * GW_BM);
  a.ptiles = (P + plan.bn - 1) / plan.bn;
  a.splits = plan.splits;
  const int64_t tiles = (int64_t)a.mtiles * a.ptiles * a.splits, pairs = device_sms() / 2;
  if (tiles > INT32_MAX) return FGQ_ERR_UNSUPPORTED;
  if (!make_map_2d(&a.w_map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, w16, (uint64_t)plan.pitch, (uint64_t)M,
                   (uint64_t)plan.pitch * 2, GW_KT, GW_BM, CU_TENSOR_MAP_SWIZZLE_128B) ||
      !make_map_2d(&a.x_map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, x16, (uint64_t)plan.pitch, (uint64_t)P,
                   (uint64_t)plan.pitch * 2, GW_KT, (uint32_t)plan.bn / 2, CU_TENSOR_MAP_SWIZZLE_128B))
    return FGQ_ERR_CUDA;
  const int grid = 2 * (int)(tiles < pairs ? tiles : pairs);
  fgq_status st = plan.bn == 256 ? launch_gw<256>(a, grid, s) : launch_gw<128>(a, grid, s);
  if (st == FGQ_OK && a.part) {
    const int rows = (P + GW_JOIN - 1) / GW_JOIN;
    const dim3 jg((unsigned)((M + 255) / 256), (unsigned)(rows < 65535 ? rows : 65535));
    st = after_launch(launch_pdl(join_splits_kernel, jg, dim3(256), 0, s, a));
  }
  return st;
}

}  // namespace fgq
