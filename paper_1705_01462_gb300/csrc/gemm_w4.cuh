// Many tokens with 4-bit weights on the tensor cores (tcgen05).
//
// y[p][m] = 2^(ex_p + ew_m) sum_k x'[p][k] w'[m][k] + bias[m], with w' = w 2^-ew_m and x' = x 2^-ex_p in fp16: a code times its scale has
// 11 bits and is exact there, down to 2^-26 of its row's largest scale.  The weights stay in 4 bits in memory, and the block's
// warps turn the 128 channels x 128 columns of a stage into the operand, in the shared memory that the MMA reads.  (Expanded
// in memory first, 4096 -> 14336 took 55 us at 64 tokens, 36 of them for the expansion.)
// A block takes a tile of 128 channels and BN tokens, or a part of its K.  Warp roles:
//   warps 0 .. W-1  (W 16 or 8) weights: warp w the row tile w % 8 of every other stage (W = 8: of each), loaded two of its stages
//                   ahead; warps 0-7 (fp32: up to all) then the epilogue: warp w reads TMEM lanes 32 (w % 4) .. (channels), an equal
//                   share of the columns (tokens), applies scales and bias and stores runs of 32 channels;
//   warp W          TMEM allocation and MMA issue;
//   warp W + 1      TMA producer of the tokens.
// Few tiles split K over blocks (fp32 partial sums, joined with scales and bias by a second kernel).
// (Pairs of SMs, cta_group::2, halve the operands' traffic, but each stage's weights then take arrivals across the pair: 1.1 us a stage of
// 64 columns, where this form takes 0.55 us for 128.)
// Bound by the instructions and shared-memory writes that turn a stage's codes into the operand: 64 tokens, 4096 -> 14336: 22.5 us
// (28 without the order of stores that meets all banks); half of the issue slots and of the shared memory's cycles are in use.
// fp32 tokens are two rows of fp16 that add up to them within 2^-22, and their sums leave the tensor memory for registers every
// 256 columns: the tensor cores cut sums off, and over 4096 columns that took outputs to 2e-6 of 64-bit sums, over 16384 to 1e-5;
// so it is 3e-7 for any length.  (2048 tokens, 4096 -> 4096: 139 us; without 133.)
// Every wait is bounded; on expiry FGQ_ERR_TIMEOUT is recorded and each role leaves its loop; copies and MMAs under way are waited
// for, and the tensor memory is freed.
#pragma once

#include <cstring>

#include "w4_many.h"

namespace fgq {
namespace w4 {

using tc::make_map_2d;

constexpr int G4_BM = 128, G4_KT = 128;  // channels and columns of a stage
constexpr int G4_EPI_WARPS = 8;
constexpr uint64_t G4_TIMEOUT_NS = 1000000000ull;  // 1 s per wait

template <int BN, int W>
struct G4Cfg {
  static constexpr int MMA_WARP = W, TMA_WARP = W + 1, THREADS = 32 * (W + 2), BLOCKS = W == 8 ? 2 : 1;  // blocks an SM
  // each operand in two halves of 64 columns (128-byte rows)
  static constexpr int A_HALF = G4_BM * 128, B_HALF = BN * 128, STAGE = 2 * (A_HALF + B_HALF);
  static constexpr int STAGES = BN == 256 || W == 8 ? 2 : (BN == 128 ? 3 : 4);
  static constexpr int SMEM = 1024 + STAGES * STAGE + 8 * (3 * STAGES + 5) + 16;
  static_assert(BLOCKS * (SMEM + 1536) <= 233472 && SMEM + 512 <= 232448, "shared memory budget");
};

struct G4Args {
  CUtensorMap x_map;
  Matrix w;
  const float* scale;  // or nullptr: 1
  const int* wexp;     // [M rounded up to row tiles]: w' = w 2^(12 - wexp)
  const float* bias;
  void* y;
  float* part;  // [splits][P][M] partial sums, or nullptr
  unsigned int* err;
  uint64_t timeout_ns;
  int P, M, mtiles, ptiles, splits, ytype;
  // GROUPED: tokens sorted by expert, a block one unit of them, or BN rows of it, and of w or of `up`; fp32 outputs without bias to y or y_up
  Matrix up;
  void* y_up;
  const Unit* units;
  const int* nunits;
  int matrices;  // 2: w and up
  int tiles;     // of BN rows, of a unit
};

// The first `live` of N values, one a row of M elements.
template <typename T, int N>
__device__ __forceinline__ void store_column(T* y, int M, int live, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < live) from_float(v[i], y[(int64_t)i * M]);
}

constexpr int TAKE = 2;  // stages of fp32 sums (see above)
// PARTS rows of x make a token (fp32: two).
// GROUPED: the rows' exponents are found by the block itself (a scan of its scales, while the kernel before it runs).
template <int BN, int PER, int PARTS, bool GROUPED, int W>
__global__ void __launch_bounds__(G4Cfg<BN, W>::THREADS, G4Cfg<BN, W>::BLOCKS) gemm_w4_kernel(const __grid_constant__ G4Args a) {
  using C = G4Cfg<BN, W>;
  constexpr int S = C::STAGES;
  // fp32: sums are taken from the tensor memory every TAKE stages, by TAKERS warps of COLUMNS columns each, from two places in turn
  constexpr bool F32 = PARTS == 2;
  constexpr int TAKERS = BN == 64 ? 8 : 16, COLUMNS = BN / (TAKERS / 4), TMEM = F32 ? 2 * BN : BN;
  extern __shared__ uint8_t smem_g4[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_g4) + 1023) & ~uintptr_t(1023));
  uint64_t* full_x = reinterpret_cast<uint64_t*>(smem + S * C::STAGE);  // the tokens have arrived
  uint64_t* full_w = full_x + S;   // the weights have been written
  uint64_t* empty = full_w + S;    // the MMAs have read both
  uint64_t* acc_full = empty + S;   // [2] sums are complete
  uint64_t* taken = acc_full + 2;  // [2] and in registers
  uint64_t* drain_bar = taken + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain_bar + 1);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  uint32_t* read = tmem_slot + 2;  // stages that MMAs were committed for
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // tile -> channels, tokens, tile columns [c0, c1): neighbours share tokens
  int id = blockIdx.x;
  const int m0 = (id % a.mtiles) * G4_BM;
  id /= a.mtiles;
  Matrix w = a.w;
  void* y = a.y;
  int sp = 0, p0, end = a.P;  // rows of tokens from p0, tokens up to `end`
  int64_t first_tile = 0;
  if constexpr (GROUPED) {
    if (id % a.matrices) w = a.up, y = a.y_up;
    id /= a.matrices;
    const int tile = id % a.tiles;
    id /= a.tiles;
    if (id >= __ldcg(a.nunits)) {  // units are those of a kernel before the one that this one waits for
      pdl_wait();  // what comes after this kernel comes after that one
      return;
    }
    const int4 u = __ldcg(reinterpret_cast<const int4*>(a.units) + id);
    first_tile = (int64_t)u.x * w.rt * w.ct;
    p0 = u.y * PARTS + tile * BN;
    end = u.y + u.z;
    if (p0 >= end * PARTS) {
      pdl_wait();
      return;
    }
  } else {
    sp = id % a.splits, p0 = (id / a.splits) * BN;
  }
  const int c0 = GROUPED ? 0 : (int)((int64_t)w.ct * sp / a.splits), n = (GROUPED ? w.ct : (int)((int64_t)w.ct * (sp + 1) / a.splits)) - c0;
  const uint64_t tmo = a.timeout_ns;

  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(&full_x[i], 1);
      mbar_init(&full_w[i], 8);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&taken[i], TAKERS);
    }
    mbar_init(drain_bar, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == C::MMA_WARP) {
    tmem_alloc(tmem_slot, TMEM);
    tmem_relinquish();
  }
  __shared__ uint32_t tops[GROUPED ? G4_BM : 1];  // GROUPED: the rows' largest scales
  if constexpr (GROUPED) {
    if (threadIdx.x < G4_BM) tops[threadIdx.x] = 0u;
    __syncthreads();
    if (warp < W) {  // as magnitudes, which compare as whole numbers: warp w row tile w % 8, every other column
      constexpr int CHUNKS = 2 * PER;  // pieces of eight scales, 8 / PER rows, of a tile
      const int d = warp & 7, rt = min(m0 / TILE_ROWS + d, w.rt - 1), chunk = lane % CHUNKS;
      const uint16_t* sc = w.scales + (first_tile + (int64_t)rt * w.ct) * (TILE_ROWS * PER) + chunk * 8;
      uint32_t top[8 / PER] = {};
      for (int c = lane / CHUNKS + 32 / CHUNKS * (warp >> 3); c < n; c += W / 8 * (32 / CHUNKS)) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(sc + (int64_t)c * (TILE_ROWS * PER)));
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i % PER < (c == n - 1 ? w.live : PER)) top[i / PER] = max(top[i / PER], (i & 1 ? u[i / 2] >> 16 : u[i / 2]) & 0x7fffu);
      }
#pragma unroll
      for (int i = 0; i < 8 / PER; ++i) {
#pragma unroll
        for (int o = CHUNKS; o < 32; o <<= 1) top[i] = max(top[i], __shfl_xor_sync(FULL_MASK, top[i], o));
        if (lane < CHUNKS) atomicMax(&tops[TILE_ROWS * d + chunk * (8 / PER) + i], top[i]);
      }
    }
  }
  // the exponent of row r's largest scale (subnormal ones: of the smallest normal)
  auto exponent = [&](int r) {
    return GROUPED ? max((int)(tops[GROUPED ? r : 0] >> 7) - 127, -126) : __ldcg(a.wexp + m0 + r);
  };
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  auto fail = [&]() {
    *abort_flag = 1;
    record_error(a.err, FGQ_ERR_TIMEOUT);
  };
  const int runs = F32 ? (n + TAKE - 1) / TAKE : 1;  // of stages that are summed in the tensor memory
  int issued = 0;  // by the producer
  bool ok = true;

  if (warp == C::TMA_WARP && lane == 0) {
    pdl_wait();  // the tokens may be those of the kernel before
    for (; issued < n; ++issued) {
      const int st = issued % S;
      if (!mbar_wait_timed(&empty[st], ((issued / S) & 1) ^ 1, tmo, abort_flag, 0)) {
        ok = false;
        break;
      }
      const uint32_t B = smem_u32(smem + st * C::STAGE + 2 * C::A_HALF);
      mbar_arrive_expect_tx(&full_x[st], 2 * C::B_HALF);
      tma_load_2d(B, &a.x_map, (c0 + issued) * G4_KT, p0, &full_x[st]);
      tma_load_2d(B + C::B_HALF, &a.x_map, (c0 + issued) * G4_KT + 64, p0, &full_x[st]);
    }
    // the last stages' commits: those before them were waited for
    for (int i = n > S ? n - S : 0; i < n && ok; ++i) ok = mbar_wait_timed(&empty[i % S], (i / S) & 1, tmo, abort_flag, 0);
    if (!ok && !*abort_flag) fail();
  }

  if (warp == C::MMA_WARP) {  // converged, an elected lane issues
    const uint32_t idesc = idesc_f16_f32(G4_BM, BN);
    int j = 0;
    for (; j < n; ++j) {
      const int st = j % S, run = F32 ? j / TAKE : 0;
      const bool fresh = F32 ? j % TAKE == 0 : j == 0;
      if (F32 && fresh && run >= 2) {
        ok = mbar_wait_warp(&taken[run & 1], ((run >> 1) & 1) ^ 1, tmo, abort_flag);
        if (!ok) break;
      }
      ok = mbar_wait_warp(&full_x[st], (j / S) & 1, tmo, abort_flag) && mbar_wait_warp(&full_w[st], (j / S) & 1, tmo, abort_flag);
      if (!ok) break;
      tc_fence_after();
      const uint32_t A = smem_u32(smem + st * C::STAGE), B = A + 2 * C::A_HALF;
      if (elect_one()) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint64_t ad = sdesc_k_sw128(A + half * C::A_HALF), bd = sdesc_k_sw128(B + half * C::B_HALF);
#pragma unroll
          for (int s = 0; s < 4; ++s) mma_f16(tmem + (uint32_t)((run & 1) * BN), ad + 2 * s, bd + 2 * s, idesc, fresh && half == 0 && s == 0 ? 0u : 1u);
        }
        mma_commit(&empty[st]);
        if (j == n - 1 || (F32 && j % TAKE == TAKE - 1)) mma_commit(&acc_full[run & 1]);
      }
      __syncwarp();
    }
    if (!ok) {
      if (lane == 0 && !*abort_flag) fail();
      if (elect_one()) mma_commit(drain_bar);
    }
    if (lane == 0) *read = (uint32_t)j;
  }

  float acc[F32 ? COLUMNS / 2 : 1];
  const int taker_column = (warp >> 2) * COLUMNS;
  if (F32) {
#pragma unroll
    for (int i = 0; i < COLUMNS / 2; ++i) acc[i] = 0.0f;
  }
  int took = 0;  // runs that this warp has
  auto take = [&]() {
    const int at = took & 1;
    ok = mbar_wait_warp(&acc_full[at], (took >> 1) & 1, tmo, abort_flag);
    if (!ok) return;
    tc_fence_after();
#pragma unroll
    for (int c = 0; c < COLUMNS; c += 32) {
      uint32_t r[32];
      tmem_ld32(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + (uint32_t)(at * BN + taker_column + c), r);
      tmem_ld_wait_regs(r);
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[c / 2 + i] += __uint_as_float(r[2 * i]) + __uint_as_float(r[2 * i + 1]);
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(&taken[at]);
    ++took;
  };

  if (warp < W) {
    const int d = warp & 7, first = warp >> 3, g = lane >> 2, t = lane & 3;
    const int own = min(TILE_ROWS * d, (w.rt - 1) * TILE_ROWS - m0);  // a row tile past the last is read as the last
    const int64_t at = first_tile + (int64_t)(m0 + own) / TILE_ROWS * w.ct + c0;
    constexpr int STEP = W / 8;  // every other stage, or each
    constexpr int AHEAD = F32 && BN == 256 ? 1 : 2;  // 32 registers are the sums'
    Tile<PER> tile[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (first + STEP * i < n) tile[i].load(w.codes, w.scales, at + first + STEP * i, lane);
    pdl_wait();  // the exponents are those of the kernel before
    // what takes the rows' scales to fp16's range, in two factors: it passes fp32's largest for tiny ones
    float up[2], up2[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int e = 12 - exponent(own + g + 8 * r);
      up[r] = pow2f(e / 2);
      up2[r] = pow2f(e - e / 2);
    }
    // lanes of odd rows take a word's neighbour first: stores of eight lanes, two rows, then meet all banks
    const int odd = g & 1, last = w.live < PER ? w.ct - 1 - c0 : -1;  // the stage with groups that are none
    for (int j0 = first; j0 < n && ok; j0 += STEP * AHEAD) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int j = j0 + STEP * i, st = j % S;
        if (j >= n || !ok) break;
        uint32_t s2[2][PER];  // scales as fp16 pairs
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int k = 0; k < PER; ++k) {
            float s = (PER == 4 && odd ? tile[i].s[r].get(k ^ 1) : tile[i].s[r].get(k)) * up[r] * up2[r];
            if (PER > 1 && j == last && (PER == 4 ? k ^ odd : k) >= w.live) s = 0.0f;
            s2[r][k] = pack2(s, s, __half());
          }
        uint4 v[2][4];
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int k = 0; k < 4; ++k) v[r][k] = scaled_codes(odd ? tile[i].word(r, k ^ 1) : tile[i].word(r, k), s2[r][k * PER / 4]);
        if (j + STEP * AHEAD < n) tile[i].load(w.codes, w.scales, at + j + STEP * AHEAD, lane);
        ok = mbar_wait_warp(&empty[st], ((j / S) & 1) ^ 1, tmo, abort_flag);
        if (!ok) break;
        uint8_t* A = smem + st * C::STAGE;
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            *reinterpret_cast<uint4*>(A + (k >> 1) * C::A_HALF + tc::sw128(TILE_ROWS * d + 8 * r + g, 4 * ((k & 1) ^ odd) + t)) = v[r][k];
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&full_w[st]);
        if (F32 && warp < TAKERS && took < j / TAKE) take();  // the run before this stage's
      }
    }
    if (F32 && warp < TAKERS)
      while (ok && took < runs) take();
    if (!ok && lane == 0 && !*abort_flag) fail();
  }

  if (warp < (F32 ? TAKERS : G4_EPI_WARPS) && ok) {
    if (!F32) {
      ok = mbar_wait_warp(acc_full, 0, tmo, abort_flag);
      if (!ok && lane == 0 && !*abort_flag) fail();
    }
    if (ok) {
      tc_fence_after();
      constexpr int OWN = F32 ? COLUMNS : BN / 2, N = 32 / PARTS;  // columns of a warp, tokens of 32 columns
      const int m = m0 + 32 * (warp & 3) + lane, column = (warp >> 2) * OWN;
      const bool mok = m < a.M;
      const float sw = mok ? pow2f(exponent(m - m0) - 12) : 0.0f;
      const float bias = mok && a.bias ? __ldg(a.bias + m) : 0.0f;
#pragma unroll(F32 ? OWN / 32 : 1)
      for (int c = 0; c < OWN; c += 32) {
        const int tok = (p0 + column + c) / PARTS;
        float v[N];
        if constexpr (F32) {
#pragma unroll
          for (int i = 0; i < N; ++i) v[i] = acc[c / 2 + i];
        }
        uint32_t r[32];
        if (!F32) tmem_ld32(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + (uint32_t)(column + c), r);
        // the tokens' scales, one a lane
        const float sx = !a.scale ? 1.0f : (lane < N && tok + lane < end ? __ldcg(a.scale + tok + lane) : 0.0f);
        if constexpr (!F32) {
          tmem_ld_wait_regs(r);
#pragma unroll
          for (int i = 0; i < N; ++i) v[i] = __uint_as_float(r[i]);
        }
        const int live = mok ? end - tok : 0;  // how many tokens there are
        if (!GROUPED && a.part) {
          store_column(a.part + ((int64_t)sp * a.P + tok) * a.M + m, a.M, live, v);
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) v[i] = fmaf(v[i], __shfl_sync(FULL_MASK, sx, i) * sw, bias);
          const int64_t out = (int64_t)tok * a.M + m;
          if constexpr (F32 || GROUPED)
            store_column(static_cast<float*>(y) + out, a.M, live, v);
          else if (a.ytype == FGQ_BF16)
            store_column(static_cast<__nv_bfloat16*>(y) + out, a.M, live, v);
          else
            store_column(static_cast<__half*>(y) + out, a.M, live, v);
        }
      }
      tc_fence_before();
    }
  }

  __syncthreads();
  if (*abort_flag && warp == C::TMA_WARP && lane == 0) {  // what is still under way: MMAs, then boxes that no MMA has read
    const int done = (int)*read;
    auto drain = [](uint64_t* bar, int phase) { mbar_wait_bounded(bar, (uint32_t)phase & 1u, 1u << 16); };
    drain(done < n ? drain_bar : &acc_full[(runs - 1) & 1], done < n ? 0 : (runs - 1) >> 1);
    for (int i = done > S ? done - S : 0; i < done; ++i) drain(&empty[i % S], i / S);
    for (int i = done; i < issued; ++i) drain(&full_x[i % S], i / S);
  }
  __syncthreads();
  if (warp == C::MMA_WARP) {
    tc_fence_after();
    tmem_dealloc(tmem, TMEM);
  }
}

template <int BN, int PER, int PARTS, bool GROUPED, int W>
fgq_status launch_g4_per(const G4Args& a, int grid, cudaStream_t s) {
  using C = G4Cfg<BN, W>;
  if (!tc::smem_attr_once<gemm_w4_kernel<BN, PER, PARTS, GROUPED, W>>(C::SMEM)) return FGQ_ERR_CUDA;
  return after_launch(launch_pdl(gemm_w4_kernel<BN, PER, PARTS, GROUPED, W>, dim3(grid), dim3(C::THREADS), C::SMEM, s, a));
}
template <int BN, int PARTS, bool GROUPED, int W>
fgq_status launch_g4(const G4Args& a, int grid, cudaStream_t s) {
  if (a.w.per == 4) return launch_g4_per<BN, 4, PARTS, GROUPED, W>(a, grid, s);
  return a.w.per == 2 ? launch_g4_per<BN, 2, PARTS, GROUPED, W>(a, grid, s) : launch_g4_per<BN, 1, PARTS, GROUPED, W>(a, grid, s);
}

}  // namespace w4
}  // namespace fgq
